"""The autograd forms of the operators against torch's own gradients of the
plain formulas in 64 bits, and the example that trains and serves with them.

Tolerances, u = 2^-24, fp32 tensors: a gradient's terms are each formed in fp32
from sums of n terms, so each term is off by (n + 16) u of its size at most; the
bounds add the sizes of the terms, taken from the formula in 64 bits."""
import pytest
import torch

from paper_2608_13966_amd import example, ste

pytestmark = pytest.mark.gpu

U, V = 2.0 ** -24, 2.0 ** -8
EPS = 1e-6


def rand(*shape, seed=0, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, device="cuda", generator=g).to(dtype)


def norm_terms(x, w, res, dy, dh):
    """Gradients of the formula in 64 bits, and the sizes of their terms."""
    n = x.shape[-1]
    x, w, dy = x.double(), w.double(), dy.double()
    h = x if res is None else x + res.double()
    rstd = ((h * h).mean(-1, keepdim=True) + EPS).rsqrt()
    c = (dy * w * h).mean(-1, keepdim=True) * rstd * rstd
    size_c = (dy * w * h).abs().mean(-1, keepdim=True) * rstd * rstd
    dx = rstd * (dy * w - h * c)
    size = rstd * ((dy * w).abs() + h.abs() * size_c)
    if dh is not None:
        dx, size = dx + dh.double(), size + dh.double().abs()
    lead = tuple(range(x.dim() - 1))
    dw, size_w = (dy * h * rstd).sum(lead), (dy * h * rstd).abs().sum(lead)
    return dx, size * (n + 16) * U + 1e-30, dw, size_w * (n + 16 + x.numel() // n) * U + 1e-30


@pytest.mark.parametrize("shape", [(7, 96), (1, 33), (3, 5, 256), (2, 1, 4, 40)])
@pytest.mark.parametrize("residual", [False, True])
def test_norm_gradients(shape, residual):
    x, w = rand(*shape, seed=1).requires_grad_(), (1 + 0.1 * rand(shape[-1], seed=2)).requires_grad_()
    res = rand(*shape, seed=3).requires_grad_() if residual else None
    dy, dh = rand(*shape, seed=4), rand(*shape, seed=5) if residual else None
    o = ste.add_rms_norm(x, w, res, eps=EPS)
    if residual:
        torch.autograd.backward(o, [dy, dh])
    else:
        o.backward(dy)
    dx, tx, dw, tw = norm_terms(x.detach(), w.detach(), None if res is None else res.detach(), dy, dh)
    assert x.grad.shape == x.shape and bool(((x.grad.double() - dx).abs() <= tx).all())
    assert bool(((w.grad.double() - dw).abs() <= tw).all())
    if residual:
        assert torch.equal(res.grad, x.grad)


def test_norm_against_torch_autograd():
    """The formula above is the gradient of the plain form."""
    x, w, res = (rand(6, 48, seed=i).double().requires_grad_() for i in (1, 2, 3))
    dy, dh = rand(6, 48, seed=4).double(), rand(6, 48, seed=5).double()
    w = rand(48, seed=2).double().requires_grad_()
    h = x + res
    y = h * ((h * h).mean(-1, keepdim=True) + EPS).rsqrt() * w
    torch.autograd.backward([y, h], [dy, dh])
    dx, _, dw, _ = norm_terms(x.detach(), w.detach(), res.detach(), dy, dh)
    assert torch.allclose(x.grad, dx, rtol=1e-12, atol=1e-13) and torch.allclose(w.grad, dw, rtol=1e-12, atol=1e-13)


def test_norm_mixed_types_and_strides():
    x = rand(9, 130, seed=1, dtype=torch.bfloat16)[:, 1:129].requires_grad_()
    x.retain_grad()
    res, w = rand(128, 9, seed=2).t().requires_grad_(), rand(128, seed=3, dtype=torch.bfloat16).requires_grad_()
    y, h = ste.add_rms_norm(x, w, res)
    assert y.dtype is torch.bfloat16 and h.dtype is torch.float32
    y.sum().backward()  # a gradient of stride 0, and none of h
    assert x.grad.dtype is torch.bfloat16 and res.grad.dtype is torch.float32 and w.grad.dtype is torch.bfloat16
    dx, tx, dw, tw = norm_terms(x.detach(), w.detach(), res.detach(), torch.ones_like(y), None)
    assert bool(((res.grad.double() - dx).abs() <= tx).all())
    assert bool(((x.grad.double() - dx).abs() <= tx + V * dx.abs()).all())
    assert bool(((w.grad.double() - dw).abs() <= tw + V * dw.abs()).all())


def test_norm_unused_outputs_and_frozen_inputs():
    x, w, res = rand(4, 64, seed=1).requires_grad_(), rand(64, seed=2).requires_grad_(), rand(4, 64, seed=3)
    y, h = ste.add_rms_norm(x, w, res)
    dh = rand(4, 64, seed=4)
    h.backward(dh)  # y took no part
    assert torch.equal(x.grad, dh) and w.grad is None
    x, w = rand(4, 64, seed=1), rand(64, seed=2).requires_grad_()
    ste.add_rms_norm(x, w).sum().backward()
    assert x.grad is None and w.grad is not None
    x, w = rand(4, 64, seed=1).requires_grad_(), rand(64, seed=2)
    ste.add_rms_norm(x, w).sum().backward()
    assert x.grad is not None and w.grad is None
    x = torch.empty(0, 64, device="cuda").requires_grad_()
    ste.add_rms_norm(x, w).sum().backward()
    assert x.grad.shape == (0, 64)


def plain_loss(z, index, teacher, tau, weight):
    z, t = z.double() / tau, teacher.double() / tau
    valid = index >= 0
    t = t.masked_fill(~valid, float("-inf"))
    logp = torch.log_softmax(t, -1).masked_fill(~valid, 0.0)
    p = logp.exp().masked_fill(~valid, 0.0)
    logq = torch.log_softmax(z, -1).gather(-1, index.clamp(min=0))
    loss = (p * (logp - logq)).sum(-1)
    return loss if weight is None else loss * weight.double()


@pytest.mark.parametrize("shape, listed", [((5, 300), 8), ((2, 3, 5000), 17), ((1, 1), 1), ((40000,), 64)])
@pytest.mark.parametrize("reduction", ["mean", "weighted", "rows"])
def test_distill_gradient(shape, listed, reduction):
    z = rand(*shape, seed=1).requires_grad_()
    index = torch.topk(rand(*shape, seed=2), min(listed, shape[-1]), dim=-1)[1]
    teacher = rand(*index.shape, seed=3)
    if listed > 1:
        index[..., -1] = -1
    weight = rand(*shape[:-1], seed=4).abs() if reduction == "weighted" else None
    zd = z.detach().double().requires_grad_()
    got = ste.distill_topk_loss(z, index, teacher, temperature=1.5, row_weight=weight)
    want = plain_loss(zd, index, teacher, 1.5, weight)
    assert got.shape == z.shape[:-1]
    # a sum over the classes and one over the list, each term off by a few u of a logit below 8
    n = shape[-1] + listed + 32
    assert bool(((got - want).abs() <= n * U * (want.abs() + 16)).all())
    g = rand(*shape[:-1], seed=5)
    (got.mean() if reduction != "rows" else (got * g).sum()).backward()
    (want.mean() if reduction != "rows" else (want * g.double()).sum()).backward()
    # q and p each relative to themselves: n u at most
    q = torch.softmax(z.detach().double() / 1.5, -1)
    scale = (1.0 if reduction != "rows" else g.double().abs()[..., None]) / 1.5
    if weight is not None:
        scale = scale * weight.double()[..., None]
    p = (zd.grad / scale - q).abs() + q if reduction == "rows" else (zd.grad * got.numel() / scale).abs() + 2 * q
    assert bool(((z.grad.double() - zd.grad).abs() <= n * U * scale * (p + q) + 1e-12).all())


def test_example_learns_and_serves_what_it_learnt():
    s, losses, t = example.run(steps=30, tokens=96, vocab=512, width=128, hidden=192, log=None)
    assert float(losses[-1]) < 0.5 * float(losses[0]), losses
    with torch.no_grad():
        want = s(t).float()
        exact, eight = example.Server(s, False)(t), example.Server(s, True)(t)
        one = example.Server(s, True)(t[5:6])
    # bf16 rows, the same r: every stored value's rounding 2^-8, at some 10 places on the way, in quadrature and
    # with a gain of 2; 8-bit rows: 2^-4 at three places instead
    assert float((exact - want).norm() / want.norm()) < 2 * 10 ** 0.5 * V
    assert float((eight - want).norm() / want.norm()) < 2 * 3 ** 0.5 * 2 ** -4
    # a token alone goes through the kernel for few tokens: the sums' order, now and then a bf16 or 8-bit step
    assert float((one[0] - eight[5]).norm() / eight[5].norm()) < 2 ** -4


def test_packed_codes_of_a_layer_are_its_r():
    from paper_2608_13966_amd import ops
    layer = ste.QuasarLinear(128, 48, bits=3, group=64)
    x = torch.eye(128, device="cuda", dtype=torch.bfloat16)
    for _ in range(2):
        y = ops.linear_codes(x, layer.packed())["y"]
        assert torch.equal(y.t(), layer.r)
        layer(rand(4, 128, seed=1)).square().sum().backward()
        layer.step()


@pytest.mark.parametrize("x_type,r_type", [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32),
                                           (torch.bfloat16, torch.bfloat16)])
@pytest.mark.parametrize("stream_too", [False, True])
def test_norm_gradients_have_their_inputs_precision(x_type, r_type, stream_too):
    """Each input's gradient is rounded to its own type once: an fp32 input's not to the other's bf16 first.  The formula
    with the h that the forward pass kept, in 64 bits; its bound as above."""
    x, res = rand(30, 200, seed=1, dtype=x_type).requires_grad_(), rand(30, 200, seed=2, dtype=r_type).requires_grad_()
    w = (1 + 0.1 * rand(200, seed=3)).requires_grad_()
    y, h = ste.add_rms_norm(x, w, res, eps=EPS)
    dy, dh = rand(30, 200, seed=4, dtype=y.dtype), rand(30, 200, seed=5, dtype=h.dtype) if stream_too else None
    torch.autograd.backward([y, h] if stream_too else [y], [dy, dh] if stream_too else [dy])
    rstd = ((x.detach().double() + res.detach().double()).square().mean(-1, keepdim=True) + EPS).rsqrt()
    n, u = h.detach().double() * rstd, dy.double() * w.detach().double()
    dx, size = rstd * (u - n * (u * n).mean(-1, keepdim=True)), rstd * (u.abs() + n.abs() * (u * n).abs().mean(-1, keepdim=True))
    if stream_too:
        dx, size = dx + dh.double(), size + dh.double().abs()
    # rstd's own error beside the others': another (200 + 16) u of each term, three times a term at most
    tol = 4 * size * (200 + 16) * U
    for t in (x, res):
        assert t.grad.dtype is t.dtype
        assert bool(((t.grad.double() - dx).abs() <= tol + (V * dx.abs() * 1.01 if t.dtype is torch.bfloat16 else 0)).all())


def test_a_frozen_input_does_not_widen_the_gradient():
    x, res, w = rand(4, 64, seed=1), rand(4, 64, seed=2, dtype=torch.bfloat16).requires_grad_(), rand(64, seed=3)
    y, h = ste.add_rms_norm(x, w, res)
    torch.autograd.backward([y, h], [rand(4, 64, seed=4), rand(4, 64, seed=5, dtype=torch.bfloat16)])
    assert res.grad.dtype is torch.bfloat16 and x.grad is None


def test_distill_takes_lists_cut_from_longer_ones():
    z = rand(2, 6, 500, seed=1)
    values, index = torch.topk(rand(2, 6, 500, seed=2), 40, dim=-1)
    runs = []
    for i, t in ((index[..., :16], values[..., :16]), (index[..., :16].contiguous(), values[..., :16].contiguous()),
                 (index.transpose(0, 1)[..., :16].contiguous().transpose(0, 1), values[..., :16])):
        a = z.clone().requires_grad_()
        loss = ste.distill_topk_loss(a, i, t, row_weight=torch.ones(12, 2, device="cuda")[:, 0].reshape(2, 6))
        loss.sum().backward()
        runs.append((loss.detach(), a.grad))
    for loss, grad in runs[1:]:
        assert torch.equal(loss, runs[0][0]) and torch.equal(grad, runs[0][1])
