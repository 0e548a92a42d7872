"""The operators of a training step together: autograd forms against torch's own
gradients of the plain formulas in 64 bits, a step captured into a graph, calls on
other streams, and the example that trains and serves with them.

Tolerances, u = 2^-24: as in the operators' own tests, a term of n summands is off
by (n + 16) u of the sum of their sizes; the bounds add the terms' sizes."""
import pytest
import torch

from paper_2608_13966_amd import example, ops as O, ste

pytestmark = pytest.mark.gpu

DEV = "cuda"
U, V = 2.0 ** -24, 2.0 ** -8
SLEEP = 1 << 21  # of torch's spinning kernel: milliseconds
E4M3 = torch.float8_e4m3fn


def rand(*shape, seed=0, dtype=torch.float32):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(shape, device=DEV, generator=g).to(dtype)


def back(o):
    return o["q"].double() * torch.exp2(o["exponent"].double() - 127).repeat_interleave(128, 1)[:, :o["q"].shape[1]]


# ---- autograd forms -----------------------------------------------------------------

@pytest.mark.parametrize("shape", [(7, 96), (1, 33), (3, 5, 256), (2, 1, 4, 40)])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("with_bias", [False, True])
def test_layer_norm_gradients(shape, residual, with_bias):
    n, rows = shape[-1], torch.Size(shape[:-1]).numel()
    x, w = rand(*shape, seed=1).requires_grad_(), (1 + 0.1 * rand(n, seed=2)).requires_grad_()
    b = rand(n, seed=6).requires_grad_() if with_bias else None
    res = rand(*shape, seed=3).requires_grad_() if residual else None
    dy, dh = rand(*shape, seed=4), rand(*shape, seed=5)
    o = ste.add_layer_norm(x, w, b, res)
    torch.autograd.backward(o if residual else [o], [dy, dh] if residual else [dy])
    xd, wd, bd, rd = (None if t is None else t.detach().double().requires_grad_() for t in (x, w, b, res))
    h = xd if rd is None else xd + rd
    y = torch.nn.functional.layer_norm(h, (n,), wd, bd, 1e-5)
    torch.autograd.backward([y, h] if residual else [y], [dy.double(), dh.double()] if residual else [dy.double()])
    with torch.no_grad():
        var, mean = torch.var_mean(h, -1, correction=0, keepdim=True)
        r = (var + 1e-5).rsqrt()
        nn, u = ((h - mean) * r), (dy.double() * wd)
        # mean and rstd are off by (n + 8) u of the row's sizes as well, through n and outright
        near = (h.abs().mean(-1, keepdim=True) * r + 1)
        size = r * near * (u.abs() + u.abs().mean(-1, keepdim=True) + (nn.abs() + near) * (u * nn).abs().mean(-1, keepdim=True)
                           + (nn.abs() + near) * u.abs().mean(-1, keepdim=True))
        size = size + (dh.abs() if residual else 0)
        lead = tuple(range(len(shape) - 1))
        size_w = (dy.double().abs() * near * (nn.abs() + 1)).sum(lead)
    assert ((x.grad.double() - xd.grad).abs() <= 4 * (n + 16) * U * size).all()
    assert ((w.grad.double() - wd.grad).abs() <= 4 * (n + rows + 16) * U * size_w).all()
    if with_bias:
        assert ((b.grad.double() - bd.grad).abs() <= (rows + 8) * U * dy.double().abs().sum(lead)).all()
    if residual:
        assert torch.equal(res.grad, x.grad)


def test_a_frozen_input_does_not_widen_the_gradient():
    x, res, w = rand(4, 64, seed=1), rand(4, 64, seed=2, dtype=torch.bfloat16).requires_grad_(), rand(64, seed=3)
    y, h = ste.add_layer_norm(x, w, None, res)
    torch.autograd.backward([y, h], [rand(4, 64, seed=4), rand(4, 64, seed=5, dtype=torch.bfloat16)])
    assert res.grad.dtype is torch.bfloat16 and x.grad is None
    res.grad = None
    _, h = ste.add_layer_norm(x, w, None, res)  # only the stream goes on
    g = rand(4, 64, seed=5, dtype=torch.bfloat16)
    h.backward(g)
    assert torch.equal(res.grad, g)


@pytest.mark.parametrize("shape", [(), (5,), (3, 7), (2, 0), (2, 3, 4)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_embed_gradients(shape, dtype):
    w = rand(20, 48, seed=1, dtype=dtype).requires_grad_()
    t = torch.randint(-1, 21, shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(2))
    y = ste.embed(t, w, scale=2.0)
    assert y.shape == (*shape, 48) and y.dtype is dtype
    dy = rand(*shape, 48, seed=3, dtype=dtype)
    y.backward(dy)
    wd = w.detach().double().requires_grad_()
    ok = (t >= 0) & (t < 20)
    want = torch.where(ok[..., None], 2.0 * wd[torch.where(ok, t, 0)], 0.0)
    want.backward(dy.double())
    assert torch.equal(y.double(), want.detach())  # a power of two
    size = torch.zeros(20, 48, device=DEV, dtype=torch.float64).index_add_(0, t[ok].reshape(-1), 2 * dy.double()[ok].abs().reshape(-1, 48))
    assert w.grad.dtype is dtype
    e = (t.numel() + 2) * U * size
    assert ((w.grad.double() - wd.grad).abs() <= e + (V if dtype is torch.bfloat16 else 0) * (wd.grad.abs() + e)).all()


@pytest.mark.parametrize("act", ["relu", "silu", "gelu"])
@pytest.mark.parametrize("shape", [(300,), (5, 200), (2, 3, 130)])
def test_activation_gradients(act, shape):
    x = rand(*shape, seed=1).requires_grad_()
    dy = rand(*shape, seed=2)
    y = ste.activation(x, act)
    y.backward(dy)
    flat = x.detach().reshape(-1, shape[-1])
    kept = back(O.checkpoint_rows(flat)).view(shape).requires_grad_()
    f = getattr(torch.nn.functional, act)
    f(kept).backward(dy.double())
    # inputs below 7: the exponential's argument is off by 7^2 u, the rest by 16 u
    assert ((y.detach().double() - f(x.detach().double())).abs() <= 80 * U * (x.detach().double().abs() + 1)).all()
    assert ((x.grad.double() - kept.grad).abs() <= 80 * U * dy.double().abs() * (x.detach().abs() + 1)).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(128,), (9, 128), (2, 70, 128)])
def test_linear_keeps_its_input_in_8_bits(dtype, shape):
    layer = ste.QuasarLinear(128, 48, bits=4, group=64, checkpoint=True)
    plain = ste.QuasarLinear(128, 48, bits=4, group=64)
    plain.load_state_dict(layer.state_dict())
    x = rand(*shape, seed=1, dtype=dtype)
    a, b = x.clone().requires_grad_(), x.clone().requires_grad_()
    dy = rand(*shape[:-1], 48, seed=2, dtype=dtype)
    ya, yb = layer(a), plain(b)
    assert torch.equal(ya, yb)
    saved = [t for t in ya.grad_fn.saved_tensors]
    assert sorted(t.dtype.itemsize for t in saved) == [1, 1, 2]  # q, its exponents and r
    ya.backward(dy)
    yb.backward(dy)
    assert torch.equal(a.grad, b.grad)
    k = back(O.checkpoint_rows(x.reshape(-1, 128)))
    g = dy.reshape(-1, 48).double()
    want, size = g.t() @ k, g.abs().t() @ k.abs()
    assert layer.weight.grad.dtype is torch.float32
    assert ((layer.weight.grad.double() - want).abs() <= 2 * (3 * len(g) + 4) * U * size).all()
    layer.step()
    assert layer.weight.grad is None and layer.t == 1


def test_frozen_parts_of_a_linear_that_keeps_8_bits():
    layer = ste.QuasarLinear(128, 48, bits=4, group=64, checkpoint=True)
    x = rand(5, 128, seed=1)
    layer(x).sum().backward()                     # x takes no gradient
    assert layer.weight.grad is not None
    layer.weight.requires_grad_(False)
    layer.weight.grad = None
    x.requires_grad_()
    layer(x).sum().backward()
    assert x.grad is not None and layer.weight.grad is None


# ---- calls on other streams, and captured ones -----------------------------------------

def _ln():
    x, res, w, b = rand(700, 1537, seed=1), rand(700, 1537, seed=2), rand(1537, seed=3), rand(1537, seed=4)
    return lambda **kw: O.add_layer_norm(x, w, b, res, quantize=True, **kw)


def _ln_backward():
    x, dy, w = rand(3000, 1537, seed=1), rand(3000, 1537, seed=2), rand(1537, seed=3)
    o = O.add_layer_norm(x, w)
    return lambda **kw: O.add_layer_norm_backward(dy, x, w, o["mean"], o["rstd"], **kw)


def _embed():
    w, t = rand(5000, 300, seed=1), torch.randint(-1, 5000, (3000,), device=DEV)
    return lambda **kw: O.embed(t, w, scale=3.0, **kw)


def _embed_backward(n=3000, rows=5000):
    dy, t = rand(n, 300, seed=1), torch.randint(-1, rows, (n,), device=DEV)
    return lambda **kw: O.embed_backward(dy, t, rows, **kw)


def _keep():
    x = rand(700, 1537, seed=1, dtype=torch.bfloat16)
    return lambda **kw: O.checkpoint_rows(x, act="gelu", **kw)


def _keep_backward():
    k, dy = O.checkpoint_rows(rand(700, 1537, seed=1)), rand(700, 1537, seed=2)
    return lambda **kw: O.checkpoint_backward(dy, k["q"], k["exponent"], act="silu", **kw)


def _weight(t, n, k, dtype):
    o, dy = O.checkpoint_rows(rand(t, k, seed=1, dtype=torch.bfloat16)), rand(t, n, seed=2, dtype=dtype)
    return lambda **kw: O.linear_weight_grad(dy, o["q"], o["exponent"], **kw)


CALLS = {"norm": _ln, "norm_backward": _ln_backward, "embed": _embed, "embed_backward": _embed_backward,
         "embed_backward_long": lambda: _embed_backward(30000, 70), "keep": _keep, "keep_backward": _keep_backward,
         "weight_small": lambda: _weight(3000, 200, 300, torch.bfloat16),
         "weight_fp32": lambda: _weight(3000, 200, 300, torch.float32),
         "weight_large": lambda: _weight(1500, 4096, 4096, torch.bfloat16),
         "weight_odd": lambda: _weight(1500, 4099, 4100, torch.bfloat16)}


def bits(o):
    return {k: v.clone().view(torch.uint8) for k, v in o.items() if torch.is_tensor(v) and k != "workspace"}


def stream_of_memory(t):
    """The handle of the stream that the caching allocator keeps t's memory for."""
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("not the allocator's")


@pytest.mark.parametrize("name", CALLS)
def test_another_stream(name):
    """The same bits; what is allocated belongs to the stream, and what was dropped before the stream's work came is
    nobody's loss."""
    call = CALLS[name]()
    want = bits(call())
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for turn in range(3):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            torch.cuda._sleep(SLEEP)
        o = call(stream=s.cuda_stream)
        for k, t in o.items():
            if torch.is_tensor(t) and k != "h":
                assert stream_of_memory(t) == s.cuda_stream, k
        space = o.pop("workspace", None)
        size = 0 if space is None else space.numel()
        del space
        junk = [torch.full((max(size, 512),), 255, device=DEV, dtype=torch.uint8) for _ in range(4)]
        s.synchronize()
        for k, t in want.items():
            assert torch.equal(o[k].view(torch.uint8), t), (k, turn)
        assert all(int(j[0]) == 255 for j in junk)


@pytest.mark.parametrize("name", CALLS)
def test_two_streams_at_once(name):
    call = CALLS[name]()
    want = bits(call())
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[call(stream=s.cuda_stream) for s in streams] for _ in range(4)]
    torch.cuda.synchronize()
    for turn in got:
        for o in turn:
            for k, t in want.items():
                assert torch.equal(o[k].view(torch.uint8), t), k


@pytest.mark.parametrize("name", CALLS)
def test_out_of_an_earlier_call_and_a_graph(name):
    """The dict of an earlier call is written again, eagerly and by the replays of two captured calls in turn."""
    call = CALLS[name]()
    want = bits(call())
    outs = [call() for _ in range(2)]
    torch.cuda.synchronize()
    graphs = []
    for o in outs:
        for k in want:
            o[k].view(torch.uint8).fill_(0xA5)
        again = call(out=o)
        assert all(again[k] is o[k] for k in want)
        torch.cuda.synchronize()
        assert all(torch.equal(o[k].view(torch.uint8), want[k]) for k in want)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(out=o)
        graphs.append(g)
    for rep in range(4):
        for o in outs:
            for k in list(want) + ["workspace"] * (o.get("workspace") is not None):
                o[k].view(torch.uint8).fill_(0xA5 + rep)
        eager = bits(call())
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for o in [eager] + outs:
            for k in want:
                assert torch.equal(o[k].view(torch.uint8), want[k]), (k, rep)


def test_a_captured_step_replays():
    """Embedding, layer norm, a product, GELU from 8 bits and back, as one graph: every replay gives the eager bits."""
    vocab, width, hidden, n = 700, 256, 384, 300
    w, wb, b = rand(vocab, width, seed=1, dtype=torch.bfloat16), rand(width, seed=2), rand(width, seed=3)
    r = rand(hidden, width, seed=4, dtype=torch.bfloat16)
    tok = torch.randint(-1, vocab, (n,), device=DEV, generator=torch.Generator(device=DEV).manual_seed(5))
    dy = rand(n, hidden, seed=6, dtype=torch.bfloat16)

    def step():
        x = O.embed(tok, w, scale=4.0)["y"]
        y = O.add_layer_norm(x, wb, b)
        kx = O.checkpoint_rows(y["y"])
        a = O.checkpoint_rows(y["y"] @ r.t(), act="gelu")
        da = O.checkpoint_backward(dy, a["q"], a["exponent"], act="gelu")["dx"]
        dw = O.linear_weight_grad(da, kx["q"], kx["exponent"])["dw"]
        g = O.add_layer_norm_backward(da @ r, y["h"], wb, y["mean"], y["rstd"])
        return [a["y"], dw, g["dw"], g["db"], O.embed_backward(g["dx"], tok, vocab, scale=4.0)["dw"]]

    want = [t.clone() for t in step()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(4):
        for t in got:
            t.zero_()
        junk = [t.clone() for t in step()]
        graph.replay()
        torch.cuda.synchronize()
        for x, y, z in zip(want, got, junk):
            assert torch.equal(x, y) and torch.equal(x, z)


def test_devices():
    if torch.cuda.device_count() < 2:
        pytest.skip("one GPU")
    x, w = rand(30, 100, seed=1), rand(100, seed=2)
    want = O.add_layer_norm(x, w)
    with torch.cuda.device(0):
        o = O.add_layer_norm(x.to("cuda:1"), w.to("cuda:1"))
        assert torch.cuda.current_device() == 0 and o["y"].device.index == 1
    assert torch.equal(o["y"].cpu(), want["y"].cpu())


# ---- the example -----------------------------------------------------------------------

def _students(**kw):
    make = dict(vocab=512, width=128, hidden=192, **kw)
    return example.Student(**make, checkpoint=True), example.Student(**make)


def test_example_runs_and_serves():
    s, losses, t = example.run(steps=6, tokens=96, vocab=512, width=128, hidden=192, norm="layer", embed_scale=2.0, checkpoint=True,
                               log=None)
    assert losses.isfinite().all()
    with torch.no_grad():
        want = s(t).float()
        exact, eight = example.Server(s, False)(t), example.Server(s, True)(t)
    # bf16 rows, the same r: every stored value's rounding 2^-8, at some 10 places on the way, in quadrature and
    # with a gain of 2; 8-bit rows: 2^-4 at three places instead
    assert float((exact - want).norm() / want.norm()) < 2 * 10 ** 0.5 * V
    assert float((eight - want).norm() / want.norm()) < 2 * 3 ** 0.5 * 2 ** -4


@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_example_gradients(norm):
    """Logits are the same bits whatever is kept; the gradients are those of kept activations: within 2^-4 a stored value,
    at most at five places on the way back, in quadrature and with a gain of 2."""
    kept, plain = _students(norm=norm, embed_scale=2.0)
    t = torch.randint(0, 512, (200,), device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    a, b = kept(t), plain(t)
    g = rand(200, 512, seed=2, dtype=torch.bfloat16)
    # GELU is made in fp32 and rounded once by one, by torch for the other: a last place now and then
    assert float((a - b).detach().float().norm() / b.detach().float().norm()) < 2 * 5 ** 0.5 * V
    a.backward(g)
    b.backward(g)
    for (name, x), y in zip(kept.named_parameters(), plain.parameters()):
        assert x.grad.shape == y.grad.shape
        assert float((x.grad - y.grad).float().norm() / y.grad.float().norm()) < 2 * 5 ** 0.5 * 2 ** -4, name


def test_example_without_the_options_is_as_before():
    """The same layers and parameters, and torch's own lookup."""
    s = example.Student(vocab=128, width=64, hidden=64)
    assert len(s.biases) == 0 and not any(layer.checkpoint for layer in s.linears())
    t = torch.arange(10, device=DEV)
    assert "biases" not in " ".join(s.state_dict()) and s(t).shape == (10, 128)
