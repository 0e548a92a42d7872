"""The distillation loss and its gradient against their formulas in 64 bits.

Tolerances, u = 2^-24: an exponential exp(a) in fp32 carries its argument's
rounding, (|a| + 2) u relative, with |a| below the row's span of logits / tau; a
sum of n terms in any order n u at worst, here taken as 64 u of its (positive)
terms, what trees and short chains of additions leave; gradients in bf16 have
their own rounding, 2^-8."""
import math

import pytest
import torch

from paper_2608_13966_amd import ops as O
from paper_2608_13966_amd import quasar as Q

pytestmark = pytest.mark.gpu

DEV = "cuda"
U, VB = 2.0 ** -24, 2.0 ** -8
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def make(t, v, k, dtype="bf16", teacher="fp32", index=torch.int64, seed=0, pad=0, off=0, scale=2.5):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    buf = torch.zeros(t * (v + pad) + off, device=DEV, dtype=DT[dtype])
    z = buf[off:].view(t, v + pad)[:, :v]
    z.copy_(scale * torch.randn(t, v, generator=g, device=DEV))
    s = z.float() + 0.7 * torch.randn(t, v, generator=g, device=DEV)
    kk = min(k, v)
    top = torch.topk(s, kk, dim=1)
    idx = torch.full((t, k), -1, device=DEV, dtype=index)
    val = torch.zeros(t, k, device=DEV)
    idx[:, :kk], val[:, :kk] = top.indices.to(index), top.values
    return z, idx, val.to(DT[teacher])


def reference(z, idx, val, tau=1.0, wt=None, gl=None):
    """(loss, lse, grad) in 64 bits, masked rows 0."""
    t, v = z.shape
    ok = (idx >= 0) & (idx < v)
    tt = torch.where(ok, val.double() / tau, -math.inf)
    m = tt.amax(1, keepdim=True)
    live = m[:, 0] > -math.inf
    w = torch.ones(t, device=DEV, dtype=torch.float64) if wt is None else wt.double()
    live = live & (w != 0)
    e = torch.where(ok, (tt - m).exp(), 0.0)
    p = torch.where(live[:, None], e / e.sum(1, keepdim=True), 0.0)
    zz = z.double() / tau
    lse = torch.logsumexp(zz, 1)
    at = torch.where(ok, idx, 0).long()
    term = torch.where(p > 0, p * (p.clamp_min(1e-300).log() - zz.gather(1, at) + lse[:, None]), 0.0)
    loss = torch.where(live, w * term.sum(1), 0.0)
    grad = (zz - lse[:, None]).exp()
    grad = grad - torch.zeros_like(grad).scatter_add_(1, at, p)
    g = w / tau * (1.0 if gl is None else gl if isinstance(gl, float) else gl.double())
    grad = torch.where(live[:, None], g[:, None] * grad, 0.0)
    return loss, torch.where(live, lse, 0.0), grad, term.abs().sum(1) * w.abs(), p, at


def check(z, idx, val, o, tau=1.0, wt=None, gl=None, what=("loss", "lse", "grad")):
    loss, lse, grad, _, p, at = reference(z, idx, val, tau, wt, gl)
    zz = (z.double() / tau)
    zz = zz.masked_fill(~torch.isfinite(zz), 0.0)
    span = (zz.amax(1) - zz.amin(1)).clamp_min(1.0)
    e = (span + 66) * U                                  # of lse's sum, and of any exponential
    top = lse.abs() + zz.abs().amax(1)
    if "lse" in what:
        assert ((o["lse"].double() - lse).abs() <= e + 4 * U * top).all()
    if "loss" in what:
        # each term p (log p - z + lse): the three parts' sizes, times p's own error
        w = 1.0 if wt is None else wt.double().abs()
        tspan = (torch.where(p > 0, p.log().abs(), 0.0)).amax(1) + 2
        tol = w * (e + 8 * U * (top + tspan) + (tspan + 66) * U * (top + tspan))
        assert ((o["loss"].double() - loss).abs() <= tol).all(), float((o["loss"].double() - loss).abs().max())
    if "grad" in what:
        w = (1.0 if wt is None else wt.double().abs()) / tau
        g = (w if torch.is_tensor(w) else torch.full_like(lse, w)) * (1.0 if gl is None else abs(gl) if isinstance(gl, float) else gl.double().abs())
        q = torch.zeros_like(grad).scatter_add_(1, at, p)
        size = (zz - lse[:, None]).exp() + q
        tspan = torch.where(p > 0, p.log().abs(), 0.0).amax(1) + 2
        tol = g[:, None] * size * (2 * e + 8 * U * top + (tspan + 66) * U)[:, None]
        tol = tol + grad.abs() * (VB if z.dtype is torch.bfloat16 else U) * 1.01 + 1e-37
        assert o["grad"].dtype is z.dtype
        bad = ~((o["grad"].double() - grad).abs() <= tol)
        assert not bad.any(), (int(bad.sum()), float((o["grad"].double() - grad).abs().max()))


def all_three(z, idx, val, tau=1.0, wt=None, gl=0.25):
    """The three entry points on the same rows; each against the formula."""
    f = O.distill_topk(z, idx, val, temperature=tau, row_weight=wt)
    check(z, idx, val, f, tau, wt, what=("loss", "lse"))
    b = O.distill_topk_backward(z, idx, val, f["lse"], temperature=tau, row_weight=wt, grad_scale=gl)
    check(z, idx, val, b, tau, wt, gl, what=("grad",))
    o = O.distill_topk_grad(z, idx, val, temperature=tau, row_weight=wt, grad_scale=gl)
    check(z, idx, val, o, tau, wt, gl)
    return o


@pytest.mark.parametrize("t,v,k", [(1, 1, 1), (2, 3, 2), (3, 8, 1), (2, 9, 9), (1, 1000, 20), (5, 1023, 64), (3, 4096, 256),
                                   (2, 16384, 16), (2, 16385, 64), (300, 2000, 33), (3, 50021, 1024), (2, 131072, 64),
                                   (1, 160001, 100), (260, 33000, 64), (2, 300000, 8)])
@pytest.mark.parametrize("dtype,teacher,index,tau", [("bf16", "bf16", torch.int32, 1.0), ("fp32", "fp32", torch.int64, 2.0)])
def test_sizes(t, v, k, dtype, teacher, index, tau):
    z, idx, val = make(t, v, k, dtype, teacher, index, seed=v + k)
    all_three(z, idx, val, tau)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("pad,off", [(1, 0), (0, 1), (5, 3), (64, 8)])
def test_strides_and_offsets(dtype, pad, off):
    """Rows of a wider buffer at odd elements, the gradient's too; nothing beside it is written."""
    t, v = 7, 3001
    z, idx, val = make(t, v, 20, dtype, seed=3, pad=pad, off=off)
    buf = torch.full((t * (v + 2 + pad) + off,), 9.0, device=DEV, dtype=DT[dtype])
    grad = buf[off:].view(t, v + 2 + pad)[:, :v]
    want = all_three(z, idx, val)
    o = O.distill_topk_grad(z, idx, val, grad_scale=0.25,
                            out={"grad": grad, "loss": torch.empty(t, device=DEV), "lse": torch.empty(t, device=DEV)})
    assert o["grad"] is grad and torch.equal(grad, want["grad"])
    assert (buf[:off] == 9).all() and (buf[off:].view(t, -1)[:, v:] == 9).all()


@pytest.mark.parametrize("t,v", [(3, 1000), (2, 40000), (300, 17000), (4, 140001)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_in_place(t, v, dtype):
    z, idx, val = make(t, v, 64, dtype, seed=5)
    want = O.distill_topk_grad(z, idx, val, grad_scale=0.5, temperature=1.5)
    wb = O.distill_topk_backward(z, idx, val, want["lse"], grad_scale=0.5, temperature=1.5)
    zz = z.clone()
    o = O.distill_topk_grad(zz, idx, val, grad_scale=0.5, temperature=1.5,
                            out={"grad": zz, "loss": torch.empty(t, device=DEV), "lse": torch.empty(t, device=DEV)})
    for k in ("loss", "lse", "grad"):
        assert torch.equal(o[k], want[k]), k
    zz = z.clone()
    b = O.distill_topk_backward(zz, idx, val, want["lse"], grad_scale=0.5, temperature=1.5, out={"grad": zz})
    assert torch.equal(b["grad"], wb["grad"])


@pytest.mark.parametrize("t,v", [(12, 500), (12, 40000), (600, 1000)])
def test_masked_rows(t, v):
    """Weight 0, nothing listed, everything listed at -inf: exact zeros, also where the row's logits are NaN."""
    z, idx, val = make(t, v, 16, seed=6)
    wt = torch.rand(t, device=DEV) + 0.5
    wt[1] = 0.0
    z[1, 3] = float("nan")
    z[1, 4] = float("inf")
    idx[2] = -1
    z[2, 0] = float("nan")
    val[3] = -math.inf
    z[3] = float("nan")
    wt[4], wt[5] = -0.0, -1.5
    wt[6] = 0.0
    val[6] = float("nan")
    dead = [1, 2, 3, 4, 6]
    z[dead, 5] = float("nan")
    o = O.distill_topk_grad(z, idx, val, row_weight=wt, grad_scale=0.25)
    f = O.distill_topk(z, idx, val, row_weight=wt)
    b = O.distill_topk_backward(z, idx, val, f["lse"], row_weight=wt, grad_scale=0.25)
    for x in (o["loss"], o["lse"], o["grad"], f["loss"], f["lse"], b["grad"]):
        assert (x[dead] == 0).all()
    keep = [i for i in range(t) if i not in dead]
    sub = {k: o[k][keep] for k in ("loss", "lse", "grad")}
    check(z[keep], idx[keep], val[keep], sub, 1.0, wt[keep], 0.25)


def test_entries_out_of_range_and_listed_twice():
    z, idx, val = make(9, 2000, 24, seed=7)
    idx[0, 3:] = -1
    idx[1, ::2] = 2000                      # the first class past the end
    idx[2, 5] = torch.iinfo(torch.int64).max
    idx[3, 1] = torch.iinfo(torch.int64).min
    idx[4] = idx[4, 0]                      # one class, 24 times
    idx[5, 10:14] = idx[5, 3]
    val[6, 2:20] = -math.inf
    val[7, 0] = 80.0                        # all but one vanish
    idx[8, 0], idx[8, 1] = 0, 1999
    all_three(z, idx, val)
    o = all_three(z, idx, val, tau=0.5)
    # a class listed by several entries has their probabilities' sum
    assert float(o["grad"][4].double().sum().abs()) < 1e-2
    i32 = idx.clamp(-1, 2000).to(torch.int32)
    assert torch.equal(O.distill_topk_grad(z, i32, val, temperature=0.5, grad_scale=0.25)["grad"], o["grad"])


@pytest.mark.parametrize("t,v,k,distinct", [(4, 70, 64, 8), (3, 5000, 1024, 64), (300, 3000, 200, 40), (2, 140001, 1000, 100),
                                            (2, 2 ** 20 + 7, 512, 500)])
@pytest.mark.parametrize("dtype,index", [("bf16", torch.int64), ("fp32", torch.int32)])
def test_lists_that_name_classes_often(t, v, k, distinct, dtype, index):
    """A class's entries add up, a few tens of them at most (what the bound of a sum allows)."""
    z, _, val = make(t, v, k, dtype, "fp32", index, seed=k)
    g = torch.Generator(device=DEV).manual_seed(distinct)
    classes = torch.stack([torch.randperm(v, generator=g, device=DEV)[:distinct] for _ in range(t)])
    classes[:, 0], classes[:, -1] = 0, v - 1
    idx = classes.gather(1, torch.randint(0, distinct, (t, k), generator=g, device=DEV)).to(index)
    idx[:, ::7] = -1
    all_three(z, idx, val, 1.5)


@pytest.mark.parametrize("t,v,k", [(1024, 1, 1), (1025, 9, 5), (3080, 1023, 64), (1024, 2048, 256), (1100, 2049, 7),
                                   (1031, 4096, 64), (1024, 4097, 64), (1024, 2000, 257), (6200, 300, 20), (1023, 4096, 40),
                                   (1500, 8192, 30), (1040, 8193, 8), (1040, 6001, 300)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_many_short_rows(t, v, k, dtype):
    """A wavefront or a few a row, several rows in turn; masked rows among them; the gradient in the logits' place."""
    z, idx, val = make(t, v, k, dtype, index=torch.int32, seed=t + k)
    wt = torch.rand(t, device=DEV) + 0.5
    wt[5::17] = 0.0
    idx[3::19] = -1
    dead = (wt == 0) | (idx < 0).all(1)
    o = all_three(z, idx, val, 1.5, wt)
    for x in o["loss"], o["lse"], o["grad"]:
        assert (x[dead] == 0).all()
    zz = z.clone()
    a = O.distill_topk_grad(zz, idx, val, temperature=1.5, row_weight=wt, grad_scale=0.25,
                            out={"grad": zz, "loss": torch.empty(t, device=DEV), "lse": torch.empty(t, device=DEV)})
    assert all(torch.equal(a[x], o[x]) for x in ("loss", "lse", "grad"))
    few = O.distill_topk_grad(z[:40], idx[:40], val[:40], temperature=1.5, row_weight=wt[:40], grad_scale=0.25)
    check(z[:40], idx[:40], val[:40], few, 1.5, wt[:40], 0.25)


@pytest.mark.parametrize("v", [700, 33000])
def test_student_logits_at_minus_infinity(v):
    """Classes that the student cannot take: probability 0 and gradient 0 where the teacher does not list them; a
    listed one makes the loss infinite and its gradient -p."""
    z, idx, val = make(4, v, 8, "fp32", seed=8)
    z[0, :v // 2] = -math.inf
    z[1] = torch.where(torch.arange(v, device=DEV) == 17, 1.0, -math.inf)
    low = torch.finfo(torch.float32).min
    z[3, v // 3:] = low
    o = O.distill_topk_grad(z, idx, val)
    ref = reference(z, idx, val)
    for r in range(4):
        assert torch.equal(torch.isinf(o["loss"][r]), torch.isinf(ref[0][r]))
    g = o["grad"].double()
    assert torch.isfinite(g).all()
    # q - p may cancel where a class is listed: each of the two has its own error
    p = torch.zeros_like(g).scatter_add_(1, ref[5], ref[4])
    assert ((g - ref[2]).abs() <= 3e-5 * (ref[2].abs() + 2 * p) + 1e-9).all()
    assert abs(float(o["lse"][1]) - 1.0) < 1e-6


def test_nan_keeps_to_its_row():
    z, idx, val = make(5, 5000, 8, seed=9)
    clean = O.distill_topk_grad(z, idx, val)
    z[1, 4001] = float("nan")
    val[3, 2] = float("nan")
    o = O.distill_topk_grad(z, idx, val)
    for k in ("loss", "lse", "grad"):
        assert torch.equal(o[k][[0, 2, 4]], clean[k][[0, 2, 4]])
    assert torch.isnan(o["loss"][1]) and torch.isnan(o["lse"][1]) and torch.isnan(o["grad"][1].float()).all()
    assert torch.isnan(o["loss"][3]) and torch.isfinite(o["lse"][3])


def test_wide_spans():
    """Logits hundreds apart: the running maximum grows over the row, sums do not overflow."""
    z, idx, val = make(6, 20000, 8, "fp32", seed=10)
    z[0] = torch.linspace(-300, 300, 20000, device=DEV)
    z[1] = torch.linspace(300, -300, 20000, device=DEV)
    z[2] *= 100.0
    z[3] = 5.0
    z[4, 19999] = 3000.0
    idx[:] = torch.arange(8, device=DEV) * 2500
    all_three(z, idx, val)


def test_no_rows():
    z = torch.empty(0, 100, device=DEV)
    i, t = torch.empty(0, 4, device=DEV, dtype=torch.int64), torch.empty(0, 4, device=DEV)
    o = O.distill_topk_grad(z, i, t)
    assert o["loss"].shape == (0,) and o["grad"].shape == (0, 100)
    assert O.distill_topk(z, i, t)["lse"].shape == (0,)
    assert O.distill_topk_backward(z, i, t, o["lse"])["grad"].shape == (0, 100)


@pytest.mark.parametrize("v", [40, 3000])
def test_gradient_against_differences(v):
    """Central differences of the 64-bit loss along random directions, at 1e-4: the second-order rest is below 1e-7
    of the gradient's size."""
    z, idx, val = make(4, v, 8, "fp32", seed=11)
    wt = torch.tensor([1.0, 0.5, 2.0, 1.0], device=DEV)
    gl = torch.tensor([0.3, 1.0, -2.0, 0.0], device=DEV)
    f = O.distill_topk(z, idx, val, temperature=1.7, row_weight=wt)
    o = O.distill_topk_backward(z, idx, val, f["lse"], temperature=1.7, row_weight=wt, grad_loss=gl)
    check(z, idx, val, o, 1.7, wt, gl, what=("grad",))
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    d = torch.randn(4, v, generator=g, device=DEV, dtype=torch.float64)
    at = lambda s: reference(z.double() + s * d, idx, val, 1.7, wt)[0]  # noqa: E731
    want = gl.double() * (at(1e-4) - at(-1e-4)) / 2e-4
    got = (o["grad"].double() * d).sum(1)
    size = (o["grad"].double() * d).abs().sum(1)
    assert ((got - want).abs() <= 2e-5 * size + 1e-9).all()
    assert (o["grad"][3] == 0).all()


def test_offsets_past_32_bits():
    stride, v = (1 << 31) + 24, 3000
    z, idx, val = make(3, v, 8, seed=12)
    big = torch.zeros(2 * stride + v, device=DEV, dtype=torch.bfloat16)
    far = big.as_strided((3, v), (stride, 1))
    far.copy_(z)
    o, want = O.distill_topk_grad(far, idx, val), O.distill_topk_grad(z, idx, val)
    assert torch.equal(o["grad"], want["grad"]) and torch.equal(o["loss"], want["loss"])
    O.distill_topk_grad(far, idx, val, out={"grad": far, "loss": o["loss"], "lse": o["lse"]})
    assert torch.equal(far, want["grad"])


def test_many_rows():
    """More rows than a grid's second dimension holds."""
    z, idx, val = make(70000, 24, 4, seed=13)
    all_three(z, idx, val)


@pytest.mark.parametrize("t,v", [(40, 20000), (700, 3000)])
def test_determinism_other_stream_and_graph(t, v):
    z, idx, val = make(t, v, 32, seed=14)
    want = O.distill_topk_grad(z, idx, val)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        o = O.distill_topk_grad(z, idx, val)
    s.synchronize()
    for k in ("loss", "lse", "grad"):
        assert torch.equal(o[k], want[k])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        O.distill_topk_grad(z, idx, val, out=o)
    for _ in range(3):
        o["grad"].zero_()
        o["loss"].zero_()
        graph.replay()
        torch.cuda.synchronize()
        for k in ("loss", "lse", "grad"):
            assert torch.equal(o[k], want[k])


def test_refusals():
    z, idx, val = make(2, 100, 4, seed=15)
    for kw in (dict(temperature=0.0), dict(temperature=float("nan")), dict(grad_scale=float("inf"))):
        with pytest.raises(Q.QuasarError) as e:
            O.distill_topk_grad(z, idx, val, **kw)
        assert e.value.status == Q.ERR_ARG


def test_more_rows_than_a_grid_takes():
    """The gradient alone takes a workgroup of 256 threads a row: from 2^24 rows on more than 2^32 threads."""
    t, v = (1 << 24) + 7, 8
    z, idx, val = make(t, v, 2, "bf16", "bf16", torch.int32, seed=16)
    wt, gl = torch.rand(t, device=DEV), torch.randn(t, device=DEV)
    wt[5::31] = 0.0
    lse = O.distill_topk(z, idx, val, row_weight=wt, temperature=1.5)["lse"]
    o = O.distill_topk_backward(z, idx, val, lse, row_weight=wt, grad_loss=gl, temperature=1.5)
    cut = (1 << 24) - 3
    for s in (slice(0, cut), slice(cut, t)):
        part = O.distill_topk_backward(z[s], idx[s], val[s], lse[s], row_weight=wt[s], grad_loss=gl[s], temperature=1.5)
        assert torch.equal(o["grad"][s], part["grad"])
    s = slice(t - 50, t)
    check(z[s], idx[s], val[s], {"grad": o["grad"][s], "lse": lse[s]}, 1.5, wt[s], gl[s], what=("grad", "lse"))


@pytest.mark.parametrize("t,v,k", [(1100, 1200, 200), (300, 17000, 64), (5, 9000, 1000), (3, 140001, 64), (2, 200, 200)])
@pytest.mark.parametrize("tau", [1.0, 0.7])
def test_loss_has_no_error_of_the_logits_size(t, v, k, tau):
    """The loss depends on differences of logits alone.  On a grid of 1/64 these are exact in fp32 whatever is added to
    all, so adding 512 to the student's row, or to the teacher's, changes no bit of it; and it is off from the formula
    in 64 bits by no more than its parts' errors, which know no 512: with y = (z - max) / tau, d = (t - max) / tau,
      log q: 3 u |y| + log of the sum, whose terms are off by (3 |y| + 4) u and their sum by 64 u more;
      log p: likewise from d; and the products' and the sum's own, p's error included: (3 |d| + 72) u of their size."""
    z, idx, val = make(t, v, k, "fp32", "fp32", torch.int32, seed=17)
    z, val = (64 * z).round() / 64, (64 * val).round() / 64
    idx[0, k // 2:] = -1
    runs = [O.distill_topk(a, idx, b, temperature=tau)["loss"] for a, b in ((z, val), (z + 512, val), (z, val - 512))]
    runs += [O.distill_topk_grad(z + 512, idx, val + 512, temperature=tau)["loss"]]
    assert all(torch.equal(r, runs[0]) for r in runs)
    loss, _, _, _, _, at = reference(z, idx, val, tau)
    y = (z.double() - z.double().amax(1, keepdim=True)) / tau
    d = torch.where(idx >= 0, val.double(), -math.inf)
    d = (d - d.amax(1, keepdim=True)) / tau
    p, q = torch.softmax(d, 1), torch.softmax(y, 1)
    d = torch.where(idx >= 0, d, 0.0)
    yk, lq = y.gather(1, at).abs(), torch.log_softmax(y, 1).gather(1, at)
    lp = torch.where(idx >= 0, p.clamp_min(1e-300).log(), 0.0)
    sum_q = ((q * (3 * y.abs() + 4)).sum(1) + 64 + 2 * torch.logsumexp(y, 1).abs())[:, None]
    sum_p = ((p * (3 * d.abs() + 4)).sum(1) + 64 + 2 * torch.where(idx >= 0, lp - d, 0.0).abs().amax(1))[:, None]
    tol = (p * (3 * yk + sum_q + 3 * d.abs() + sum_p + (lp - lq).abs() * (3 * d.abs() + 72 + sum_p))).sum(1) * U
    off = (runs[0].double() - loss).abs()
    assert (off <= tol).all(), float((off / tol).max())


@pytest.mark.parametrize("t,v", [(1100, 1203), (1100, 4097), (300, 17003), (6, 9000), (6, 140003)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_student_logits_at_plus_infinity(t, v, dtype):
    """As the formula has it: the log-sum is +inf, the loss +inf (NaN where the infinite class is listed: inf - inf), the
    gradient -p of the finite classes and NaN of the infinite one.  A NaN beside it makes all of them NaN."""
    z, idx, val = make(t, v, 8, dtype, seed=18)
    inf = float("inf")
    free = [c for c in range(v - 1, -1, -1)]
    at = [next(c for c in free[a:] if c not in idx[r].tolist()) for r, a in ((0, 0), (1, v - 3), (2, 0), (3, v // 2))]
    z[0, at[0]] = inf                      # past the whole pieces
    z[1, at[1]] = inf                      # in the first piece
    z[2, int(idx[2, 3])] = inf             # listed, and one that is not
    z[2, at[2]] = inf
    z[3, at[3]], z[3, at[3] - 1] = inf, float("nan")
    f = O.distill_topk(z, idx, val, temperature=1.5)
    o = O.distill_topk_grad(z, idx, val, temperature=1.5, grad_scale=0.25)
    b = O.distill_topk_backward(z, idx, val, f["lse"], temperature=1.5, grad_scale=0.25)
    loss, lse, grad, _, p, listed = reference(z, idx, val, 1.5, None, 0.25)
    for x in (f, o):
        assert (x["lse"][:3] == inf).all() and x["lse"][3].isnan()
        assert (x["loss"][:2] == inf).all() and x["loss"][2:4].isnan().all()
    for x in (o["grad"], b["grad"]):
        g = x[:3].double()
        assert torch.equal(g.isnan(), grad[:3].isnan())
        where = ~g.isnan()
        assert ((g - grad[:3]).abs()[where] <= (VB if dtype == "bf16" else 1e-5) * grad[:3].abs()[where]).all()
        assert x[3].isnan().all()
    rest = slice(4, t)
    check(z[rest], idx[rest], val[rest], {k: o[k][rest] for k in ("loss", "lse", "grad")}, 1.5, None, 0.25)


@pytest.mark.parametrize("t,v", [(3, 140001), (40, 60000)])
def test_loss_workspace_is_reused(t, v):
    g = torch.Generator(device=DEV).manual_seed(24)
    z = torch.randn(t, v, device=DEV, generator=g)
    values, idx = torch.topk(z + torch.randn(t, v, device=DEV, generator=g), 16, dim=1)
    want = {k: a.clone() for k, a in O.distill_topk_grad(z, idx, values).items()}
    o = O.distill_topk_grad(z, idx, values)
    space = o["workspace"].fill_(255)
    a = O.distill_topk_grad(z, idx, values, out=o)
    assert a["workspace"].data_ptr() == space.data_ptr()
    assert all(torch.equal(a[k], want[k]) for k in ("loss", "lse", "grad"))
