"""Activations kept in 8 bits: checkpoint_rows bit for bit against its definition,
the activations' gradients and the linear layer's weight gradient against theirs
in 64 bits.

Tolerances, u = 2^-24, v = 2^-8.  GELU's tail at |x| = t is off by its fit and a
dozen roundings (16 u) and by the rounding of the exponential's argument t^2 / 2
(1.2 t^2 u); SiLU by 8 u.  Their derivatives: each term as much, and its products.
The hardware's exponential gives 0 for results below 2^-126 (at -87.5, say, where
it is 9.98e-39): what it is multiplied by there, |x| at most, is lost with it.
The weight gradient: its products are exact, a sum of n terms is off by n steps
of 2 u at most, however a matrix instruction adds them."""
import math

import pytest
import torch

from paper_2608_13966_amd import ops as O

pytestmark = pytest.mark.gpu

DEV = "cuda"
U, V = 2.0 ** -24, 2.0 ** -8
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
E4M3 = torch.float8_e4m3fn
INF, NAN = float("inf"), float("nan")


def gen(shape, dtype, seed, scale=1.0, pad=0, off=0):
    """Normal values with rows and columns of other sizes among them, in rows of a wider buffer."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    t = torch.randn(shape, generator=g, device=DEV) * scale
    t *= torch.exp2(torch.randint(-6, 7, (shape[0], 1), generator=g, device=DEV).float())
    t *= torch.where(torch.rand(1, shape[1], generator=g, device=DEV) < 0.05, 30.0, 1.0)
    buf = torch.empty(shape[0] * (shape[1] + pad) + off, device=DEV, dtype=dtype)
    v = buf[off:].view(shape[0], shape[1] + pad)[:, :shape[1]]
    v.copy_(t)
    return v


def rnd(dtype):
    return V if dtype is torch.bfloat16 else U


def kept_ref(x):
    """(q as numbers, exponents) by the definition, in 64 bits."""
    rows, cols = x.shape
    n = -(-cols // 128)
    b = torch.nn.functional.pad(x.double(), (0, n * 128 - cols)).view(rows, n, 128)
    top = torch.where(b.isfinite(), b.abs(), 0.0).amax(2)
    m, e = torch.frexp(top / 448)
    e = torch.where(m == 0.5, e - 1, e)
    e = torch.where(top == 0, -120, e).clamp(-120, 120)
    v = b * torch.exp2(-e.double())[:, :, None]
    step = torch.exp2(v.abs().clamp_min(2.0 ** -6).log2().floor() - 3)
    q = torch.where(v.isfinite(), torch.round(v / step) * step, NAN)
    q = torch.where((e == 120)[:, :, None], q.clamp(-240, 240), q)  # 256 * 2^120 would not be finite
    return q.view(rows, n * 128)[:, :cols], (e + 127).to(torch.uint8)


def back(q, e):
    return q.double() * torch.exp2(e.double() - 127).repeat_interleave(128, 1)[:, :q.shape[1]]


def lost(x):
    """What an exponential below 2^-126 that is given as 0 takes away."""
    return (x.abs() + 1) * 2.0 ** -126


def act_ref(act, x):
    """act(x) and how far the kernels' may be from it."""
    x = x.double()
    if act == "relu":
        return torch.where(x < 0, 0.0, x), torch.zeros_like(x)
    if act == "silu":
        y = x * torch.sigmoid(x)
        return y, 8 * U * y.abs() + lost(x)
    tail = 0.5 * torch.special.erfc(x.abs() / math.sqrt(2))
    y = torch.where(x > 0, x - x * tail, x * tail)
    return y, (x.abs() * tail) * (16 + 1.2 * x * x) * U + 2 * U * y.abs() + lost(x)


def grad_ref(act, x):
    if act == "relu":
        return (x > 0).double(), torch.zeros_like(x)
    if act == "silu":
        s, r = torch.sigmoid(x), torch.sigmoid(-x)
        return s + x * s * r, (10 * s + 16 * x.abs() * s * r) * U + lost(x)
    tail = 0.5 * torch.special.erfc(x.abs() / math.sqrt(2))
    dens = x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    cdf = torch.where(x > 0, 1 - tail, tail)
    return cdf + dens, (tail * (16 + 1.2 * x * x) + dens.abs() * (8 + 1.2 * x * x) + 4 * cdf) * U + lost(x)


SHAPES = [(1, 1), (3, 7), (2, 127), (5, 128), (4, 129), (17, 300), (33, 1000), (8, 4096), (3, 14337), (1, 40000), (70000, 3)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("xt,yt,act", [("bf16", None, "none"), ("fp32", None, "gelu"), ("bf16", None, "gelu"), ("bf16", "fp32", "silu"),
                                       ("fp32", "bf16", "relu")])
def test_rows(shape, xt, yt, act):
    x = gen(shape, DT[xt], 1, pad=shape[1] % 4, off=shape[1] % 3)
    o = O.checkpoint_rows(x, act=act, y_dtype=yt)
    q, e = kept_ref(x)
    assert o["q"].dtype is E4M3 and torch.equal(o["exponent"], e)
    assert torch.equal(o["q"].double(), q)
    k = back(o["q"], e)  # four significant bits, or 2^-10 of the stretch's scale
    f = torch.exp2(e.double() - 127).repeat_interleave(128, 1)[:, :shape[1]]
    assert ((k - x.double()).abs() <= torch.maximum(x.double().abs() * 2.0 ** -4, f * 2.0 ** -10)).all()
    if act == "none":
        assert o["y"] is None
        same = O.checkpoint_rows(x, want_y=True)
        assert torch.equal(same["y"], x) and torch.equal(same["q"].view(torch.uint8), o["q"].view(torch.uint8))
    else:
        y, tol = act_ref(act, x)
        assert o["y"].dtype is DT[yt or xt]
        assert ((o["y"].double() - y).abs() <= tol + rnd(o["y"].dtype) * (y.abs() + tol)).all()


def test_rows_at_the_edges():
    """The exponent where the largest value is 448 times a power of two or next to it, at both ends of the range, and in
    stretches of zeros; halfway values go to the even code."""
    tops = []
    for p in (-149, -126, -125, -113, -112, -111, -20, 0, 1, 100, 127):
        for m in (1.0, 1.75, 1.75 - 2.0 ** -23, 1.75 + 2.0 ** -23, 2 - 2.0 ** -23):
            v = math.ldexp(m, p)
            tops.append(v)
    tops.append(0.0)
    x = torch.zeros(len(tops), 256, device=DEV)
    x[:, 77] = torch.tensor(tops, dtype=torch.float64).float().to(DEV)
    x[:, 78] = -x[:, 77] / 3
    x[:, 200] = 1.0 + 2.0 ** -4                                  # between 1 and 1.125
    x[:, 201] = 1.0 + 3 * 2.0 ** -4
    x[:, 202] = -448.0
    o = O.checkpoint_rows(x)
    q, e = kept_ref(x)
    assert torch.equal(o["exponent"], e) and torch.equal(o["q"].double(), q)
    assert (o["exponent"][-1, 0] == 7) and (e[:, 1] == 127).all()
    assert (o["q"][:, 200].float() == 1.0).all() and (o["q"][:, 201].float() == 1.25).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_what_is_not_finite_stays_by_itself(dtype):
    x = gen((5, 400), dtype, 1)
    x[0, 3], x[1, 130], x[2, 399], x[3, :128] = NAN, INF, -INF, NAN
    x[4, 256:384] = INF
    o = O.checkpoint_rows(x, act="relu")
    q, e = kept_ref(x)
    assert torch.equal(o["exponent"], e)
    bad = ~x.isfinite()
    assert o["q"].float()[bad].isnan().all() and torch.equal(o["q"].double()[~bad], q[~bad])
    assert torch.equal(o["y"].isnan(), x.isnan()) and o["y"][1, 130] == INF and o["y"][2, 399] == 0


def formula(act, x):
    """The header's formulas as they stand, in 64 bits."""
    x = x.double()
    return {"none": x, "relu": torch.where(x < 0, 0.0, x), "silu": x / (1 + torch.exp(-x)),
            "gelu": x * (1 + torch.erf(x / math.sqrt(2))) / 2}[act]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
def test_activations_of_what_is_not_finite(act, dtype):
    """As IEEE arithmetic takes them through the formulas: SiLU and GELU of -infinity are -infinity times 0.  Neighbours are
    what they are without them."""
    clean = gen((5, 400), dtype, 1)
    x = clean.clone()
    x[0, 3], x[1, 130], x[2, 399], x[3, :128], x[4, 256:384] = NAN, INF, -INF, NAN, -INF
    x[1, 131] = -INF
    bad = ~x.isfinite()
    y, want = O.checkpoint_rows(x, act=act, want_y=True)["y"], formula(act, x)
    assert torch.equal(y.isnan()[bad], want.isnan()[bad])
    there = bad & ~want.isnan()
    assert torch.equal(y[there].double(), want[there])
    assert torch.equal(y[~bad], O.checkpoint_rows(clean, act=act, want_y=True)["y"][~bad])


def test_outputs_in_wider_buffers_and_in_place():
    x = gen((9, 300), torch.bfloat16, 1, pad=3, off=1)
    want = O.checkpoint_rows(x, act="gelu")
    qb, eb = torch.full((9, 307), 7, device=DEV, dtype=torch.uint8), torch.full((9, 5), 9, device=DEV, dtype=torch.uint8)
    y = x.clone()
    o = O.checkpoint_rows(y, act="gelu", out={"q": qb[:, 2:302].view(E4M3), "exponent": eb[:, 1:4], "y": y})
    assert o["y"] is y and torch.equal(y, want["y"])
    assert torch.equal(qb[:, 2:302], want["q"].view(torch.uint8)) and torch.equal(eb[:, 1:4], want["exponent"])
    assert (qb[:, :2] == 7).all() and (qb[:, 302:] == 7).all() and (eb[:, [0, 4]] == 9).all()
    dy = gen((9, 300), torch.bfloat16, 2)
    dx = O.checkpoint_backward(dy, o["q"], o["exponent"], act="gelu")["dx"]
    assert torch.equal(dx, O.checkpoint_backward(dy, want["q"], want["exponent"], act="gelu")["dx"])
    g = dy.clone()
    assert O.checkpoint_backward(g, o["q"], o["exponent"], act="gelu", out={"dx": g})["dx"] is g and torch.equal(g, dx)


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("gt,xt,act", [("bf16", None, "gelu"), ("fp32", None, "gelu"), ("bf16", "fp32", "silu"), ("fp32", "bf16", "relu"),
                                       ("fp32", None, "silu")])
def test_backward(shape, gt, xt, act):
    kept = O.checkpoint_rows(gen(shape, torch.float32, 1, 0.3))
    dy = gen(shape, DT[gt], 2, pad=shape[1] % 4, off=shape[1] % 3)
    o = O.checkpoint_backward(dy, kept["q"], kept["exponent"], act=act, dx_dtype=xt)
    assert o["dx"].dtype is DT[xt or gt]
    d, tol = grad_ref(act, back(kept["q"], kept["exponent"]))
    want, tol = dy.double() * d, dy.double().abs() * (tol + 2 * U * d.abs())
    assert ((o["dx"].double() - want).abs() <= tol + rnd(o["dx"].dtype) * (want.abs() + tol) + 1e-37).all()


@pytest.mark.parametrize("act", ["relu", "silu", "gelu"])
def test_derivatives_over_the_whole_range(act):
    """Every E4M3 number at every exponent, as far as it is finite in fp32: the derivative is finite, and NaN only for the
    NaN codes."""
    codes = torch.arange(256, device=DEV, dtype=torch.uint8).repeat(241, 1)
    e = torch.arange(7, 248, device=DEV, dtype=torch.uint8)[:, None].repeat(1, 2)
    q = codes.view(E4M3)
    dx = O.checkpoint_backward(torch.ones(241, 256, device=DEV), q, e, act=act)["dx"].double()
    x = back(q, e)
    nan, kept = x.isnan(), ~(x.abs() >= 2.0 ** 128)
    assert torch.equal(dx.isnan()[kept], nan[kept])
    nan |= ~kept
    assert dx[~nan].isfinite().all()
    d, tol = grad_ref(act, torch.where(nan, 0.0, x.clamp(-1e4, 1e4)))
    assert ((dx - d).abs() <= tol + 2 * U * d.abs())[~nan].all()


def test_derivatives_against_differences():
    x = torch.linspace(-6, 6, 241, dtype=torch.float64)
    for act in ("silu", "gelu"):
        d, _ = grad_ref(act, x)
        diff = (act_ref(act, x + 1e-5)[0] - act_ref(act, x - 1e-5)[0]) / 2e-5
        assert (d - diff).abs().max() < 1e-9, act  # h^2 of the third derivative, 1e-16 / h


# ---- the weight gradient ------------------------------------------------------------

def check_weight(dy, q, e, dw):
    k, g = back(q, e), dy.double()
    want, size = g.t().contiguous() @ k, g.abs().t().contiguous() @ k.abs()
    n = dy.shape[0] * (3 if dy.dtype is torch.float32 else 1) + 4
    tol = 2 * n * U * size
    assert dw.shape == want.shape
    bad = ~((dw.double() - want).abs() <= tol + rnd(dw.dtype) * (want.abs() + tol) + 1e-37)
    assert not bad.any(), (int(bad.sum()), float((dw.double() - want).abs().max()))


TNK = [(1, 1, 1), (1, 64, 64), (3, 7, 5), (63, 64, 129), (64, 65, 64), (65, 200, 300), (130, 128, 128), (200, 129, 72), (777, 100, 1544),
       (1000, 256, 256), (4097, 64, 40), (256, 1030, 520)]


@pytest.mark.parametrize("t,n,k", TNK)
@pytest.mark.parametrize("gt,wt", [("bf16", "fp32"), ("fp32", "fp32"), ("bf16", "bf16"), ("fp32", "bf16")])
def test_weight_grad(t, n, k, gt, wt):
    kept = O.checkpoint_rows(gen((t, k), torch.bfloat16, 1))
    dy = gen((t, n), DT[gt], 2, 1e-3, pad=n % 4, off=n % 3)
    out = {"dw": torch.full((n, k), NAN, device=DEV, dtype=DT[wt])}
    o = O.linear_weight_grad(dy, kept["q"], kept["exponent"], dw_dtype=wt, out=out)
    assert o["dw"] is out["dw"]
    check_weight(dy, kept["q"], kept["exponent"], o["dw"])
    again = O.linear_weight_grad(dy, kept["q"], kept["exponent"], dw_dtype=wt)
    assert torch.equal(again["dw"], o["dw"])


@pytest.mark.parametrize("t,n,k", [(300, 2048, 4096), (1, 4096, 4096), (513, 4096, 4104), (1025, 2056, 8192), (4100, 1000, 2000),
                                   (127, 5000, 3333)])
@pytest.mark.parametrize("gt", ["bf16", "fp32"])
def test_large_weight_grad(t, n, k, gt):
    kept = O.checkpoint_rows(gen((t, k), torch.bfloat16, 1))
    dy = gen((t, n), DT[gt], 2, 1e-3)
    check_weight(dy, kept["q"], kept["exponent"], O.linear_weight_grad(dy, kept["q"], kept["exponent"])["dw"])


@pytest.mark.parametrize("t,n,k", [(100, 72, 136), (700, 4096, 4096)])
@pytest.mark.parametrize("pads", [(1, 3, 1), (8, 8, 0), (13, 5, 2)])
def test_weight_grad_strides(t, n, k, pads):
    """Rows of wider buffers, which hold NaN; what is beside the result stays."""
    gp, qp, ep = pads
    kept = O.checkpoint_rows(gen((t, k), torch.bfloat16, 1))
    blocks = -(-k // 128)
    dyb = torch.full((t, n + gp), NAN, device=DEV, dtype=torch.bfloat16)
    qb, eb = torch.full((t, k + qp), 0x7f, device=DEV, dtype=torch.uint8), torch.full((t, blocks + ep), 255, device=DEV, dtype=torch.uint8)
    dyb[:, :n], qb[:, :k], eb[:, :blocks] = gen((t, n), torch.bfloat16, 2), kept["q"].view(torch.uint8), kept["exponent"]
    dwb = torch.full((n, k + gp), 7.0, device=DEV)
    dy, q, e, dw = dyb[:, :n], qb[:, :k].view(E4M3), eb[:, :blocks], dwb[:, :k]
    O.linear_weight_grad(dy, q, e, out={"dw": dw})
    check_weight(dy, q, e, dw)
    assert (dwb[:, k:] == 7).all()


FEW = [(1, 3126, 4372), (2, 8, 33000), (3, 16400, 9), (31, 1500, 2700), (32, 2047, 2049), (33, 2049, 2047), (64, 2061, 2560), (65, 1281, 1803),
       (96, 1030, 3001), (97, 2056, 1416), (128, 1999, 1289)]


@pytest.mark.parametrize("t,n,k", FEW)
@pytest.mark.parametrize("gt,wt", [("bf16", "fp32"), ("fp32", "fp32"), ("bf16", "bf16"), ("fp32", "bf16")])
def test_weight_grad_of_few_tokens(t, n, k, gt, wt):
    """Rows of wider buffers, which hold NaN, as does what lies before and after them; what is beside the result stays."""
    kept, blocks = O.checkpoint_rows(gen((t, k), torch.bfloat16, 1)), -(-k // 128)
    dyb = torch.full((t + 2, n + 3), NAN, device=DEV, dtype=DT[gt])
    qb = torch.full((t + 2, k + 5), 0x7f, device=DEV, dtype=torch.uint8)
    eb = torch.full((t + 2, blocks + 1), 255, device=DEV, dtype=torch.uint8)
    dwb = torch.full((n + 2, k + 5), 7.0, device=DEV, dtype=DT[wt])
    dy, q, e, dw = dyb[1:-1, 1:n + 1], qb[1:-1, 1:k + 1], eb[1:-1, 1:], dwb[1:-1, 3:k + 3]
    dy.copy_(gen((t, n), DT[gt], 2, 1e-3)), q.copy_(kept["q"].view(torch.uint8)), e.copy_(kept["exponent"])
    assert O.linear_weight_grad(dy, q.view(E4M3), e, dw_dtype=wt, out={"dw": dw})["workspace"] is None
    check_weight(dy, q.view(E4M3), e, dw)
    again = O.linear_weight_grad(dy.contiguous(), kept["q"], kept["exponent"], dw_dtype=wt)["dw"]
    assert torch.equal(again, dw)
    dw.fill_(7.0)
    assert (dwb == 7).all()


@pytest.mark.parametrize("gt", ["bf16", "fp32"])
@pytest.mark.parametrize("t,n,k", [(1, 2050, 3001), (70, 3001, 1030)])
def test_what_is_not_finite_among_few_tokens(gt, t, n, k):
    kept, dy = O.checkpoint_rows(gen((t, k), torch.bfloat16, 1).clamp_min(0.5)), gen((t, n), DT[gt], 2)
    want = O.linear_weight_grad(dy, kept["q"], kept["exponent"])["dw"].clone()
    dy[t - 1, n - 2], dy[0, 0] = INF, NAN
    kept["q"].view(torch.uint8)[t - 1, k - 1] = 0x7f
    dw = O.linear_weight_grad(dy, kept["q"], kept["exponent"])["dw"]
    assert (dw[n - 2, :k - 1] == INF).all() and dw[0].isnan().all() and dw[:, k - 1].isnan().all()
    rows = [i for i in range(n) if i not in (0, n - 2)]
    assert torch.equal(dw[rows, :k - 1], want[rows, :k - 1])


@pytest.mark.parametrize("gt", ["bf16", "fp32"])
@pytest.mark.parametrize("n,k", [(300, 200), (4096, 4096)])
def test_one_hot_tokens_read_what_was_kept(gt, n, k):
    """dy with one 1 a row: the gradient's rows are the activations that were kept, bit for bit."""
    t = 130
    kept = O.checkpoint_rows(gen((t, k), torch.bfloat16, 1))
    dy = torch.zeros(t, n, device=DEV, dtype=DT[gt])
    at = torch.randperm(n, generator=torch.Generator(device=DEV).manual_seed(3), device=DEV)[:t]
    dy[torch.arange(t, device=DEV), at] = 1.0
    dw = O.linear_weight_grad(dy, kept["q"], kept["exponent"])["dw"]
    assert torch.equal(dw[at].double(), back(kept["q"], kept["exponent"]))
    assert int(dw.count_nonzero()) == int((kept["q"].float() != 0).sum())


@pytest.mark.parametrize("n,k", [(300, 200), (4096, 4096)])
def test_fp32_gradients_are_taken_whole(n, k):
    """One token, x = 1: dweight is dy itself, all 24 bits of it; and infinity and NaN."""
    x = torch.ones(1, k, device=DEV)
    kept = O.checkpoint_rows(x)
    dy = gen((1, n), torch.float32, 1)
    dy[0, 5], dy[0, 6], dy[0, 7], dy[0, 8] = INF, NAN, 3.4028234663852886e38, -1e-30
    dw = O.linear_weight_grad(dy, kept["q"], kept["exponent"])["dw"]
    assert torch.equal(dw.nan_to_num(12.5), dy.nan_to_num(12.5)[0][:, None].expand(n, k))


@pytest.mark.parametrize("t,n,k,parts", [(100, 4096, 4096, 0), (150, 300, 200, 0), (130, 4096, 4096, 3), (191, 4096, 4096, 3),
                                         (700, 4096, 4096, 3), (1500, 4099, 4104, 3)])
def test_all_parts_of_an_fp32_gradient(t, n, k, parts):
    """One value of 24 significant bits a token, each in a row of dweight of its own, and x a power of two: dweight's rows
    are those values, scaled, bit for bit, in each form, whichever steps and shares their three parts fall to."""
    g = torch.Generator(device=DEV).manual_seed(1)
    blocks, rows = -(-k // 128), min(n, t)
    powers = torch.randint(-20, 20, (t, blocks), generator=g, device=DEV)
    x = torch.exp2(powers.float()).repeat_interleave(128, 1)[:, :k].contiguous()
    kept = O.checkpoint_rows(x)
    assert torch.equal(back(kept["q"], kept["exponent"]), x.double())
    value = torch.randn(t, generator=g, device=DEV)
    value = (value.view(torch.int32) | 0x010101).view(torch.float32)  # no part is 0
    at = torch.randperm(n, generator=g, device=DEV)[:rows]
    dy = torch.zeros(t, n, device=DEV)
    tok = torch.randperm(t, generator=g, device=DEV)[:rows]
    dy[tok, at] = value[tok]
    o = O.linear_weight_grad(dy, kept["q"], kept["exponent"])
    if parts:  # the form that spreads dy's parts over its workspace
        assert o["workspace"].numel() >= parts * -(-t // 64) * 64 * n * 2
    want = torch.zeros(n, k, device=DEV, dtype=torch.float64)
    want[at] = value[tok].double()[:, None] * x[tok].double()
    assert torch.equal(o["dw"].double(), want)


@pytest.mark.parametrize("gt", ["bf16", "fp32"])
@pytest.mark.parametrize("t,n,k", [(150, 200, 300), (700, 4096, 4096)])
@pytest.mark.parametrize("x_size,dy_size", [(2.0 ** -100, 2.0 ** 90), (2.0 ** 120, 2.0 ** -100)])
def test_weight_grad_at_the_ends_of_the_range(gt, t, n, k, x_size, dy_size):
    g = torch.Generator(device=DEV).manual_seed(1)
    x = (torch.rand(t, k, generator=g, device=DEV) + 0.5) * x_size
    dy = ((torch.randn(t, n, generator=g, device=DEV) + 3) * dy_size).to(DT[gt])
    kept = O.checkpoint_rows(x)
    assert (back(kept["q"], kept["exponent"]) != 0).all()
    check_weight(dy, kept["q"], kept["exponent"], O.linear_weight_grad(dy, kept["q"], kept["exponent"])["dw"])


@pytest.mark.parametrize("n,k", [(64, 200), (4096, 2048)])
def test_weight_grad_with_far_apart_rows(n, k):
    """Strides past what 32-bit offsets of a step take."""
    t, stride = 100, (1 << 22) + 24
    kept = O.checkpoint_rows(gen((t, k), torch.bfloat16, 1))
    buf = torch.empty(t * stride, device=DEV, dtype=torch.bfloat16)
    dy = buf.view(t, stride)[:, :n]
    dy.copy_(gen((t, n), torch.bfloat16, 2))
    check_weight(dy, kept["q"], kept["exponent"], O.linear_weight_grad(dy, kept["q"], kept["exponent"])["dw"])
    qb = torch.empty(t * stride, device=DEV, dtype=torch.uint8)
    q = qb.view(t, stride)[:, :k]
    q.copy_(kept["q"].view(torch.uint8))
    check_weight(dy, q.view(E4M3), kept["exponent"], O.linear_weight_grad(dy, q.view(E4M3), kept["exponent"])["dw"])


@pytest.mark.parametrize("t,n,k", TNK + [(128, 2048, 4096), (300, 2048, 4096), (513, 4096, 4104), (1025, 2056, 8192), (4100, 1000, 2000),
                                         (1500, 4099, 4100), (8191, 2304, 2050), (16385, 300, 77)])
@pytest.mark.parametrize("gt,wt", [("bf16", "fp32"), ("fp32", "fp32")])
def test_sums_of_integers_are_exact(t, n, k, gt, wt):
    """Every product and every sum is an integer below 2^24: no order rounds, and a token that is lost or counted twice
    shows in any list."""
    g = torch.Generator(device=DEV).manual_seed(1)
    x, dy = torch.randint(-15, 16, (t, k), generator=g, device=DEV), torch.randint(-60, 61, (t, n), generator=g, device=DEV)
    assert 15 * 60 * t < 2 ** 24
    kept = O.checkpoint_rows(x.to(torch.bfloat16))
    assert torch.equal(back(kept["q"], kept["exponent"]).long(), x)
    dw = O.linear_weight_grad(dy.to(DT[gt]), kept["q"], kept["exponent"], dw_dtype=wt)["dw"]
    assert torch.equal(dw.double(), dy.double().t().contiguous() @ x.double())


def test_weight_grad_of_the_longest_rows():
    """dy's rows of 2^22 elements, 64 of them a step, in the form for large weights."""
    t, n, k = 130, 1 << 22, 264
    kept = O.checkpoint_rows(gen((t, k), torch.bfloat16, 1))
    dy = gen((t, n), torch.bfloat16, 2)
    o = O.linear_weight_grad(dy, kept["q"], kept["exponent"])
    assert o["workspace"].numel() >= 192 * k * 2
    some = torch.randperm(n, generator=torch.Generator(device=DEV).manual_seed(3), device=DEV)[:2000]
    for rows in (slice(0, 600), slice(n - 600, n), some):
        check_weight(dy[:, rows], kept["q"], kept["exponent"], o["dw"][rows])


@pytest.mark.parametrize("gt", ["bf16", "fp32"])
@pytest.mark.parametrize("t,n,k", [(70, 200, 300), (191, 4096, 4096)])
def test_what_is_not_finite_reaches_its_row_and_column(gt, t, n, k):
    x = gen((t, k), torch.bfloat16, 1)
    x[x == 0] = 1.0
    kept = O.checkpoint_rows(x)
    dy = gen((t, n), DT[gt], 2)
    want = O.linear_weight_grad(dy, kept["q"], kept["exponent"])["dw"]
    dy[t - 1, n - 2] = INF
    x[3, k - 1] = NAN
    kept = O.checkpoint_rows(x)
    dw = O.linear_weight_grad(dy, kept["q"], kept["exponent"])["dw"]
    q = kept["q"].float()[t - 1]
    row = torch.where(q == 0, NAN, torch.copysign(torch.full_like(q, INF), q))
    row[k - 1] = NAN
    assert torch.equal(dw[n - 2].nan_to_num(0.5), row.nan_to_num(0.5)) and dw[:, k - 1].isnan().all()
    rest = torch.ones(n, device=DEV, dtype=torch.bool)
    rest[n - 2] = False
    assert torch.equal(dw[rest, :k - 1], want[rest, :k - 1])


def test_no_tokens():
    q, e = torch.empty(0, 300, device=DEV, dtype=torch.uint8).view(E4M3), torch.empty(0, 3, device=DEV, dtype=torch.uint8)
    out = {"dw": torch.full((40, 300), 7.0, device=DEV)}
    dw = O.linear_weight_grad(torch.empty(0, 40, device=DEV), q, e, out=out)["dw"]
    assert (dw == 0).all()
    o = O.checkpoint_rows(torch.empty(0, 300, device=DEV), act="gelu")
    assert o["q"].shape == (0, 300) and o["exponent"].shape == (0, 3) and o["y"].shape == (0, 300)
    assert O.checkpoint_backward(torch.empty(0, 300, device=DEV), q, e, act="relu")["dx"].shape == (0, 300)
