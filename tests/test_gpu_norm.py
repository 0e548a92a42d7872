"""add_rms_norm and its gradients against their formulas in 64 bits.

Tolerances, u = 2^-24 (fp32), v = 2^-8 (bf16, 8 significant bits):
h is one fp32 addition; rstd has a sum of n squares (any order: n u at worst,
sqrt is halved) and three more roundings; y two more products; the outputs'
own rounding on top.  The bounds below take (n + 8) u for sums, which no
order of summation exceeds."""
import numpy as np
import pytest
import torch

from paper_2608_13966_amd import ops as O
from paper_2608_13966_amd import quasar as Q

pytestmark = pytest.mark.gpu

DEV = "cuda"
U, V = 2.0 ** -24, 2.0 ** -8
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-6


def gen(shape, dtype, seed, scale=1.0, pad=0, off=0):
    """Normal values, as rows of a wider buffer (pad) that starts `off` elements into its storage."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    buf = torch.empty(shape[0] * (shape[1] + pad) + off, device=DEV, dtype=dtype)
    t = buf[off:].view(shape[0], shape[1] + pad)[:, :shape[1]]
    t.copy_(torch.randn(shape, generator=g, device=DEV) * scale)
    return t


def rnd(dtype):
    return V if dtype is torch.bfloat16 else U


def close(got, want, tol):
    """|got - want| <= tol elementwise (tol: a tensor or a number)."""
    got = got.double()
    assert got.shape == want.shape
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), float((got - want).abs().max()))


def forward_ref(x, w, res):
    h = x.double() + (0 if res is None else res.double())
    rstd = ((h * h).mean(1) + EPS).rsqrt()
    return h, rstd, h * rstd[:, None] * w.double()


def check_forward(x, w, res, o, quantize=True, want_y=True):
    n = x.shape[1]
    h, rstd, y = forward_ref(x, w, res)
    e = (n + 8) * U
    close(o["rstd"], rstd, rstd * e)
    if res is not None:
        close(o["h"], h, h.abs() * (rnd(res.dtype) + U) + 1e-38)
    if want_y:
        close(o["y"], y, y.abs() * (rnd(o["y"].dtype) + e) + 1e-38)
    if quantize:
        top = y.abs().amax(1)
        s = (top / 448).clamp_min(2.0 ** -120)
        close(o["scale"], s, s * (e + 2 * U))
        # E4M3 to nearest: half an ulp is 2^-4 of a normal value and 2^-10 below the smallest; plus y's own error
        q = o["q"].float().double()
        t = y / s[:, None]
        close(q, t, t.abs() * (2.0 ** -4 + 2 * e) + 2.0 ** -10 + 1e-6)


SHAPES = [(1, 1), (3, 7), (5, 64), (2, 511), (2, 513), (4, 1000), (9, 1024), (3, 2049), (7, 4096), (5, 4097), (2, 8195),
          (3, 16384), (2, 32768)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("xt,rt,wt,yt", [("bf16", "bf16", "bf16", None), ("bf16", "fp32", "fp32", "bf16"),
                                         ("fp32", "bf16", "fp32", "fp32"), ("fp32", "fp32", "bf16", "bf16"),
                                         ("bf16", None, "fp32", "fp32"), ("fp32", None, "bf16", None)])
def test_forward(shape, xt, rt, wt, yt):
    x = gen(shape, DT[xt], 1, 1.7)
    w = gen((1, shape[1]), DT[wt], 2)[0]
    res = gen(shape, DT[rt], 3, 0.8) if rt else None
    o = O.add_rms_norm(x, w, res, eps=EPS, y_dtype=yt, quantize=True)
    assert o["y"].dtype is DT[yt or xt]
    if res is None:
        assert o["h"] is x
    check_forward(x, w, res, o)


@pytest.mark.parametrize("shape", [(7, 1537), (4, 4096), (33, 72)], ids=str)
@pytest.mark.parametrize("pad,off", [(0, 1), (3, 0), (8, 8), (5, 3)])
def test_forward_strides_and_offsets(shape, pad, off):
    """Rows of wider buffers, at odd elements; outputs likewise, and nothing beside them is touched."""
    x = gen(shape, torch.bfloat16, 4, pad=pad, off=off)
    res = gen(shape, torch.float32, 5, pad=pad, off=off)
    w = gen((1, shape[1]), torch.bfloat16, 6, off=off)[0]
    mark = 7.0
    outs, bufs = {}, {}
    for name, dt in (("h", torch.float32), ("y", torch.bfloat16), ("q", torch.uint8)):
        b = torch.full((shape[0] * (shape[1] + pad + 2) + off,), mark, device=DEV).to(dt)
        t = b[off:].view(shape[0], shape[1] + pad + 2)[:, :shape[1]]
        outs[name], bufs[name] = t, b
    outs["q"] = outs["q"].view(torch.float8_e4m3fn)
    outs["rstd"], outs["scale"] = (torch.empty(shape[0], device=DEV) for _ in range(2))
    o = O.add_rms_norm(x, w, res, eps=EPS, quantize=True, out=outs)
    assert o["y"] is outs["y"] and o["q"] is outs["q"]
    check_forward(x, w, res, o)
    for b in bufs.values():
        rest = b[off:].view(shape[0], -1)[:, shape[1]:]
        assert (rest == mark).all() and (b[:off] == mark).all()


def test_stream_updated_in_place():
    x, res = gen((19, 1000), torch.bfloat16, 7), gen((19, 1000), torch.bfloat16, 8)
    w = gen((1, 1000), torch.float32, 9)[0]
    want = O.add_rms_norm(x, w, res)
    o = O.add_rms_norm(x, w, res, out={"h": res, "rstd": want["rstd"].clone(), "y": want["y"].clone()})
    assert o["h"] is res
    for k in ("h", "y", "rstd"):
        assert torch.equal(o[k], want[k]), k


def test_no_rows():
    x = torch.empty(0, 64, device=DEV, dtype=torch.bfloat16)
    w = torch.ones(64, device=DEV)
    o = O.add_rms_norm(x, w, x, quantize=True)
    assert o["y"].shape == (0, 64) and o["scale"].shape == (0,)
    b = O.add_rms_norm_backward(x, x, w, o["rstd"])
    assert b["dx"].shape == (0, 64) and torch.equal(b["dw"], torch.zeros(64, device=DEV))


def test_zero_tiny_and_huge_rows():
    x = gen((6, 300), torch.float32, 10)
    x[0] = 0.0
    x[1] *= 1e-30
    x[2] *= 1e15
    x[3] = 0.0
    x[3, 17] = 1e-20
    w = torch.ones(300, device=DEV)
    o = O.add_rms_norm(x, w, eps=EPS, quantize=True)
    check_forward(x, w, None, o)
    assert (o["q"][0].float() == 0).all() and (o["y"][0] == 0).all() and o["scale"][0] > 0
    assert torch.isfinite(o["q"].float()).all()


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_a_row_that_is_not_finite_keeps_to_itself(value):
    x = gen((5, 700), torch.bfloat16, 11)
    w = torch.ones(700, device=DEV)
    clean = O.add_rms_norm(x, w, quantize=True)
    x[2, 333] = value
    o = O.add_rms_norm(x, w, quantize=True)
    keep = [0, 1, 3, 4]
    for k in ("y", "scale", "rstd"):
        assert torch.equal(o[k][keep], clean[k][keep])
    assert torch.equal(o["q"][keep].float(), clean["q"][keep].float())
    assert torch.isnan(o["scale"][2]) and torch.isnan(o["q"][2].float()).all() and torch.isnan(o["y"][2, 333])


def backward_ref(dy, h, w, rstd, dh):
    n = h.double() * rstd.double()[:, None]
    u = dy.double() * w.double()
    dot = (u * n).mean(1, keepdim=True)
    dx = rstd.double()[:, None] * (u - n * dot)
    if dh is not None:
        dx = dx + dh.double()
    return dx, (dy.double() * n).sum(0), n, u


def check_backward(dy, h, w, rstd, dh, o):
    cols, rows = dy.shape[1], dy.shape[0]
    dx, dw, n, u = backward_ref(dy, h, w, rstd, dh)
    r = rstd.double()[:, None]
    # u and n one product each; the mean's sum cols u of its terms' sizes; then four operations
    size = r * (u.abs() + n.abs() * (u * n).abs().mean(1, keepdim=True))
    tol = (cols + 12) * U * r * n.abs() * (u * n).abs().mean(1, keepdim=True) + 8 * U * size
    if dh is not None:
        tol = tol + U * (dh.double().abs() + dx.abs())
    close(o["dx"], dx, tol + rnd(o["dx"].dtype) * dx.abs() * (1 + 2 * V) + 1e-38)
    if o["dw"] is not None:
        close(o["dw"], dw, (rows + 4) * U * (dy.double() * n).abs().sum(0) + 1e-38)


@pytest.mark.parametrize("shape", SHAPES + [(2500, 96), (1300, 4096), (4099, 640)], ids=str)
@pytest.mark.parametrize("gt,ht,wt,dt", [("bf16", "bf16", "bf16", "bf16"), ("bf16", "fp32", "fp32", "fp32"),
                                         ("fp32", "bf16", "bf16", None), ("fp32", "fp32", "fp32", "bf16")])
def test_backward(shape, gt, ht, wt, dt):
    dy, h = gen(shape, DT[gt], 12, 1e-2, pad=3, off=1), gen(shape, DT[ht], 13, 1.3)
    w = gen((1, shape[1]), DT[wt], 14)[0]
    rstd = (h.double().square().mean(1) + EPS).rsqrt().float()
    dh = gen(shape, DT[dt], 15, 1e-2, pad=5) if dt else None
    o = O.add_rms_norm_backward(dy, h, w, rstd, dh)
    assert o["dx"].dtype is (DT[dt] if dt else h.dtype)
    check_backward(dy, h, w, rstd, dh, o)
    again = O.add_rms_norm_backward(dy, h, w, rstd, dh)
    assert torch.equal(again["dx"], o["dx"]) and torch.equal(again["dw"], o["dw"])


def test_backward_options():
    dy, h = gen((65, 500), torch.bfloat16, 16), gen((65, 500), torch.bfloat16, 17)
    w = torch.ones(500, device=DEV)
    rstd = (h.double().square().mean(1) + EPS).rsqrt().float()
    a = O.add_rms_norm_backward(dy, h, w, rstd)
    b = O.add_rms_norm_backward(dy, h, w, rstd, want_dweight=False, dx_dtype="fp32")
    assert b["dw"] is None and b["dx"].dtype is torch.float32
    assert torch.equal(b["dx"].bfloat16(), a["dx"])
    dh = gen((65, 500), torch.bfloat16, 18)
    want = O.add_rms_norm_backward(dy, h, w, rstd, dh)["dx"]
    o = O.add_rms_norm_backward(dy, h, w, rstd, dh, out={"dx": dh, "dw": a["dw"]})   # the stream's gradient in place
    assert torch.equal(o["dx"], want)


@pytest.mark.parametrize("cols", [5, 130, 1000])
def test_backward_against_differences(cols):
    """Directional differences of the 64-bit formula: L = sum(gy y) + sum(gh h), x and weight moved along random
    directions.  A central difference at 1e-5 leaves about 1e-9 of L'' beside fp32's errors."""
    x, res = gen((6, cols), torch.float32, 19), gen((6, cols), torch.float32, 20)
    w = gen((1, cols), torch.float32, 21)[0]
    gy, gh = gen((6, cols), torch.float32, 22), gen((6, cols), torch.float32, 23)
    f = O.add_rms_norm(x, w, res, eps=EPS)
    o = O.add_rms_norm_backward(gy, f["h"], w, f["rstd"], gh)
    dx_dir, dw_dir = gen((6, cols), torch.float32, 24).double(), gen((1, cols), torch.float32, 25)[0].double()

    def loss(t):
        h = x.double() + t * dx_dir + res.double()
        y = h * ((h * h).mean(1, keepdim=True) + EPS).rsqrt() * (w.double() + t * dw_dir)
        return float((gy.double() * y).sum() + (gh.double() * h).sum())

    want = (loss(1e-5) - loss(-1e-5)) / 2e-5
    got = float((o["dx"].double() * dx_dir).sum() + (o["dw"].double() * dw_dir).sum())
    size = float((o["dx"].double() * dx_dir).abs().sum() + (o["dw"].double() * dw_dir).abs().sum())
    assert abs(got - want) <= size * (2 * cols + 40) * U + 1e-6 * size


def test_offsets_past_32_bits():
    """Rows more than 2^31 elements apart."""
    stride, cols = (1 << 31) + 8, 200
    big = torch.zeros(2 * stride + cols, device=DEV, dtype=torch.bfloat16)
    x = big.as_strided((3, cols), (stride, 1))
    x.copy_(gen((3, cols), torch.bfloat16, 26))
    w = torch.ones(cols, device=DEV)
    near = x.contiguous()
    o, want = O.add_rms_norm(x, w, quantize=True), O.add_rms_norm(near, w, quantize=True)
    assert torch.equal(o["y"], want["y"]) and torch.equal(o["q"].float(), want["q"].float())
    b, wb = O.add_rms_norm_backward(x, x, w, o["rstd"]), O.add_rms_norm_backward(near, near, w, o["rstd"])
    assert torch.equal(b["dx"], wb["dx"]) and torch.equal(b["dw"], wb["dw"])


def test_another_stream_and_graph():
    """On a stream of its own, and replayed from a captured graph: the same bits."""
    x, res = gen((300, 1537), torch.bfloat16, 27), gen((300, 1537), torch.bfloat16, 28)
    w = gen((1, 1537), torch.float32, 29)[0]
    want = O.add_rms_norm(x, w, res, quantize=True)
    wb = O.add_rms_norm_backward(want["y"], want["h"], w, want["rstd"], want["h"])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        o = O.add_rms_norm(x, w, res, quantize=True)
        b = O.add_rms_norm_backward(o["y"], o["h"], w, o["rstd"], o["h"])
    s.synchronize()
    assert torch.equal(o["y"], want["y"]) and torch.equal(b["dw"], wb["dw"]) and torch.equal(b["dx"], wb["dx"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        O.add_rms_norm(x, w, res, quantize=True, out=o)
        O.add_rms_norm_backward(o["y"], o["h"], w, o["rstd"], o["h"], out=b)
    for _ in range(3):
        for t in (o["y"], o["h"], b["dx"], b["dw"]):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o["y"], want["y"]) and torch.equal(o["h"], want["h"])
        assert torch.equal(b["dw"], wb["dw"]) and torch.equal(b["dx"], wb["dx"])


def test_strided_by_zero_is_refused():
    x = torch.ones(1, 64, device=DEV).expand(4, 64)
    with pytest.raises(Q.QuasarError) as e:
        O.add_rms_norm(x, torch.ones(64, device=DEV))
    assert e.value.status == Q.ERR_SHAPE
    assert np.isfinite(float(x.sum()))


@pytest.mark.parametrize("shape", [(64, 4096), (300, 1537), (40, 9000), (1000, 70)], ids=str)
@pytest.mark.parametrize("residual", [False, True])
def test_eight_bit_rows_are_the_rounded_quotients(shape, residual):
    """scale = max |y| / 448 and q = E4M3(y / scale) of the y of the same call, each one fp32 division: bit for bit what
    those give on the CPU.  (y times the reciprocal falls on the neighbouring byte for one value in millions: half of
    each row lies at the edges between bytes, where a rounding of the reciprocal decides.)"""
    x = gen(shape, torch.float32, 30)
    w = torch.ones(shape[1], device=DEV)
    n = shape[1] // 2
    edge = (2.0 + torch.arange(n, device=DEV) % 14 + 0.5) / 16  # halves of the last bit of E4M3
    x[:, :n] = edge * torch.exp2(-(torch.arange(n, device=DEV) % 5).float())
    x[:, n] = 448.0 / 64  # the largest: x at an edge is y / scale at an edge but for rounding
    o = O.add_rms_norm(x, w, torch.zeros_like(x) if residual else None, eps=EPS, quantize=True)
    y = o["y"].cpu()
    scale = y.abs().amax(1) / 448
    assert torch.equal(o["scale"].cpu(), scale)
    want = (y / scale[:, None]).to(torch.float8_e4m3fn)
    assert torch.equal(o["q"].cpu().view(torch.uint8), want.view(torch.uint8))


def test_more_rows_than_a_grid_takes():
    """2^26 rows, four a workgroup of 256 threads, would be 2^32 threads: rows on either side of that."""
    rows, cols = (1 << 26) + 6, 8
    g = torch.Generator(device=DEV).manual_seed(31)
    x, res = (torch.randn(rows, cols, device=DEV, generator=g, dtype=torch.bfloat16) for _ in range(2))
    w = gen((1, cols), torch.float32, 32)[0]
    o = O.add_rms_norm(x, w, res, eps=EPS, quantize=True)
    cut = (1 << 26) - 4
    for a, b in ((0, cut), (cut, rows)):
        part = O.add_rms_norm(x[a:b], w, res[a:b], eps=EPS, quantize=True)
        for k in ("h", "y", "q", "scale", "rstd"):
            assert torch.equal(o[k][a:b].view(torch.uint8), part[k].view(torch.uint8)), k
    check_forward(x[-40:], w, res[-40:], {k: o[k][-40:] for k in ("h", "y", "q", "scale", "rstd")})


@pytest.mark.parametrize("size", [2.0 ** -100, 2.0 ** -85, 2.0 ** -40, 1.0, 2.0 ** 60, 2.0 ** 110])
def test_eight_bit_rows_of_any_size(size):
    """The quotients of the last test with y as large or small as fp32 has it (a weight of that size)."""
    n = 300
    x = gen((50, n), torch.float32, 33)
    x[:, ::2] = ((2.0 + torch.arange(n // 2, device=DEV) % 14 + 0.5) / 16)
    x[:, 1] = 7.0
    w = torch.full((n,), size, device=DEV)
    o = O.add_rms_norm(x, w, eps=EPS, quantize=True)
    y = o["y"].cpu()
    scale = y.abs().amax(1) / 448
    assert torch.equal(o["scale"].cpu(), scale)
    want = (y / scale[:, None]).to(torch.float8_e4m3fn)
    assert torch.equal(o["q"].cpu().view(torch.uint8), want.view(torch.uint8))
    # a weight that makes one column overflow: its scale is infinite, finite values are 0 of it
    w[5] = float("inf")
    o = O.add_rms_norm(x, w, eps=EPS, quantize=True)
    assert (o["scale"] == float("inf")).all()
    q = o["q"].float()
    assert q[:, 5].isnan().all() and (q[:, :5] == 0).all() and (q[:, 6:] == 0).all()
