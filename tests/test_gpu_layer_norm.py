"""add_layer_norm and its gradients against their formulas in 64 bits.

Tolerances, u = 2^-24 (fp32), v = 2^-8 (bf16).  A sum of n fp32 terms in any order
is off by n u of the sum of their sizes at most, so the mean by (n + 4) u mean|h|
(h itself is rounded once); a deviation by that, its h's rounding and its own; the
variance by the deviations' errors and n u of itself; rstd by half of the
variance's relative error and three roundings; y by those of its factors."""
import pytest
import torch

from paper_2608_13966_amd import ops as O

pytestmark = pytest.mark.gpu

DEV = "cuda"
U, V = 2.0 ** -24, 2.0 ** -8
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-5


def gen(shape, dtype, seed, scale=1.0, pad=0, off=0, mean=0.0):
    """Normal values, as rows of a wider buffer (pad) that starts `off` elements into its storage."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    buf = torch.empty(shape[0] * (shape[1] + pad) + off, device=DEV, dtype=dtype)
    t = buf[off:].view(shape[0], shape[1] + pad)[:, :shape[1]]
    t.copy_(torch.randn(shape, generator=g, device=DEV) * scale + mean)
    return t


def rnd(dtype):
    return V if dtype is torch.bfloat16 else U


def close(got, want, tol):
    got = got.double()
    assert got.shape == want.shape
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), float((got - want).abs().max()))


def check_forward(x, w, b, res, o, quantize=False, want_y=True):
    n = x.shape[1]
    h = x.double() + (0 if res is None else res.double())
    mean = h.mean(1, keepdim=True)
    d = h - mean
    var = (d * d).mean(1, keepdim=True)
    rstd = (var + EPS).rsqrt()
    y = d * rstd * w.double() + (0 if b is None else b.double())
    e_mean = (n + 4) * U * h.abs().mean(1, keepdim=True)
    e_d = e_mean + U * h.abs() + U * d.abs()
    e_var = (2 * d.abs() * e_d + e_d * e_d).mean(1, keepdim=True) * 1.01 + (n + 4) * U * var
    e_rstd = rstd * (0.55 * e_var / (var + EPS) + 4 * U)
    e_y = w.double().abs() * (rstd * e_d + d.abs() * e_rstd) * 1.01 + 4 * U * ((d * rstd * w.double()).abs() + y.abs()) + 1e-38
    close(o["mean"], mean[:, 0], e_mean[:, 0] + 1e-38)
    close(o["rstd"], rstd[:, 0], e_rstd[:, 0])
    if res is not None:
        close(o["h"], h, h.abs() * (rnd(res.dtype) + U) + 1e-38)
    if want_y:
        close(o["y"], y, y.abs() * rnd(o["y"].dtype) + e_y * 1.01)
    if quantize:
        s = (y.abs().amax(1) / 448).clamp_min(2.0 ** -120)
        e_top = e_y.amax(1)
        close(o["scale"], s, e_top / 448 + 2 * U * s)
        # E4M3 to nearest: half an ulp is 2^-4 of a normal value and 2^-10 below the smallest; plus y's and the scale's errors
        t = y / s[:, None]
        off = (e_y + t.abs() * e_top[:, None] / 448) / s[:, None] * 1.1 + 4 * U * t.abs()
        close(o["q"].float(), t, t.abs() * 2.0 ** -4 + 2.0 ** -10 + off)


SHAPES = [(1, 1), (3, 7), (5, 64), (33, 128), (17, 129), (9, 250), (2, 511), (2, 513), (4, 1000), (9, 1024), (3, 2049), (7, 4096),
          (5, 4097), (2, 8195), (3, 16384), (2, 32768)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("xt,rt,wt,bt,yt", [("bf16", "bf16", "bf16", "bf16", None), ("bf16", "fp32", "fp32", None, "bf16"),
                                            ("fp32", "bf16", "fp32", "bf16", "fp32"), ("fp32", "fp32", "bf16", "fp32", "bf16"),
                                            ("bf16", None, "fp32", "fp32", "fp32"), ("fp32", None, "bf16", None, None)])
def test_forward(shape, xt, rt, wt, bt, yt):
    x, w = gen(shape, DT[xt], 1, 1.7, mean=0.6), gen((1, shape[1]), DT[wt], 2)[0]
    b = gen((1, shape[1]), DT[bt], 4)[0] if bt else None
    res = gen(shape, DT[rt], 3, 0.8) if rt else None
    o = O.add_layer_norm(x, w, b, res, eps=EPS, y_dtype=yt, quantize=True)
    assert o["y"].dtype is DT[yt or xt]
    if res is None:
        assert o["h"] is x
    check_forward(x, w, b, res, o, quantize=True)


@pytest.mark.parametrize("shape", [(7, 1537), (4, 4096), (33, 72)], ids=str)
@pytest.mark.parametrize("pad,off", [(0, 1), (3, 0), (8, 8), (5, 3)])
def test_forward_strides_and_offsets(shape, pad, off):
    """Rows of wider buffers, at odd elements; outputs likewise, and nothing beside them is touched."""
    x, res = gen(shape, torch.bfloat16, 4, pad=pad, off=off), gen(shape, torch.float32, 5, pad=pad, off=off)
    w, b = gen((1, shape[1]), torch.bfloat16, 6, off=off)[0], gen((1, shape[1]), torch.float32, 7, off=off)[0]
    mark, outs, bufs = 7.0, {}, {}
    for name, dt in (("h", torch.float32), ("y", torch.bfloat16), ("q", torch.uint8)):
        buf = torch.full((shape[0] * (shape[1] + pad + 2) + off,), mark, device=DEV).to(dt)
        outs[name], bufs[name] = buf[off:].view(shape[0], shape[1] + pad + 2)[:, :shape[1]], buf
    outs["q"] = outs["q"].view(torch.float8_e4m3fn)
    outs["mean"], outs["rstd"], outs["scale"] = (torch.empty(shape[0], device=DEV) for _ in range(3))
    o = O.add_layer_norm(x, w, b, res, eps=EPS, quantize=True, out=outs)
    assert o["y"] is outs["y"] and o["q"] is outs["q"]
    check_forward(x, w, b, res, o, quantize=True)
    for buf in bufs.values():
        assert (buf[off:].view(shape[0], -1)[:, shape[1]:] == mark).all() and (buf[:off] == mark).all()


def test_a_large_mean_does_not_cancel():
    """Deviations of 2^-8 around 1000: sum(h^2) - n mean^2 in fp32 would have nothing left."""
    x = (1000 + gen((6, 4096), torch.float32, 1, 2.0 ** -8))
    w = torch.ones(4096, device=DEV)
    check_forward(x, w, None, None, O.add_layer_norm(x, w, eps=EPS))


def test_stream_updated_in_place():
    x, res, w = gen((19, 1000), torch.bfloat16, 7), gen((19, 1000), torch.bfloat16, 8), gen((1, 1000), torch.float32, 9)[0]
    want = O.add_layer_norm(x, w, w, res)
    o = O.add_layer_norm(x, w, w, res, out={"h": res, **{k: torch.empty_like(want[k]) for k in ("mean", "rstd", "y")}})
    assert o["h"] is res
    for k in ("h", "y", "mean", "rstd"):
        assert torch.equal(o[k], want[k]), k


def test_rows_that_are_constant_or_not_finite():
    x = gen((6, 300), torch.float32, 1)
    x[1], x[2, 5], x[3, 299], x[4] = 3.25, float("nan"), float("inf"), 0.0
    w, b = torch.ones(300, device=DEV), torch.full((300,), 0.5, device=DEV)
    o = O.add_layer_norm(x, w, b, eps=EPS, quantize=True)
    good = [0, 1, 4, 5]
    check_forward(x[good], w, b, None, {k: o[k][good] for k in ("mean", "rstd", "y", "q", "scale")}, quantize=True)
    assert (o["y"][[1, 4]] == 0.5).all()
    assert o["y"][2:4].isnan().all() and o["scale"][2:4].isnan().all() and o["q"][2:4].float().isnan().all()


def test_no_rows():
    e = torch.empty(0, 64, device=DEV)
    w = torch.ones(64, device=DEV)
    o = O.add_layer_norm(e, w, quantize=True)
    assert o["y"].shape == (0, 64) and o["mean"].shape == (0,)
    g = O.add_layer_norm_backward(e, e, w, o["mean"], o["rstd"])
    assert g["dx"].shape == (0, 64) and (g["dw"] == 0).all() and (g["db"] == 0).all()


def check_backward(dy, h, w, mean, rstd, dh, o):
    rows, n = dy.shape
    g, hd, wd, r = dy.double(), h.double(), w.double(), rstd.double()[:, None]
    d = hd - mean.double()[:, None]
    nn, u = d * r, g * wd
    mu, m = u.mean(1, keepdim=True), (u * nn).mean(1, keepdim=True)
    dx = r * (u - mu - nn * m)
    size_mu, size_m = u.abs().mean(1, keepdim=True), (u * nn).abs().mean(1, keepdim=True)
    e = r * ((n + 8) * U * (size_mu + nn.abs() * size_m) + 10 * U * (u.abs() + size_mu + nn.abs() * size_m))
    if dh is not None:
        dx = dx + dh.double()
        e = e + U * (dx.abs() + dh.double().abs())
    close(o["dx"], dx, (e + rnd(o["dx"].dtype) * (dx.abs() + e)) * 1.01 + 1e-38)
    if o["dw"] is not None:
        close(o["dw"], (g * nn).sum(0), (rows + 8) * U * (g * nn).abs().sum(0) + 1e-38)
    if o["db"] is not None:
        close(o["db"], g.sum(0), (rows + 8) * U * g.abs().sum(0) + 1e-38)


def stats(h):
    var, mean = torch.var_mean(h.double(), 1, correction=0)
    return mean.float(), (var + EPS).rsqrt().float()


@pytest.mark.parametrize("shape", SHAPES + [(1500, 96), (3000, 200), (1100, 2048), (1030, 4096), (2050, 1000)], ids=str)
@pytest.mark.parametrize("gt,ht,wt,dt", [("bf16", "bf16", "bf16", "bf16"), ("fp32", "fp32", "fp32", None),
                                         ("bf16", "fp32", "fp32", "fp32"), ("fp32", "bf16", "bf16", "bf16")])
def test_backward(shape, gt, ht, wt, dt):
    dy, h = gen(shape, DT[gt], 1), gen(shape, DT[ht], 2, 1.3, mean=0.4)
    w, dh = gen((1, shape[1]), DT[wt], 3)[0], gen(shape, DT[dt], 4) if dt else None
    mean, rstd = stats(h)
    o = O.add_layer_norm_backward(dy, h, w, mean, rstd, dh)
    check_backward(dy, h, w, mean, rstd, dh, o)
    again = O.add_layer_norm_backward(dy, h, w, mean, rstd, dh)
    for k in ("dx", "dw", "db"):
        assert torch.equal(o[k], again[k]), k
    for want in ("dweight", "dbias"):  # one of the sums alone: the same bits
        one = O.add_layer_norm_backward(dy, h, w, mean, rstd, dh, **{f"want_{want}": False})
        key, other = ("dw", "db") if want == "dweight" else ("db", "dw")
        assert one[key] is None and torch.equal(one[other], o[other]) and torch.equal(one["dx"], o["dx"])


@pytest.mark.parametrize("pad,off", [(3, 1), (8, 8), (13, 5)])
def test_backward_strides_and_in_place(pad, off):
    shape = (41, 1537)
    dy, h, dh = (gen(shape, torch.float32, i, pad=pad, off=off) for i in (1, 2, 3))
    w = gen((1, shape[1]), torch.float32, 4, off=off)[0]
    mean, rstd = stats(h)
    want = O.add_layer_norm_backward(dy, h, w, mean, rstd, dh)
    check_backward(dy, h, w, mean, rstd, dh, want)
    for name, t in (("dh", dh), ("dy", dy), ("h", h)):
        copies = {"dy": dy.clone(), "h": h.clone(), "dh": dh.clone()}
        o = O.add_layer_norm_backward(copies["dy"], copies["h"], w, mean, rstd, copies["dh"],
                                      out={"dx": copies[name], "dw": torch.empty_like(w), "db": torch.empty_like(w)})
        for k in ("dx", "dw", "db"):
            assert torch.equal(o[k], want[k]), (name, k)


def test_gradient_against_differences():
    """The formula in 64 bits against central differences of the plain form."""
    g = torch.Generator().manual_seed(0)
    x, w, b, dy = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((4, 9), (9,), (9,), (4, 9)))

    def loss(x, w, b):
        d = x - x.mean(1, keepdim=True)
        return (dy * (d / (d.square().mean(1, keepdim=True) + EPS).sqrt() * w + b)).sum()

    var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
    r = (var + EPS).rsqrt()
    n, u = (x - mean) * r, dy * w
    want = {"x": r * (u - u.mean(1, keepdim=True) - n * (u * n).mean(1, keepdim=True)), "w": (dy * n).sum(0), "b": dy.sum(0)}
    for name, t in (("x", x), ("w", w), ("b", b)):
        got = torch.zeros_like(t)
        for i in range(t.numel()):
            e = torch.zeros(t.numel(), dtype=torch.float64)
            e[i] = 1e-5
            args = {"x": x, "w": w, "b": b}
            up, down = dict(args, **{name: t + e.view_as(t)}), dict(args, **{name: t - e.view_as(t)})
            got.view(-1)[i] = (loss(**up) - loss(**down)) / 2e-5
        assert (got - want[name]).abs().max() < 1e-8  # differences: h^2 of the third derivative and 1e-16 / h


@pytest.mark.parametrize("cols", [1, 5, 7, 8, 9, 15, 60, 65, 70, 127, 131, 198, 260, 511, 700, 1027, 1537, 2047, 3333, 4099, 8191, 9001, 16383])
@pytest.mark.parametrize("typ", ["bf16", "fp32"])
def test_widths_that_cut_a_piece(cols, typ):
    """Rows whose last piece is short, between NaN on the way in and values that stay on the way out."""
    def inside(seed, rows=9, scale=1.0):
        buf = torch.full((rows + 2, cols + 5), float("nan"), device=DEV, dtype=DT[typ])
        buf[1:-1, 2:cols + 2] = gen((rows, cols), DT[typ], seed, scale)
        return buf[1:-1, 2:cols + 2]

    def around(dtype=DT[typ]):
        buf = torch.full((11, cols + 5), 7.0, device=DEV, dtype=dtype)
        return buf, buf[1:-1, 2:cols + 2]

    x, res, w, b = inside(1), inside(2), inside(3, 1)[0], inside(4, 1)[0]
    (yb, y), (hb, h) = around(), around()
    o = O.add_layer_norm(x, w, b, res, eps=EPS, out={"y": y, "h": h, "mean": torch.empty(9, device=DEV), "rstd": torch.empty(9, device=DEV)})
    check_forward(x, w, b, res, o)
    dy, dh, (dxb, dx) = inside(5), inside(6), around()
    out = O.add_layer_norm_backward(dy.contiguous(), h.contiguous(), w.contiguous(), o["mean"], o["rstd"], dh.contiguous())
    kept = {k: out[k].clone() for k in ("dw", "db")}
    got = O.add_layer_norm_backward(dy, h, w, o["mean"], o["rstd"], dh, out={**kept, "dx": dx})
    check_backward(dy, h, w, o["mean"], o["rstd"], dh, got)
    assert all(torch.equal(got[k], out[k]) for k in ("dx", "dw", "db"))
    for buf, t in ((yb, y), (hb, h), (dxb, dx)):
        t.fill_(7.0)
        assert (buf == 7).all()


# ---- means that are large against the deviations ----------------------------------------
# Here the bounds above say nothing: n u of the mean is more than the deviations.  No value of the kernels' sums goes
# through more than 32 additions in a thread, 6 in a wavefront and 16 between them, so D = 64 takes n's place; and what the
# mean is off by is known, since all deviations have it: taken off, only the errors of that are left.
D = 64


def about_a_large_mean(h, w, b):
    """(mean, rstd, y) of fp32 rows in 64 bits, and how far from them a form may be that takes the mean's error off."""
    hd, wd = h.double(), w.double()
    mean = hd.mean(1, keepdim=True)
    d = hd - mean
    size, var = d.abs().mean(1, keepdim=True), (d * d).mean(1, keepdim=True)
    rstd = (var + EPS).rsqrt()
    n = d * rstd
    y = n * wd + b.double()
    e_mean = (D + 2) * U * hd.abs().mean(1, keepdim=True)
    e_dev = U * (d.abs() + e_mean)                           # of a deviation, about the mean that is off
    e_rest = (D + 3) * U * (size + e_mean)                   # of what it is off by
    e_var = 2 * (D + 4) * U * (var + e_mean ** 2) + 2 * e_mean * e_rest
    e_rel = 0.55 * e_var / (var + EPS) + 4 * U               # of rstd
    e_y = wd.abs() * rstd * (e_rest + e_dev + U * d.abs()) + (n * wd).abs() * (e_rel + 3 * U) + U * y.abs()
    return (mean[:, 0], rstd[:, 0], y), (U * mean[:, 0].abs() + 1.01 * e_rest[:, 0], rstd[:, 0] * e_rel[:, 0] * 1.1, e_y * 1.1)


LARGE_MEANS = [(1000.0, 2.0 ** -8), (-100.0, 2.0 ** -4), (1000.0, 1.0), (12345.678, 0.05), (33333.3, 0.0), (0.0, 1.0)]


@pytest.mark.parametrize("cols", [60, 100, 250, 511, 1000, 2047, 4096, 8191, 16384, 32768])
@pytest.mark.parametrize("mean,size", LARGE_MEANS)
@pytest.mark.parametrize("typ", ["fp32", "bf16"])
def test_the_mean_is_taken_off_whole(cols, mean, size, typ):
    """y, rstd and mean of rows with a large mean: fp32 alone, and the same mean in an fp32 stream that bf16 comes to."""
    w, b = gen((1, cols), torch.float32, 2, 0.2, mean=1.0)[0], gen((1, cols), torch.float32, 3, 0.1)[0]
    if typ == "fp32":
        x, res = gen((9, cols), torch.float32, 1, size, mean=mean), None
        h = x
    else:
        x, res = gen((9, cols), torch.bfloat16, 1, size), gen((9, cols), torch.float32, 4, size, mean=mean)
        h = x.float() + res
    o = O.add_layer_norm(x, w, b, res, eps=EPS, y_dtype="fp32")
    for name, want, tol in zip(("mean", "rstd", "y"), *about_a_large_mean(h, w, b)):
        assert o[name].isfinite().all(), name
        close(o[name], want, tol)


@pytest.mark.parametrize("rows,cols", [(1, 64), (7, 4096), (777, 1537), (3000, 200), (5000, 60), (1030, 4096), (1100, 9000), (300, 20000)])
@pytest.mark.parametrize("typ", ["bf16", "fp32"])
def test_sums_over_rows_of_integers_are_exact(rows, cols, typ):
    """mean 0, rstd 1 and integers: dweight = sum dy h and dbias = sum dy have no rounding, whichever row is lost."""
    g = torch.Generator(device=DEV).manual_seed(1)
    dy, h = (torch.randint(-9, 10, (rows, cols), generator=g, device=DEV) for _ in range(2))
    assert 81 * rows < 2 ** 24
    o = O.add_layer_norm_backward(dy.to(DT[typ]), h.to(DT[typ]), torch.ones(cols, device=DEV), torch.zeros(rows, device=DEV),
                                  torch.ones(rows, device=DEV))
    assert torch.equal(o["dw"].long(), (dy * h).sum(0)) and torch.equal(o["db"].long(), dy.sum(0))


# ---- in place, where a row's end cuts a piece ----------------------------------------------
# Such a piece comes as the row's last eight elements, some of which another lane, perhaps of another wavefront, owns and
# writes: they have to be read before that.  Odd widths for each number of threads a row, rows for several rounds.

CUT_WIDTHS = [9, 61, 127, 199, 301, 1023, 1537, 2047, 3333, 4095, 5001, 8191, 16383, 20001]


@pytest.mark.parametrize("cols", CUT_WIDTHS)
@pytest.mark.parametrize("typ", ["bf16", "fp32"])
def test_forward_in_place_with_a_cut_piece(cols, typ):
    rows = 600 if cols < 8192 else 300
    x, res = gen((rows, cols), DT[typ], 1), gen((rows, cols), DT[typ], 2, mean=0.5)
    w, b = gen((1, cols), DT[typ], 3)[0], gen((1, cols), DT[typ], 4)[0]
    want = O.add_layer_norm(x, w, b, res, eps=EPS)
    for turn in range(3):
        for name in ("x", "res"):
            t = {"x": x.clone(), "res": res.clone()}
            out = {"h": t[name], "y": torch.full_like(x, float("nan")), "mean": torch.empty(rows, device=DEV), "rstd": torch.empty(rows, device=DEV)}
            o = O.add_layer_norm(t["x"], w, b, t["res"], eps=EPS, out=out)
            assert o["h"] is t[name]
            for k in ("h", "y", "mean", "rstd"):
                assert torch.equal(o[k], want[k]), (name, k, turn)


@pytest.mark.parametrize("cols", CUT_WIDTHS)
@pytest.mark.parametrize("typ", ["bf16", "fp32"])
def test_backward_in_place_with_a_cut_piece(cols, typ):
    rows = 1500 if cols < 4096 else 600
    dy, h, dh = gen((rows, cols), DT[typ], 1), gen((rows, cols), DT[typ], 2, 1.3, mean=0.4), gen((rows, cols), DT[typ], 3)
    w = gen((1, cols), DT[typ], 4)[0]
    mean, rstd = stats(h)
    want = O.add_layer_norm_backward(dy, h, w, mean, rstd, dh)
    for turn in range(3):
        for name in ("dh", "dy", "h"):
            t = {"dy": dy.clone(), "h": h.clone(), "dh": dh.clone()}
            o = O.add_layer_norm_backward(t["dy"], t["h"], w, mean, rstd, t["dh"],
                                          out={"dx": t[name], "dw": torch.empty(cols, device=DEV), "db": torch.empty(cols, device=DEV)})
            assert o["dx"] is t[name]
            for k in ("dx", "dw", "db"):
                assert torch.equal(o[k], want[k]), (name, k, turn)
