"""The product from packed codes.

One-hot activations read r out: y is then r's columns, and has to be the r that
quasar_reconstruct gave, bit for bit, for every format and from both sides of
every choice the library makes by the number of tokens.  Other activations are
held to the 64-bit product within K u sum |x r| (u = 2^-24: no order of the fp32
sums is worse) and the epilogue's and output's roundings."""
import math

import pytest
import torch

from paper_2608_13966_amd import ops as O
from paper_2608_13966_amd import quasar as Q
from paper_2608_13966_amd import synth

pytestmark = pytest.mark.gpu

DEV = "cuda"
U = 2.0 ** -24
FORMATS = [("int", 2, 64), ("int", 2, 128), ("int", 3, 64), ("int", 3, 128), ("int", 4, 64), ("int", 4, 128),
           ("int_sym", 2, 64), ("int_sym", 3, 128), ("int_sym", 4, 64), ("nvfp4", 4, 16), ("rubin", 3, 512)]
CLIPS = tuple(synth.clip_grid(1.0, 0.7, 4))


def layer(n, k, fmt, bits, group, seed=0):
    """(PackedWeight, r in bf16) of a reconstruction."""
    W, v, _ = synth.gen_matrix(n, k, seed, w_bf16=True, ema=False, device=DEV)
    out = Q.reconstruct(W, v, fmt=fmt, bits=bits, group=group, clips=CLIPS)
    return O.PackedWeight.of(out), out["r"]


def acts(t, k, seed, dtype="bf16", pad=0, off=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    x = torch.randn(t, k, generator=g, device=DEV) * torch.exp(0.5 * torch.randn(t, 1, generator=g, device=DEV))
    s = None
    dt = torch.bfloat16
    if dtype == "fp8":
        s = x.abs().amax(1) / 448
        x, dt = (x / s[:, None]), torch.float8_e4m3fn
    buf = torch.zeros(t * (k + pad) + off, device=DEV).to(dt)
    v = buf[off:].view(t, k + pad)[:, :k]
    v.copy_(x.to(dt))
    return v, s


def act64(v, act):
    if act == "relu":
        return v.clamp_min(0)
    if act == "silu":
        return v * torch.sigmoid(v)
    if act == "gelu":
        return 0.5 * v * torch.special.erfc(-v / math.sqrt(2))
    return v


def check(y, x, r, s=None, bias=None, res=None, act="none"):
    xd, rd = x.double(), r.double()
    k = rd.shape[1]
    v = xd @ rd.t()
    e = (k + 4) * U * (xd.abs() @ rd.abs().t())
    if s is not None:
        v, e = v * s.double()[:, None], e * s.double()[:, None]
    if bias is not None:
        v = v + bias.double()
    e = e + 2 * U * v.abs()
    a = act64(v, act)
    if act in ("silu", "gelu"):
        e = 1.2 * e + 16 * U * (a.abs() + v.abs() * 0.1)  # slopes below 1.13; fp32 exp, erf and quotient
    if res is not None:
        a = a + res.double()
        e = e + U * a.abs()
    e = e + a.abs() * (2.0 ** -8 if y.dtype is torch.bfloat16 else U) * 1.01 + 1e-38
    bad = ~((y.double() - a).abs() <= e)
    assert not bad.any(), (int(bad.sum()), float((y.double() - a).abs().max()))


@pytest.mark.parametrize("fmt,bits,group", FORMATS)
@pytest.mark.parametrize("tokens", [1, 5, 16, 33, 64, 65, 200])
def test_one_hot_tokens_read_the_trained_weights(fmt, bits, group, tokens):
    n, k = (72, 512) if fmt == "rubin" else (75, 512)
    w, r = layer(n, k, fmt, bits, group, seed=bits)
    assert r.dtype is torch.bfloat16
    for at in (0, k // 2, k - 1 - tokens if tokens < k else 0):
        cols = (torch.arange(tokens, device=DEV) * 7 + at) % k
        x = torch.nn.functional.one_hot(cols, k).to(torch.bfloat16)
        want = r[:, cols].t()
        assert torch.equal(O.linear_codes(x, w)["y"], want + 0.0)
        assert torch.equal(O.linear_codes(x, w, y_dtype="fp32")["y"], want.float())
        assert torch.equal(O.linear_codes(x.to(torch.float8_e4m3fn), w)["y"], want + 0.0)


def test_a_constant_group_and_a_zero_matrix():
    W = torch.full((16, 256), 0.375, device=DEV, dtype=torch.bfloat16)
    W[3] = 0.0
    v = torch.ones(16, 256, device=DEV)
    for fmt, bits, group in FORMATS:
        w = O.PackedWeight.of(Q.reconstruct(W, v, fmt=fmt, bits=bits, group=group, clips=CLIPS))
        r = Q.reconstruct(W, v, fmt=fmt, bits=bits, group=group, clips=CLIPS)["r"]
        for tokens in (2, 100):
            x, _ = acts(tokens, 256, 1)
            check(O.linear_codes(x, w, y_dtype="fp32")["y"], x, r)


SIZES = [(1, 1, 64), (1, 16, 128), (2, 17, 192), (16, 40, 256), (17, 33, 320), (31, 129, 128), (48, 8, 4096), (64, 100, 1088),
         (65, 130, 64), (96, 257, 448), (128, 128, 128), (129, 300, 1024), (255, 1000, 256), (513, 70, 640), (1000, 520, 2048)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("xt", ["bf16", "fp8"])
def test_sizes(m, n, k, xt):
    w, r = layer(n, k, "int", 4, 64, seed=m)
    x, s = acts(m, k, n, xt)
    check(O.linear_codes(x, w, x_scale=s)["y"], x, r, s)
    check(O.linear_codes(x, w, x_scale=s, y_dtype="fp32")["y"], x, r, s)


@pytest.mark.parametrize("fmt,bits,group", FORMATS)
@pytest.mark.parametrize("m", [3, 40, 150, 300])
def test_formats(fmt, bits, group, m):
    n, k = 144, 1024
    w, r = layer(n, k, fmt, bits, group, seed=m)
    for xt in ("bf16", "fp8"):
        x, s = acts(m, k, bits, xt)
        check(O.linear_codes(x, w, x_scale=s, y_dtype="fp32")["y"], x, r, s)


@pytest.mark.parametrize("k", [16, 48, 80, 144, 208, 1040])
@pytest.mark.parametrize("m", [1, 7, 60, 70, 130])
def test_nvfp4_columns_that_are_no_multiple_of_a_tile(k, m):
    w, r = layer(37, k, "nvfp4", 4, 16, seed=k)
    for xt in ("bf16", "fp8"):
        x, s = acts(m, k, k + m, xt)
        check(O.linear_codes(x, w, x_scale=s, y_dtype="fp32")["y"], x, r, s)


@pytest.mark.parametrize("fmt,bits,group", FORMATS)
@pytest.mark.parametrize("m,k", [(1, 8192), (6, 8256), (13, 12224), (32, 33024), (84, 14400)])
def test_few_outputs_of_many_columns(fmt, bits, group, m, k):
    """The columns are shared out over workgroups."""
    k = k // 128 * 128 if group > 64 and fmt != "rubin" else k
    n = 40 if fmt == "rubin" else 35
    w, r = layer(n, k, fmt, bits, group, seed=m)
    x, s = acts(m, k, k, "fp8")
    g = torch.Generator(device=DEV).manual_seed(7)
    bias = torch.randn(n, generator=g, device=DEV)
    res = torch.randn(m, n, generator=g, device=DEV)
    y = O.linear_codes(x, w, x_scale=s, bias=bias, residual=res, act="silu", y_dtype="fp32")["y"]
    check(y, x, r, s, bias, res, "silu")
    x, _ = acts(m, k, k + 1)
    y = O.linear_codes(x, w)["y"]
    check(y, x, r)
    assert torch.equal(y, O.linear_codes(x, w)["y"])


@pytest.mark.parametrize("m,n,k,fmt,bits,group", [
    (179, 1040, 11904, "int", 3, 128), (250, 2250, 9088, "int_sym", 3, 64), (60, 4000, 1040, "nvfp4", 4, 16),
    (301, 1500, 4160, "rubin", 3, 512), (300, 5000, 1024, "int", 4, 64), (700, 500, 2944, "int", 2, 64),
    (47, 1581, 560, "nvfp4", 4, 16), (96, 8200, 640, "int", 4, 64)])
@pytest.mark.parametrize("xt", ["bf16", "fp8"])
def test_columns_shared_out_unevenly(m, n, k, fmt, bits, group, xt):
    """Shares of any number, the last of fewer steps than the others."""
    n = n // 8 * 8 if fmt == "rubin" else n
    w, r = layer(n, k, fmt, bits, group, seed=m)
    x, s = acts(m, k, n, xt)
    g = torch.Generator(device=DEV).manual_seed(9)
    bias, res = torch.randn(n, generator=g, device=DEV), torch.randn(m, n, generator=g, device=DEV)
    y = O.linear_codes(x, w, x_scale=s, bias=bias, residual=res, act="gelu", y_dtype="fp32")["y"]
    check(y, x, r, s, bias, res, "gelu")
    check(O.linear_codes(x, w, x_scale=s)["y"], x, r, s)


@pytest.mark.parametrize("m,n,k", [(768, 13600, 192), (1025, 8200, 320), (1030, 3336, 8256)])
@pytest.mark.parametrize("fmt,bits,group", FORMATS)
def test_many_tokens(m, n, k, fmt, bits, group):
    """r is written out first; whole tiles and ragged ones, the columns of the last case shared out."""
    k = (k + 127) // 128 * 128 if group == 128 else k + 16 if fmt == "nvfp4" else k
    w, r = layer(n, k, fmt, bits, group, seed=m)
    g = torch.Generator(device=DEV).manual_seed(10)
    bias, res = torch.randn(n, generator=g, device=DEV), torch.randn(m, n, generator=g, device=DEV)
    x, s = acts(m, k, n, "fp8")
    check(O.linear_codes(x, w, x_scale=s, bias=bias, residual=res, act="silu", y_dtype="fp32")["y"], x, r, s, bias, res,
          "silu")
    x, _ = acts(m, k, n + 1)
    y = O.linear_codes(x, w)["y"]
    check(y, x, r)
    # rows that the kernel cannot load as they are, the residual's buffer as y's
    far, _ = acts(m, k, n + 1, pad=3, off=5)
    far.copy_(x)
    out = {"y": res.clone()}
    check(O.linear_codes(far, w, residual=out["y"], y_dtype="fp32", out=out)["y"], x, r, res=res)
    x[7], x[m - 1, 3] = float("nan"), float("inf")
    z = O.linear_codes(x, w)["y"]
    keep = [t for t in range(m) if t not in (7, m - 1)]
    assert z[7].isnan().all() and torch.equal(z[keep], y[keep])


@pytest.mark.parametrize("fmt,bits,group", FORMATS)
@pytest.mark.parametrize("m", [17, 32])
@pytest.mark.parametrize("n", [8200, 8224])
def test_many_outputs_of_few_tokens(fmt, bits, group, m, n):
    """Two blocks of 16 outputs a workgroup, the last of them past the matrix or not."""
    k = 384 if fmt != "nvfp4" else 400
    w, r = layer(n, k, fmt, bits, group, seed=m)
    x, _ = acts(m, k, n)
    g = torch.Generator(device=DEV).manual_seed(8)
    bias, res = torch.randn(n, generator=g, device=DEV), torch.randn(m, n, generator=g, device=DEV)
    y = O.linear_codes(x, w, bias=bias, residual=res, act="gelu", y_dtype="fp32")["y"]
    check(y, x, r, None, bias, res, "gelu")
    check(O.linear_codes(x, w)["y"], x, r)


@pytest.mark.parametrize("m", [4, 30, 140])
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("bt,rt,yt", [("fp32", "bf16", "bf16"), ("bf16", "fp32", "fp32"), (None, "bf16", "fp32"),
                                      ("bf16", None, "bf16")])
def test_epilogue(m, act, bt, rt, yt):
    dt = {"bf16": torch.bfloat16, "fp32": torch.float32}
    n, k = 203, 512
    w, r = layer(n, k, "int", 3, 128, seed=1)
    x, s = acts(m, k, 2, "fp8")
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    bias = torch.randn(n, generator=g, device=DEV).to(dt[bt]) if bt else None
    res = torch.randn(m, n, generator=g, device=DEV).to(dt[rt]) if rt else None
    y = O.linear_codes(x, w, x_scale=s, bias=bias, residual=res, act=act, y_dtype=yt)["y"]
    assert y.dtype is dt[yt]
    check(y, x, r, s, bias, res, act)


@pytest.mark.parametrize("m", [2, 50, 180])
@pytest.mark.parametrize("xt", ["bf16", "fp8"])
@pytest.mark.parametrize("pad,off", [(1, 0), (8, 8), (3, 5)])
def test_strides_and_offsets(m, xt, pad, off):
    n, k = 135, 384
    w, r = layer(n, k, "int", 4, 128, seed=4)
    x, s = acts(m, k, 5, xt, pad, off)
    buf = torch.full((m * (n + pad) + off,), 3.0, device=DEV, dtype=torch.bfloat16)
    y = buf[off:].view(m, n + pad)[:, :n]
    res = torch.zeros(m * (n + pad) + off, device=DEV)[off:].view(m, n + pad)[:, :n]
    res.copy_(torch.randn(m, n, device=DEV))
    o = O.linear_codes(x, w, x_scale=s, residual=res, out={"y": y})
    assert o["y"] is y
    check(y, x, r, s, res=res)
    assert (buf[:off] == 3).all() and (buf[off:].view(m, -1)[:, n:] == 3).all()


@pytest.mark.parametrize("m", [3, 20, 140])
def test_residual_in_place_and_workspace_reuse(m):
    n, k = 200, 256
    w, r = layer(n, k, "int", 2, 64, seed=6)
    x, _ = acts(m, k, 7)
    res = torch.randn(m, n, device=DEV).bfloat16()
    want = O.linear_codes(x, w, residual=res)
    y = res.clone()
    o = O.linear_codes(x, w, residual=y, out={"y": y, "workspace": want["workspace"]})
    assert o["y"] is y and torch.equal(y, want["y"])
    if want["workspace"] is not None:
        assert o["workspace"] is want["workspace"]


@pytest.mark.parametrize("m", [16, 60, 190])
def test_a_token_that_is_not_finite_keeps_to_itself(m):
    n, k = 100, 512
    w, _ = layer(n, k, "int", 4, 128, seed=8)
    x, _ = acts(m, k, 9)
    clean = O.linear_codes(x, w)["y"]
    x[m // 2, 100], x[m - 1, 511] = float("nan"), float("inf")
    y = O.linear_codes(x, w)["y"]
    keep = [i for i in range(m) if i not in (m // 2, m - 1)]
    assert torch.equal(y[keep], clean[keep])
    assert torch.isnan(y[m // 2].float()).all() and not torch.isfinite(y[m - 1].float()).all()


def test_no_tokens():
    w, _ = layer(64, 128, "int", 4, 128)
    y = O.linear_codes(torch.empty(0, 128, device=DEV, dtype=torch.bfloat16), w)["y"]
    assert y.shape == (0, 64)


@pytest.mark.parametrize("m", [1, 8, 64, 100, 257])
def test_results_do_not_depend_on_the_company(m):
    """A token's result alone and among others: the same up to the order of the fp32 sums."""
    n, k = 264, 2048
    w, r = layer(n, k, "int", 4, 128, seed=10)
    x, _ = acts(257, k, 11)
    many, few = O.linear_codes(x, w, y_dtype="fp32")["y"][:m], O.linear_codes(x[:m], w, y_dtype="fp32")["y"]
    size = x[:m].double().abs() @ r.double().abs().t()
    assert ((many.double() - few.double()).abs() <= 2 * (k + 4) * U * size).all()


@pytest.mark.parametrize("m", [5, 40, 300])
def test_another_stream_and_graph(m):
    n, k = 300, 1024
    w, _ = layer(n, k, "int", 3, 128, seed=12)
    x, s = acts(m, k, 13, "fp8")
    bias = torch.randn(n, device=DEV)
    want = O.linear_codes(x, w, x_scale=s, bias=bias, act="silu")["y"]
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        o = O.linear_codes(x, w, x_scale=s, bias=bias, act="silu")
    st.synchronize()
    assert torch.equal(o["y"], want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        O.linear_codes(x, w, x_scale=s, bias=bias, act="silu", out=o)
    for _ in range(3):
        o["y"].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o["y"], want)


def test_offsets_past_32_bits():
    """Tokens of x and y more than 2^31 elements apart."""
    n, k, stride = 40, 256, (1 << 31) + 16
    w, r = layer(n, k, "int", 4, 128, seed=14)
    x, _ = acts(2, k, 15)
    bx = torch.zeros(stride + k, device=DEV, dtype=torch.bfloat16)
    by = torch.zeros(stride + n, device=DEV, dtype=torch.bfloat16)
    fx, fy = bx.as_strided((2, k), (stride, 1)), by.as_strided((2, n), (stride, 1))
    fx.copy_(x)
    O.linear_codes(fx, w, out={"y": fy})
    assert torch.equal(fy, O.linear_codes(x, w)["y"])


def test_norm_into_product():
    """The norm's 8-bit rows and their scales, as the product takes them."""
    n, k, m = 256, 512, 9
    w, r = layer(n, k, "int", 4, 128, seed=16)
    x, _ = acts(m, k, 17)
    f = O.add_rms_norm(x, torch.ones(k, device=DEV), want_y=False, quantize=True)
    y = O.linear_codes(f["q"], w, x_scale=f["scale"], y_dtype="fp32")["y"]
    check(y, f["q"].float(), r, f["scale"])


def test_more_activations_than_a_grid_has_threads():
    """2^28 tokens of 128 columns in 8 bits (34 GB): eight a thread they are 2^32 threads' work."""
    n, k, m = 8, 128, 1 << 28
    w, r = layer(n, k, "int", 4, 128, seed=18)
    torch.cuda.empty_cache()
    g = torch.Generator(device=DEV).manual_seed(19)
    x = torch.randint(0, 0x58, (m, k), device=DEV, generator=g, dtype=torch.uint8).view(torch.float8_e4m3fn)
    y = O.linear_codes(x, w)["y"]
    rt = r.float().t().contiguous()
    for a in range(0, m, 1 << 24):
        part = x[a:a + (1 << 24)].float()
        want = part @ rt
        size = part.abs_() @ rt.abs()
        # both sums in fp32, k u of their terms' sizes each at worst; y's own rounding
        assert ((y[a:a + (1 << 24)].float() - want).abs() <= 2 * (k + 4) * U * size + 2.0 ** -8 * 1.01 * want.abs()).all(), a
        del part, want, size
    check(y[-500:], x[-500:].float(), r)
    del x, y
    torch.cuda.empty_cache()


@pytest.mark.parametrize("m", [1, 20, 60, 1100])
def test_silu_to_the_last_bits(m):
    """Of values that are exact (bias, x being 0), in fp32: an exponential's 2 u, four roundings more, 8 u at most."""
    n, k = 40000 if m > 1000 else 4096, 64
    g = torch.Generator(device=DEV).manual_seed(20)
    codes = torch.randint(0, 256, (n * k // 2,), device=DEV, generator=g, dtype=torch.uint8)
    scales, zeros = torch.rand(n, device=DEV, generator=g), torch.randn(n, device=DEV, generator=g)
    w = O.PackedWeight(n, k, codes, scales, zeros, bits=4, group=64)
    bias = torch.linspace(-60, 60, n, device=DEV)
    bias[::3] = 2 * torch.randn(bias[::3].shape, device=DEV, generator=g)
    inf = float("inf")
    bias[:6] = torch.tensor([-1000.0, 1000.0, 0.0, inf, -inf, float("nan")], device=DEV)
    y = O.linear_codes(torch.zeros(m, k, device=DEV, dtype=torch.bfloat16), w, bias=bias, act="silu", y_dtype="fp32")["y"]
    assert (y[:, 0].abs() < 1e-37).all() and (y[:, 1] == 1000).all() and (y[:, 2] == 0).all() and (y[:, 3] == inf).all()
    assert y[:, 4:6].isnan().all()  # -inf / (1 + inf), and NaN
    v = bias[6:].double()
    want = v / (1 + (-v).exp())
    assert ((y[:, 6:].double() - want).abs() <= 8 * U * want.abs()).all(), float(((y[:, 6:].double() / want - 1).abs() / U).max())


@pytest.mark.parametrize("m,n,k", [(1, 40, 8192), (20, 200, 16384), (140, 200, 4096), (500, 130, 9088), (1500, 3000, 8192)])
@pytest.mark.parametrize("rt,yt", [("bf16", "bf16"), ("fp32", "fp32"), ("fp32", "bf16")])
def test_residual_in_place_through_shared_columns(m, n, k, rt, yt):
    """Where workgroups share the columns their sums meet in the workspace, and the residual is read when they are
    joined: in y's place where it has its type.  What the workspace held before does not matter."""
    dt = {"bf16": torch.bfloat16, "fp32": torch.float32}
    w, r = layer(n, k, "int", 4, 64, seed=21)
    x, _ = acts(m, k, 22)
    g = torch.Generator(device=DEV).manual_seed(23)
    res, bias = torch.randn(m, n, device=DEV, generator=g).to(dt[rt]), torch.randn(n, device=DEV, generator=g)
    want = O.linear_codes(x, w, residual=res, bias=bias, act="gelu", y_dtype=yt)
    check(want["y"], x, r, bias=bias, res=res, act="gelu")
    space = want["workspace"]
    assert space is not None
    space.fill_(255)  # NaN
    y = res.clone() if rt == yt else torch.full_like(want["y"], float("nan"))
    o = O.linear_codes(x, w, residual=y if rt == yt else res, bias=bias, act="gelu", y_dtype=yt,
                       out={"y": y, "workspace": space})
    assert o["y"] is y and o["workspace"].data_ptr() == space.data_ptr()
    assert torch.equal(y, want["y"])
    small = torch.empty(space.numel() - 1, device=DEV, dtype=torch.uint8)  # too small: a new one is taken
    o = O.linear_codes(x, w, residual=res, bias=bias, act="gelu", y_dtype=yt, out={"y": y, "workspace": small})
    assert o["workspace"].numel() >= space.numel() and torch.equal(y, want["y"])
