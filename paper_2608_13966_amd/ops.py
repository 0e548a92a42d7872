"""The operators around the reconstruction (the C ABI in include/quasar_ops.h):
the RMS norm with the residual's addition and an 8-bit output, the loss against
a teacher's top logits, and the product from packed codes.

Argument checks and marshalling only, as in ``quasar``: the work runs in the HIP
kernels behind the C entry points, there is no CPU path, and every call is
asynchronous on ``stream`` (default: torch's current stream on the tensors'
device).  Tensors are 2-D with unit stride in the last dimension; rows may have
any stride.  Each function returns a dict of tensors; a dict it returned may be
passed as ``out`` to a later call of the same sizes and arguments, whose results
then overwrite it and which allocates nothing.

The functions named ``quasar_*`` (``EXPORTS``) mirror the C entry points.
``ste`` has the autograd forms (``add_rms_norm``, ``distill_topk_loss``).
"""
from __future__ import annotations

import ctypes as C

from . import quasar as Q

E4M3 = 3
MAX_LISTED = 1024
NORM_MAX_COLS = 32768
ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}

EXPORTS = ("quasar_add_rms_norm", "quasar_add_rms_norm_check", "quasar_add_rms_norm_backward",
           "quasar_add_rms_norm_backward_check", "quasar_add_rms_norm_backward_workspace_bytes",
           "quasar_distill_topk", "quasar_distill_topk_backward", "quasar_distill_topk_grad",
           "quasar_distill_topk_check", "quasar_distill_topk_workspace_bytes",
           "quasar_linear_codes", "quasar_linear_codes_check", "quasar_linear_codes_workspace_bytes")

_vp, _i64, _i32, _f32, _sz = C.c_void_p, C.c_int64, C.c_int32, C.c_float, C.c_size_t


class Norm(C.Structure):
    """quasar_norm"""
    _fields_ = [("rows", _i64), ("cols", _i64), ("x", _vp), ("residual", _vp), ("weight", _vp), ("h", _vp), ("y", _vp),
                ("q", _vp), ("scale", _vp), ("rstd", _vp), ("x_stride", _i64), ("residual_stride", _i64),
                ("h_stride", _i64), ("y_stride", _i64), ("q_stride", _i64), ("x_dtype", _i32),
                ("residual_dtype", _i32), ("weight_dtype", _i32), ("y_dtype", _i32), ("eps", _f32)]


class NormBackward(C.Structure):
    """quasar_norm_backward"""
    _fields_ = [("rows", _i64), ("cols", _i64), ("dy", _vp), ("h", _vp), ("weight", _vp), ("rstd", _vp), ("dh", _vp),
                ("dx", _vp), ("dweight", _vp), ("workspace", _vp), ("workspace_bytes", _sz), ("dy_stride", _i64),
                ("h_stride", _i64), ("dh_stride", _i64), ("dx_stride", _i64), ("dy_dtype", _i32), ("h_dtype", _i32),
                ("weight_dtype", _i32), ("dx_dtype", _i32)]


class Distill(C.Structure):
    """quasar_distill"""
    _fields_ = [("rows", _i64), ("classes", _i64), ("listed", _i32), ("logits_dtype", _i32), ("teacher_dtype", _i32),
                ("index_bits", _i32), ("logits", _vp), ("index", _vp), ("teacher", _vp), ("row_weight", _vp),
                ("grad_loss", _vp), ("loss", _vp), ("lse", _vp), ("grad", _vp), ("workspace", _vp),
                ("workspace_bytes", _sz), ("logits_stride", _i64), ("grad_stride", _i64), ("temperature", _f32),
                ("grad_scale", _f32)]


class Linear(C.Structure):
    """quasar_linear"""
    _fields_ = [("tokens", _i64), ("x", _vp), ("x_scale", _vp), ("codes", _vp), ("scales", _vp), ("zeros", _vp),
                ("tensor_scale", _vp), ("bias", _vp), ("residual", _vp), ("y", _vp), ("workspace", _vp),
                ("workspace_bytes", _sz), ("x_stride", _i64), ("residual_stride", _i64), ("y_stride", _i64),
                ("x_dtype", _i32), ("bias_dtype", _i32), ("residual_dtype", _i32), ("y_dtype", _i32), ("act", _i32)]


_lib = None


def lib():
    """The library of ``quasar.lib()`` with these entry points' signatures."""
    global _lib
    if _lib is None:
        L = Q.lib()
        np_, bp, dp, lp, desc = (C.POINTER(t) for t in (Norm, NormBackward, Distill, Linear, Q.Desc))
        for name, args, res in (
                ("quasar_add_rms_norm", [np_, _vp], C.c_int), ("quasar_add_rms_norm_check", [np_], C.c_int),
                ("quasar_add_rms_norm_backward", [bp, _vp], C.c_int),
                ("quasar_add_rms_norm_backward_check", [bp], C.c_int),
                ("quasar_add_rms_norm_backward_workspace_bytes", [_i64, _i64], _sz),
                ("quasar_distill_topk", [dp, _vp], C.c_int), ("quasar_distill_topk_backward", [dp, _vp], C.c_int),
                ("quasar_distill_topk_grad", [dp, _vp], C.c_int),
                ("quasar_distill_topk_check", [dp, C.c_int], C.c_int),
                ("quasar_distill_topk_workspace_bytes", [_i64, _i64], _sz),
                ("quasar_linear_codes", [desc, lp, _vp], C.c_int), ("quasar_linear_codes_check", [desc, lp], C.c_int),
                ("quasar_linear_codes_workspace_bytes", [desc, _i64, _i32], _sz)):
            f = getattr(L, name)
            f.argtypes, f.restype = args, res
        _lib = L
    return _lib


def quasar_add_rms_norm(a: Norm, stream) -> int:
    return lib().quasar_add_rms_norm(C.byref(a), stream)


def quasar_add_rms_norm_check(a: Norm) -> int:
    return lib().quasar_add_rms_norm_check(C.byref(a))


def quasar_add_rms_norm_backward(a: NormBackward, stream) -> int:
    return lib().quasar_add_rms_norm_backward(C.byref(a), stream)


def quasar_add_rms_norm_backward_check(a: NormBackward) -> int:
    return lib().quasar_add_rms_norm_backward_check(C.byref(a))


def quasar_add_rms_norm_backward_workspace_bytes(rows: int, cols: int) -> int:
    return int(lib().quasar_add_rms_norm_backward_workspace_bytes(int(rows), int(cols)))


def quasar_distill_topk(a: Distill, stream) -> int:
    return lib().quasar_distill_topk(C.byref(a), stream)


def quasar_distill_topk_backward(a: Distill, stream) -> int:
    return lib().quasar_distill_topk_backward(C.byref(a), stream)


def quasar_distill_topk_grad(a: Distill, stream) -> int:
    return lib().quasar_distill_topk_grad(C.byref(a), stream)


def quasar_distill_topk_check(a: Distill, what: int) -> int:
    return lib().quasar_distill_topk_check(C.byref(a), int(what))


def quasar_distill_topk_workspace_bytes(rows: int, classes: int) -> int:
    return int(lib().quasar_distill_topk_workspace_bytes(int(rows), int(classes)))


def quasar_linear_codes(d: Q.Descriptor, a: Linear, stream) -> int:
    return lib().quasar_linear_codes(d.ref, C.byref(a), stream)


def quasar_linear_codes_check(d: Q.Descriptor, a: Linear) -> int:
    return lib().quasar_linear_codes_check(d.ref, C.byref(a))


def quasar_linear_codes_workspace_bytes(d: Q.Descriptor, tokens: int, x_dtype: int) -> int:
    return int(lib().quasar_linear_codes_workspace_bytes(d.ref, int(tokens), int(x_dtype)))


# ---- argument checks ----------------------------------------------------------

_torch = None


def _t():
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


def _code(t, what, e4m3=False) -> int:
    """The dtype code of a tensor: fp32, bf16 or, where allowed, E4M3."""
    torch = _t()
    d = t.dtype
    if d is torch.bfloat16:
        return Q.BF16
    if d is torch.float32 and not e4m3:
        return Q.F32
    if e4m3 and d is torch.float8_e4m3fn:
        return E4M3
    raise TypeError(f"{what}: unsupported dtype {d}")


def _dtype(name, what):
    torch = _t()
    if name in ("bf16", torch.bfloat16):
        return torch.bfloat16
    if name in ("fp32", torch.float32):
        return torch.float32
    raise TypeError(f"{what}: unsupported dtype {name}")


def _matrix(t, what, shape, device):
    """t: [rows, cols] on the device with unit stride in the last dimension."""
    if t.dim() != 2 or tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what} must be a tensor of shape {tuple(shape)}, not {tuple(t.shape)}")
    if t.device != device:
        raise ValueError(f"{what} is on {t.device}, not on {device}")
    if t.stride(1) != 1 and shape[1] > 1:
        raise ValueError(f"{what}: the last dimension must have unit stride")
    return t


def _vector(t, what, n, device, dtype=None):
    if t.dim() != 1 or t.shape[0] != n or t.device != device or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous tensor of {n} elements on {device}")
    if dtype is not None and t.dtype is not dtype:
        raise ValueError(f"{what} must be {dtype}, not {t.dtype}")
    return t


def _ptr(t):
    return None if t is None else t.data_ptr()


def _row_stride(t):
    return 0 if t is None else t.stride(0)


def _workspace(n, device, out):
    if n == 0:
        return None
    w = out.get("workspace") if out else None
    if w is not None and w.numel() >= n and w.device == device:
        return w
    return _t().empty(n, dtype=_t().uint8, device=device)


def _result(out, name, shape, dtype, device):
    """The buffer of one output: out's where it has one of this shape and type, else a new one."""
    if out is None:
        return _t().empty(shape, dtype=dtype, device=device)
    t = out.get(name)
    if t is None or tuple(t.shape) != tuple(shape) or t.dtype is not dtype or t.device != device:
        raise ValueError(f"out[{name!r}] must be a {dtype} tensor of shape {tuple(shape)} on {device}")
    if t.dim() == 1 and not t.is_contiguous() or t.dim() == 2 and t.stride(1) != 1 and shape[1] > 1:
        raise ValueError(f"out[{name!r}] must have unit stride in its last dimension")
    if t.dim() == 2 and shape[0] > 1 and t.stride(0) < shape[1]:
        raise ValueError(f"out[{name!r}]: its rows overlap")
    return t


# ---- RMS norm with the residual's addition ------------------------------------

def add_rms_norm(x, weight, residual=None, *, eps=1e-6, y_dtype=None, want_y=True, quantize=False, out=None,
                 stream=None):
    """h = x + residual; y = h / sqrt(mean(h^2) + eps) * weight, row by row.

    Returns ``h`` (in residual's type; x itself without a residual), ``rstd``
    (fp32, one per row), ``y`` (``want_y``; in ``y_dtype``, default x's) and,
    with ``quantize``, ``q`` (torch.float8_e4m3fn) with ``scale`` (fp32, one per
    row): y is q * scale to 8 bits.  x, residual and weight are fp32 or bf16,
    each its own.  A given ``out`` may hold ``residual`` itself as ``out["h"]``:
    the stream is then updated in place.
    """
    torch = _t()
    if x.dim() != 2:
        raise ValueError("add_rms_norm: x must be 2-D")
    rows, cols = x.shape
    dev = x.device
    _matrix(x, "x", (rows, cols), dev)
    _vector(weight, "weight", cols, dev)
    xc, wc = _code(x, "x"), _code(weight, "weight")
    rc = 0
    if residual is not None:
        _matrix(residual, "residual", (rows, cols), dev)
        rc = _code(residual, "residual")
    o = {"h": x, "y": None, "q": None, "scale": None}
    if residual is not None:
        o["h"] = _result(out, "h", (rows, cols), residual.dtype, dev)
    o["rstd"] = _result(out, "rstd", (rows,), torch.float32, dev)
    yd = x.dtype if y_dtype is None else _dtype(y_dtype, "y_dtype")
    if want_y:
        o["y"] = _result(out, "y", (rows, cols), yd, dev)
    if quantize:
        o["q"] = _result(out, "q", (rows, cols), torch.float8_e4m3fn, dev)
        o["scale"] = _result(out, "scale", (rows,), torch.float32, dev)
    h = o["h"] if residual is not None else None
    a = Norm(rows, cols, x.data_ptr(), _ptr(residual), weight.data_ptr(), _ptr(h), _ptr(o["y"]), _ptr(o["q"]),
             _ptr(o["scale"]), o["rstd"].data_ptr(), x.stride(0), _row_stride(residual), _row_stride(h),
             _row_stride(o["y"]), _row_stride(o["q"]), xc, rc, wc, Q.BF16 if yd is torch.bfloat16 else Q.F32, eps)
    s = quasar_add_rms_norm(a, Q._stream(x) if stream is None else stream)
    if s != Q.OK:
        raise Q.QuasarError(s, "quasar_add_rms_norm")
    return o


def add_rms_norm_backward(dy, h, weight, rstd, dh=None, *, dx_dtype=None, want_dweight=True, out=None, stream=None):
    """The gradients of ``add_rms_norm``: ``dx`` (of x and of residual alike; in
    dh's type, else ``dx_dtype``, default h's) and ``dw`` (fp32).

    dy is y's gradient, h and rstd what the forward call returned, dh the
    gradient of h itself (the rest of the stream's), or None.
    """
    torch = _t()
    if dy.dim() != 2:
        raise ValueError("add_rms_norm_backward: dy must be 2-D")
    rows, cols = dy.shape
    dev = dy.device
    _matrix(dy, "dy", (rows, cols), dev)
    _matrix(h, "h", (rows, cols), dev)
    _vector(weight, "weight", cols, dev)
    _vector(rstd, "rstd", rows, dev, torch.float32)
    xd = h.dtype if dx_dtype is None else _dtype(dx_dtype, "dx_dtype")
    if dh is not None:
        _matrix(dh, "dh", (rows, cols), dev)
        if dx_dtype is not None and xd is not dh.dtype:
            raise ValueError("add_rms_norm_backward: dx has dh's type")
        xd = dh.dtype
        _code(dh, "dh")
    gc, hc, wc = _code(dy, "dy"), _code(h, "h"), _code(weight, "weight")
    o = {"dx": _result(out, "dx", (rows, cols), xd, dev), "dw": None, "workspace": None}
    nb = 0
    if want_dweight:
        o["dw"] = _result(out, "dw", (cols,), torch.float32, dev)
        nb = quasar_add_rms_norm_backward_workspace_bytes(rows, cols)
        o["workspace"] = _workspace(nb, dev, out)
        if rows == 0:
            o["dw"].zero_()
    a = NormBackward(rows, cols, dy.data_ptr(), h.data_ptr(), weight.data_ptr(), rstd.data_ptr(), _ptr(dh),
                     o["dx"].data_ptr(), _ptr(o["dw"]), _ptr(o["workspace"]), nb, dy.stride(0), h.stride(0),
                     _row_stride(dh), o["dx"].stride(0), gc, hc, wc, Q.BF16 if xd is torch.bfloat16 else Q.F32)
    s = quasar_add_rms_norm_backward(a, Q._stream(dy) if stream is None else stream)
    if s != Q.OK:
        raise Q.QuasarError(s, "quasar_add_rms_norm_backward")
    return o


# ---- distillation from a teacher's top logits -----------------------------------

def _distill(what, logits, index, teacher, temperature, row_weight, lse, grad_loss, grad_scale, out, stream, where):
    torch = _t()
    if logits.dim() != 2:
        raise ValueError(f"{where}: logits must be 2-D")
    rows, classes = logits.shape
    dev = logits.device
    _matrix(logits, "logits", (rows, classes), dev)
    lc = _code(logits, "logits")
    if index.dim() != 2 or index.shape[0] != rows:
        raise ValueError(f"{where}: index must be [rows, listed]")
    k = index.shape[1]
    if index.dtype is torch.int64:
        bits = 64
    elif index.dtype is torch.int32:
        bits = 32
    else:
        raise TypeError(f"index: unsupported dtype {index.dtype}")
    for t, n in ((index, "index"), (teacher, "teacher")):
        if tuple(t.shape) != (rows, k) or t.device != dev or not t.is_contiguous():
            raise ValueError(f"{where}: {n} must be a contiguous tensor of shape {(rows, k)} on {dev}")
    tc = _code(teacher, "teacher")
    if row_weight is not None:
        _vector(row_weight, "row_weight", rows, dev, torch.float32)
    o = {"workspace": None}
    nb = 0
    if what == 1:
        _vector(lse, "lse", rows, dev, torch.float32)
        if grad_loss is not None:
            _vector(grad_loss, "grad_loss", rows, dev, torch.float32)
    else:
        o["loss"] = _result(out, "loss", (rows,), torch.float32, dev)
        o["lse"] = lse = _result(out, "lse", (rows,), torch.float32, dev)
        nb = quasar_distill_topk_workspace_bytes(rows, classes)
        o["workspace"] = _workspace(nb, dev, out)
    if what != 0:
        o["grad"] = _result(out, "grad", (rows, classes), logits.dtype, dev)
    g = o.get("grad")
    a = Distill(rows, classes, k, lc, tc, bits, logits.data_ptr(), index.data_ptr(), teacher.data_ptr(),
                _ptr(row_weight), _ptr(grad_loss), _ptr(o.get("loss")), _ptr(lse), _ptr(g), _ptr(o["workspace"]), nb,
                logits.stride(0), _row_stride(g), temperature, grad_scale)
    f = (quasar_distill_topk, quasar_distill_topk_backward, quasar_distill_topk_grad)[what]
    s = f(a, Q._stream(logits) if stream is None else stream)
    if s != Q.OK:
        raise Q.QuasarError(s, f.__name__)
    return o


def distill_topk(logits, index, teacher, *, temperature=1.0, row_weight=None, out=None, stream=None):
    """Forward KL of the student's logits [rows, classes] to a teacher known by
    its values ``teacher`` [rows, listed] (logits or log-probabilities, fp32 or
    bf16) at the classes ``index`` [rows, listed] (int32 or int64; -1: no entry),
    renormalised over the list, at ``temperature``, times ``row_weight``.

    Returns ``loss`` and ``lse`` (the log-sum of exp(logits / temperature)),
    fp32, one per row.  A row of weight 0, or with nothing listed, is masked:
    its loss and gradient are 0 whatever its logits hold.
    """
    return _distill(0, logits, index, teacher, temperature, row_weight, None, None, 1.0, out, stream, "distill_topk")


def distill_topk_backward(logits, index, teacher, lse, *, temperature=1.0, row_weight=None, grad_loss=None,
                          grad_scale=1.0, out=None, stream=None):
    """``grad``, the gradient of the logits in their type, from the forward
    call's arguments and its ``lse``; ``grad_loss`` is the gradient of each
    row's loss [rows], or None: ``grad_scale`` for every row.  ``out["grad"]``
    may be ``logits`` itself."""
    return _distill(1, logits, index, teacher, temperature, row_weight, lse, grad_loss, grad_scale, out, stream,
                    "distill_topk_backward")


def distill_topk_grad(logits, index, teacher, *, temperature=1.0, row_weight=None, grad_scale=1.0, out=None,
                      stream=None):
    """Both in one call, the gradient of each row's loss being ``grad_scale``
    (1 / rows for a mean, times a loss scale): ``loss``, ``lse`` and ``grad``.
    ``out["grad"]`` may be ``logits`` itself."""
    return _distill(2, logits, index, teacher, temperature, row_weight, None, None, grad_scale, out, stream,
                    "distill_topk_grad")


# ---- product from packed codes ---------------------------------------------------

class PackedWeight:
    """The packed form of a weight matrix [rows = out, cols = in], as a
    reconstruction gives it: ``PackedWeight.of(quasar.reconstruct(...))``, or
    from buffers that were stored.  Holds the tensors; copies nothing.
    """

    def __init__(self, rows, cols, codes, scales, zeros=None, tensor_scale=None, *, fmt="int", bits=4, group=128):
        torch = _t()
        d = self.desc = Q.Descriptor(rows, cols, fmt=fmt, bits=bits, group=group)
        if Q.quasar_num_groups(d) == 0:
            raise ValueError(f"PackedWeight: no {fmt} weight of {bits} bits in groups of {group} is {rows} x {cols}")
        self.fmt, self.rows, self.cols, self.device = fmt, int(rows), int(cols), codes.device
        ng = Q.quasar_num_groups(d)
        eight = fmt in ("nvfp4", "rubin")
        zeros = zeros if fmt == "int" else None
        tensor_scale = tensor_scale if fmt == "nvfp4" else None
        self._check(codes, "codes", torch.uint8, Q.quasar_codes_bytes(d))
        self._check(scales, "scales", torch.uint8 if eight else torch.float32, ng * 8 if fmt == "rubin" else ng)
        if fmt == "int":
            self._check(zeros, "zeros", torch.float32, ng)
        if fmt == "nvfp4":
            self._check(tensor_scale, "tensor_scale", torch.float32, 1, more=True)
        self.codes, self.scales, self.zeros, self.tensor_scale = codes, scales, zeros, tensor_scale

    def _check(self, t, name, dtype, n, more=False):
        if t is None or t.dtype is not dtype or not t.is_contiguous() or t.device != self.device or \
                (t.numel() < n if more else t.numel() != n):
            raise ValueError(f"PackedWeight: {name} must be a contiguous {dtype} tensor of {n} elements on the codes' "
                             "device")

    @classmethod
    def of(cls, out):
        """From the dict that ``quasar.reconstruct`` (or a batched or AdamW form) returned."""
        d = out["desc"].desc
        fmt = {Q.INT: "int", Q.INT_SYM: "int_sym", Q.NVFP4: "nvfp4", Q.RUBIN_INT3: "rubin"}[d.format]
        return cls(d.rows, d.cols, out["codes"], out["scales"], out["zeros"], out["tensor_scale"], fmt=fmt,
                   bits=d.bits, group=d.group)


def linear_codes(x, weight: PackedWeight, *, x_scale=None, bias=None, residual=None, act="none", y_dtype="bf16",
                 out=None, stream=None):
    """``y`` = act(x_scale * (x r^T) + bias) + residual, with r [out, in] the
    bf16 reconstruction that ``weight``'s codes stand for.

    x [tokens, in]: bf16, or torch.float8_e4m3fn with ``x_scale`` (fp32, one per
    token: the ``q`` and ``scale`` of ``add_rms_norm``).  bias [out] and residual
    [tokens, out]: fp32 or bf16.  act: "none", "relu", "silu" or "gelu" (the
    exact one, with erf).  y is bf16 or fp32; ``out["y"]`` may be ``residual``.
    """
    if x.dim() != 2:
        raise ValueError("linear_codes: x must be 2-D")
    tokens = x.shape[0]
    dev = weight.device
    _matrix(x, "x", (tokens, weight.cols), dev)
    xc = _code(x, "x", e4m3=True)
    torch = _t()
    if x_scale is not None:
        _vector(x_scale, "x_scale", tokens, dev, torch.float32)
    bc = rc = 0
    if bias is not None:
        bc = _code(_vector(bias, "bias", weight.rows, dev), "bias")
    if residual is not None:
        rc = _code(_matrix(residual, "residual", (tokens, weight.rows), dev), "residual")
    if act not in ACTS:
        raise ValueError(f"linear_codes: act must be one of {', '.join(ACTS)}")
    yd = _dtype(y_dtype, "y_dtype")
    y = _result(out, "y", (tokens, weight.rows), yd, dev)
    d = weight.desc
    nb = quasar_linear_codes_workspace_bytes(d, tokens, xc)
    ws = _workspace(nb, dev, out)
    a = Linear(tokens, x.data_ptr(), _ptr(x_scale), weight.codes.data_ptr(), weight.scales.data_ptr(),
               _ptr(weight.zeros), _ptr(weight.tensor_scale), _ptr(bias), _ptr(residual), y.data_ptr(), _ptr(ws), nb,
               x.stride(0), _row_stride(residual), y.stride(0), xc, bc, rc, Q.BF16 if yd is torch.bfloat16 else Q.F32,
               ACTS[act])
    s = quasar_linear_codes(d, a, Q._stream(x) if stream is None else stream)
    if s != Q.OK:
        raise Q.QuasarError(s, "quasar_linear_codes")
    return {"y": y, "workspace": ws}
