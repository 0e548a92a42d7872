"""The operators around the reconstruction (the C ABI in include/quasar_ops.h):
the RMS norm with the residual's addition and an 8-bit output, the loss against
a teacher's top logits, and the product from packed codes.

Argument checks and marshalling only, as in ``quasar`` (in C++, ``_ops_binding``):
the work runs in the HIP kernels behind the C entry points, there is no CPU path,
and every call is asynchronous on ``stream`` (a ``hipStream_t`` as an int, as a
torch stream's ``cuda_stream``; default: torch's current stream on the tensors'
device).  What a call allocates belongs to that stream, as if it were torch's
current one.  Matrices have unit stride in the last dimension and rows of any
stride that keeps them apart; the teacher's lists are contiguous.  Each function
returns a dict of tensors; a dict it returned may be passed as ``out`` to a later
call of the same sizes and arguments, whose results then overwrite it and which
allocates nothing.

The functions named ``quasar_*`` (``EXPORTS``) mirror the C entry points.
``ste`` has the autograd forms (``add_rms_norm``, ``distill_topk_loss``).
"""
from __future__ import annotations

import ctypes as C
import os

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


# ---- the calls --------------------------------------------------------------------

BINDING_PATH = os.path.join(Q.HERE, "_ops_binding.so")
_binding = None


def _load():
    """The extension module behind the functions below (built in-tree by ``paper_2608_13966_amd.build``)."""
    global _binding
    if _binding is None:
        lib()
        if not os.path.exists(BINDING_PATH):
            raise RuntimeError(f"{BINDING_PATH} is missing: build it with `python -m paper_2608_13966_amd.build` "
                               "(there is no fallback path)")
        import torch  # noqa: F401  the module's own libraries
        from . import _ops_binding as m
        m.set_stream_functions(Q._stream, Q._torch_stream)
        _binding = m
    return _binding


def _dtype(name, what) -> int:
    """The code of "bf16", "fp32" or torch's own dtypes; -1 for None."""
    if name is None:
        return -1
    if isinstance(name, str):
        c = {"bf16": Q.BF16, "fp32": Q.F32}.get(name)
    else:
        import torch
        c = {torch.bfloat16: Q.BF16, torch.float32: Q.F32}.get(name)
    if c is None:
        raise TypeError(f"{what}: unsupported dtype {name}")
    return c


def _done(o, where):
    if type(o) is int:
        raise Q.QuasarError(o, where)
    return o


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
    return _done((_binding or _load()).add_rms_norm(x, weight, residual, eps, _dtype(y_dtype, "y_dtype"), want_y, quantize,
                                                   out, stream), "quasar_add_rms_norm")


def add_rms_norm_backward(dy, h, weight, rstd, dh=None, *, dx_dtype=None, want_dweight=True, out=None, stream=None):
    """The gradients of ``add_rms_norm``: ``dx`` (of x and of residual alike; in
    dh's type, else ``dx_dtype``, default h's) and ``dw`` (fp32).

    dy is y's gradient, h and rstd what the forward call returned, dh the
    gradient of h itself (the rest of the stream's), or None.
    """
    return _done((_binding or _load()).add_rms_norm_backward(dy, h, weight, rstd, dh, _dtype(dx_dtype, "dx_dtype"),
                                                            want_dweight, out, stream), "quasar_add_rms_norm_backward")


# ---- distillation from a teacher's top logits -----------------------------------

def distill_topk(logits, index, teacher, *, temperature=1.0, row_weight=None, out=None, stream=None):
    """Forward KL of the student's logits [rows, classes] to a teacher known by
    its values ``teacher`` [rows, listed] (logits or log-probabilities, fp32 or
    bf16) at the classes ``index`` [rows, listed] (int32 or int64; -1: no entry),
    renormalised over the list, at ``temperature``, times ``row_weight``.

    Returns ``loss`` and ``lse`` (the log-sum of exp(logits / temperature)),
    fp32, one per row.  A row of weight 0, or with nothing listed, is masked:
    its loss and gradient are 0 whatever its logits hold.
    """
    return _done((_binding or _load()).distill(0, logits, index, teacher, temperature, row_weight, None, None, 1.0, out,
                                              stream), "quasar_distill_topk")


def distill_topk_backward(logits, index, teacher, lse, *, temperature=1.0, row_weight=None, grad_loss=None,
                          grad_scale=1.0, out=None, stream=None):
    """``grad``, the gradient of the logits in their type, from the forward
    call's arguments and its ``lse``; ``grad_loss`` is the gradient of each
    row's loss [rows], or None: ``grad_scale`` for every row.  ``out["grad"]``
    may be ``logits`` itself."""
    return _done((_binding or _load()).distill(1, logits, index, teacher, temperature, row_weight, lse, grad_loss,
                                              grad_scale, out, stream), "quasar_distill_topk_backward")


def distill_topk_grad(logits, index, teacher, *, temperature=1.0, row_weight=None, grad_scale=1.0, out=None,
                      stream=None):
    """Both in one call, the gradient of each row's loss being ``grad_scale``
    (1 / rows for a mean, times a loss scale): ``loss``, ``lse`` and ``grad``.
    ``out["grad"]`` may be ``logits`` itself."""
    return _done((_binding or _load()).distill(2, logits, index, teacher, temperature, row_weight, None, None, grad_scale,
                                              out, stream), "quasar_distill_topk_grad")


# ---- product from packed codes ---------------------------------------------------

class PackedWeight:
    """The packed form of a weight matrix [rows = out, cols = in], as a
    reconstruction gives it: ``PackedWeight.of(quasar.reconstruct(...))``, or
    from buffers that were stored.  Holds the tensors; copies nothing.
    """

    def __init__(self, rows, cols, codes, scales, zeros=None, tensor_scale=None, *, fmt="int", bits=4, group=128):
        import torch
        d = self.desc = Q.Descriptor(rows, cols, fmt=fmt, bits=bits, group=group)
        ng = Q.quasar_num_groups(d)
        if ng == 0:
            raise ValueError(f"PackedWeight: no {fmt} weight of {bits} bits in groups of {group} is {rows} x {cols}")
        self.fmt, self.rows, self.cols, self.device = fmt, int(rows), int(cols), codes.device
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
        self._packed = _load().Packed(self.rows, self.cols, d.desc.format, d.desc.bits, d.desc.group, codes, scales, zeros,
                                      tensor_scale)

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
    code = ACTS.get(act)
    if code is None:
        raise ValueError(f"linear_codes: act must be one of {', '.join(ACTS)}")
    return _done((_binding or _load()).linear_codes(x, weight._packed, x_scale, bias, residual, code,
                                                   _dtype(y_dtype, "y_dtype"), out, stream), "quasar_linear_codes")
