"""C-ABI contract of the operators of include/quasar_ops.h, checked without a
GPU: exports, the statuses of invalid arguments (the *_check functions touch no
device memory), structure sizes and the refusals of the Python wrappers."""
import ctypes
import os
import re

import pytest
import torch

from paper_2608_13966_amd import ops as O
from paper_2608_13966_amd import quasar as Q

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 0x10000


def _header():
    src = open(os.path.join(ROOT, "include", "quasar_ops.h")).read()
    return re.sub(r"/\*.*?\*/", "", src, flags=re.S)


def test_library_exports_every_declared_operator():
    names = set(re.findall(r"\b(quasar_[a-z_]+)\s*\(", _header()))
    assert names == set(O.EXPORTS)
    for n in names:
        assert hasattr(O.lib(), n) and callable(getattr(O, n)), n


def test_constants_are_the_headers():
    src = _header()
    got = dict(re.findall(r"#define (QUASAR_[A-Z0-9_]+) (\d+)", src))
    assert got == {"QUASAR_E4M3": str(O.E4M3), "QUASAR_NORM_MAX_COLS": str(O.NORM_MAX_COLS),
                   "QUASAR_DISTILL_MAX_LISTED": str(O.MAX_LISTED)}
    acts = {k.lower(): int(v) for k, v in re.findall(r"QUASAR_ACT_([A-Z]+) = (\d)", src)}
    assert acts == O.ACTS


@pytest.mark.parametrize("cls,name", [(O.Norm, "quasar_norm"), (O.NormBackward, "quasar_norm_backward"),
                                      (O.Distill, "quasar_distill"), (O.Linear, "quasar_linear")])
def test_structures_follow_the_header(cls, name):
    """The fields in the header's order, with its types."""
    src = _header()
    end = src.index("} %s;" % name)
    body = src[src.rindex("{", 0, end) + 1:end]
    size = {"int64_t": 8, "int32_t": 4, "float": 4, "size_t": 8}
    want = []
    for decl in body.split(";"):
        decl = decl.strip()
        if not decl:
            continue
        typ, rest = re.match(r"(?:const )?(\w+)\s*(.*)", decl, flags=re.S).groups()
        for f in rest.split(","):
            f = f.strip()
            want.append((f.lstrip("* "), 8 if f.startswith("*") or rest.startswith("*") else size[typ]))
    assert want == [(f, ctypes.sizeof(t)) for f, t in cls._fields_]


def _norm(**kw):
    p = dict(rows=4, cols=100, x=A, residual=A, weight=A, h=A, y=A, q=A, scale=A, rstd=A, x_stride=100,
             residual_stride=100, h_stride=100, y_stride=100, q_stride=100, x_dtype=Q.BF16, residual_dtype=Q.BF16,
             weight_dtype=Q.F32, y_dtype=Q.BF16, eps=1e-6)
    p.update(kw)
    return O.quasar_add_rms_norm_check(O.Norm(**p))


@pytest.mark.parametrize("kw,status", [
    (dict(), Q.OK), (dict(rows=0, x=None, weight=None), Q.OK), (dict(rows=-1), Q.ERR_SHAPE),
    (dict(cols=0), Q.ERR_SHAPE), (dict(cols=O.NORM_MAX_COLS + 1), Q.ERR_SHAPE), (dict(rows=1 << 31), Q.ERR_SHAPE),
    (dict(x=None), Q.ERR_ARG), (dict(weight=None), Q.ERR_ARG), (dict(q=None), Q.ERR_ARG), (dict(scale=None), Q.ERR_ARG),
    (dict(q=None, scale=None, y=None, h=None, rstd=None), Q.OK), (dict(residual=None), Q.ERR_ARG),
    (dict(residual=None, h=None), Q.OK), (dict(eps=-1.0), Q.ERR_ARG), (dict(eps=float("nan")), Q.ERR_ARG),
    (dict(eps=float("inf")), Q.ERR_ARG), (dict(eps=0.0), Q.OK), (dict(x_dtype=Q.F16), Q.ERR_FORMAT),
    (dict(residual_dtype=7), Q.ERR_FORMAT), (dict(weight_dtype=O.E4M3), Q.ERR_FORMAT), (dict(y_dtype=-1), Q.ERR_FORMAT),
    (dict(x_stride=99), Q.ERR_SHAPE), (dict(rows=1, x_stride=0, h_stride=3), Q.OK), (dict(h_stride=99), Q.ERR_SHAPE),
    (dict(q_stride=1 << 41), Q.ERR_SHAPE), (dict(x=A + 2), Q.OK), (dict(x=A + 1), Q.ERR_ALIGN),
    (dict(x=A + 2, x_dtype=Q.F32), Q.ERR_ALIGN), (dict(q=A + 1), Q.OK), (dict(scale=A + 2), Q.ERR_ALIGN),
    (dict(weight=A + 2), Q.ERR_ALIGN), (dict(rstd=A + 1), Q.ERR_ALIGN)])
def test_norm_arguments(kw, status):
    assert _norm(**kw) == status


def _norm_backward(**kw):
    rows, cols = kw.get("rows", 64), kw.get("cols", 4096)
    p = dict(rows=rows, cols=cols, dy=A, h=A, weight=A, rstd=A, dh=A, dx=A, dweight=A, workspace=A,
             workspace_bytes=O.quasar_add_rms_norm_backward_workspace_bytes(rows, cols), dy_stride=4096, h_stride=4096,
             dh_stride=4096, dx_stride=4096, dy_dtype=Q.BF16, h_dtype=Q.F32, weight_dtype=Q.F32, dx_dtype=Q.F32)
    p.update(kw)
    return O.quasar_add_rms_norm_backward_check(O.NormBackward(**p))


@pytest.mark.parametrize("kw,status", [
    (dict(), Q.OK), (dict(dh=None), Q.OK), (dict(dweight=None, workspace=None, workspace_bytes=0), Q.OK),
    (dict(workspace=None), Q.ERR_WORKSPACE), (dict(workspace_bytes=15), Q.ERR_WORKSPACE),
    (dict(rows=1, workspace=None, workspace_bytes=0), Q.OK), (dict(rows=0, dy=None, dx=None), Q.OK),
    (dict(dy=None), Q.ERR_ARG), (dict(h=None), Q.ERR_ARG), (dict(rstd=None), Q.ERR_ARG), (dict(dx=None), Q.ERR_ARG),
    (dict(weight=None), Q.ERR_ARG), (dict(dx_dtype=Q.F16), Q.ERR_FORMAT), (dict(dy_dtype=O.E4M3), Q.ERR_FORMAT),
    (dict(dh_stride=4095), Q.ERR_SHAPE), (dict(cols=40000), Q.ERR_SHAPE), (dict(dh=A + 2), Q.ERR_ALIGN),
    (dict(dy=A + 2), Q.OK), (dict(workspace=A + 8), Q.ERR_ALIGN)])
def test_norm_backward_arguments(kw, status):
    assert _norm_backward(**kw) == status


def _distill(what=2, **kw):
    p = dict(rows=5, classes=1000, listed=8, logits_dtype=Q.BF16, teacher_dtype=Q.F32, index_bits=64, logits=A, index=A,
             teacher=A, row_weight=A, grad_loss=None, loss=A if what != 1 else None, lse=A,
             grad=A + 2 if what else None, workspace=A, workspace_bytes=1 << 20, logits_stride=1000, grad_stride=1000,
             temperature=1.0, grad_scale=1.0)
    p.update(kw)
    return O.quasar_distill_topk_check(O.Distill(**p), what)


@pytest.mark.parametrize("what", [0, 1, 2])
@pytest.mark.parametrize("kw,status", [
    (dict(), Q.OK), (dict(row_weight=None), Q.OK), (dict(rows=0, logits=None, lse=None), Q.OK),
    (dict(rows=-1), Q.ERR_SHAPE), (dict(classes=0), Q.ERR_SHAPE), (dict(classes=1 << 31), Q.ERR_SHAPE),
    (dict(listed=0), Q.ERR_SHAPE), (dict(listed=O.MAX_LISTED + 1), Q.ERR_SHAPE),
    (dict(rows=1 << 31, classes=1 << 20, logits_stride=1 << 20, grad_stride=1 << 20), Q.ERR_SHAPE),
    (dict(logits_dtype=Q.F16), Q.ERR_FORMAT), (dict(teacher_dtype=5), Q.ERR_FORMAT), (dict(index_bits=16), Q.ERR_FORMAT),
    (dict(temperature=0.0), Q.ERR_ARG), (dict(temperature=-1.0), Q.ERR_ARG), (dict(temperature=float("nan")), Q.ERR_ARG),
    (dict(temperature=float("inf")), Q.ERR_ARG), (dict(temperature=1e-45), Q.ERR_ARG),
    (dict(grad_scale=float("inf")), Q.ERR_ARG), (dict(logits=None), Q.ERR_ARG), (dict(index=None), Q.ERR_ARG),
    (dict(teacher=None), Q.ERR_ARG), (dict(lse=None), Q.ERR_ARG), (dict(logits_stride=999), Q.ERR_SHAPE),
    (dict(logits=A + 1), Q.ERR_ALIGN), (dict(index=A + 4), Q.ERR_ALIGN), (dict(teacher=A + 2), Q.ERR_ALIGN),
    (dict(lse=A + 2), Q.ERR_ALIGN), (dict(workspace=A + 4), Q.ERR_ALIGN)])
def test_distill_arguments(what, kw, status):
    assert _distill(what, **kw) == status


def test_distill_outputs_and_workspace():
    assert _distill(0, loss=None) == Q.ERR_ARG and _distill(0, grad=A) == Q.ERR_ARG
    assert _distill(1, loss=A) == Q.ERR_ARG and _distill(1, grad=None) == Q.ERR_ARG
    assert _distill(2, loss=None) == Q.ERR_ARG and _distill(2, grad=None) == Q.ERR_ARG
    assert _distill(0, grad_loss=A) == Q.ERR_ARG and _distill(2, grad_loss=A) == Q.ERR_ARG
    assert _distill(1, grad_loss=A) == Q.OK and _distill(1, workspace=None, workspace_bytes=0) == Q.OK
    assert _distill(2, grad=A, grad_stride=1000) == Q.OK                # in place
    assert _distill(2, grad=A, grad_stride=1008) == Q.ERR_ARG           # ... row by row, or not at all
    assert _distill(3) == Q.ERR_ARG and _distill(-1) == Q.ERR_ARG
    for rows, classes in ((1, 1000), (3, 131072), (4096, 131072), (1, 1 << 24)):
        need = O.quasar_distill_topk_workspace_bytes(rows, classes)
        if need:
            kw = dict(rows=rows, classes=classes, logits_stride=classes, grad_stride=classes)
            assert _distill(2, workspace_bytes=need, **kw) == Q.OK
            assert _distill(2, workspace_bytes=need - 1, **kw) == Q.ERR_WORKSPACE
            assert _distill(0, workspace=None, **kw) == Q.ERR_WORKSPACE
    assert O.quasar_distill_topk_workspace_bytes(0, 10) == 0 and O.quasar_distill_topk_workspace_bytes(1, 0) == 0


def _linear(d=None, **kw):
    d = d or Q.Descriptor(200, 256, fmt="int", bits=4, group=128)
    t = kw.get("tokens", 300)
    nv = d.desc.format == Q.NVFP4
    xd = kw.get("x_dtype", Q.BF16)
    p = dict(tokens=t, x=A, x_scale=A, codes=A, scales=A, zeros=A if d.desc.format == Q.INT else None,
             tensor_scale=A if nv else None, bias=A, residual=A, y=A, workspace=A,
             workspace_bytes=O.quasar_linear_codes_workspace_bytes(d, t, xd), x_stride=256, residual_stride=200,
             y_stride=200, x_dtype=xd, bias_dtype=Q.F32, residual_dtype=Q.BF16, y_dtype=Q.BF16, act=0)
    p.update(kw)
    return O.quasar_linear_codes_check(d, O.Linear(**p))


@pytest.mark.parametrize("kw,status", [
    (dict(), Q.OK), (dict(x_scale=None, bias=None, residual=None), Q.OK), (dict(x_dtype=O.E4M3), Q.OK),
    (dict(tokens=0, x=None, y=None), Q.OK), (dict(tokens=-1), Q.ERR_SHAPE), (dict(x=None), Q.ERR_ARG),
    (dict(y=None), Q.ERR_ARG), (dict(codes=None), Q.ERR_ARG), (dict(scales=None), Q.ERR_ARG),
    (dict(zeros=None), Q.ERR_ARG), (dict(tensor_scale=A), Q.ERR_ARG), (dict(act=4), Q.ERR_ARG), (dict(act=-1), Q.ERR_ARG),
    (dict(x_dtype=Q.F32), Q.ERR_FORMAT), (dict(y_dtype=O.E4M3), Q.ERR_FORMAT), (dict(bias_dtype=9), Q.ERR_FORMAT),
    (dict(residual_dtype=Q.F16), Q.ERR_FORMAT), (dict(bias=None, bias_dtype=9), Q.OK), (dict(x_stride=255), Q.ERR_SHAPE),
    (dict(y_stride=199), Q.ERR_SHAPE), (dict(x=A + 2), Q.OK), (dict(x=A + 1), Q.ERR_ALIGN), (dict(codes=A + 8), Q.ERR_ALIGN),
    (dict(x_scale=A + 2), Q.ERR_ALIGN), (dict(bias=A + 2), Q.ERR_ALIGN), (dict(y=A + 1), Q.ERR_ALIGN)])
def test_linear_arguments(kw, status):
    assert _linear(**kw) == status


def test_linear_formats_and_workspace():
    for fmt, bits, group in (("int", 2, 64), ("int_sym", 3, 128), ("nvfp4", 4, 16), ("rubin", 3, 512)):
        d = Q.Descriptor(200, 256, fmt=fmt, bits=bits, group=group)
        assert _linear(d) == Q.OK, fmt
        need = O.quasar_linear_codes_workspace_bytes(d, 300, Q.BF16)
        if need:
            assert _linear(d, workspace_bytes=need - 1) == Q.ERR_WORKSPACE
            assert _linear(d, workspace=None) == Q.ERR_WORKSPACE
    assert _linear(Q.Descriptor(200, 256, fmt="nvfp4"), tensor_scale=None) == Q.ERR_ARG
    assert _linear(Q.Descriptor(200, 200, fmt="int")) == Q.ERR_SHAPE      # not whole groups
    assert _linear(Q.Descriptor(200, 256, fmt="int", bits=5)) == Q.ERR_FORMAT
    assert O.quasar_linear_codes_workspace_bytes(Q.Descriptor(200, 200), 300, Q.BF16) == 0
    assert O.quasar_linear_codes_check(Q.Descriptor(8, 128), O.Linear(tokens=0, codes=A, scales=A, zeros=A, x_dtype=1,
                                                                      y_dtype=1)) == Q.OK


def test_wrappers_refuse_before_launch():
    """CPU tensors: the checks run first, so no device is touched."""
    x, w = torch.zeros(4, 64), torch.zeros(64)
    with pytest.raises(ValueError, match="2-D"):
        O.add_rms_norm(w, w)
    with pytest.raises(ValueError, match="weight"):
        O.add_rms_norm(x, w[:63])
    with pytest.raises(ValueError, match="residual"):
        O.add_rms_norm(x, w, x[:3])
    with pytest.raises(ValueError, match="unit stride"):
        O.add_rms_norm(torch.zeros(64, 4).t(), w)
    with pytest.raises(TypeError, match="dtype"):
        O.add_rms_norm(x.half(), w)
    with pytest.raises(TypeError, match="dtype"):
        O.add_rms_norm(x, w, y_dtype="fp16")
    with pytest.raises(ValueError, match="out"):
        O.add_rms_norm(x, w, out={"rstd": torch.zeros(4), "y": torch.zeros(4, 65)})
    with pytest.raises(ValueError, match="rstd"):
        O.add_rms_norm_backward(x, x, w, torch.zeros(3))
    with pytest.raises(ValueError, match="dh's type"):
        O.add_rms_norm_backward(x, x, w, torch.zeros(4), x, dx_dtype="bf16")
    ix, t = torch.zeros(4, 3, dtype=torch.int64), torch.zeros(4, 3)
    with pytest.raises(TypeError, match="index"):
        O.distill_topk(x, ix.short(), t)
    with pytest.raises(ValueError, match="teacher"):
        O.distill_topk(x, ix, t[:, :2])
    with pytest.raises(ValueError, match="index"):
        O.distill_topk(x, ix[:3], t)
    with pytest.raises(ValueError, match="row_weight"):
        O.distill_topk_grad(x, ix, t, row_weight=torch.zeros(4, dtype=torch.float64))
    with pytest.raises(ValueError, match="lse"):
        O.distill_topk_backward(x, ix, t, torch.zeros(5))
    c, s = torch.zeros(8 * 64, dtype=torch.uint8), torch.zeros(8)
    with pytest.raises(ValueError, match="zeros"):
        O.PackedWeight(8, 128, c, s, None, fmt="int", bits=4)
    with pytest.raises(ValueError, match="codes"):
        O.PackedWeight(8, 128, c[:-1], s, s, fmt="int", bits=4)
    with pytest.raises(ValueError, match="no int weight"):
        O.PackedWeight(8, 100, c, s, s, fmt="int", bits=4)
    pw = O.PackedWeight(8, 128, c, s, s, fmt="int", bits=4)
    xb = torch.zeros(4, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="x must"):
        O.linear_codes(xb[:, :64], pw)
    with pytest.raises(TypeError, match="x"):
        O.linear_codes(xb.float(), pw)
    with pytest.raises(ValueError, match="act"):
        O.linear_codes(xb, pw, act="tanh")
    with pytest.raises(ValueError, match="x_scale"):
        O.linear_codes(xb, pw, x_scale=torch.zeros(3))
    with pytest.raises(ValueError, match="bias"):
        O.linear_codes(xb, pw, bias=torch.zeros(9))
    with pytest.raises(ValueError, match="residual"):
        O.linear_codes(xb, pw, residual=torch.zeros(4, 9))


def test_backward_without_the_saved_log_sum_is_refused():
    x, ix, t = torch.zeros(4, 64), torch.zeros(4, 3, dtype=torch.int64), torch.zeros(4, 3)
    with pytest.raises(TypeError, match="lse"):
        O.distill_topk_backward(x, ix, t, None)


def test_tensors_off_the_gpu_are_refused_as_torch_does():
    x = torch.zeros(4, 64)
    with pytest.raises(Exception) as want:
        torch.cuda.current_stream(x.device)
    with pytest.raises(want.type) as got:
        O.add_rms_norm(x, torch.ones(64))
    assert str(got.value) == str(want.value)


def test_tensors_off_the_gpu_are_refused_with_a_stream_too():
    """Their pointers would go to a kernel.  No rows: where it is not refused nothing is launched either."""
    x, w, one = torch.zeros(0, 64), torch.ones(64), torch.zeros(0)
    i, t = torch.zeros(0, 3, dtype=torch.int64), torch.zeros(0, 3)
    c, s = torch.zeros(8 * 64, dtype=torch.uint8), torch.zeros(8)
    pw = O.PackedWeight(8, 128, c, s, s, fmt="int", bits=4)
    for call in (lambda: O.add_rms_norm(x, w, stream=1), lambda: O.add_rms_norm_backward(x, x, w, one, stream=1),
                 lambda: O.distill_topk(x, i, t, stream=1), lambda: O.distill_topk_grad(x, i, t, stream=1),
                 lambda: O.distill_topk_backward(x, i, t, one, stream=0),
                 lambda: O.linear_codes(torch.zeros(0, 128, dtype=torch.bfloat16), pw, stream=0)):
        with pytest.raises(ValueError, match="cpu"):
            call()


def test_linear_sizes_that_no_grid_takes():
    """HIP takes fewer than 2^32 threads in a grid: what has more is refused by the check, not by the launch."""
    def status(rows, cols, tokens, xd=Q.BF16):
        d = Q.Descriptor(rows, cols, fmt="int", bits=2, group=64)
        return _linear(d, tokens=tokens, x_dtype=xd, x_stride=cols, y_stride=rows, residual_stride=rows)

    # 16 outputs a workgroup of 512 threads, or 32 (17 to 32 tokens in bf16)
    assert status((1 << 27) - 16, 64, 1) == Q.OK and status((1 << 27) - 15, 64, 1) == Q.ERR_SHAPE
    assert status(1 << 27, 64, 32, O.E4M3) == Q.ERR_SHAPE and status(1 << 27, 64, 32) == Q.OK
    assert status((1 << 28) - 32, 64, 20) == Q.OK and status(1 << 28, 64, 20) == Q.ERR_SHAPE
    # 256 x 256 outputs a workgroup of 512 threads
    assert status(2048, 64, (1 << 28) - 256) == Q.OK and status(2049, 64, (1 << 28) - 256) == Q.ERR_SHAPE
    assert status(256, 128, 1 << 28, O.E4M3) == Q.OK  # many more activations than threads
    # every size that was accepted before, and that a card holds
    assert status(1 << 20, 1 << 14, 1000) == Q.OK and status(1 << 22, 4096, 8192) == Q.OK
