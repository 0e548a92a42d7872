"""C-ABI contract of the layer norm, the embedding and the activations kept in 8
bits (include/quasar_ops.h), checked without a GPU: structures, the statuses of
invalid arguments, workspace sizes and the refusals of the Python wrappers."""
import ctypes
import os
import re

import pytest
import torch

from paper_2608_13966_amd import ops as O
from paper_2608_13966_amd import quasar as Q
from paper_2608_13966_amd import ste

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 0x10000
E4M3 = torch.float8_e4m3fn


@pytest.mark.parametrize("cls,name", [
    (O.LayerNorm, "quasar_layer_norm"), (O.LayerNormBackward, "quasar_layer_norm_backward"),
    (O.Embedding, "quasar_embedding"), (O.EmbeddingBackward, "quasar_embedding_backward"),
    (O.Checkpoint, "quasar_checkpoint"), (O.CheckpointGrad, "quasar_checkpoint_grad"),
    (O.WeightGrad, "quasar_weight_grad")])
def test_structures_follow_the_header(cls, name):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "quasar_ops.h")).read(), flags=re.S)
    end = src.index("} %s;" % name)
    body = src[src.rindex("{", 0, end) + 1:end]
    size = {"int64_t": 8, "int32_t": 4, "float": 4, "size_t": 8}
    want = []
    for decl in filter(None, map(str.strip, body.split(";"))):
        typ, rest = re.match(r"(?:const )?(\w+)\s*(.*)", decl, flags=re.S).groups()
        for f in map(str.strip, rest.split(",")):
            want.append((f.lstrip("* "), 8 if f.startswith("*") or rest.startswith("*") else size[typ]))
    assert want == [(f, ctypes.sizeof(t)) for f, t in cls._fields_]


def _norm(**kw):
    p = dict(rows=4, cols=100, x=A, residual=A, weight=A, bias=A, h=A, y=A, q=A, scale=A, mean=A, rstd=A, x_stride=100,
             residual_stride=100, h_stride=100, y_stride=100, q_stride=100, x_dtype=Q.BF16, residual_dtype=Q.BF16,
             weight_dtype=Q.F32, bias_dtype=Q.F32, y_dtype=Q.BF16, eps=1e-5)
    p.update(kw)
    return O.quasar_add_layer_norm_check(O.LayerNorm(**p))


@pytest.mark.parametrize("kw,status", [
    (dict(), Q.OK), (dict(rows=0, x=None, weight=None), Q.OK), (dict(rows=-1), Q.ERR_SHAPE), (dict(cols=0), Q.ERR_SHAPE),
    (dict(cols=O.NORM_MAX_COLS + 1), Q.ERR_SHAPE), (dict(rows=1 << 31), Q.ERR_SHAPE), (dict(x=None), Q.ERR_ARG),
    (dict(weight=None), Q.ERR_ARG), (dict(bias=None, bias_dtype=9), Q.OK), (dict(bias_dtype=9), Q.ERR_FORMAT),
    (dict(bias=A + 2), Q.ERR_ALIGN), (dict(bias=A + 2, bias_dtype=Q.BF16), Q.OK), (dict(q=None), Q.ERR_ARG),
    (dict(scale=None), Q.ERR_ARG), (dict(q=None, scale=None, y=None, h=None, mean=None, rstd=None), Q.OK),
    (dict(residual=None), Q.ERR_ARG), (dict(residual=None, h=None), Q.OK), (dict(eps=-1.0), Q.ERR_ARG),
    (dict(eps=float("nan")), Q.ERR_ARG), (dict(eps=0.0), Q.OK), (dict(x_dtype=Q.F16), Q.ERR_FORMAT),
    (dict(weight_dtype=O.E4M3), Q.ERR_FORMAT), (dict(y_dtype=-1), Q.ERR_FORMAT), (dict(x_stride=99), Q.ERR_SHAPE),
    (dict(rows=1, x_stride=0, h_stride=3), Q.OK), (dict(y_stride=1 << 41), Q.ERR_SHAPE), (dict(x=A + 2), Q.OK),
    (dict(x=A + 1), Q.ERR_ALIGN), (dict(mean=A + 2), Q.ERR_ALIGN), (dict(rstd=A + 1), Q.ERR_ALIGN)])
def test_layer_norm_arguments(kw, status):
    assert _norm(**kw) == status


def _norm_backward(**kw):
    rows, cols = kw.get("rows", 64), kw.get("cols", 4096)
    p = dict(rows=rows, cols=cols, dy=A, h=A, weight=A, mean=A, rstd=A, dh=A, dx=A, dweight=A, dbias=A, workspace=A,
             workspace_bytes=O.quasar_add_layer_norm_backward_workspace_bytes(rows, cols), dy_stride=4096, h_stride=4096,
             dh_stride=4096, dx_stride=4096, dy_dtype=Q.BF16, h_dtype=Q.F32, weight_dtype=Q.F32, dx_dtype=Q.F32)
    p.update(kw)
    return O.quasar_add_layer_norm_backward_check(O.LayerNormBackward(**p))


@pytest.mark.parametrize("kw,status", [
    (dict(), Q.OK), (dict(dh=None), Q.OK), (dict(dweight=None), Q.OK), (dict(dbias=None), Q.OK),
    (dict(dweight=None, dbias=None, workspace=None, workspace_bytes=0), Q.OK), (dict(workspace=None), Q.ERR_WORKSPACE),
    (dict(dbias=None, workspace_bytes=15), Q.ERR_WORKSPACE), (dict(rows=1, workspace=None, workspace_bytes=0), Q.OK),
    (dict(rows=0, dy=None, dx=None), Q.OK), (dict(dy=None), Q.ERR_ARG), (dict(mean=None), Q.ERR_ARG),
    (dict(rstd=None), Q.ERR_ARG), (dict(dx=None), Q.ERR_ARG), (dict(dx_dtype=Q.F16), Q.ERR_FORMAT),
    (dict(dh_stride=4095), Q.ERR_SHAPE), (dict(cols=40000), Q.ERR_SHAPE), (dict(dh=A + 2), Q.ERR_ALIGN),
    (dict(dbias=A + 2), Q.ERR_ALIGN), (dict(dy=A + 2), Q.OK), (dict(workspace=A + 8), Q.ERR_ALIGN)])
def test_layer_norm_backward_arguments(kw, status):
    assert _norm_backward(**kw) == status


def _embed(**kw):
    p = dict(rows=1000, cols=64, tokens=10, index=A, weight=A, y=A, weight_stride=64, y_stride=64, index_bits=64,
             weight_dtype=Q.BF16, y_dtype=Q.F32, scale=8.0)
    p.update(kw)
    return O.quasar_embed_check(O.Embedding(**p))


@pytest.mark.parametrize("kw,status", [
    (dict(), Q.OK), (dict(tokens=0, index=None, weight=None, y=None), Q.OK), (dict(rows=0), Q.ERR_SHAPE),
    (dict(cols=0), Q.ERR_SHAPE), (dict(cols=(1 << 20) + 1), Q.ERR_SHAPE), (dict(rows=1 << 31), Q.ERR_SHAPE),
    (dict(tokens=-1), Q.ERR_SHAPE), (dict(tokens=(1 << 28) + 1), Q.ERR_SHAPE), (dict(index_bits=16), Q.ERR_FORMAT),
    (dict(weight_dtype=Q.F16), Q.ERR_FORMAT), (dict(y_dtype=O.E4M3), Q.ERR_FORMAT), (dict(scale=float("inf")), Q.ERR_ARG),
    (dict(scale=float("nan")), Q.ERR_ARG), (dict(scale=-0.5), Q.OK), (dict(index=None), Q.ERR_ARG),
    (dict(weight=None), Q.ERR_ARG), (dict(y=None), Q.ERR_ARG), (dict(weight_stride=63), Q.ERR_SHAPE),
    (dict(y_stride=63), Q.ERR_SHAPE), (dict(index=A + 4), Q.ERR_ALIGN), (dict(index=A + 4, index_bits=32), Q.OK),
    (dict(weight=A + 2), Q.OK), (dict(y=A + 2), Q.ERR_ALIGN)])
def test_embed_arguments(kw, status):
    assert _embed(**kw) == status


def _embed_backward(**kw):
    rows, cols, tokens = kw.get("rows", 1000), kw.get("cols", 64), kw.get("tokens", 10)
    p = dict(rows=rows, cols=cols, tokens=tokens, index=A, dy=A, dweight=A, workspace=A,
             workspace_bytes=O.quasar_embed_backward_workspace_bytes(rows, cols, tokens), dy_stride=64, dweight_stride=64,
             index_bits=32, dy_dtype=Q.BF16, dweight_dtype=Q.F32, scale=1.0)
    p.update(kw)
    return O.quasar_embed_backward_check(O.EmbeddingBackward(**p))


@pytest.mark.parametrize("kw,status", [
    (dict(), Q.OK), (dict(tokens=0, index=None, dy=None), Q.OK), (dict(tokens=0, workspace=None), Q.ERR_WORKSPACE),
    (dict(workspace=None), Q.ERR_WORKSPACE), (dict(workspace_bytes=15), Q.ERR_WORKSPACE), (dict(rows=0), Q.ERR_SHAPE),
    (dict(cols=1 << 21), Q.ERR_SHAPE), (dict(tokens=-1), Q.ERR_SHAPE), (dict(index=None), Q.ERR_ARG),
    (dict(dy=None), Q.ERR_ARG), (dict(dweight=None), Q.ERR_ARG), (dict(index_bits=8), Q.ERR_FORMAT),
    (dict(dy_dtype=Q.F16), Q.ERR_FORMAT), (dict(dweight_dtype=O.E4M3), Q.ERR_FORMAT), (dict(scale=float("nan")), Q.ERR_ARG),
    (dict(dy_stride=63), Q.ERR_SHAPE), (dict(dweight_stride=63), Q.ERR_SHAPE), (dict(index=A + 2), Q.ERR_ALIGN),
    (dict(dy=A + 2), Q.OK), (dict(dweight=A + 2), Q.ERR_ALIGN), (dict(workspace=A + 8), Q.ERR_ALIGN)])
def test_embed_backward_arguments(kw, status):
    assert _embed_backward(**kw) == status


def test_embed_backward_workspace():
    for rows, cols, tokens in ((1, 1, 0), (1, 1, 1), (131072, 4096, 32768), (2 ** 31 - 1, 1, 5), (10, 1 << 20, 3)):
        need = O.quasar_embed_backward_workspace_bytes(rows, cols, tokens)
        kw = dict(rows=rows, cols=cols, tokens=tokens, dy_stride=cols, dweight_stride=cols)
        assert need > 0 and _embed_backward(**kw) == Q.OK
        assert _embed_backward(workspace_bytes=need - 1, **kw) == Q.ERR_WORKSPACE
    # parts for every stretch of the sorted tokens, not for every token
    assert O.quasar_embed_backward_workspace_bytes(131072, 4096, 32768) < 32768 * 4096 * 2
    # more workgroups than a grid takes
    kw = dict(rows=5, cols=1 << 20, tokens=1 << 28, dy_stride=1 << 20, dweight_stride=1 << 20)
    assert _embed_backward(**kw) == Q.ERR_SHAPE and O.quasar_embed_backward_workspace_bytes(5, 1 << 20, 1 << 28) == 0


def test_embed_backward_takes_the_tokens_that_memory_holds():
    """Up to 2^28 tokens, where dy in bf16 is at most 288 GB."""
    for cols, tokens in ((1, 1 << 28), (8, 1 << 28), (257, 1 << 28), (512, 1 << 28), (513, 1 << 28), (520, 270000000), (1025, 1 << 27),
                         (4096, 35000000), (4097, 35000000), (1 << 20, 137000)):
        tokens = min(tokens, 1 << 28)
        kw = dict(rows=1000, cols=cols, tokens=tokens, dy_stride=cols, dweight_stride=cols)
        assert _embed_backward(**kw) == Q.OK, (cols, tokens)
        assert O.quasar_embed_backward_workspace_bytes(1000, cols, tokens) > 16 * tokens
    for cols, tokens, status in ((1024, 1 << 28, Q.OK), (1025, 1 << 28, Q.ERR_SHAPE), (1 << 20, 32 * 8193, Q.ERR_SHAPE)):
        kw = dict(rows=1000, cols=cols, tokens=tokens, dy_stride=cols, dweight_stride=cols)
        assert _embed_backward(**kw) == status, (cols, tokens)


def _checkpoint(**kw):
    p = dict(rows=4, cols=300, x=A, y=A, q=A, exponent=A, x_stride=300, y_stride=300, q_stride=300, exponent_stride=3,
             x_dtype=Q.BF16, y_dtype=Q.BF16, act=3)
    p.update(kw)
    return O.quasar_checkpoint_rows_check(O.Checkpoint(**p))


@pytest.mark.parametrize("kw,status", [
    (dict(), Q.OK), (dict(y=None, y_dtype=9), Q.OK), (dict(act=0), Q.OK), (dict(act=4), Q.ERR_ARG), (dict(act=-1), Q.ERR_ARG),
    (dict(rows=0, x=None, q=None, exponent=None), Q.OK), (dict(rows=-1), Q.ERR_SHAPE), (dict(cols=0), Q.ERR_SHAPE),
    (dict(cols=(1 << 24) + 1), Q.ERR_SHAPE), (dict(x=None), Q.ERR_ARG), (dict(q=None), Q.ERR_ARG),
    (dict(exponent=None), Q.ERR_ARG), (dict(x_dtype=O.E4M3), Q.ERR_FORMAT), (dict(y_dtype=Q.F16), Q.ERR_FORMAT),
    (dict(x_stride=299), Q.ERR_SHAPE), (dict(q_stride=299), Q.ERR_SHAPE), (dict(exponent_stride=2), Q.ERR_SHAPE),
    (dict(rows=1, exponent_stride=0), Q.OK), (dict(x=A + 1), Q.ERR_ALIGN), (dict(q=A + 1, exponent=A + 3), Q.OK)])
def test_checkpoint_arguments(kw, status):
    assert _checkpoint(**kw) == status


def _checkpoint_backward(**kw):
    p = dict(rows=4, cols=300, dy=A, q=A, exponent=A, dx=A, dy_stride=300, q_stride=300, exponent_stride=3, dx_stride=300,
             dy_dtype=Q.BF16, dx_dtype=Q.F32, act=1)
    p.update(kw)
    return O.quasar_checkpoint_backward_check(O.CheckpointGrad(**p))


@pytest.mark.parametrize("kw,status", [
    (dict(), Q.OK), (dict(act=0), Q.ERR_ARG), (dict(act=4), Q.ERR_ARG), (dict(rows=0, dy=None, dx=None), Q.OK),
    (dict(dy=None), Q.ERR_ARG), (dict(q=None), Q.ERR_ARG), (dict(exponent=None), Q.ERR_ARG), (dict(dx=None), Q.ERR_ARG),
    (dict(dy_dtype=Q.F16), Q.ERR_FORMAT), (dict(dx_dtype=O.E4M3), Q.ERR_FORMAT), (dict(dx_stride=299), Q.ERR_SHAPE),
    (dict(exponent_stride=2), Q.ERR_SHAPE), (dict(dx=A + 2), Q.ERR_ALIGN), (dict(cols=0), Q.ERR_SHAPE)])
def test_checkpoint_backward_arguments(kw, status):
    assert _checkpoint_backward(**kw) == status


def _weight_args(**kw):
    t, n, k = kw.get("tokens", 777), kw.get("rows", 200), kw.get("cols", 300)
    p = dict(tokens=t, rows=n, cols=k, dy=A, q=A, exponent=A, dweight=A, workspace=A, dy_stride=n, q_stride=k,
             exponent_stride=(k + 127) // 128, dweight_stride=k, dy_dtype=Q.BF16, dweight_dtype=Q.F32)
    p.update(kw)
    a = O.WeightGrad(**p)
    if "workspace_bytes" not in kw:
        a.workspace_bytes = O.quasar_linear_weight_grad_workspace_bytes(a)
    return a


def _weight(**kw):
    return O.quasar_linear_weight_grad_check(_weight_args(**kw))


@pytest.mark.parametrize("kw,status", [
    (dict(), Q.OK), (dict(tokens=0, dy=None, q=None, exponent=None), Q.OK), (dict(tokens=-1), Q.ERR_SHAPE),
    (dict(rows=0), Q.ERR_SHAPE), (dict(cols=0), Q.ERR_SHAPE), (dict(rows=(1 << 22) + 1), Q.ERR_SHAPE),
    (dict(cols=(1 << 22) + 1), Q.ERR_SHAPE), (dict(tokens=(1 << 28) + 1), Q.ERR_SHAPE), (dict(dy=None), Q.ERR_ARG),
    (dict(q=None), Q.ERR_ARG), (dict(exponent=None), Q.ERR_ARG), (dict(dweight=None), Q.ERR_ARG),
    (dict(dy_dtype=Q.F16), Q.ERR_FORMAT), (dict(dweight_dtype=O.E4M3), Q.ERR_FORMAT), (dict(dy_stride=199), Q.ERR_SHAPE),
    (dict(q_stride=299), Q.ERR_SHAPE), (dict(exponent_stride=2), Q.ERR_SHAPE), (dict(dweight_stride=299), Q.ERR_SHAPE),
    (dict(dy=A + 1), Q.ERR_ALIGN), (dict(dy=A + 2, q=A + 1, exponent=A + 1), Q.OK), (dict(dweight=A + 2), Q.ERR_ALIGN),
    (dict(workspace=A + 8), Q.ERR_ALIGN)])
def test_weight_grad_arguments(kw, status):
    assert _weight(**kw) == status


@pytest.mark.parametrize("dt", [Q.BF16, Q.F32])
def test_weight_grad_workspace(dt):
    some = 0
    for t, n, k in ((1, 1, 1), (64, 64, 64), (5000, 200, 300), (8192, 14336, 4096), (16384, 256, 256), (2000, 4000, 4100)):
        kw = dict(tokens=t, rows=n, cols=k, dy_dtype=dt)
        need = _weight_args(**kw).workspace_bytes
        assert _weight(**kw) == Q.OK
        if need:
            some += 1
            assert _weight(workspace_bytes=need - 1, **kw) == Q.ERR_WORKSPACE
            assert _weight(workspace=None, **kw) == Q.ERR_WORKSPACE
    assert some > 0
    assert _weight_args(tokens=-1).workspace_bytes == 0 and _weight_args(dy_dtype=O.E4M3).workspace_bytes == 0


@pytest.mark.parametrize("dt", [Q.BF16, Q.F32])
@pytest.mark.parametrize("wt", [Q.BF16, Q.F32])
def test_weight_grad_takes_what_memory_holds(dt, wt):
    """Every call whose tensors the card's 288 GB hold, sizes up to the largest; the workspace is x in bf16 and dy's three
    parts at most, and the shares' sums."""
    most = 1 << 22
    for t in (1, 64, 129, 200, 10 ** 4, 10 ** 6, 10 ** 7, 10 ** 8, 1 << 28):
        for n in (1, 7, 64, 1000, 4096, 10 ** 5, most - 1, most):
            for k in (1, 7, 64, 1000, 16384, 10 ** 5, most - 1, most):
                dy, x, dw = t * n * (2 if dt == Q.BF16 else 4), t * k + t * -(-k // 128), n * k * (2 if wt == Q.BF16 else 4)
                if dy + x + dw > 288e9:
                    continue
                a = _weight_args(tokens=t, rows=n, cols=k, dy_dtype=dt, dweight_dtype=wt)
                assert O.quasar_linear_weight_grad_check(a) == Q.OK, (t, n, k)
                rows = -(-t // 64) * 64
                assert a.workspace_bytes <= rows * (2 * (k + 7) + 6 * (n + 7)) + 33 * max(256 * 256 * 4 * 256, n * (k + 7) * 4), (t, n, k)


def test_weight_grad_copies_dy_only_where_it_has_to():
    kw = dict(tokens=8192, rows=14336, cols=4096)
    plain, whole = _weight_args(**kw).workspace_bytes, 8192 * 14336 * 2
    assert plain < whole
    for more in (dict(dy=A + 2), dict(dy_stride=14337), dict(dy_dtype=Q.F32)):
        need = _weight_args(**kw, **more).workspace_bytes
        assert need >= plain + whole
        assert _weight(**kw, **more) == Q.OK and _weight(**kw, **more, workspace_bytes=plain) == Q.ERR_WORKSPACE


def test_wrappers_refuse_before_launch():
    """CPU tensors: the checks run first, so no device is touched."""
    x, w, one = torch.zeros(4, 64), torch.zeros(64), torch.zeros(4)
    q, e, tok = x.to(E4M3), torch.zeros(4, 1, dtype=torch.uint8), torch.zeros(4, dtype=torch.int64)
    V, T = ValueError, TypeError
    for call, kind, text in (
            (lambda: O.add_layer_norm(w, w), V, "2-D"), (lambda: O.add_layer_norm(x, w[:63]), V, "weight"),
            (lambda: O.add_layer_norm(x, w, w[:3]), V, "bias"), (lambda: O.add_layer_norm(x, w, w, x[:3]), V, "residual"),
            (lambda: O.add_layer_norm(torch.zeros(64, 4).t(), w), V, "unit stride"),
            (lambda: O.add_layer_norm(x.half(), w), T, "dtype"), (lambda: O.add_layer_norm(x, w, w.half()), T, "dtype"),
            (lambda: O.add_layer_norm(x, w, y_dtype="fp16"), T, "dtype"),
            (lambda: O.add_layer_norm(x, w, out={"mean": one, "rstd": one, "y": torch.zeros(4, 65)}), V, "out"),
            (lambda: O.add_layer_norm_backward(x, x, w, one[:3], one), V, "mean"),
            (lambda: O.add_layer_norm_backward(x, x, w, one, one[:3]), V, "rstd"),
            (lambda: O.add_layer_norm_backward(x, x, w, one, one, x, dx_dtype="bf16"), V, "dh's type"),
            (lambda: O.embed(tok.short(), x), T, "tokens"), (lambda: O.embed(tok[None], x), V, "1-D"),
            (lambda: O.embed(torch.zeros(8, dtype=torch.int64)[::2], x), V, "contiguous"),
            (lambda: O.embed(tok, w), V, "2-D"), (lambda: O.embed(tok, x.half()), T, "dtype"),
            (lambda: O.embed(tok, x, out={"y": torch.zeros(4, 63)}), V, "out"),
            (lambda: O.embed_backward(x, tok[:3], 10), V, "dy"), (lambda: O.embed_backward(x, tok, 0), V, "rows"),
            (lambda: O.embed_backward(x, tok, -5), V, "rows"), (lambda: O.embed_backward(x, tok, 10, dw_dtype="fp16"), T, "dtype"),
            (lambda: O.checkpoint_rows(w), V, "2-D"), (lambda: O.checkpoint_rows(x.half()), T, "dtype"),
            (lambda: O.checkpoint_rows(x, act="tanh"), V, "act"),
            (lambda: O.checkpoint_rows(x, out={"q": q, "exponent": e[:, :0]}), V, "exponent"),
            (lambda: O.checkpoint_backward(x, q, e, act="none"), V, "act"),
            (lambda: O.checkpoint_backward(x, x, e, act="gelu"), T, "q"),
            (lambda: O.checkpoint_backward(x, q, e.int(), act="gelu"), T, "exponent"),
            (lambda: O.checkpoint_backward(x, q[:, :5], e, act="gelu"), V, "q"),
            (lambda: O.linear_weight_grad(x, q[:3], e), V, "q"), (lambda: O.linear_weight_grad(x, q, e[:3]), V, "exponent"),
            (lambda: O.linear_weight_grad(x.half(), q, e), T, "dtype"), (lambda: O.linear_weight_grad(w, q, e), V, "2-D"),
            (lambda: O.linear_weight_grad(x, q, e, out={"dw": torch.zeros(64, 63)}), V, "out"),
            (lambda: ste.activation(x, "none"), V, "act")):
        with pytest.raises(kind, match=text):
            call()


@pytest.mark.parametrize("stream", [None, 0, 1])
def test_tensors_off_the_gpu_are_refused(stream):
    """No rows: where it is not refused nothing is launched either."""
    x, w, one = torch.zeros(0, 64), torch.ones(64), torch.zeros(0)
    q, e, tok = x.to(E4M3), torch.zeros(0, 1, dtype=torch.uint8), torch.zeros(0, dtype=torch.int32)
    kw = {} if stream is None else {"stream": stream}
    for call in (lambda: O.add_layer_norm(x, w, **kw), lambda: O.add_layer_norm_backward(x, x, w, one, one, **kw),
                 lambda: O.embed(tok, torch.zeros(5, 64), **kw), lambda: O.embed_backward(x, tok, 5, **kw),
                 lambda: O.checkpoint_rows(x, **kw), lambda: O.checkpoint_backward(x, q, e, act="silu", **kw),
                 lambda: O.linear_weight_grad(x, q, e, **kw)):
        with pytest.raises(Exception, match="cpu|CUDA|HIP|NVIDIA|device"):
            call()
