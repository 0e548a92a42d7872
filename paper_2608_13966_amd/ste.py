"""Training through the reconstruction: a linear layer whose forward pass uses
QUASAR's reconstruction r of latent weights W, with the straight-through
estimator (Sec. 3.2: the gradient is evaluated at r and applied to W), and
whose optimiser step is the fused AdamW + reconstruction of libquasar.so.

The forward/backward products are ordinary torch matmuls (the model around
the path); the optimiser update and the reconstruction run in the HIP kernels
behind ``quasar_adamw_reconstruct``.  A layer made with ``checkpoint=True`` keeps
its input for the backward pass in 8 bits, and its weight gradient is the
product from those (``ops.linear_weight_grad``).

``embed``, ``add_rms_norm``, ``add_layer_norm``, ``activation`` and
``distill_topk_loss`` are the autograd forms of the operators of ``ops`` that
training uses; their tensors may have any number of leading dimensions.  A backward
pass may be captured into a HIP graph; drop what still holds an eager graph of the
same parameters (a loss that was kept) first: torch accumulates gradients on the
stream that such a graph was made on, which a capture may not wait for.
"""
from __future__ import annotations

import math

import torch

from . import ops
from . import quasar as Q


class _STELinear(torch.autograd.Function):
    """y = x r^T; dL/dx = dL/dy r; dL/dW := dL/dr = dL/dy^T x (straight through)."""

    @staticmethod
    def forward(ctx, x, weight, r):
        ctx.save_for_backward(x, r)
        return x @ r.to(x.dtype).t()

    @staticmethod
    def backward(ctx, gy):
        x, r = ctx.saved_tensors
        gx = gy @ r.to(gy.dtype)
        gw = gy.reshape(-1, gy.shape[-1]).t() @ x.reshape(-1, x.shape[-1])
        return gx, gw.to(torch.float32), None


class _STELinearKept(torch.autograd.Function):
    """The same, x kept in 8 bits: dL/dr = dL/dy^T of what was kept, in fp32.  Of a frozen weight nothing is kept but r."""

    @staticmethod
    def forward(ctx, x, weight, r):
        kept = ()
        if ctx.needs_input_grad[1]:
            o = ops.checkpoint_rows(_rows(x))
            kept = o["q"], o["exponent"]
        ctx.save_for_backward(*kept, r)
        return x @ r.to(x.dtype).t()

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, gy):
        *kept, r = ctx.saved_tensors
        need_x, need_w = ctx.needs_input_grad[:2]
        gx = gy @ r.to(gy.dtype) if need_x else None
        gw = ops.linear_weight_grad(_rows(gy), *kept)["dw"] if need_w else None
        return gx, gw, None


class QuasarLinear(torch.nn.Module):
    """Linear layer (no bias) with fp32 latent weights trained by AdamW and
    quantised by QUASAR at every step.

    ``weight`` is the latent W (a Parameter, so autograd delivers its
    gradient); ``m`` and ``v`` are AdamW's moments; ``r`` (bf16) is the
    reconstruction the forward pass uses; ``codes``/``scales``/``zeros`` are
    the deployable form of r.  Call :meth:`step` after ``backward()``.
    ``checkpoint``: x is kept for the backward pass in 8 bits (x in fp32 or bf16).
    """

    checkpoint = False

    def __init__(self, in_features: int, out_features: int, *, fmt="int", bits=4, group=128,
                 clips=(1.0, 0.95, 0.9, 0.85, 0.8, 0.75, 0.7, 0.65), lr=1e-3, betas=(0.9, 0.999), eps=1e-8,
                 weight_decay=0.0, weighting="h", device="cuda", generator=None, checkpoint=False):
        super().__init__()
        if fmt == "nvfp4":
            raise ValueError("QuasarLinear supports the INT formats (NVFP4 needs the tensor amax state)")
        w = torch.empty(out_features, in_features, device=device, dtype=torch.float32)
        torch.nn.init.kaiming_uniform_(w, a=math.sqrt(5), generator=generator)
        self.weight = torch.nn.Parameter(w)
        self.register_buffer("m", torch.zeros_like(w))
        self.register_buffer("v", torch.zeros_like(w))
        self.cfg = dict(fmt=fmt, bits=bits, group=group, clips=tuple(clips), weighting=weighting)
        self.hp = dict(lr=lr, beta1=betas[0], beta2=betas[1], eps=eps, weight_decay=weight_decay)
        self.t = 0
        if checkpoint:
            self.checkpoint = True
        # initial reconstruction: no saliency yet (v = 0), so every group keeps
        # the min-max RTN dequantiser of the first clip (Standard QAT)
        out = Q.reconstruct(self.weight.data, self.v.clone(), None, want_diag=True, **self.cfg)
        self.register_buffer("r", out["r"].to(torch.bfloat16))
        self._out = None
        self.codes, self.scales, self.zeros = out["codes"], out["scales"], out["zeros"]

    def forward(self, x):
        # without gradients the plain form, which keeps nothing then
        kept = self.checkpoint and torch.is_grad_enabled()
        return (_STELinearKept if kept else _STELinear).apply(x, self.weight, self.r)

    @torch.no_grad()
    def step(self):
        """One fused AdamW step on the latent weights from their gradient,
        then the reconstruction of the result into ``r`` (in place)."""
        weight = self.weight
        g = weight.grad
        if g is None:
            raise RuntimeError("no gradient: call backward() first")
        # Module.__setattr__ looks through every registration (1.5 us a name): a
        # plain attribute is counted in place, and the results are assigned
        # only when they are not the objects already there
        own = self.__dict__
        if "t" in own:
            own["t"] += 1
        else:  # a buffer of a subclass
            self.t += 1
        W = weight.data
        out = self._out
        if out is None:
            d = Q.Descriptor(*W.shape, w_dtype=Q.F32, g_dtype=Q.F32, **self.cfg)
            out = Q.alloc_outputs(d, W, want_r=False, want_diag=True, has_amax=True)
            out["r"] = self.r
            self._out = out
        Q.adamw_reconstruct(W, self.m, self.v, g.contiguous(), step=self.t, out=out, r_dtype="bf16", **self.cfg,
                            **self.hp)
        if (own.get("codes", own) is not out["codes"] or own.get("scales", own) is not out["scales"]
                or own.get("zeros", own) is not out["zeros"]):
            self.codes, self.scales, self.zeros = out["codes"], out["scales"], out["zeros"]
        weight.grad = None

    def packed(self):
        """The layer's codes as ``ops.linear_codes`` takes them.  It holds the
        layer's own tensors: ask again after a step."""
        cfg = self.cfg
        return ops.PackedWeight(*self.weight.shape, self.codes, self.scales, self.zeros, fmt=cfg["fmt"],
                                bits=cfg["bits"], group=cfg["group"])


# ---- autograd forms ----------------------------------------------------------------

def _rows(t):
    """t as the operators take it: 2-D, rows that do not overlap, unit stride in the last dimension."""
    t = t.reshape(math.prod(t.shape[:-1]), t.shape[-1])
    return t if t.stride(1) == 1 and t.stride(0) >= t.shape[1] else t.contiguous()


class _AddRMSNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, residual, eps):
        ctx.set_materialize_grads(False)
        o = ops.add_rms_norm(_rows(x), weight, None if residual is None else _rows(residual), eps=eps)
        ctx.save_for_backward(o["h"], weight, o["rstd"])
        ctx.types = x.dtype, None if residual is None else residual.dtype
        y = o["y"].view(x.shape)
        return y if residual is None else (y, o["h"].view(x.shape))

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, dh=None):
        h, weight, rstd = ctx.saved_tensors
        x_type, r_type = ctx.types
        need_x, need_w, need_r = ctx.needs_input_grad[:3]
        if dy is None:  # only the stream went on
            return (dh.to(x_type) if need_x and dh is not None else None, None,
                    dh if need_r else None, None)
        # in the widest type that an input takes it in
        wide = torch.float32 in (need_x and x_type, need_r and r_type)
        dx_type = torch.float32 if wide else r_type or x_type
        o = ops.add_rms_norm_backward(_rows(dy), h, weight, rstd, None if dh is None else _rows(dh.to(dx_type)),
                                      dx_dtype=dx_type, want_dweight=need_w)
        dx = o["dx"].view(dy.shape)
        return (dx.to(x_type) if need_x else None, o["dw"].to(weight.dtype) if need_w else None,
                dx.to(r_type) if need_r else None, None)


def add_rms_norm(x, weight, residual=None, *, eps=1e-6):
    """``ops.add_rms_norm`` with gradients: y, or (y, h) with a residual, where
    h = x + residual is the stream that goes on; y has x's type, h residual's."""
    return _AddRMSNorm.apply(x, weight, residual, eps)


class _AddLayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, residual, eps):
        ctx.set_materialize_grads(False)
        o = ops.add_layer_norm(_rows(x), weight, bias, None if residual is None else _rows(residual), eps=eps)
        ctx.save_for_backward(o["h"], weight, o["mean"], o["rstd"])
        ctx.types = x.dtype, None if bias is None else bias.dtype, None if residual is None else residual.dtype
        y = o["y"].view(x.shape)
        return y if residual is None else (y, o["h"].view(x.shape))

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, dh=None):
        h, weight, mean, rstd = ctx.saved_tensors
        x_type, b_type, r_type = ctx.types
        need_x, need_w, need_b, need_r = ctx.needs_input_grad[:4]
        if dy is None:  # only the stream went on
            return (dh.to(x_type) if need_x and dh is not None else None, None, None, dh if need_r else None, None)
        # in the widest type that an input takes it in
        wide = torch.float32 in (need_x and x_type, need_r and r_type)
        dx_type = torch.float32 if wide else r_type or x_type
        o = ops.add_layer_norm_backward(_rows(dy), h, weight, mean, rstd, None if dh is None else _rows(dh.to(dx_type)),
                                        dx_dtype=dx_type, want_dweight=need_w, want_dbias=need_b)
        dx = o["dx"].view(dy.shape)
        return (dx.to(x_type) if need_x else None, o["dw"].to(weight.dtype) if need_w else None,
                o["db"].to(b_type) if need_b else None, dx.to(r_type) if need_r else None, None)


def add_layer_norm(x, weight, bias=None, residual=None, *, eps=1e-5):
    """``ops.add_layer_norm`` with gradients: y, or (y, h) with a residual, as ``add_rms_norm``."""
    return _AddLayerNorm.apply(x, weight, bias, residual, eps)


class _Embed(torch.autograd.Function):
    @staticmethod
    def forward(ctx, tokens, weight, scale):
        flat = tokens.reshape(-1).contiguous()
        ctx.save_for_backward(flat)
        ctx.table, ctx.scale = (weight.shape[0], weight.dtype), scale
        return ops.embed(flat, weight, scale=scale)["y"].view(*tokens.shape, weight.shape[1])

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        rows, dtype = ctx.table
        return None, ops.embed_backward(_rows(dy), ctx.saved_tensors[0], rows, scale=ctx.scale, dw_dtype=dtype)["dw"], None


def embed(tokens, weight, *, scale=1.0):
    """``ops.embed`` with the table's gradient, for tokens of any shape."""
    return _Embed.apply(tokens, weight, scale)


class _Activation(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, act):
        o = ops.checkpoint_rows(_rows(x), act=act, want_y=True)
        ctx.save_for_backward(o["q"], o["exponent"])
        ctx.act, ctx.dtype = act, x.dtype
        return o["y"].view(x.shape)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        q, exponent = ctx.saved_tensors
        return ops.checkpoint_backward(_rows(dy), q, exponent, act=ctx.act, dx_dtype=ctx.dtype)["dx"].view(dy.shape), None


def activation(x, act="gelu"):
    """act(x) ("relu", "silu" or "gelu"), x kept for the backward pass in 8 bits (``ops.checkpoint_rows``)."""
    if act not in ("relu", "silu", "gelu"):
        raise ValueError("activation: act must be one of relu, silu, gelu")
    return _Activation.apply(x, act)


class _DistillTopK(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, index, teacher, temperature, row_weight):
        flat, index, teacher = _rows(logits), _rows(index).contiguous(), _rows(teacher).contiguous()
        row_weight = None if row_weight is None else row_weight.reshape(-1).contiguous()
        o = ops.distill_topk(flat, index, teacher, temperature=temperature, row_weight=row_weight)
        ctx.save_for_backward(flat, index, teacher, o["lse"], row_weight)
        ctx.shape, ctx.temperature = logits.shape, temperature
        return o["loss"].view(logits.shape[:-1])

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_loss):
        flat, index, teacher, lse, row_weight = ctx.saved_tensors
        if not ctx.needs_input_grad[0]:
            return None, None, None, None, None
        o = ops.distill_topk_backward(flat, index, teacher, lse, temperature=ctx.temperature, row_weight=row_weight,
                                      grad_loss=grad_loss.reshape(-1).contiguous())
        return o["grad"].view(ctx.shape), None, None, None, None


def distill_topk_loss(logits, index, teacher, *, temperature=1.0, row_weight=None):
    """``ops.distill_topk`` with the gradient of the logits: the loss of each
    row, for any reduction.  Two passes over the logits; where the loss is a
    plain mean or sum, ``ops.distill_topk_grad`` makes loss and gradient in one
    (``logits.backward(grad)``)."""
    return _DistillTopK.apply(logits, index, teacher, temperature, row_weight)
