"""A small network trained by distillation and served from its codes:

    python -m paper_2608_13966_amd.example

Residual blocks of norm -> linear -> GELU -> linear and a head, all linears
``ste.QuasarLinear``.  Training: the residual's addition and the norm in one
pass (``ste.add_rms_norm``), loss and gradient against the teacher's top logits
in one pass (``ops.distill_topk_grad``), the products through the
reconstruction, one fused AdamW + reconstruction a layer.  Serving: the norm
writes 8-bit rows with their scales, which ``ops.linear_codes`` multiplies by
the packed codes; nothing of the latent weights is read.  The teacher is a
seeded random network of the same shape, the tokens are random.
"""
from __future__ import annotations

import torch

from . import ops, ste


class Student(torch.nn.Module):
    def __init__(self, vocab=2048, width=256, hidden=512, blocks=2, bits=4, group=64, lr=1e-3, device="cuda",
                 seed=0):
        super().__init__()
        gen = torch.Generator(device=device).manual_seed(seed)
        make = dict(bits=bits, group=group, lr=lr, device=device, generator=gen)
        self.embed = torch.nn.Parameter(
            torch.randn(vocab, width, device=device, generator=gen).to(torch.bfloat16))
        self.norms = torch.nn.ParameterList(torch.ones(width, device=device) for _ in range(blocks + 1))
        self.up = torch.nn.ModuleList(ste.QuasarLinear(width, hidden, **make) for _ in range(blocks))
        self.down = torch.nn.ModuleList(ste.QuasarLinear(hidden, width, **make) for _ in range(blocks))
        self.head = ste.QuasarLinear(width, vocab, **make)

    def linears(self):
        return [*self.up, *self.down, self.head]

    def forward(self, tokens):
        stream, branch = self.embed[tokens], None
        for norm, up, down in zip(self.norms, self.up, self.down):
            if branch is None:
                y = ste.add_rms_norm(stream, norm)
            else:
                y, stream = ste.add_rms_norm(branch, norm, stream)
            branch = down(torch.nn.functional.gelu(up(y)))
        y, _ = ste.add_rms_norm(branch, self.norms[-1], stream)
        return self.head(y)


class Trainer:
    """One step: forward, loss and gradient of the logits in one pass, backward,
    the linears' fused AdamW + reconstruction, torch's AdamW for the rest."""

    def __init__(self, student, temperature=1.0, lr=1e-3):
        self.student, self.temperature = student, temperature
        self.rest = torch.optim.AdamW([student.embed, *student.norms], lr=lr)

    def step(self, tokens, index, teacher, row_weight=None):
        logits = self.student(tokens)
        o = ops.distill_topk_grad(logits.detach(), index, teacher, temperature=self.temperature,
                                  row_weight=row_weight, grad_scale=1.0 / logits.shape[0])
        logits.backward(o["grad"])
        for layer in self.student.linears():
            layer.step()
        self.rest.step()
        self.rest.zero_grad(set_to_none=True)
        return o["loss"].mean()


class Server:
    """The student from its packed codes, norms and embedding.  ``eight`` sends
    the norms' rows to the products in 8 bits with a scale each."""

    def __init__(self, student, eight=True):
        self.embed = student.embed.detach()
        self.norms = [w.detach() for w in student.norms]
        self.up, self.down = ([layer.packed() for layer in part] for part in (student.up, student.down))
        self.head, self.eight = student.head.packed(), eight

    def _linear(self, n, weight, **kw):
        if self.eight:
            return ops.linear_codes(n["q"], weight, x_scale=n["scale"], **kw)["y"]
        return ops.linear_codes(n["y"], weight, **kw)["y"]

    def _norm(self, x, weight, residual=None):
        return ops.add_rms_norm(x, weight, residual, want_y=not self.eight, quantize=self.eight)

    def __call__(self, tokens):
        x, stream = self.embed[tokens], None
        for norm, up, down in zip(self.norms, self.up, self.down):
            n = self._norm(x, norm, stream)
            stream = n["h"]
            x = ops.linear_codes(self._linear(n, up, act="gelu"), down)["y"]
        return self._linear(self._norm(x, self.norms[-1], stream), self.head, y_dtype="fp32")


def top_logits(tokens, vocab, listed, seed=1, width=64, device="cuda"):
    """The teacher's ``listed`` largest logits of each token and their classes:
    a seeded random map of low rank."""
    gen = torch.Generator(device=device).manual_seed(seed)
    a = torch.randn(vocab, width, device=device, generator=gen)
    b = torch.randn(width, vocab, device=device, generator=gen) / width ** 0.5
    values, index = torch.topk(3.0 * (a[tokens] @ b), listed, dim=1)
    return index, values


def run(steps=40, tokens=512, vocab=2048, listed=32, device="cuda", log=print, **student):
    """Trains and returns the student, the losses, and the tokens."""
    s = Student(vocab=vocab, device=device, **student)
    trainer = Trainer(s)
    gen = torch.Generator(device=device).manual_seed(2)
    t = torch.randint(0, vocab, (tokens,), device=device, generator=gen)
    index, teacher = top_logits(t, vocab, listed, device=device)
    losses = []
    for i in range(steps):
        losses.append(trainer.step(t, index, teacher))
        if log and (i + 1) % 10 == 0:
            log(f"step {i + 1}: loss {float(losses[-1]):.4f}")
    return s, torch.stack(losses), t


def main():
    s, _, t = run()
    with torch.no_grad():
        want = s(t).float()
        for eight in (False, True):
            got = Server(s, eight)(t)
            one = Server(s, eight)(t[:1])
            print(f"served from codes, {8 if eight else 16}-bit rows: logits differ by "
                  f"{float((got - want).norm() / want.norm()):.2e}, the same first class for "
                  f"{float((got.argmax(1) == want.argmax(1)).float().mean()):.1%} of {len(t)} tokens; "
                  f"one token alone by {float((one[0] - got[0]).norm() / got[0].norm()):.2e}")


if __name__ == "__main__":
    main()
