"""A small language model distilled from stored teacher logits, with the model operators
and the whole optimizer together.

One transformer layer with a tied token embedding: scaled embedding lookup, queries and
keys normalised per head and rotated, causal attention, a feed-forward pair, and the
table again as output head.  The teacher is a fixed table of next-token logits (its
largest entries for each token, as they would be stored on disk), positions before
`prompt` do not count, and a step is

  lookup -> layer (torch products, qk_norm) -> logits -> loss and gradient in one pass
  -> gradients back to the lookup, the table's added to the head's -> MALT on the
  matrices and AdamW on the table and the gains.

torch forms the matrix products and the attention; lookup, norms, loss and the three
gradients are the library's kernels, like the optimizer's step.
"""
from __future__ import annotations

import dataclasses
import math

import torch

from . import malt, model_ops


@dataclasses.dataclass(frozen=True)
class Config:
    vocab: int = 512
    dim: int = 128
    heads: int = 4
    batch: int = 8
    seq: int = 64
    top: int = 16               # teacher logits kept per token
    prompt: int = 4             # positions of a sequence that do not count
    temperature: float = 2.0
    dtype: torch.dtype = torch.bfloat16     # of activations and of the weights' copies


class _QKNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_gain, k_gain, cos, sin):
        ctx.save_for_backward(q, k, q_gain, k_gain, cos, sin)
        return model_ops.qk_norm(q, k, q_gain, k_gain, cos, sin)

    @staticmethod
    def backward(ctx, dq_out, dk_out):
        grads = model_ops.qk_norm_grad(dq_out.contiguous(), dk_out.contiguous(), *ctx.saved_tensors)
        return (*grads, None, None)


class Teacher:
    """Next-token logits of a bigram model: for each token its `top` largest entries."""

    def __init__(self, cfg: Config, seed: int = 0):
        g = torch.Generator().manual_seed(seed)
        full = torch.randn(cfg.vocab, cfg.vocab, generator=g) * 3.0
        logits, ids = full.topk(cfg.top, dim=1)
        self.ids, self.logits = ids.to(torch.int32).cuda(), logits.cuda()

    def entries(self, tokens):
        """(ids, logits) of the rows of `tokens`, [tokens, top] each."""
        flat = tokens.reshape(-1)
        return self.ids[flat], self.logits[flat]


class Model:
    """fp32 master weights with their copies, gradients and optimizer."""

    def __init__(self, cfg: Config, seed: int = 1):
        self.cfg = cfg
        g = torch.Generator().manual_seed(seed)
        d, hd = cfg.dim, cfg.dim // cfg.heads

        def normal(rows, cols):
            return (torch.randn(rows, cols, generator=g) * (0.5 / math.sqrt(cols))).cuda()

        self.matrices = {"qkv": normal(3 * d, d), "out": normal(d, d), "up": normal(4 * d, d), "down": normal(d, 4 * d)}
        self.others = {"table": (torch.randn(cfg.vocab, d, generator=g) * 0.05).cuda(),
                       "q_gain": torch.ones(hd).cuda(), "k_gain": torch.ones(hd).cuda()}
        self.grads = {n: torch.zeros_like(w) for n, w in (self.matrices | self.others).items()}
        bf16 = cfg.dtype == torch.bfloat16
        copied = self.matrices | {"table": self.others["table"]}
        self.copies = {n: w.to(cfg.dtype) if bf16 else w for n, w in copied.items()}
        vec = lambda n: torch.empty(n, device="cuda")
        mats = [(w, self.grads[n], torch.empty_like(w), vec(w.shape[0]), vec(w.shape[1]))
                for n, w in self.matrices.items()]
        rest = [(w, self.copies[n] if bf16 and n == "table" else None, self.grads[n], torch.empty_like(w),
                 torch.empty_like(w), 0.1 if n == "table" else 0.0) for n, w in self.others.items()]
        mat_copies = [self.copies[n] for n in self.matrices] if bf16 else None
        self.optimizer = malt.WholeOptimizer(mats, rest, copies=mat_copies)
        angle = torch.arange(cfg.seq)[:, None] * 100.0 ** (-torch.arange(hd // 2) / (hd // 2))[None, :]
        self.cos, self.sin = angle.cos().cuda(), angle.sin().cuda()

    def layer(self, h, qkv, out, up, down, q_gain, k_gain):
        c = self.cfg
        b, n, d = h.shape
        rows = (h @ qkv.t()).view(b, n, 3, c.heads, d // c.heads)
        q, k = _QKNorm.apply(rows[:, :, 0], rows[:, :, 1], q_gain, k_gain, self.cos, self.sin)
        score = torch.einsum("bihd,bjhd->bhij", q, k) / math.sqrt(d // c.heads)
        score = score.masked_fill(torch.ones(n, n, dtype=torch.bool, device=h.device).triu(1), float("-inf"))
        mixed = torch.einsum("bhij,bjhd->bihd", score.softmax(-1), rows[:, :, 2]).reshape(b, n, d)
        h = h + mixed @ out.t()
        return h + torch.relu(h @ up.t()).square() @ down.t()

    def loss_and_gradients(self, tokens, teacher: Teacher):
        """The mean loss of the positions that count; every gradient lands in self.grads."""
        c, w = self.cfg, self.copies
        scale = math.sqrt(c.dim)
        with torch.no_grad():
            h0 = model_ops.embed(w["table"], tokens, scale=scale)
        names = ("qkv", "out", "up", "down", "q_gain", "k_gain")
        leaves = [h0.requires_grad_()] + [(w[n] if n in w else self.others[n]).detach().requires_grad_() for n in names]
        with torch.enable_grad():
            h = self.layer(*leaves)
        with torch.no_grad():
            hidden = h.detach().reshape(-1, c.dim)
            logits = hidden @ w["table"].t()
            counts = (torch.arange(c.seq, device=h.device) >= c.prompt).float().repeat(c.batch)
            ids, top = teacher.entries(tokens)
            loss, dlogits = model_ops.distill_loss_grad(logits, ids, top, weight=counts / counts.sum(),
                                                        temperature=c.temperature, dlogits=logits)
            dh = (dlogits @ w["table"]).view_as(h)
        grads = torch.autograd.grad(h, leaves, dh)
        with torch.no_grad():
            for n, g in zip(names, grads[1:]):
                self.grads[n].copy_(g)
            # the head's gradient of the table, then the lookup's added to it
            self.grads["table"].copy_(dlogits.t() @ hidden)
            model_ops.embed_grad(grads[0], tokens, c.vocab, scale=scale, out=self.grads["table"], accumulate=True)
        return loss.sum()

    def step(self, lr: float = 0.02, adam_lr: float = 3e-3):
        self.optimizer.step(malt.hparams(lr=lr), malt.adamw_hparams(lr=adam_lr))


def train(steps: int = 60, cfg: Config = Config(), seed: int = 0):
    """Losses of `steps` training steps (host floats)."""
    teacher, model = Teacher(cfg, seed), Model(cfg, seed + 1)
    g = torch.Generator().manual_seed(seed + 2)
    losses = []
    for _ in range(steps):
        tokens = torch.randint(0, cfg.vocab, (cfg.batch, cfg.seq), generator=g).cuda()
        losses.append(model.loss_and_gradients(tokens, teacher))
        model.step()
    out = [float(x) for x in losses]
    status = model.optimizer.check()
    model.optimizer.close()
    if status != malt.MALT_OK:
        raise RuntimeError(f"toy distillation failed: {malt.status_string(status)}")
    return out


if __name__ == "__main__":
    trace = train()
    print("loss", " ".join(f"{x:.3f}" for x in trace[::6]), f"{trace[-1]:.3f}")
