"""A small decoder trained with the step operators, its gradients and weights
through the compression path: ``python -m paper_2410_15526_amd.decoder``.

One worker's share of a sharded data-parallel step, end to end: the forward
and backward pass run norm and rotation of queries and keys, bias + dropout
+ residual, and the loss with its gradient through the library, with torch's
matrix products between them; the gradients then take the two-level path of
:class:`~paper_2410_15526_amd.pipeline.HotPath` (one peer at each level, so
what comes out is the worker's own gradient after both quantizations), the
optimizer updates the float32 main weights, and the bfloat16 model weights
follow by 4-bit weight differences.
"""
from __future__ import annotations

import argparse
from dataclasses import dataclass

import torch

from . import autograd
from .pipeline import HotPath


@dataclass(frozen=True)
class Config:
    vocab: int = 1000
    width: int = 1024        # of the logits: the vocabulary padded for the output product
    hidden: int = 256
    heads: int = 4
    layers: int = 2
    seq: int = 64
    batch: int = 16
    dropout: float = 0.1
    lr: float = 3e-3
    group: int = 128
    hadamard_block: int = 128


class Decoder:
    """Model weights are views of one flat bfloat16 buffer, the one that the
    weight differences update in place."""

    def __init__(self, cfg: Config = Config(), seed: int = 0):
        self.cfg, self.seed, self.steps = cfg, seed, 0
        h, d = cfg.hidden, cfg.hidden // cfg.heads
        shapes = [("embed", (cfg.width, h))]
        for i in range(cfg.layers):
            shapes += [(f"{i}.qkv", (3 * h, h)), (f"{i}.q_norm", (d,)), (f"{i}.k_norm", (d,)), (f"{i}.out", (h, h)),
                       (f"{i}.out_bias", (h,)), (f"{i}.up", (4 * h, h)), (f"{i}.down", (h, 4 * h)), (f"{i}.down_bias", (h,))]
        count = sum(torch.Size(s).numel() for _, s in shapes)
        n = -(-count // cfg.group) * cfg.group
        self.path = HotPath(n, cfg.group, cfg.hadamard_block, 1, 1, cfg.group, "bf16")
        for b in (self.path.w_new, self.path.grad):
            b.zero_()
        self.weights, self.main, self.grads, at = {}, {}, {}, 0
        g = torch.Generator(device="cuda").manual_seed(seed)
        for name, shape in shapes:
            size = torch.Size(shape).numel()
            part = slice(at, at + size)
            self.main[name] = self.path.w_new[part].view(shape)
            if name.endswith("_norm"):
                self.main[name].fill_(1.0)
            elif not name.endswith("_bias"):
                self.main[name].copy_(torch.randn(shape, device="cuda", generator=g) * shape[-1] ** -0.5)
            self.weights[name] = self.path.w_prev[part].view(shape)
            self.grads[name] = self.path.grad[part].view(shape)
            at += size
        self.path.w_prev.copy_(self.path.w_new)
        self.moments = [torch.zeros(n, device="cuda") for _ in range(2)]
        self.table = autograd.rope_table(cfg.seq, d)
        self.mask = torch.full((cfg.seq, cfg.seq), float("-inf"), device="cuda").triu(1)

    def logits(self, tokens, weights, step: int, p: float):
        """Logits [batch * seq, width] of tokens [batch, seq]."""
        c = self.cfg
        rows, d = tokens.numel(), c.hidden // c.heads
        norm = lambda v: v * torch.rsqrt((v.float() ** 2).mean(1, keepdim=True) + 1e-6).to(v.dtype)  # noqa: E731
        positions = torch.arange(c.seq, device="cuda").repeat(tokens.shape[0])
        x = weights["embed"][tokens.reshape(-1)]
        for i in range(c.layers):
            w = {k[len(f"{i}."):]: v for k, v in weights.items() if k.startswith(f"{i}.")}
            # masks of this step, layer and place: a range of element numbers each
            offset = [(((step * c.layers + i) * 2 + j) * rows * c.hidden) for j in range(2)]
            qkv = (norm(x) @ w["qkv"].t()).view(rows, 3 * c.heads, d)
            q, k = autograd.qk_norm_rope(qkv[:, :c.heads], qkv[:, c.heads:2 * c.heads], w["q_norm"], w["k_norm"], 1e-6,
                                         self.table, positions)
            q, k, v = (t.reshape(-1, c.seq, c.heads, d).transpose(1, 2).float().contiguous()
                       for t in (q, k, qkv[:, 2 * c.heads:]))
            a = torch.softmax(q @ k.transpose(2, 3).contiguous() * d ** -0.5 + self.mask, -1) @ v
            a = a.transpose(1, 2).reshape(rows, c.hidden).to(x.dtype)
            x = autograd.dropout_add(a @ w["out"].t(), w["out_bias"], x, p, self.seed, offset[0])
            u = torch.nn.functional.gelu(norm(x) @ w["up"].t())
            x = autograd.dropout_add(u @ w["down"].t(), w["down_bias"], x, p, self.seed, offset[1])
        return norm(x) @ weights["embed"].t()

    def backward(self, tokens, targets, p: float | None = None):
        """Mean loss over the targets (negative: none); fills ``grads``."""
        c = self.cfg
        leaves = {k: v.detach().requires_grad_() for k, v in self.weights.items()}
        z = self.logits(tokens, leaves, self.steps, c.dropout if p is None else p)
        t = targets.reshape(-1)
        has = (t >= 0).float()
        loss, dz = autograd.token_loss(z.detach(), t, has / has.sum().clamp(min=1), c.vocab)
        z.backward(dz)
        for k, v in leaves.items():
            self.grads[k].copy_(v.grad)
        return loss

    def step(self, tokens, targets):
        """One training step; returns the loss before it."""
        loss = self.backward(tokens, targets)
        self.path.gradient_variant("tlq_hs")
        self.steps += 1
        g, (m, v) = self.path.out, self.moments
        m.lerp_(g, 0.1)
        v.lerp_(g * g, 0.01)
        rate = self.cfg.lr * (1 - 0.99 ** self.steps) ** 0.5 / (1 - 0.9 ** self.steps)
        self.path.w_new.addcdiv_(m, v.sqrt() + 1e-8, value=-rate)
        self.path.qwd_encode()
        self.path.qwd_decode()
        return loss


def sequences(cfg: Config, count: int, seed: int):
    """Tokens [count, seq] and next tokens of walks along a fixed random map, from random starts."""
    g = torch.Generator(device="cuda").manual_seed(1)
    after = torch.randperm(cfg.vocab, device="cuda", generator=g)
    g.manual_seed(2 + seed)
    t = [torch.randint(0, cfg.vocab, (count,), device="cuda", generator=g)]
    for _ in range(cfg.seq):
        t.append(after[t[-1]])
    t = torch.stack(t, 1)
    return t[:, :-1].contiguous(), t[:, 1:].contiguous()


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=200)
    a = ap.parse_args()
    model = Decoder()
    for i in range(a.steps):
        loss = model.step(*sequences(model.cfg, model.cfg.batch, i))
        if i % 20 == 0 or i == a.steps - 1:
            print(f"step {i:4d}  loss {float(loss):.4f}", flush=True)


if __name__ == "__main__":
    main()
