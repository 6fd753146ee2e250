"""The training-step operators as torch functions with gradients.

Each function allocates its outputs (and a workspace where the call needs
one) and calls the entry points of :mod:`paper_2410_15526_amd.sdp4`; a
program that keeps its buffers, wants alternatives or has gradients by entropy
and logsumexp for the loss in one pass calls those directly.  Broadcast or
transposed arguments are copied; what else must hold of them is checked there:
matrices have two dimensions, heads three, and norm weights the type of the
heads.  The gradients have no gradients themselves: torch raises where one is
asked for.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import sdp4


def _workspace(nbytes: int, device):
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


def _f32(device, *shape):
    return torch.empty(*shape, dtype=torch.float32, device=device)   # whatever the program's default type is


def _laid_out(x):
    """x, or a contiguous copy where it is broadcast or its last dimension is
    strided (gradients often are)."""
    ok = (x.shape[-1] <= 1 or x.stride(-1) == 1) and all(s >= x.shape[-1] or n <= 1
                                                          for n, s in zip(x.shape[:-1], x.stride()[:-1]))
    return x if ok else x.contiguous()


def _dense(x):
    """x contiguous, or None."""
    return None if x is None else x.contiguous()


class _DropoutAdd(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, bias, residual, p, seed, offset):
        like = x if residual is None else residual
        y = torch.empty(x.shape, dtype=like.dtype, device=x.device)
        sdp4.sdp4_dropout_add(x, bias, residual, p, seed, offset, y)
        ctx.args = (p, seed, offset, x.dtype, None if bias is None else bias.dtype, residual is not None)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        p, seed, offset, dtype, bias_dtype, with_residual = ctx.args
        if not any(ctx.needs_input_grad[:2]):
            return None, None, dy, None, None, None
        dy = _laid_out(dy)
        dx = torch.empty(dy.shape, dtype=dtype, device=dy.device)
        dbias = work = None
        if bias_dtype is not None and ctx.needs_input_grad[1]:
            dbias = _f32(dy.device, dy.shape[1])
            work = _workspace(sdp4.sdp4_dropout_grad_workspace(*dy.shape), dy.device)
        sdp4.sdp4_dropout_add_grad(dy, p, seed, offset, dx, dbias, work)
        return dx, None if dbias is None else dbias.to(bias_dtype), dy if with_residual else None, None, None, None


def dropout_add(x, bias, residual, p: float, seed: int, offset: int):
    """residual + dropout(x + bias) of matrices [rows, cols]; bias and residual
    may be None.  (seed, offset) name the mask, see ``sdp4_dropout_add``: a step
    captured in a HIP graph draws the same one in every replay."""
    return _DropoutAdd.apply(_laid_out(x), _dense(bias), None if residual is None else _laid_out(residual), p, seed, offset)


class _QkNormRope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, eps, table, positions, interleaved):
        empty = lambda x: torch.empty(x.shape, dtype=x.dtype, device=x.device)  # noqa: E731
        q_out, k_out = empty(q), empty(k)
        sdp4.sdp4_qk_norm_rope(q, k, q_weight, k_weight, eps, table, positions, q_out, k_out, interleaved)
        ctx.save_for_backward(*((None, None) if eps is None else (q, k)), q_weight, k_weight, table, positions)
        ctx.args = (eps, interleaved)
        return q_out, k_out

    @staticmethod
    @once_differentiable
    def backward(ctx, dq_out, dk_out):
        q, k, q_weight, k_weight, table, positions = ctx.saved_tensors
        eps, interleaved = ctx.args
        dq_out, dk_out = _laid_out(dq_out), _laid_out(dk_out)
        dq, dk = (torch.empty(d.shape, dtype=d.dtype, device=d.device) for d in (dq_out, dk_out))
        dws = [_f32(w.device, *w.shape) if w is not None and needed else None
               for w, needed in zip((q_weight, k_weight), ctx.needs_input_grad[2:4])]
        work = None
        if any(w is not None for w in dws):
            tokens, heads, dim = dq_out.shape
            work = _workspace(sdp4.sdp4_qk_grad_workspace(tokens, heads, dk_out.shape[1], dim), dq.device)
        sdp4.sdp4_qk_norm_rope_grad(dq_out, dk_out, q, k, q_weight, k_weight, eps, table, positions, dq, dk, *dws, work,
                                    interleaved)
        dws = [None if d is None else d.to(w.dtype) for d, w in zip(dws, (q_weight, k_weight))]
        return dq, dk, *dws, None, None, None, None


def qk_norm_rope(q, k, q_weight, k_weight, eps, table, positions, interleaved: bool = False):
    """RMS norm (none if eps is None) and rotation of query and key heads
    [tokens, heads, head_dim], see ``sdp4_qk_norm_rope``."""
    return _QkNormRope.apply(_laid_out(q), _laid_out(k), _dense(q_weight), _dense(k_weight), eps, _dense(table),
                             _dense(positions), interleaved)


class _TokenLogprob(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets, vocab):
        rows = logits.shape[0]
        out = [_f32(logits.device, rows) for _ in range(3)]
        work = _workspace(sdp4.sdp4_token_logprob_workspace(rows, vocab or logits.shape[1]), logits.device)
        sdp4.sdp4_token_logprob(logits, targets, 0, *out, workspace=work, vocab=vocab)
        ctx.save_for_backward(logits, targets, out[1], out[2])
        ctx.vocab = vocab
        ctx.set_materialize_grads(False)      # no gradient by the entropy: the form without it
        return tuple(out)

    @staticmethod
    @once_differentiable
    def backward(ctx, g_logp, g_lse, g_entropy):
        logits, targets, lse, entropy = ctx.saved_tensors
        d = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        sdp4.sdp4_token_logprob_grad(logits, targets, lse, entropy, _dense(g_logp), _dense(g_entropy), _dense(g_lse), d,
                                     vocab=ctx.vocab)
        return d, None, None


def token_logprob(logits, targets, vocab: int | None = None):
    """(logp, lse, entropy) of each row, see ``sdp4_token_logprob``."""
    return _TokenLogprob.apply(_laid_out(logits), _dense(targets), vocab)


def token_loss(logits, targets, weights, vocab: int | None = None):
    """The weighted loss -sum(weights * logp) and its gradient by the logits,
    computed together (the logits are read once): for
    ``logits.backward(gradient)``.  Returns (loss, gradient)."""
    with torch.no_grad():
        logits = _laid_out(logits)
        rows, width = logits.shape
        logp, lse, entropy = (_f32(logits.device, rows) for _ in range(3))
        d = torch.empty(rows, width, dtype=logits.dtype, device=logits.device)
        work = _workspace(sdp4.sdp4_token_logprob_workspace(rows, vocab or width), logits.device)
        sdp4.sdp4_token_loss(logits, _dense(targets), _dense(-weights), None, None, logp, lse, entropy, d, work, vocab=vocab)
        return -(weights * logp).sum(), d


def rope_table(rows: int, rot_dim: int, base: float = 10000.0, stretch: float = 1.0, ramp: tuple | None = None,
               scale: float = 1.0, start: int = 0, device="cuda"):
    """Table of ``sdp4_qk_norm_rope`` for positions start .. start + rows - 1.

    Frequencies are base^(-2i / rot_dim).  For contexts ``stretch`` times as
    long as trained for, all are divided by it (positions interpolated), or,
    with ramp = (slow, fast, length), only those that turn less than ``slow``
    times over ``length`` positions, those above ``fast`` times not at all and
    the ones between by a linear ramp.  ``scale`` multiplies cosines and sines.
    """
    i = torch.arange(rot_dim // 2, dtype=torch.float64)
    inv = base ** (-2.0 * i / rot_dim)
    if ramp is None:
        inv = inv / stretch
    else:
        slow, fast, length = ramp
        turns = length * inv / (2 * torch.pi)
        keep = ((turns - slow) / (fast - slow)).clamp(0.0, 1.0)
        inv = inv * keep + inv / stretch * (1 - keep)
    table = _f32(device, rows, rot_dim)
    sdp4.sdp4_rope_table(inv.to(device), table, start, scale)
    return table
