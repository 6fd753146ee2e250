"""Plain 64-bit forms of the training-step operators (numpy, on the host) and
the error bounds the GPU tests hold the float32 kernels to.

The bounds follow from the arithmetic: U is half a unit in the last place of
float32 (2^-24), V of bfloat16 (2^-8: 8 significant bits); a value rounded to bfloat16 at the end
adds V of itself.  A sum of n positive float32 terms is off by at most n U of
itself.
"""
from __future__ import annotations

import numpy as np

U, V = 2.0 ** -24, 2.0 ** -8
TINY = 2.0 ** -126          # results below the smallest normal float32 may be flushed
LN2 = np.log(2.0)


def rounding(dtype: str) -> float:
    return V * (1 + 2.0 ** -7) if dtype == "bf16" else U


# -- the generator -------------------------------------------------------------
def philox_words(seed: int, blocks: np.ndarray) -> np.ndarray:
    """Philox4x32-10 of counters (block, 0, 0): uint32 [len(blocks), 4].  Pinned
    by the known answers in tests/golden."""
    m = np.uint64(0xFFFFFFFF)
    c = [blocks.astype(np.uint64) & m, blocks.astype(np.uint64) >> np.uint64(32),
         np.zeros(len(blocks), np.uint64), np.zeros(len(blocks), np.uint64)]
    k0, k1 = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), p1 & m, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), p0 & m]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(c, 1).astype(np.uint32)


def keep_mask(rows, cols, p, seed, offset):
    """(mask [rows, cols], scale)."""
    pitch = (cols + 7) // 8
    w = philox_words(seed, np.arange(rows * pitch, dtype=np.uint64) + np.uint64(offset // 8))
    h = np.stack([w & 0xFFFF, w >> 16], 2).reshape(rows, 8 * pitch)[:, :cols]
    t = int(np.rint(float(np.float32(p)) * 65536))
    return h >= t, (65536.0 / (65536 - t) if t < 65536 else 0.0)


# -- dropout ---------------------------------------------------------------------
def dropout_add(x, bias, residual, p, seed, offset, dtype):
    """(y, bound) for float64 arrays."""
    keep, s = keep_mask(*x.shape, p, seed, offset)
    v = x if bias is None else x + bias
    with np.errstate(invalid="ignore"):
        part = np.where(keep, v * s, 0.0)
    y = part if residual is None else residual + part
    # sum, scale (itself rounded), product, sum
    mag = np.abs(part) + (0 if residual is None else np.abs(residual)) + np.where(keep, s * (np.abs(x) + (
        0 if bias is None else np.abs(bias))), 0.0)
    return y, 4 * U * mag + rounding(dtype) * np.abs(y) + TINY


def dropout_grad(dy, p, seed, offset, dtype):
    keep, s = keep_mask(*dy.shape, p, seed, offset)
    dx = np.where(keep, dy * s, 0.0)
    db = dx.sum(0)
    return (dx, 3 * U * np.abs(dx) + rounding(dtype) * np.abs(dx) + TINY), \
        (db, (dy.shape[0] + 3) * U * np.abs(dx).sum(0) + TINY)


# -- token log probabilities -------------------------------------------------------
def shifted(x):
    """(reference value of each row, log of the sum of exp(x - reference), -inf for rows without a finite logit)."""
    with np.errstate(divide="ignore"):
        m = x.max(1)
        ref = np.where(np.isinf(m), 0.0, m)
        return ref, np.log(np.exp(x - ref[:, None]).sum(1))


def log_probs(x):
    """log p of every element; -inf in rows without a finite logit."""
    ref, ln_s = shifted(x)
    with np.errstate(invalid="ignore"):
        return np.where(np.isneginf(ln_s)[:, None], -np.inf, (x - ref[:, None]) - ln_s[:, None])


def token_stats(x, targets):
    """(logp, lse, entropy) of float64 rows, finite logits or -inf."""
    ref, ln_s = shifted(x)
    lq = log_probs(x)
    p = np.exp(lq)
    ent = -(p * np.where(p > 0, lq, 0.0)).sum(1)
    t = np.clip(targets, 0, x.shape[1] - 1)
    logp = np.where(targets < 0, 0.0, np.where(targets >= x.shape[1], np.nan, lq[np.arange(len(x)), t]))
    return logp, ref + ln_s, ent


def stats_bounds(x, logp, ent):
    """A term of S is off by (|t| + 2) U, by its weight in the sum at most (log2 vocab + 4) U; 64 terms are added one
    after the other, then the lanes' and the slices' sums in 6 steps each and the wave or slice sums."""
    rel = (64 + 6 + 16 + np.log2(x.shape[1]) + 8) * U
    ref, ln_s = shifted(x)
    ln_s = np.where(np.isfinite(ln_s), ln_s, 0.0)
    b_lse = rel + 3 * U * (np.abs(ref) + ln_s)
    b_logp = rel + 3 * U * (np.where(np.isfinite(logp), np.abs(logp), 0) + 2 * ln_s)
    b_ent = 2 * rel * (1 + ln_s + np.abs(ent))
    return b_logp, b_lse, b_ent


def token_grad(x, targets, ent, g_logp, g_ent, g_lse, width, dtype, lse_given=True):
    """(dlogits, bound).  p is off by the rounding of lse where that is given, else by the error of the statistics."""
    n, vocab = x.shape
    z = np.zeros(n)
    ga, ge, gl = (z if g is None else g for g in (g_logp, g_ent, g_lse))
    ga = np.where(targets < 0, 0.0, ga)
    ref, ln_s = shifted(x)
    empty = np.isneginf(ln_s)
    ln_s = np.where(empty, 0.0, ln_s)
    d = log_probs(x)
    p = np.exp(d)
    dd = np.where(p > 0, d, 0.0)
    v = p * ((gl - ga)[:, None] - ge[:, None] * (dd + ent[:, None]))
    mag = p * ((np.abs(gl) + np.abs(ga) + np.abs(ge) * np.abs(ent))[:, None] + np.abs(ge[:, None] * dd))
    if lse_given:
        base = 2 * U * np.abs(ref + ln_s) / LN2
    else:
        base = (64 + 6 + 16 + np.log2(vocab) + 8) * U * 3 + 6 * U * ln_s
    bound = mag * (U * (2 * np.abs(dd) / LN2 + 10) + base[:, None])
    bound += p * (np.abs(ge) * 2 * (base * (1 + ln_s + np.abs(ent))))[:, None]
    hit = (targets >= 0) & (targets < vocab) & ~empty
    v[np.nonzero(hit)[0], targets[hit]] += ga[hit]
    bound[np.nonzero(hit)[0], targets[hit]] += 2 * U * np.abs(ga[hit])
    v[empty] = 0.0
    out, b = np.zeros((n, width)), np.zeros((n, width))
    out[:, :vocab], b[:, :vocab] = v, bound + rounding(dtype) * np.abs(v) + TINY
    return out, b


def top(x, k):
    return np.argsort(-x, axis=1, kind="stable")[:, :k]


# -- norm and rotation ----------------------------------------------------------------
def _pairs(dim, rot, inter):
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if inter else (i, i + rot // 2)


def rotate(u, table, positions, inter, back=False):
    """(rotated, magnitude) of [tokens, heads, dim]."""
    out, mag = u.copy(), np.abs(u)
    if table is None:
        return out, mag
    rot = table.shape[1]
    a, b = _pairs(u.shape[2], rot, inter)
    c, s = table[positions][:, None, :rot // 2], table[positions][:, None, rot // 2:]
    s = -s if back else s
    out[..., a], out[..., b] = u[..., a] * c - u[..., b] * s, u[..., b] * c + u[..., a] * s
    mag[..., a] = np.abs(u[..., a] * c) + np.abs(u[..., b] * s)
    mag[..., b] = np.abs(u[..., b] * c) + np.abs(u[..., a] * s)
    return out, mag


def qk(x, w, eps, table, positions, inter, dtype):
    """(y, bound): the sum of squares is off by 2 W + 6 additions at most (16 + 6), r by half of that and 3 U."""
    u = x
    if eps is not None:
        u = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (1 if w is None else w)
    y, mag = rotate(u, table, positions, inter)
    return y, 20 * U * mag + rounding(dtype) * np.abs(y) + TINY


def qk_grad(dy, x, w, eps, table, positions, inter, dtype):
    """((dx, bound), (dw, bound))."""
    g, gm = rotate(dy, table, positions, inter, back=True)
    if eps is None:
        return (g, 3 * U * gm + rounding(dtype) * np.abs(g) + TINY), None
    wv = 1.0 if w is None else w
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    xr = x * r
    dot = (wv * g * xr).mean(-1, keepdims=True)
    dx = r * (wv * g - xr * dot)
    dot_mag = (np.abs(wv) * gm * np.abs(xr)).mean(-1, keepdims=True)
    bound = 64 * U * r * (np.abs(wv) * gm + np.abs(xr) * dot_mag) + rounding(dtype) * np.abs(dx) + TINY
    n = dy.shape[0] * dy.shape[1]
    dw = (g * xr).sum((0, 1))
    return (dx, bound), (dw, (n + 24) * U * (gm * np.abs(xr)).sum((0, 1)) + TINY)
