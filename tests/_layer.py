"""Plain 64-bit forms of attention, block norms and the embedding (numpy, on
the host) and the error bounds the GPU tests hold the kernels to.

Bounds as in :mod:`tests._step`: U and V are half a step of float32 and
bfloat16, a float32 dot product or sum of n terms is off by at most n U of the
sum of its terms' magnitudes.
"""
from __future__ import annotations

import numpy as np

from tests._step import TINY, U, V, rounding


# -- attention -------------------------------------------------------------------
def spans(lengths):
    a = 0
    for n in lengths:
        if n:
            yield a, a + n
        a += n


def _scores(q, k, scale):
    """Masked scores of one sequence and head and the largest error of each: a product of d terms, c = scale log2(e) and its
    product rounded, the exponential."""
    d = q.shape[1]
    s, mag = scale * q @ k.T, scale * np.abs(q) @ np.abs(k).T
    seen = np.tril(np.ones(s.shape, bool))
    err = (d + 2) * U * mag + 4 * U * np.abs(s)
    return np.where(seen, s, -np.inf), np.where(seen, err, 0.0), seen


def attention(q, k, v, lengths, scale, dtype):
    """((out, bound), (lse, bound)) for [tokens, heads, dim]; NaN in rows of no sequence."""
    n, hq, d = q.shape
    group = hq // k.shape[1]
    out, b_out = np.full((n, hq, d), np.nan), np.zeros((n, hq, d))
    lse, b_lse = np.full((hq, n), np.nan), np.zeros((hq, n))
    for a, b in spans(lengths):
        for h in range(hq):
            s, err, seen = _scores(q[a:b, h], k[a:b, h // group], scale)
            m = s.max(1, keepdims=True)
            e = np.exp(s - m)
            total = e.sum(1, keepdims=True)
            p = e / total
            val = v[a:b, h // group]
            o = p @ val
            m_n = b - a
            # the worst relative error of a probability; the reference's rounding is common to all
            rel = err.max(1, keepdims=True) + 6 * U * np.abs(np.where(seen, s, 0.0)).max(1, keepdims=True) + 8 * U
            mag = p @ np.abs(val)
            low = V * (1 + 2.0 ** -7) if dtype == "bf16" else 0.0          # probabilities rounded for the product
            out[a:b, h] = o
            b_out[a:b, h] = mag * (2 * rel + (m_n + m_n / 16 + 16) * U + low) + rounding(dtype) * np.abs(o) + TINY
            ln = (m + np.log(total))[:, 0]
            lse[h, a:b] = ln
            b_lse[h, a:b] = rel[:, 0] + (m_n + m_n / 16 + 16) * U + 4 * U * (np.abs(m[:, 0]) + np.abs(ln))
    return (out, b_out), (lse, b_lse)


def attention_grad(dout, q, k, v, out, lse, lengths, scale, dtype):
    """((dq, bound), (dk, bound), (dv, bound)) from out and lse as given."""
    n, hq, d = q.shape
    group = hq // k.shape[1]
    res = [(np.full(x.shape, np.nan), np.zeros(x.shape)) for x in (q, k, v)]
    low = V * (1 + 2.0 ** -7) if dtype == "bf16" else 0.0
    for a, b in spans(lengths):
        for x, e in res:
            x[a:b] = 0.0
        for h in range(hq):
            kh = h // group
            qq, kk, vv, gg, oo = q[a:b, h], k[a:b, kh], v[a:b, kh], dout[a:b, h], out[a:b, h]
            s, err, seen = _scores(qq, kk, scale)
            ls = lse[h, a:b][:, None]
            p = np.where(seen, np.exp(s - ls), 0.0)
            rel = err + 4 * U * (np.abs(np.where(seen, s, 0.0)) + np.abs(ls)) + 4 * U
            dp, along = gg @ vv.T, (gg * oo).sum(1, keepdims=True)
            dp_mag, along_mag = np.abs(gg) @ np.abs(vv).T, np.abs(gg * oo).sum(1, keepdims=True)
            ds = p * (dp - along)
            e_ds = p * (rel * np.abs(dp - along) + (d + 4) * U * (dp_mag + along_mag)) + low * np.abs(ds)
            m = b - a
            res[0][0][a:b, h] = scale * ds @ kk
            res[0][1][a:b, h] = scale * (e_ds + (m + 4) * U * np.abs(ds)) @ np.abs(kk)
            res[1][0][a:b, kh] += scale * ds.T @ qq
            res[1][1][a:b, kh] += scale * (e_ds + (m * group + 4) * U * np.abs(ds)).T @ np.abs(qq)
            res[2][0][a:b, kh] += p.T @ gg
            res[2][1][a:b, kh] += (p * (rel + low + (m * group + 4) * U)).T @ np.abs(gg)
    return [(x, e + rounding(dtype) * np.abs(x) + TINY) for x, e in res]


# -- block norms -------------------------------------------------------------------
SUM = 100 * U      # of a row's sum of squares, relative: at most 64 terms of a lane, 6 steps over lanes, 16 waves, the square


def block_norm(branch, residual, post_eps, post_weight, gate, branch_scale, residual_scale, pre_eps, pre_weight, x_dtype, y_dtype):
    """((y, bound), (h, bound)) of float64 matrices; None where there is none."""
    part = mag = 0.0
    if branch is not None:
        u = branch
        if post_eps is not None:
            u = branch / np.sqrt((branch ** 2).mean(1, keepdims=True) + post_eps)
        if post_weight is not None:
            u = u * post_weight
        part = branch_scale * (1 if gate is None else gate[:, None]) * u
        mag = (SUM + 10 * U) * np.abs(part)
    y = part
    if residual is not None:
        y = residual_scale * residual + part
        mag = mag + 3 * U * np.abs(residual_scale * residual)
    e_y = mag + 2 * U * np.abs(y)
    r = 1 / np.sqrt((y ** 2).mean(1, keepdims=True) + pre_eps)
    w = 1.0 if pre_weight is None else pre_weight
    h = y * r * w
    rel_r = np.sqrt((e_y ** 2).mean(1, keepdims=True)) * r + SUM
    return (y, e_y + rounding(y_dtype) * np.abs(y) + TINY), \
        (h, np.abs(w) * r * e_y + np.abs(h) * (rel_r + 6 * U) + rounding(x_dtype) * np.abs(h) + TINY)


def block_norm_grad(dh, dy, branch, y, post_eps, post_weight, gate, branch_scale, residual_scale, pre_eps, pre_weight, x_dtype,
                    y_dtype):
    """{name: (gradient, bound)}; dh, dy, branch, y may be None as the entry point allows."""
    shape = (dy if dh is None else dh).shape
    t, mag = np.zeros(shape), np.zeros(shape)
    out = {}
    w2 = 1.0 if pre_weight is None else pre_weight
    if dh is not None:
        r = 1 / np.sqrt((y ** 2).mean(1, keepdims=True) + pre_eps)
        yh, g = y * r, dh * w2
        t = r * (g - yh * (g * yh).mean(1, keepdims=True))
        mag = r * (np.abs(g) + np.abs(yh) * np.abs(g * yh).mean(1, keepdims=True))
        out["dpre_weight"] = ((dh * yh).sum(0), (shape[0] + 16) * U * np.abs(dh * yh).sum(0) + SUM * np.abs(dh * yh).sum(0) + TINY)
    if dy is not None:
        t, mag = t + dy, mag + np.abs(dy)
    e_t = (2 * SUM + 16 * U) * mag
    dres = residual_scale * t
    out["dresidual"] = (dres, np.abs(residual_scale) * e_t + (2 * U + rounding(y_dtype)) * np.abs(dres) + TINY)
    by = branch_scale * (np.ones((shape[0], 1)) if gate is None else gate[:, None])
    w1 = 1.0 if post_weight is None else post_weight
    s, e_s = by * t * w1, np.abs(by * w1) * (e_t + 4 * U * np.abs(t))
    if branch is not None:
        rb = 1 / np.sqrt((branch ** 2).mean(1, keepdims=True) + post_eps) if post_eps is not None else np.ones((shape[0], 1))
        bh = branch * rb
        rel = SUM + 8 * U
        terms, e_terms = by * t * bh, np.abs(by * bh) * (e_t + rel * np.abs(t))
        out["dpost_weight"] = (terms.sum(0), (e_terms + (shape[0] + 16) * U * np.abs(terms)).sum(0) + TINY)
        terms, e_terms = branch_scale * t * bh * w1, np.abs(branch_scale * bh * w1) * (e_t + (2 * rel + SUM) * np.abs(t))
        out["dgate"] = (terms.sum(1), e_terms.sum(1) + TINY)
        if post_eps is not None:
            dot, dot_mag = (s * bh).mean(1, keepdims=True), np.abs(s * bh).mean(1, keepdims=True)
            e_dot = (e_s * np.abs(bh)).mean(1, keepdims=True) + (2 * rel + SUM) * dot_mag
            s, e_s = rb * (s - bh * dot), rb * (e_s + np.abs(bh) * e_dot + 2 * rel * (np.abs(s) + np.abs(bh) * dot_mag))
    out["dbranch"] = (s, e_s + 4 * U * np.abs(s) + rounding(x_dtype) * np.abs(s) + TINY)
    return out


# -- embedding ---------------------------------------------------------------------
def embedding(tokens, table, scale, dtype):
    rows = np.zeros((len(tokens), table.shape[1]))
    ok = (tokens >= 0) & (tokens < len(table))
    rows[ok] = table[tokens[ok]] * scale
    rows[tokens >= len(table)] = np.nan
    return rows, 2 * U * np.abs(rows) + rounding(dtype) * np.abs(rows) + TINY


def embedding_grad(tokens, dout, scale, vocab, before, dtype):
    total, mag, count = np.zeros((vocab, dout.shape[1])), np.zeros((vocab, dout.shape[1])), np.zeros((vocab, 1))
    ok = (tokens >= 0) & (tokens < vocab)
    np.add.at(total, tokens[ok], dout[ok] * scale)
    np.add.at(mag, tokens[ok], np.abs(dout[ok] * scale))
    np.add.at(count, tokens[ok], 1.0)
    bound = (count + 4) * U * mag
    if before is not None:
        total, bound = total + before, bound + 2 * U * np.abs(before)
    return total, bound + rounding(dtype) * np.abs(total) + TINY
