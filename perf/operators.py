"""The training-step operators beside the compression path: cases, inputs,
plain forms and definitions in 64 bits.

Three operators, each with its backward pass, that a sharded data-parallel
training step runs between its matrix products and that make the gradients
the compression path takes:

* ``dropout_add`` / ``dropout_add_grad``: bias, dropout from a counter-based
  generator and residual in one pass; the mask is drawn again backward.
* ``token_logprob`` / ``token_logprob_grad`` / ``token_loss``: log
  probabilities of given tokens with logsumexp, entropy and the largest
  alternatives; their gradient; both in one pass over the logits.
* ``qk_norm_rope`` / ``qk_norm_rope_grad``: RMS norm of each query and key
  head and the position rotation in one pass.

``run`` computes them with elementary torch operations, or, where ``own`` is
true, through the library's entry points.
"""
import math

import numpy as np
import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


def listed():
    return [
        # one new token's residual in a 125M-parameter decoder (hidden 768): a call's latency
        dict(name="dropout_one_token", op="dropout_add", rows=1, cols=768, x="bf16", y="bf16", p=0.1),
        # the attention output of 4 sequences of 2048 tokens in the 13B model (hidden 5120)
        dict(name="dropout_block", op="dropout_add", rows=8192, cols=5120, x="bf16", y="bf16", p=0.1),
        # bfloat16 activations joined to a float32 residual stream; an odd width, so rows start at odd addresses
        dict(name="dropout_wide_residual", op="dropout_add", rows=2047, cols=4097, x="bf16", y="f32", p=0.25),
        # backward of a block of the 1.3B model (hidden 2048) in float32, bias gradient included
        dict(name="dropout_grad", op="dropout_add_grad", rows=4095, cols=2048, x="f32", y="f32", p=0.1),
        # four next-token distributions scored, with alternatives: few rows of a large vocabulary
        dict(name="logprob_scoring", op="token_logprob", rows=4, vocab=131072, width=131072, x="bf16", top=8),
        # evaluation of two sequences of 2048 tokens; unpadded vocabulary of odd size
        dict(name="logprob_batch", op="token_logprob", rows=4096, vocab=50001, width=50001, x="bf16", top=5),
        # policy gradient with an entropy bonus and a penalty on the logsumexp: all three gradients, float32 logits
        dict(name="logprob_grad", op="token_logprob_grad", rows=2048, vocab=32768, width=32768, x="f32", ent=True),
        # the training loss of 4 sequences of 2048 tokens with its gradient, vocabulary padded for the output product
        dict(name="loss_batch", op="token_loss", rows=8192, vocab=50000, width=50176, x="bf16", ent=False),
        # eight tokens being generated: 40 query and 8 key heads of 128
        dict(name="qk_decode", op="qk_norm_rope", tokens=8, heads=40, kv_heads=8, dim=128, rot=128, inter=False,
             x="bf16", packed=True),
        # 4 sequences of 2048 tokens of the 13B model's width, queries and keys inside the packed projection
        dict(name="qk_block", op="qk_norm_rope", tokens=8192, heads=40, kv_heads=8, dim=128, rot=128, inter=False,
             x="bf16", packed=True),
        # their backward, weight gradients included
        dict(name="qk_grad", op="qk_norm_rope_grad", tokens=8192, heads=40, kv_heads=8, dim=128, rot=128, inter=False,
             x="bf16", packed=True),
        # a float32 run with 12 heads of 80, rotated in half of the head as neighbouring pairs
        dict(name="qk_partial_grad", op="qk_norm_rope_grad", tokens=1023, heads=12, kv_heads=12, dim=80, rot=40,
             inter=True, x="f32", packed=False),
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


_LIMIT = 0.9 * 8192 * (50000 + 50176) * 2   # bytes: a little less than the largest listed case


def draw(rng):
    op = rng.choice(["dropout_add", "dropout_add_grad", "token_logprob", "token_logprob_grad", "token_loss",
                     "qk_norm_rope", "qk_norm_rope_grad"])
    while True:
        x = rng.choice(["f32", "bf16"])
        if op.startswith("dropout"):
            y = "f32" if x == "f32" else rng.choice(["f32", "bf16"])
            c = dict(op=op, rows=_log_uniform(rng, 1, 16384), cols=_log_uniform(rng, 64, 8192), x=x, y=y,
                     p=rng.choice([0.0, 0.05, 0.1, 0.25, 0.5]))
        elif op.startswith("token"):
            vocab = _log_uniform(rng, 500, 131072)
            width = vocab if rng.random() < 0.5 else -(-vocab // 128) * 128
            c = dict(op=op, rows=_log_uniform(rng, 1, 8192), vocab=vocab, width=width, x=x)
            if op == "token_logprob":
                c["top"] = rng.choice([0, 1, 5, 8, 20])
            else:
                c["ent"] = rng.random() < 0.5
        else:
            dim = rng.choice([64, 80, 96, 128, 128, 256])
            kv = rng.choice([1, 2, 4, 8, 12])
            c = dict(op=op, tokens=_log_uniform(rng, 1, 8192), heads=kv * rng.choice([1, 2, 4, 5]), kv_heads=kv, dim=dim,
                     rot=rng.choice([dim, dim, dim // 2]), inter=rng.random() < 0.5, x=x, packed=rng.random() < 0.7)
        if work(c)["bytes"] <= _LIMIT:
            return c


def work(case):
    """Bytes (inputs read once, outputs written once) and floating-point
    operations (the generator's and the selection's integer work not counted)."""
    op = case["op"]
    if op.startswith("dropout"):
        n, sx, sy = case["rows"] * case["cols"], SIZE[case["x"]], SIZE[case["y"]]
        if op == "dropout_add":
            return {"bytes": n * (sx + 2 * sy) + case["cols"] * sx, "flops": 3 * n}
        return {"bytes": n * (sx + sy) + 4 * case["cols"], "flops": 2 * n}
    if op.startswith("token"):
        r, v, w, s = case["rows"], case["vocab"], case["width"], SIZE[case["x"]]
        if op == "token_logprob":
            return {"bytes": r * (v * s + 8 + 12 + 12 * case["top"]), "flops": 6 * r * v}
        if op == "token_logprob_grad":
            return {"bytes": r * ((v + w) * s + 8 + 8 + (12 if case["ent"] else 4)), "flops": 6 * r * v}
        return {"bytes": r * ((v + w) * s + 8 + 12 + (12 if case["ent"] else 4)), "flops": 10 * r * v}
    t, h, d, s = case["tokens"], case["heads"] + case["kv_heads"], case["dim"], SIZE[case["x"]]
    n = t * h * d
    small = t * (8 + 4 * case["rot"]) + 2 * d * s
    if op == "qk_norm_rope":
        return {"bytes": 2 * n * s + small, "flops": 7 * n}
    return {"bytes": 3 * n * s + small + 8 * d, "flops": 14 * n}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _bytes(n):
    return torch.empty(max(int(n), 16), dtype=torch.uint8, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]

    def normal(*shape, dtype=torch.float32, scale=1.0):
        return (torch.randn(*shape, device="cuda", generator=g) * scale).to(dtype)

    s = dict(case)
    if op.startswith("dropout"):
        rows, cols, xt, yt = case["rows"], case["cols"], DT[case["x"]], DT[case["y"]]
        s["seed"] = (0x9E3779B97F4A7C15 * (seed + 1)) % (1 << 64)
        s["offset"] = 8 * (seed % 1000) * (1 << 31)             # further layers and micro-batches came before
        if op == "dropout_add":
            s["x"], s["bias"] = normal(rows, cols, dtype=xt), normal(cols, dtype=xt, scale=0.1)
            s["residual"], s["y"] = normal(rows, cols, dtype=yt, scale=3.0), torch.empty(rows, cols, dtype=yt, device="cuda")
        else:
            s["dy"], s["dx"] = normal(rows, cols, dtype=yt, scale=1e-3), torch.empty(rows, cols, dtype=xt, device="cuda")
            s["dbias"] = torch.empty(cols, device="cuda")
            if own:
                from paper_2410_15526_amd import sdp4
                s["workspace"] = _bytes(sdp4.sdp4_dropout_grad_workspace(rows, cols))
        return s

    if op.startswith("token"):
        rows, vocab, width, dt = case["rows"], case["vocab"], case["width"], DT[case["x"]]
        s["logits"] = torch.empty(rows, width, dtype=dt, device="cuda")
        for a in range(0, rows, 1024):                          # float32 draws of a part of the rows at a time
            s["logits"][a:a + 1024] = torch.randn(min(1024, rows - a), width, device="cuda", generator=g) * 2.5
        s["logits"][:, vocab:] = 1e4                            # what the padding holds must not count
        t = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
        hit = torch.rand(rows, device="cuda", generator=g)
        s["logits"].scatter_add_(1, t[:, None], (6 * hit.to(dt))[:, None])   # trained: targets more likely than others
        t[torch.rand(rows, device="cuda", generator=g) < 0.1] = -100  # tokens without a loss (prompts, padding)
        s["targets"] = t
        f = lambda *n: torch.empty(*n, device="cuda")  # noqa: E731
        s["logp"], s["lse"], s["entropy"] = f(rows), f(rows), f(rows)
        if op == "token_logprob":
            s["top_logp"] = f(rows, case["top"])
            s["top_ids"] = torch.empty(rows, case["top"], dtype=torch.int64, device="cuda")
        else:
            s["g_logp"] = -torch.rand(rows, device="cuda", generator=g) / max(1, rows // 8)
            s["g_entropy"] = normal(rows, scale=0.01) if case["ent"] else None
            s["g_lse"] = normal(rows, scale=0.01) if case["ent"] else None
            s["dlogits"] = torch.empty(rows, width, dtype=dt, device="cuda")
            if op == "token_logprob_grad":                      # what the forward pass left
                for a in range(0, rows, 256):
                    x = s["logits"][a:a + 256, :vocab].double()
                    lse = torch.logsumexp(x, 1)
                    s["lse"][a:a + 256] = lse
                    s["entropy"][a:a + 256] = lse - (torch.exp(x - lse[:, None]) * x).sum(1)
        if own and op != "token_logprob_grad":
            from paper_2410_15526_amd import sdp4
            s["workspace"] = _bytes(sdp4.sdp4_token_logprob_workspace(rows, vocab, case.get("top", 0)))
        return s

    tokens, hq, hk, d, dt = case["tokens"], case["heads"], case["kv_heads"], case["dim"], DT[case["x"]]
    if case["packed"]:                                          # views into one projection: queries, keys, values
        qkv = normal(tokens, hq + 2 * hk, d, dtype=dt, scale=1.5)
        s["q"], s["k"] = qkv[:, :hq], qkv[:, hq:hq + hk]
    else:
        s["q"], s["k"] = normal(tokens, hq, d, dtype=dt, scale=1.5), normal(tokens, hk, d, dtype=dt, scale=1.5)
    s["q_weight"], s["k_weight"] = 1 + normal(d, scale=0.1), 1 + normal(d, scale=0.1)
    s["q_weight"], s["k_weight"] = s["q_weight"].to(dt), s["k_weight"].to(dt)
    s["eps"] = 1e-6
    half = case["rot"] // 2
    freq = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half) / 4  # stretched to 4 times the length
    ang = torch.arange(8192, dtype=torch.float64, device="cuda")[:, None] * freq
    s["table"] = torch.cat([torch.cos(ang), torch.sin(ang)], 1).float()
    start = int(torch.randint(0, 64, (1,), device="cuda", generator=g))
    s["positions"] = (torch.arange(tokens, device="cuda") + start) % 2048 + (seed % 3) * 2048
    e = lambda h: torch.empty(tokens, h, d, dtype=dt, device="cuda")  # noqa: E731
    if op == "qk_norm_rope":
        s["q_out"], s["k_out"] = e(hq), e(hk)
    else:
        s["dq_out"], s["dk_out"] = normal(tokens, hq, d, dtype=dt, scale=1e-2), normal(tokens, hk, d, dtype=dt, scale=1e-2)
        s["dq"], s["dk"] = e(hq), e(hk)
        s["dq_weight"], s["dk_weight"] = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
        if own:
            from paper_2410_15526_amd import sdp4
            s["workspace"] = _bytes(sdp4.sdp4_qk_grad_workspace(tokens, hq, hk, d))
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(s):
    return (_own if own else _plain)[s["op"]](s)


def _own_dropout_add(s):
    from paper_2410_15526_amd import sdp4
    sdp4.sdp4_dropout_add(s["x"], s["bias"], s["residual"], s["p"], s["seed"], s["offset"], s["y"])
    return s["y"]


def _own_dropout_add_grad(s):
    from paper_2410_15526_amd import sdp4
    sdp4.sdp4_dropout_add_grad(s["dy"], s["p"], s["seed"], s["offset"], s["dx"], s["dbias"], s["workspace"])
    return s["dx"], s["dbias"]


def _own_token_logprob(s):
    from paper_2410_15526_amd import sdp4
    sdp4.sdp4_token_logprob(s["logits"], s["targets"], s["top"], s["logp"], s["lse"], s["entropy"], s["top_logp"],
                            s["top_ids"], s["workspace"], vocab=s["vocab"])
    return s["logp"], s["lse"], s["entropy"], s["top_logp"], s["top_ids"]


def _own_token_logprob_grad(s):
    from paper_2410_15526_amd import sdp4
    sdp4.sdp4_token_logprob_grad(s["logits"], s["targets"], s["lse"], s["entropy"], s["g_logp"], s["g_entropy"],
                                 s["g_lse"], s["dlogits"], vocab=s["vocab"])
    return s["dlogits"]


def _own_token_loss(s):
    from paper_2410_15526_amd import sdp4
    sdp4.sdp4_token_loss(s["logits"], s["targets"], s["g_logp"], s["g_entropy"], s["g_lse"], s["logp"], s["lse"],
                         s["entropy"], s["dlogits"], s["workspace"], vocab=s["vocab"])
    return s["logp"], s["lse"], s["entropy"], s["dlogits"]


def _own_qk_norm_rope(s):
    from paper_2410_15526_amd import sdp4
    sdp4.sdp4_qk_norm_rope(s["q"], s["k"], s["q_weight"], s["k_weight"], s["eps"], s["table"], s["positions"],
                           s["q_out"], s["k_out"], interleaved=s["inter"])
    return s["q_out"], s["k_out"]


def _own_qk_norm_rope_grad(s):
    from paper_2410_15526_amd import sdp4
    sdp4.sdp4_qk_norm_rope_grad(s["dq_out"], s["dk_out"], s["q"], s["k"], s["q_weight"], s["k_weight"], s["eps"],
                                s["table"], s["positions"], s["dq"], s["dk"], s["dq_weight"], s["dk_weight"],
                                s["workspace"], interleaved=s["inter"])
    return s["dq"], s["dk"], s["dq_weight"], s["dk_weight"]


# -- plain forms: elementary torch operations in float32 ----------------------
M32 = 0xFFFFFFFF


def _keep(s, rows, cols):
    """Dropout mask [rows, cols]: Philox4x32-10, eight 16-bit uniforms a block,
    rows at multiples of the width rounded up to 8."""
    pitch = -(-cols // 8) * 8
    blk = torch.arange(rows * (pitch // 8), device="cuda") + s["offset"] // 8
    c = [blk & M32, blk >> 32, torch.zeros_like(blk), torch.zeros_like(blk)]
    k0, k1 = s["seed"] & M32, s["seed"] >> 32
    for r in range(10):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57       # wraps at 64 bits
        c = [(p1 >> 32) & M32 ^ c[1] ^ k0, p1 & M32, (p0 >> 32) & M32 ^ c[3] ^ k1, p0 & M32]
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    h = torch.stack([v for w in c for v in (w & 0xFFFF, w >> 16)], 1).view(rows, pitch)[:, :cols]
    t = round(s["p"] * 65536)
    return h >= t, (65536.0 / (65536 - t) if t < 65536 else 0.0)


def _plain_dropout_add(s):
    keep, scale = _keep(s, s["rows"], s["cols"])
    v = torch.where(keep, (s["x"].float() + s["bias"].float()) * scale, 0.0)
    return (v + s["residual"].float()).to(s["y"].dtype)


def _plain_dropout_add_grad(s):
    keep, scale = _keep(s, s["rows"], s["cols"])
    v = torch.where(keep, s["dy"].float() * scale, 0.0)
    return v.to(s["dx"].dtype), v.sum(0)


def _plain_stats(s):
    x = s["logits"][:, :s["vocab"]].float()
    m = x.amax(1, keepdim=True)
    d = x - m
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    log_total = torch.log(total)
    ent = (log_total - (e * d).sum(1, keepdim=True) / total)[:, 0]
    t = s["targets"]
    logp = torch.where(t >= 0, (d.gather(1, t.clamp(min=0)[:, None]) - log_total)[:, 0], 0.0)
    return x, logp, (m + log_total)[:, 0], ent, m + log_total


def _plain_token_logprob(s):
    x, logp, lse, ent, ref = _plain_stats(s)
    k = s["top"]
    if k == 0:
        return logp, lse, ent, s["top_logp"], s["top_ids"]
    v, i = torch.sort(x, dim=1, descending=True, stable=True)
    return logp, lse, ent, v[:, :k] - ref, i[:, :k].contiguous()


def _plain_gradient(s, x, lse, ent):
    d = x - lse[:, None]
    w = -s["g_logp"][:, None] * (s["targets"] >= 0)[:, None]
    if s["g_lse"] is not None:
        w = w + s["g_lse"][:, None]
    if s["g_entropy"] is not None:
        w = w - s["g_entropy"][:, None] * (d + ent[:, None])
    v = torch.exp(d) * w
    v.scatter_add_(1, s["targets"].clamp(min=0)[:, None], torch.where(s["targets"] >= 0, s["g_logp"], 0.0)[:, None])
    out = torch.zeros(s["rows"], s["width"], dtype=s["dlogits"].dtype, device="cuda")
    out[:, :s["vocab"]] = v
    return out


def _plain_token_logprob_grad(s):
    return _plain_gradient(s, s["logits"][:, :s["vocab"]].float(), s["lse"], s["entropy"])


def _plain_token_loss(s):
    x, logp, lse, ent, _ = _plain_stats(s)
    return logp, lse, ent, _plain_gradient(s, x, lse, ent)


def _pairs(u, s):
    """The two members of every rotated pair, and the elements left alone."""
    rot = s["table"].shape[1]
    if s["inter"]:
        return u[..., 0:rot:2], u[..., 1:rot:2], u[..., rot:]
    return u[..., :rot // 2], u[..., rot // 2:rot], u[..., rot:]


def _join(a, b, rest, s):
    if s["inter"]:
        return torch.cat([torch.stack([a, b], -1).flatten(-2), rest], -1)
    return torch.cat([a, b, rest], -1)


def _angles(s):
    half = s["table"].shape[1] // 2
    t = s["table"][s["positions"]]
    return t[:, None, :half], t[:, None, half:]


def _plain_qk_norm_rope(s):
    c, n = _angles(s)
    out = []
    for x, w in ((s["q"].float(), s["q_weight"].float()), (s["k"].float(), s["k_weight"].float())):
        u = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"]) * w
        a, b, rest = _pairs(u, s)
        out.append(_join(a * c - b * n, b * c + a * n, rest, s).to(s["q"].dtype))
    return tuple(out)


def _plain_qk_norm_rope_grad(s):
    c, n = _angles(s)
    dxs, dws = [], []
    for dy, x, w in ((s["dq_out"], s["q"], s["q_weight"]), (s["dk_out"], s["k"], s["k_weight"])):
        dy, x, w = dy.float(), x.float(), w.float()
        a, b, rest = _pairs(dy, s)
        g = _join(a * c + b * n, b * c - a * n, rest, s)
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"])
        xr = x * r
        dws.append((g * xr).sum((0, 1)))
        g = g * w
        dxs.append((r * (g - xr * (g * xr).mean(-1, keepdim=True))).to(s["q"].dtype))
    return dxs[0], dxs[1], dws[0], dws[1]


_OPS = ("dropout_add", "dropout_add_grad", "token_logprob", "token_logprob_grad", "token_loss", "qk_norm_rope",
        "qk_norm_rope_grad")
_own = {op: globals()["_own_" + op] for op in _OPS}
_plain = {op: globals()["_plain_" + op] for op in _OPS}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def _uniforms(seed, offset, rows, cols):
    """16-bit uniforms [rows, cols] of the generator, in numpy's unsigned words."""
    u32, u64 = np.uint32, np.uint64
    per_row = (cols + 7) // 8
    counter = np.arange(rows * per_row, dtype=u64) + u64(offset // 8)
    w0, w1 = counter.astype(u32), (counter >> u64(32)).astype(u32)
    w2, w3 = np.zeros_like(w0), np.zeros_like(w0)
    keys = [(seed + r * 0x9E3779B9) & M32 for r in range(10)], [((seed >> 32) + r * 0xBB67AE85) & M32 for r in range(10)]
    for ka, kb in zip(*keys):
        a, b = w0.astype(u64) * u64(0xD2511F53), w2.astype(u64) * u64(0xCD9E8D57)
        w0, w2 = (b >> u64(32)).astype(u32) ^ w1 ^ u32(ka), (a >> u64(32)).astype(u32) ^ w3 ^ u32(kb)
        w1, w3 = b.astype(u32), a.astype(u32)
    words = np.stack([w0, w1, w2, w3], axis=1).astype("<u4").view("<u2")     # low half first
    return words.reshape(rows, 8 * per_row)[:, :cols]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op.startswith("dropout"):
        drop = round(case["p"] * 65536)
        mask = torch.from_numpy(_uniforms(s["seed"], s["offset"], case["rows"], case["cols"]).astype(np.int32) >= drop).cuda()
        mask = mask.double() / (1 - drop / 65536)
        if op == "dropout_add":
            return s["residual"].double() + mask * (s["x"].double() + s["bias"].double())
        dx = mask * s["dy"].double()
        return dx, dx.sum(0)

    if op.startswith("token"):
        vocab, width, t = case["vocab"], case["width"], s["targets"]
        stats, tops, ids, grads = [], [], [], []
        step = max(1, (1 << 27) // width)
        for a in range(0, case["rows"], step):
            x = s["logits"][a:a + step, :vocab].double()
            ta = t[a:a + step]
            logq = torch.log_softmax(x, 1)
            q = torch.exp(logq)
            has = (ta >= 0).double()
            at = ta.clamp(min=0)[:, None]
            ent = -(q * logq).sum(1)
            stats.append(torch.stack([has * logq.gather(1, at)[:, 0], torch.logsumexp(x, 1), ent]))
            if op == "token_logprob":
                order = torch.argsort(-x, dim=1, stable=True)[:, :case["top"]]
                ids.append(order)
                tops.append(logq.gather(1, order))
            else:
                ga = s["g_logp"][a:a + step].double() * has
                d = -ga[:, None] * q
                d.scatter_add_(1, at, ga[:, None])
                if case["ent"]:
                    d -= s["g_entropy"][a:a + step].double()[:, None] * q * (logq + ent[:, None])
                    d += s["g_lse"][a:a + step].double()[:, None] * q
                grads.append(torch.nn.functional.pad(d, (0, width - vocab)))
        logp, lse, ent = torch.cat(stats, 1)
        if op == "token_logprob":
            return logp, lse, ent, torch.cat(tops), torch.cat(ids)
        if op == "token_logprob_grad":
            return torch.cat(grads)
        return logp, lse, ent, torch.cat(grads)

    # the rotation as a product with unit complex numbers times their length
    half = case["rot"] // 2
    tab = s["table"].double()[s["positions"]]
    unit = torch.complex(tab[:, :half], tab[:, half:])[:, None]

    def turn(u, by):
        part, rest = u[..., :2 * half], u[..., 2 * half:]
        part = part.unflatten(-1, (half, 2)) if case["inter"] else part.unflatten(-1, (2, half)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(part.contiguous()) * by)
        z = z.flatten(-2) if case["inter"] else z.transpose(-1, -2).flatten(-2)
        return torch.cat([z, rest], -1)

    outs, dws = [], []
    for n in ("q", "k"):
        x, w = s[n].double(), s[n + "_weight"].double()
        inv = (x.square().sum(-1, keepdim=True) / case["dim"] + s["eps"]) ** -0.5
        if op == "qk_norm_rope":
            outs.append(turn(x * inv * w, unit))
            continue
        g = turn(s["d" + n + "_out"].double(), unit.conj())
        dws.append((g * x * inv).sum((0, 1)))
        gw = g * w
        outs.append(gw * inv - x * inv ** 3 * (gw * x).sum(-1, keepdim=True) / case["dim"])
    return tuple(outs + dws)
