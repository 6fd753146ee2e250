"""Attention, block norms and the embedding as torch functions, and the small
decoder with norms behind its blocks, which trains on all of them."""
import pytest

pytestmark = pytest.mark.gpu


def leaves(seed, *shapes, dtype=None):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(*s, device="cuda", generator=g).to(dtype or torch.float32).requires_grad_() for s in shapes]


def grads(ts):
    out = [t.grad.clone() for t in ts]
    for t in ts:
        t.grad = None
    return out


def near(a, b, tol):
    """float32 chains of a few hundred terms against float64: relative to the largest value."""
    a, b = a.detach(), b.detach()
    assert float((a.double() - b.double()).abs().max()) <= tol * max(float(b.double().abs().max()), 1e-30), \
        (float((a.double() - b.double()).abs().max()), float(b.double().abs().max()))


def test_attention_function():
    import torch

    from paper_2410_15526_amd import autograd
    lengths, n = [20, 0, 33, 1], 60
    q, k, v = leaves(1, (n, 4, 40), (n, 2, 40), (n, 2, 40))
    off = torch.tensor([0, 20, 20, 53, 54], device="cuda")
    out = autograd.attention(q, k, v, off, 0.2)
    w = torch.randn_like(out)
    (out * w).sum().backward()
    got = grads([q, k, v])
    z = [t.detach().double().requires_grad_() for t in (q, k, v)]
    seq = torch.cat([torch.full((m,), i) for i, m in enumerate(lengths)] + [torch.arange(100, 106)]).cuda()
    pos = torch.arange(n, device="cuda")
    seen = (seq[:, None] == seq[None]) & (pos[:, None] >= pos[None])
    s = torch.einsum("nhd,mhd->hnm", z[0], z[1].repeat_interleave(2, 1)) * 0.2
    o = torch.einsum("hnm,mhd->nhd", torch.softmax(s.masked_fill(~seen, -torch.inf), -1), z[2].repeat_interleave(2, 1))
    (o[:54] * w[:54].double()).sum().backward()
    near(out[:54], o[:54], 1e-6)
    assert bool((out[54:] == 0).all())
    for a, b in zip(got, z):
        near(a, b.grad, 2e-6)
        assert bool((a[54:] == 0).all())
    one = autograd.attention(q[:20], k[:20], v[:20], scale=0.2)        # one sequence, no offsets
    assert torch.equal(one, out[:20])
    wide = leaves(2, (9, 1, 16))[0]                                    # a broadcast head, and a gradient that comes broadcast
    autograd.attention(wide.expand(9, 4, 16), wide.expand(9, 2, 16), wide.expand(9, 2, 16)).sum().backward()
    assert wide.grad.shape == wide.shape and bool(torch.isfinite(wide.grad).all())
    flat = autograd.attention(q.transpose(0, 1).contiguous().transpose(0, 1), k, v, off, 0.2)    # laid out head by head
    assert torch.equal(flat, out)


def test_block_norm_function():
    import torch

    from paper_2410_15526_amd import autograd
    unit = lambda x, e: x * torch.rsqrt((x * x).mean(1, keepdim=True) + e)  # noqa: E731
    for post, with_gate in ((1e-5, True), (None, False)):
        ts = leaves(3, (30, 90), (30, 90), (90,), (90,), (30,))
        b, x, w1, w2, gate = ts
        y, h = autograd.block_norm(b, x, w2, 1e-6, post_weight=w1, post_eps=post, gate=gate if with_gate else None, branch_scale=0.5,
                                   residual_scale=1.2)
        cy, ch = torch.randn_like(y), torch.randn_like(h)
        ((y * cy).sum() + (h * ch).sum()).backward()
        used = ts if with_gate else ts[:4]
        got = grads(used)
        z = [t.detach().double().requires_grad_() for t in used]
        u = (unit(z[0], post) if post else z[0]) * z[2] * (z[4][:, None] if with_gate else 1.0)
        yy = 1.2 * z[1] + 0.5 * u
        hh = unit(yy, 1e-6) * z[3]
        ((yy * cy.double()).sum() + (hh * ch.double()).sum()).backward()
        near(y, yy, 1e-6)
        near(h, hh, 1e-6)
        for a, t in zip(got, z):
            near(a, t.grad, 5e-6)
    x, w = leaves(4, (7, 50), (50,))
    y, h = autograd.block_norm(None, x, w)
    assert torch.equal(y, x)
    h.sum().backward()                                                  # a broadcast gradient; none by y
    z = [t.detach().double().requires_grad_() for t in (x, w)]
    (unit(z[0], 1e-6) * z[1]).sum().backward()
    near(x.grad, z[0].grad, 1e-5)
    near(w.grad, z[1].grad, 1e-5)
    x.grad = w.grad = None
    y, h = autograd.block_norm(None, x, w)
    (y * 2).sum().backward()                                            # none by h
    assert bool((x.grad == 2).all()) and bool((w.grad == 0).all())
    mixed = autograd.block_norm(x.detach().bfloat16(), x.detach(), dtype=torch.float32)
    assert mixed[0].dtype == torch.float32 and mixed[1].dtype == torch.bfloat16


def test_embedding_function():
    import torch

    from paper_2410_15526_amd import autograd
    table, = leaves(5, (50, 33))
    ids = torch.tensor([3, 49, -1, 3, 0, 3, 17], device="cuda")
    out = autograd.embedding(ids, table, 2.0)
    w = torch.randn_like(out)
    (out * w).sum().backward()
    want = torch.zeros(50, 33, device="cuda", dtype=torch.float64)
    for i, t in enumerate(ids.tolist()):
        if t >= 0:
            want[t] += 2.0 * w[i].double()
    near(table.grad, want, 1e-6)
    assert torch.equal(out[0], 2 * table[3]) and bool((out[2] == 0).all())
    half = autograd.embedding(ids, table, 1.0, torch.bfloat16)
    assert half.dtype == torch.bfloat16 and torch.equal(half[1], table[49].bfloat16())


@pytest.mark.parametrize("name", ["attention", "block_norm", "embedding"])
def test_gradients_of_gradients_are_refused(name):
    import torch

    from paper_2410_15526_amd import autograd
    x, = leaves(6, (8, 2, 16))
    f = {"attention": lambda: autograd.attention(x, x, x), "block_norm": lambda: autograd.block_norm(None, x.view(8, 32))[1],
         "embedding": lambda: autograd.embedding(torch.arange(8, device="cuda"), x.view(8, 32))}[name]
    g, = torch.autograd.grad((f() ** 2).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()


def test_under_another_default_type():
    import torch

    from paper_2410_15526_amd import autograd
    x, w = leaves(7, (6, 2, 16), (32,))
    ids = torch.arange(6, device="cuda") % 3
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float64)
    try:
        y = autograd.attention(x, x, x).view(6, 32)
        y, h = autograd.block_norm(y, y.detach(), w, post_weight=w, post_eps=1e-6)
        e = autograd.embedding(ids, h[:3])
        e.sum().backward()
    finally:
        torch.set_default_dtype(before)
    assert bool(torch.isfinite(x.grad).all()) and bool(torch.isfinite(w.grad).all())


def plain_loss(model, tokens, targets, weights):
    """The model with norms behind its blocks in float32 with elementary torch operations, without dropout."""
    import torch
    c = model.cfg
    rows, d = tokens.numel(), c.hidden // c.heads
    norm = lambda v, e=1e-6: v * torch.rsqrt((v * v).mean(-1, keepdim=True) + e)  # noqa: E731
    pos = torch.arange(c.seq, device="cuda").repeat(tokens.shape[0])
    cos, sin = model.table[pos][:, None, :d // 2], model.table[pos][:, None, d // 2:]
    rot = lambda u: torch.cat([u[..., :d // 2] * cos - u[..., d // 2:] * sin,  # noqa: E731
                               u[..., d // 2:] * cos + u[..., :d // 2] * sin], -1)
    x = weights["embed"][tokens.reshape(-1)]
    for i in range(c.layers):
        w = {k[len(f"{i}."):]: v for k, v in weights.items() if k.startswith(f"{i}.")}
        qkv = (norm(x) @ w["qkv"].t()).view(rows, 3 * c.heads, d)
        q, k = rot(norm(qkv[:, :c.heads]) * w["q_norm"]), rot(norm(qkv[:, c.heads:2 * c.heads]) * w["k_norm"])
        q, k, v = (t.reshape(-1, c.seq, c.heads, d).transpose(1, 2) for t in (q, k, qkv[:, 2 * c.heads:]))
        a = torch.softmax(q @ k.transpose(2, 3) * d ** -0.5 + model.mask, -1) @ v
        x = x + norm(a.transpose(1, 2).reshape(rows, c.hidden) @ w["out"].t() + w["out_bias"]) * w["attention_norm"]
        x = x + norm(torch.nn.functional.gelu(norm(x) @ w["up"].t()) @ w["down"].t() + w["down_bias"]) * w["mlp_norm"]
    z = (norm(x) @ weights["embed"].t())[:, :c.vocab]
    return torch.nn.functional.cross_entropy(z, targets.reshape(-1))


def test_decoder_with_norms_behind_its_blocks():
    """Gradients of every weight against float32, to the same 30 roundings of 2^-9 as the decoder without these norms."""
    import torch

    from paper_2410_15526_amd.decoder import Config, Decoder, sequences
    model = Decoder(Config(batch=4, post_norm=True), seed=3)
    assert any(k.endswith("mlp_norm") for k in model.weights)
    tokens, targets = sequences(model.cfg, 4, 0)
    loss = model.backward(tokens, targets, p=0.0)
    want_leaves = {k: v.detach().float().requires_grad_() for k, v in model.weights.items()}
    want = plain_loss(model, tokens, targets, want_leaves)
    want.backward()
    assert abs(float(loss) - float(want.detach())) < 0.02 * float(want.detach())
    for k, v in want_leaves.items():
        rel = float((model.grads[k] - v.grad).norm() / v.grad.norm())
        assert rel < 0.06, (k, rel)
    again = {k: v.clone() for k, v in model.grads.items()}
    model.backward(tokens, targets, p=0.0)
    assert all(torch.equal(model.grads[k], v) for k, v in again.items())       # the embedding's too: one order of sums
    losses = [float(model.step(tokens, targets)) for _ in range(3)]
    assert all(x == x for x in losses)
