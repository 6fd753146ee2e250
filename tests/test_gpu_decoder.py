"""The small decoder: its gradients against torch's own in float32, and that
it learns through both quantized paths."""
import pytest

pytestmark = pytest.mark.gpu


def plain_loss(model, tokens, targets, weights):
    """The same model in float32 with elementary torch operations, without dropout."""
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
        x = x + a.transpose(1, 2).reshape(rows, c.hidden) @ w["out"].t() + w["out_bias"]
        x = x + torch.nn.functional.gelu(norm(x) @ w["up"].t()) @ w["down"].t() + w["down_bias"]
    z = (norm(x) @ weights["embed"].t())[:, :c.vocab]
    t = targets.reshape(-1)
    keep = t >= 0
    return -(torch.log_softmax(z, 1).gather(1, t.clamp(min=0)[:, None])[:, 0] * keep).sum() / keep.sum()


def test_gradients_against_float32():
    """bfloat16 activations round each product's result by 2^-8 of it at most
    and 2^-9 on the whole; over the 30 or so roundings along a gradient's way
    the relative error of a whole weight's gradient stays below 30 * 2^-9 = 6 %."""
    import torch

    from paper_2410_15526_amd.decoder import Config, Decoder, sequences
    model = Decoder(Config(batch=4), seed=3)
    tokens, targets = sequences(model.cfg, 4, 0)
    targets[0, :5] = -1
    loss = model.backward(tokens, targets, p=0.0)
    leaves = {k: v.detach().float().requires_grad_() for k, v in model.weights.items()}
    want = plain_loss(model, tokens, targets, leaves)
    want.backward()
    assert abs(float(loss) - float(want.detach())) < 0.02 * float(want.detach())
    for k, v in leaves.items():
        got = model.grads[k]
        rel = float((got - v.grad).norm() / v.grad.norm())
        assert rel < 0.06, (k, rel)
    assert bool((model.grads["embed"][model.cfg.vocab:] == 0).all())          # the padding takes no gradient
    again = {k: v.clone() for k, v in model.grads.items()}
    model.backward(tokens, targets, p=0.0)
    del again["embed"]                                                        # torch adds up its rows in any order
    assert all(torch.equal(model.grads[k], v) for k, v in again.items())


def test_learns_through_both_quantized_paths():
    import torch

    from paper_2410_15526_amd.decoder import Decoder, sequences
    model = Decoder()
    first = [float(model.step(*sequences(model.cfg, model.cfg.batch, i))) for i in range(3)]
    for i in range(3, 117):
        model.step(*sequences(model.cfg, model.cfg.batch, i))
    last = [float(model.step(*sequences(model.cfg, model.cfg.batch, i))) for i in range(117, 120)]
    print(first, last, flush=True)
    assert min(first) > 6.0                                                   # log 1000 = 6.9
    assert max(last) < 3.0
    # the model weights follow the main weights to a step of the 4-bit differences
    assert float((model.path.w_prev.float() - model.path.w_new).abs().mean()) < 2e-3
    assert bool(torch.isfinite(model.path.w_new).all())


def test_autograd_functions():
    import torch

    from paper_2410_15526_amd import autograd
    g = torch.Generator(device="cuda").manual_seed(0)
    n = lambda *s: torch.randn(*s, device="cuda", generator=g).requires_grad_()  # noqa: E731
    x, b, r = n(37, 50), n(50), n(37, 50)
    y = autograd.dropout_add(x, b, r, 0.25, 5, 8)
    kept = (y - r).detach() != 0
    (y * y.detach()).sum().backward()
    want = torch.where(kept, y.detach() / 0.75, 0.0)
    assert torch.allclose(x.grad, want, rtol=1e-5, atol=1e-6) and torch.equal(r.grad, y.detach())
    assert torch.allclose(b.grad, want.sum(0), rtol=1e-4, atol=1e-4)
    z, t = n(9, 70), torch.randint(0, 64, (9,), device="cuda", generator=g)
    logp, lse, ent = autograd.token_logprob(z, t, 64)
    (2 * logp + lse - ent).sum().backward()
    got = z.grad.clone()
    z.grad = None
    lq = torch.log_softmax(z[:, :64], 1)
    (2 * lq.gather(1, t[:, None])[:, 0] + torch.logsumexp(z[:, :64], 1) + (lq.exp() * lq).sum(1)).sum().backward()
    assert torch.allclose(got, z.grad, rtol=1e-4, atol=1e-5)
    loss, d = autograd.token_loss(z.detach(), t, torch.full((9,), 1 / 9, device="cuda"), 64)
    z.grad = None
    want = torch.nn.functional.cross_entropy(z[:, :64], t)
    want.backward()
    assert torch.allclose(loss, want, rtol=1e-5) and torch.allclose(d, z.grad, rtol=1e-4, atol=1e-6)
    q, k, w = n(6, 3, 16), n(6, 2, 16), n(16)
    tab = autograd.rope_table(6, 16, stretch=4.0, ramp=(1.0, 4.0, 64))
    qo, ko = autograd.qk_norm_rope(q, k, w, w, 1e-6, tab, None)
    (qo.sum() + (ko * ko).sum()).backward()
    assert all(bool(torch.isfinite(v.grad).all()) for v in (q, k, w))
    wide = n(4, 1)                                                            # gradients that arrive broadcast
    autograd.dropout_add(wide.expand(4, 30), None, None, 0.0, 1, 0).sum().backward()
    assert torch.equal(wide.grad, torch.full((4, 1), 30.0, device="cuda"))
    u = q * torch.rsqrt((q * q).mean(-1, keepdim=True) + 1e-6) * w
    assert torch.allclose(qo.norm(dim=-1), u.norm(dim=-1), rtol=1e-5)         # a rotation keeps lengths


def test_rope_table_rules():
    import torch

    from paper_2410_15526_amd import autograd
    ang = lambda t: torch.atan2(t[1, 8:], t[1, :8]).double().cpu()  # noqa: E731
    inv = 10000.0 ** (-torch.arange(8, dtype=torch.float64) / 8)
    assert torch.allclose(ang(autograd.rope_table(2, 16)), inv, rtol=1e-6)
    assert torch.allclose(ang(autograd.rope_table(2, 16, stretch=8.0)), inv / 8, rtol=1e-6)
    got = ang(autograd.rope_table(2, 16, stretch=8.0, ramp=(1.0, 32.0, 2048)))
    turns = 2048 * inv / (2 * torch.pi)
    assert torch.allclose(got[turns > 32], inv[turns > 32], rtol=1e-6)
    assert torch.allclose(got[turns < 1], inv[turns < 1] / 8, rtol=1e-6)
    mid = (turns > 1) & (turns < 32)
    assert bool(mid.any()) and bool((got[mid] < inv[mid]).all()) and bool((got[mid] > inv[mid] / 8).all())
    assert torch.allclose(autograd.rope_table(3, 8, scale=0.5)[0, :4], torch.full((4,), 0.5, device="cuda"))


def test_loss_of_transposed_logits():
    import torch

    from paper_2410_15526_amd import autograd
    g = torch.Generator(device="cuda").manual_seed(1)
    z = torch.randn(70, 9, device="cuda", generator=g)
    t = torch.randint(0, 64, (9,), device="cuda", generator=g)
    w = torch.rand(9, 2, device="cuda", generator=g)[:, 0]
    got, want = (autograd.token_loss(x, t, w, 64) for x in (z.T, z.T.contiguous()))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("name", ["dropout_add", "token_logprob", "qk_norm_rope"])
def test_gradients_of_gradients_are_refused(name):
    import torch

    from paper_2410_15526_amd import autograd
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(6, 4, 16, device="cuda", generator=g).requires_grad_()
    if name == "dropout_add":
        y = autograd.dropout_add(x.view(24, 16), None, None, 0.5, 1, 0)
    elif name == "token_logprob":
        y = autograd.token_logprob(x.view(24, 16), torch.zeros(24, dtype=torch.int64, device="cuda"))[1]
    else:
        y = autograd.qk_norm_rope(x, x, None, None, 1e-6, None, None)[0]
    dx, = torch.autograd.grad((y * y).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        (dx.square().sum() + x.sum()).backward()
