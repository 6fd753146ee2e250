"""The torch functions of the training-step operators: arguments as programs
have them, and no more work than their gradients need."""
import pytest

pytestmark = pytest.mark.gpu


def generator(seed=0):
    import torch
    return torch.Generator(device="cuda").manual_seed(seed)


def test_strided_and_broadcast_vectors():
    """Biases, weights, targets, positions and tables that are columns, rows of other layouts or broadcast give what their
    copies give, gradients included."""
    import torch

    from paper_2410_15526_amd import autograd
    g = generator()
    n = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731

    def both(call, *args):
        """Results and gradients of the arguments as they are and as contiguous copies."""
        out = []
        for dense in (False, True):
            leaves = [(a.clone(memory_format=torch.contiguous_format) if dense else a.detach()) for a in args]
            leaves = [a.requires_grad_() if a.is_floating_point() else a for a in leaves]
            y = call(*leaves)
            y = y if isinstance(y, tuple) else (y,)
            sum((v * v).sum() for v in y).backward()
            out.append([v.detach() for v in y] + [a.grad for a in leaves if a.is_floating_point()])
        for a, b in zip(*out):
            assert torch.equal(a, b)
    x, r = n(12, 40), n(12, 40)
    for bias in (n(40, 3)[:, 1], n(1).expand(40)):
        if bias.stride(0) == 0:                       # a broadcast leaf: its gradient adds up outside
            one = n(1).requires_grad_()
            autograd.dropout_add(x, one.expand(40), r, 0.2, 3, 8).sum().backward()
            want = n(40).requires_grad_()
            autograd.dropout_add(x, want, r, 0.2, 3, 8).sum().backward()
            assert torch.allclose(one.grad, want.grad.sum()[None], rtol=1e-5)
        else:
            both(lambda a, b: autograd.dropout_add(a, b, r, 0.2, 3, 8), x, bias)
    t = torch.randint(0, 30, (12, 5), device="cuda", generator=g)[:, 2]
    both(lambda z: autograd.token_logprob(z, t, 30), n(12, 32))
    z, w = n(12, 32), n(12, 2)[:, 0]
    got, want = (autograd.token_loss(z, a, b, 30) for a, b in ((t, w), (t.contiguous(), w.contiguous())))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    pos = torch.randint(0, 9, (6, 2), device="cuda", generator=g)[:, 1]
    tab = autograd.rope_table(9, 32)[:, :16]
    for eps in (1e-6, None):
        ws = [n(16, 2)[:, 0], n(16, 4)[:, 3]] if eps else []
        both(lambda q, k, *w: autograd.qk_norm_rope(q, k, *(w or (None, None)), eps, tab, pos), n(6, 3, 16), n(6, 2, 16), *ws)


@pytest.mark.parametrize("default", ["bfloat16", "float64"])
def test_default_types_other_than_float32(default):
    """A program whose default type is another still gets float32 statistics and sums."""
    import torch

    from paper_2410_15526_amd import autograd
    g = generator(1)
    n = lambda *s: torch.randn(*s, device="cuda", generator=g, dtype=torch.float32).requires_grad_()  # noqa: E731
    torch.set_default_dtype(getattr(torch, default))
    try:
        x, b, z, q, w = n(12, 40), n(40), n(12, 32), n(6, 3, 16), n(16)
        t = torch.randint(0, 30, (12,), device="cuda", generator=g)
        y = autograd.dropout_add(x, b, None, 0.2, 3, 8)
        stats = autograd.token_logprob(z, t, 30)
        loss, d = autograd.token_loss(z.detach(), t, torch.ones(12, device="cuda", dtype=torch.float32), 30)
        tab = autograd.rope_table(6, 16)
        qo, ko = autograd.qk_norm_rope(q, q, w, w, 1e-6, tab, None)
        sum((v * v).sum() for v in (y, *stats, qo, ko)).backward()
    finally:
        torch.set_default_dtype(torch.float32)
    for v in (y, *stats, loss, d, tab, qo, ko, x.grad, b.grad, z.grad, q.grad, w.grad):
        assert v.dtype == torch.float32 and bool(torch.isfinite(v).all())


def test_only_the_gradients_that_are_needed(monkeypatch):
    """The backward passes ask the library for no gradient by outputs that a loss does not use, and for none of arguments that
    need none; those that remain keep their values."""
    import torch

    from paper_2410_15526_amd import autograd, sdp4
    g = generator(2)
    n = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    calls = []
    for name in ("sdp4_dropout_add_grad", "sdp4_token_logprob_grad", "sdp4_qk_norm_rope_grad"):
        def seen(*a, _f=getattr(sdp4, name), _n=name, **kw):
            calls.append((_n, a))
            return _f(*a, **kw)
        monkeypatch.setattr(sdp4, name, seen)
    z, t = n(12, 32).requires_grad_(), torch.randint(0, 30, (12,), device="cuda", generator=g)
    grads = []
    for used in ((True, False, False), (False, True, False), (True, True, True)):
        z.grad = None
        out = autograd.token_logprob(z, t, 30)
        sum(v.sum() for v, u in zip(out, used) if u).backward()
        a = calls.pop()[1]
        assert [v is not None for v in (a[4], a[6], a[5])] == list(used)        # by logp, lse, entropy
        grads.append(z.grad)
    lq = torch.log_softmax(z[:, :30], 1)
    for got, want in zip(grads, (lq.gather(1, t[:, None]).sum(), torch.logsumexp(z[:, :30], 1).sum())):
        assert torch.allclose(got, torch.autograd.grad(want, z, retain_graph=True)[0], rtol=1e-4, atol=1e-5)
    q, k = n(6, 3, 16).requires_grad_(), n(6, 2, 16).requires_grad_()
    qw, kw = n(16), n(16).requires_grad_()
    tab = autograd.rope_table(6, 16)

    def run(w):
        q.grad = k.grad = kw.grad = None
        qo, ko = autograd.qk_norm_rope(q, k, w, kw, 1e-6, tab, None)
        ((qo * qo).sum() + (ko * ko).sum() + ko.sum()).backward()
        return [v.grad.clone() for v in (q, k, kw)]
    got = run(qw)
    a = calls.pop()[1]
    assert a[11] is None and a[12] is not None
    for x, y in zip(got, run(qw.clone().requires_grad_())):
        assert torch.equal(x, y)
    assert calls.pop()[1][11] is not None
    qo, _ = autograd.qk_norm_rope(q, k, qw, kw.detach(), 1e-6, tab, None)
    qo.sum().backward()
    a = calls.pop()[1]
    assert a[11] is None and a[12] is None and a[13] is None                    # no sums, no workspace
    x, b, r = n(12, 40), n(40), n(12, 40).requires_grad_()
    autograd.dropout_add(x, b, r, 0.2, 3, 8).sum().backward()
    assert not calls and torch.equal(r.grad, torch.ones_like(r))
    autograd.dropout_add(x, b.requires_grad_(), r, 0.2, 3, 8).sum().backward()
    assert calls.pop()[1][5] is not None and x.grad is None and bool((b.grad > 0).all())
