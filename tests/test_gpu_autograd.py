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
