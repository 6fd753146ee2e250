"""Training-step operators without a GPU: the 64-bit forms the GPU tests
compare with, and the library's refusals (these calls never launch)."""
import ctypes as C
import math

import numpy as np
import pytest

import oracle
from paper_2410_15526_amd import sdp4
from tests import _step as ref

OK, EINVAL, EALIGN = 0, 1, 2
A = 0x7F0000000000          # made-up device addresses (never dereferenced)
B, D, E, F, W = (A + (i << 32) for i in range(1, 6))


def test_generator_is_the_oracles():
    """The mask draws the uniforms that stochastic rounding draws: with x * inv = 0.5 the rounded code is
    floor(0.5 + u), 1 exactly where u >= 1/2."""
    n, seed, offset = 4096, 0x0123456789ABCDEF, 8 * 12345
    x = np.full(n, 0.5, np.float32)
    x[::128] = 127.0                                   # the group's largest: inv = 1
    codes = np.ascontiguousarray(oracle.grad_quant_sr(x, 8, 0, 128, seed, offset)[0]).view(np.int8)
    keep, scale = ref.keep_mask(1, n, 0.5, seed, offset)
    assert scale == 2.0
    sel = np.arange(n) % 128 != 0
    assert np.array_equal(codes[sel] == 1, keep[0][sel])


def test_keep_mask_pieces_and_rows():
    whole, _ = ref.keep_mask(5, 13, 0.3, 99, 800)
    for r in range(5):
        assert np.array_equal(ref.keep_mask(1, 13, 0.3, 99, 800 + 16 * r)[0][0], whole[r])


def test_plain_token_forms_agree_with_torch():
    torch = pytest.importorskip("torch")
    r = np.random.default_rng(1)
    x = r.standard_normal((6, 40)) * 3
    t = np.array([0, 39, -100, 7, 7, 3])
    gs = [r.standard_normal(6) for _ in range(3)]
    logp, lse, ent = ref.token_stats(x, t)
    z = torch.tensor(x, requires_grad=True)
    lq = torch.log_softmax(z, 1)
    h = -(lq.exp() * lq).sum(1)
    s = torch.logsumexp(z, 1)
    tt = torch.tensor(t)
    lp = torch.where(tt >= 0, lq.gather(1, tt.clamp(min=0)[:, None])[:, 0], 0.0)
    for a, b in ((lp, logp), (s, lse), (h, ent)):
        assert np.allclose(a.detach().numpy(), b, rtol=1e-12, atol=1e-12)
    sum((g * torch.tensor(w)).sum() for g, w in zip((lp, h, s), gs)).backward()
    d, _ = ref.token_grad(x, t, ent, *gs, 40, "f32")
    assert np.allclose(z.grad.numpy(), d, rtol=1e-10, atol=1e-12)


@pytest.mark.parametrize("inter", [False, True])
def test_plain_qk_gradient_agrees_with_torch(inter):
    torch = pytest.importorskip("torch")
    r = np.random.default_rng(2)
    x, w, dy = r.standard_normal((5, 2, 12)), r.standard_normal(12), r.standard_normal((5, 2, 12))
    ang = np.arange(5)[:, None] * np.array([1.0, 0.3, 0.1, 0.01])
    tab, pos = np.concatenate([np.cos(ang), np.sin(ang)], 1), np.array([4, 0, 2, 2, 1])
    z, v = torch.tensor(x, requires_grad=True), torch.tensor(w, requires_grad=True)
    u = z * torch.rsqrt((z * z).mean(-1, keepdim=True) + 1e-5) * v
    c, s = torch.tensor(tab[pos][:, None, :4]), torch.tensor(tab[pos][:, None, 4:])
    a, b = (u[..., 0:8:2], u[..., 1:8:2]) if inter else (u[..., :4], u[..., 4:8])
    pair = [a * c - b * s, b * c + a * s]
    rot = torch.stack(pair, -1).flatten(-2) if inter else torch.cat(pair, -1)
    y = torch.cat([rot, u[..., 8:]], -1)
    assert np.allclose(ref.qk(x, w, 1e-5, tab, pos, inter, "f32")[0], y.detach().numpy(), rtol=1e-12)
    (y * torch.tensor(dy)).sum().backward()
    (dx, _), (dw, _) = ref.qk_grad(dy, x, w, 1e-5, tab, pos, inter, "f32")
    assert np.allclose(dx, z.grad.numpy(), rtol=1e-10) and np.allclose(dw, v.grad.numpy(), rtol=1e-10)


# ---------------------------------------------------------------------------
# refusals
# ---------------------------------------------------------------------------
def dropout(x=A, xt=0, xs=64, bias=None, res=B, rs=64, rows=4, cols=64, p=0.1, offset=0, y=D, yt=0, ys=64):
    return sdp4.lib().sdp4_dropout_add(x, xt, xs, bias, res, rs, rows, cols, p, 1, offset, y, yt, ys, None)


@pytest.mark.cpu_only
@pytest.mark.parametrize("kw,want", [
    (dict(xt=2), EINVAL), (dict(yt=-1), EINVAL), (dict(rows=-1), EINVAL), (dict(cols=-1), EINVAL), (dict(p=-0.1), EINVAL),
    (dict(p=1.01), EINVAL), (dict(p=math.nan), EINVAL), (dict(offset=4), EALIGN), (dict(xs=63), EINVAL), (dict(ys=0), EINVAL),
    (dict(rs=-64), EINVAL), (dict(x=None), EINVAL), (dict(y=None), EINVAL), (dict(x=A + 2), EALIGN), (dict(y=D + 1, yt=1, res=None), EALIGN),
    (dict(bias=E + 2), EALIGN), (dict(res=B + 2), EALIGN), (dict(y=A + 4), EINVAL), (dict(y=A, yt=1, res=None), EINVAL),
    (dict(y=B + 128), EINVAL), (dict(bias=D + 64), EINVAL), (dict(rows=1 << 40, cols=1 << 20, xs=1 << 20, ys=1 << 20, rs=1 << 20), EINVAL),
    (dict(cols=1 << 31, rows=1), EINVAL), (dict(rows=2, xs=1 << 60), EINVAL), (dict(rows=0), OK), (dict(cols=0, x=None, y=None, res=None), OK),
    (dict(xs=100, ys=100, y=A + 4 * 30, res=None), EINVAL),
])
def test_dropout_add_refusals(kw, want):
    assert dropout(**kw) == want


def dropout_grad(dy=A, yt=0, ys=64, rows=4, cols=64, p=0.1, offset=0, dx=B, xt=0, xs=64, db=D, ws=W, nb=1 << 20):
    return sdp4.lib().sdp4_dropout_add_grad(dy, yt, ys, rows, cols, p, 1, offset, dx, xt, xs, db, ws, nb, None)


@pytest.mark.cpu_only
@pytest.mark.parametrize("kw,want", [
    (dict(xt=3), EINVAL), (dict(p=2.0), EINVAL), (dict(offset=1), EALIGN), (dict(ys=1), EINVAL), (dict(dy=None), EINVAL),
    (dict(dx=None), EINVAL), (dict(db=D + 2), EALIGN), (dict(ws=None), EINVAL), (dict(nb=64), EINVAL), (dict(ws=W + 8), EALIGN),
    (dict(dx=A + 4), EINVAL), (dict(dx=A + 4, db=None), EINVAL), (dict(db=A), EINVAL), (dict(ws=A), EINVAL), (dict(ws=B), EINVAL),
    (dict(ws=D), EINVAL), (dict(db=B), EINVAL), (dict(cols=0), OK), (dict(rows=0, db=None), OK),
])
def test_dropout_grad_refusals(kw, want):
    assert dropout_grad(**kw) == want


def logprob(x=A, dt=0, stride=128, rows=4, vocab=100, t=B, k=3, lp=D, ls=D + 64, en=D + 128, tl=E, ti=F, ws=W, nb=1 << 20):
    return sdp4.lib().sdp4_token_logprob(x, dt, stride, rows, vocab, t, k, lp, ls, en, tl, ti, ws, nb, None)


@pytest.mark.cpu_only
@pytest.mark.parametrize("kw,want", [
    (dict(dt=5), EINVAL), (dict(stride=99), EINVAL), (dict(rows=-1), EINVAL), (dict(vocab=0), EINVAL),
    (dict(vocab=(1 << 20) + 1, stride=1 << 21), EINVAL), (dict(k=33), EINVAL), (dict(k=-1), EINVAL), (dict(k=3, vocab=2), EINVAL),
    (dict(t=None), EINVAL), (dict(x=None), EINVAL), (dict(x=A + 2), EALIGN), (dict(t=B + 4), EALIGN), (dict(tl=None), EINVAL),
    (dict(ti=None), EINVAL), (dict(ti=F + 4), EALIGN), (dict(lp=D + 1), EALIGN), (dict(ls=D + 4), EINVAL), (dict(lp=A + 40), EINVAL),
    (dict(tl=B), EINVAL), (dict(ti=E), EINVAL), (dict(rows=0), OK),
    (dict(vocab=50000, stride=50000, ws=None), EINVAL), (dict(vocab=50000, stride=50000, nb=100), EINVAL),
    (dict(vocab=50000, stride=50000, ws=W + 4), EALIGN), (dict(vocab=50000, stride=50000, ws=A), EINVAL),
])
def test_token_logprob_refusals(kw, want):
    assert logprob(**kw) == want


def grad(x=A, dt=0, stride=128, rows=4, vocab=100, t=B, ls=D, en=D + 64, g=(E, E + 64, E + 128), d=F, ds=128, width=128):
    return sdp4.lib().sdp4_token_logprob_grad(x, dt, stride, rows, vocab, t, ls, en, *g, d, ds, width, None)


def loss(x=A, dt=0, stride=128, rows=4, vocab=100, t=B, g=(E, E + 64, E + 128), lp=D, ls=D + 64, en=D + 128, d=F, ds=128,
         width=128, ws=W, nb=1 << 20):
    return sdp4.lib().sdp4_token_loss(x, dt, stride, rows, vocab, t, *g, lp, ls, en, d, ds, width, ws, nb, None)


@pytest.mark.cpu_only
@pytest.mark.parametrize("call", [grad, loss])
@pytest.mark.parametrize("kw,want", [
    (dict(dt=9), EINVAL), (dict(stride=64), EINVAL), (dict(width=99), EINVAL), (dict(ds=127), EINVAL), (dict(d=None), EINVAL),
    (dict(t=None), EINVAL), (dict(d=F + 2), EALIGN), (dict(g=(E + 2, None, None)), EALIGN), (dict(d=A + 4), EINVAL),
    (dict(d=A, ds=130), EINVAL), (dict(d=E), EINVAL), (dict(ls=None), EINVAL), (dict(en=None), EINVAL), (dict(ls=D + 66), EALIGN),
    (dict(ls=F + 16), EINVAL), (dict(vocab=0), EINVAL), (dict(rows=0), OK), (dict(d=B), EINVAL),
])
def test_token_grad_and_loss_refusals(call, kw, want):
    assert call(**kw) == want


@pytest.mark.cpu_only
def test_token_loss_workspace_refusals():
    big = dict(vocab=50000, stride=50000, width=50000, ds=50000)
    assert loss(ws=None, **big) == EINVAL and loss(nb=1, **big) == EINVAL and loss(ws=W + 2, **big) == EALIGN
    assert loss(ws=A, **big) == EINVAL and loss(ls=D, **big) == EINVAL


def heads(p, ts, hs, h):
    return sdp4.Heads(p, ts, hs, h)


def params(dt=0, dim=64, norm=1, eps=1e-6, qw=None, kw=None, table=W, rows=100, rot=64, inter=0, pos=None):
    return sdp4.QkParams(dt, dim, norm, eps, qw, kw, table, rows, rot, inter, pos)


def qk(q=(A, 512, 64, 4), k=(B, 512, 64, 2), qo=(D, 256, 64, 4), ko=(E, 128, 64, 2), tokens=8, prm=None, **kw):
    hs = [None if h is None else heads(*h) for h in (q, k, qo, ko)]
    prm = params(**kw) if prm is None else prm
    a = [None if h is None else C.addressof(h) for h in hs]
    return sdp4.lib().sdp4_qk_norm_rope(a[0], a[1], C.addressof(prm), tokens, a[2], a[3], None)


@pytest.mark.cpu_only
@pytest.mark.parametrize("kw,want", [
    (dict(dt=2), EINVAL), (dict(dim=0), EINVAL), (dict(dim=513), EINVAL), (dict(rot=3), EINVAL), (dict(rot=66), EINVAL),
    (dict(rot=-2), EINVAL), (dict(table=None), EINVAL), (dict(rows=0), EINVAL), (dict(eps=-1.0), EINVAL), (dict(eps=math.inf), EINVAL),
    (dict(eps=math.nan), EINVAL), (dict(norm=0, qw=F), EINVAL), (dict(table=W + 2), EALIGN), (dict(pos=F + 4), EALIGN),
    (dict(qw=F + 2), EALIGN), (dict(tokens=-1), EINVAL), (dict(q=None), EINVAL), (dict(qo=None), EINVAL), (dict(k=None), EINVAL),
    (dict(ko=None), EINVAL), (dict(qo=(D, 256, 64, 3)), EINVAL), (dict(q=(None, 512, 64, 4)), EINVAL), (dict(q=(A + 2, 512, 64, 4)), EALIGN),
    (dict(q=(A, 512, 63, 4)), EINVAL), (dict(q=(A, 100, 64, 4)), EINVAL), (dict(q=(A, 64, -64, 4)), EINVAL),
    (dict(q=(A, 512, 64, 0), qo=(D, 256, 64, 0)), EINVAL), (dict(qo=(A + 4, 512, 64, 4)), EINVAL), (dict(qo=(B, 256, 64, 4)), EINVAL),
    (dict(qo=(E, 256, 64, 4)), EINVAL), (dict(qo=(W, 256, 64, 4)), EINVAL), (dict(qo=(A + 4 * 128, 512, 64, 4)), EINVAL),
    (dict(tokens=0), OK), (dict(tokens=0, q=(None, 0, 0, 4)), OK),
])
def test_qk_refusals(kw, want):
    assert qk(**kw) == want


def qk_grad(gq=(A, 256, 64, 4), q=(B, 256, 64, 4), dq=(D, 256, 64, 4), w=None, ws=W + 4096 * 64, nb=1 << 20, tokens=8, **kw):
    hs = [None if h is None else heads(*h) for h in (gq, q, dq)]
    prm = params(**kw)
    a = [None if h is None else C.addressof(h) for h in hs]
    return sdp4.lib().sdp4_qk_norm_rope_grad(a[0], None, a[1], None, C.addressof(prm), tokens, a[2], None, w, None, ws, nb, None)


@pytest.mark.cpu_only
@pytest.mark.parametrize("kw,want", [
    (dict(gq=None), EINVAL), (dict(dq=None), EINVAL), (dict(q=None), EINVAL), (dict(w=E), EINVAL), (dict(w=E + 2, qw=F), EALIGN),
    (dict(w=E, qw=F, ws=None), EINVAL), (dict(w=E, qw=F, nb=16), EINVAL), (dict(w=E, qw=F, ws=W + 4096 * 64 + 4), EALIGN),
    (dict(w=F, qw=F), EINVAL), (dict(w=E, qw=F, ws=A), EINVAL), (dict(w=A, qw=F), EINVAL), (dict(dq=(A + 8, 256, 64, 4)), EINVAL),
    (dict(dq=(B + 8, 256, 64, 4)), EINVAL), (dict(q=(B, 256, 64, 3)), EINVAL), (dict(norm=0, w=E), EINVAL), (dict(tokens=0), OK),
])
def test_qk_grad_refusals(kw, want):
    assert qk_grad(**kw) == want


@pytest.mark.cpu_only
def test_rope_table_refusals():
    f = sdp4.lib().sdp4_rope_table
    assert f(A, 0, 0, 4, 1.0, B, None) == EINVAL and f(A, 257, 0, 4, 1.0, B, None) == EINVAL
    assert f(A, 8, -1, 4, 1.0, B, None) == EINVAL and f(A, 8, 0, -4, 1.0, B, None) == EINVAL
    assert f(A, 8, 0, 4, math.inf, B, None) == EINVAL and f(None, 8, 0, 4, 1.0, B, None) == EINVAL
    assert f(A + 4, 8, 0, 4, 1.0, B, None) == EALIGN and f(A, 8, 0, 4, 1.0, B + 2, None) == EALIGN
    assert f(A, 8, 0, 4, 1.0, A + 32, None) == EINVAL and f(None, 8, 0, 0, 1.0, None, None) == OK


@pytest.mark.cpu_only
def test_workspace_helpers():
    L = sdp4.lib()
    assert L.sdp4_dropout_grad_workspace(-1, 8) == -1 and L.sdp4_dropout_grad_workspace(8, 1 << 31) == -1
    assert L.sdp4_dropout_grad_workspace(0, 8) == 0 and L.sdp4_dropout_grad_workspace(8192, 5120) > 0
    assert L.sdp4_token_logprob_workspace(4, 0, 0) == -1 and L.sdp4_token_logprob_workspace(4, 10, 33) == -1
    assert L.sdp4_token_logprob_workspace(4, (1 << 20) + 1, 0) == -1 and L.sdp4_token_logprob_workspace(1, 1 << 20, 32) > 0
    assert L.sdp4_qk_grad_workspace(-1, 1, 1, 64) == -1 and L.sdp4_qk_grad_workspace(8, 1, 1, 0) == -1
    assert L.sdp4_qk_grad_workspace(0, 4, 4, 64) == 0 and L.sdp4_qk_grad_workspace(8192, 40, 8, 128) > 0


@pytest.mark.cpu_only
def test_token_workspace_serves_fewer_rows():
    """What the helper names never falls with more rows, whatever the rows' split."""
    f = sdp4.lib().sdp4_token_logprob_workspace
    for vocab in (1, 300, 513, 1000, 2049, 4096, 4097, 9001, 50001, 131072, 300007, 1 << 20):
        for k in (0, 3):
            sizes = [f(rows, vocab, min(k, vocab)) for rows in range(1, 4200)]
            assert sizes == sorted(sizes), (vocab, k)
            assert f(100000, vocab, min(k, vocab)) >= sizes[-1]


@pytest.mark.cpu_only
@pytest.mark.parametrize("qo,ko", [(A + 4 * 32, E), (A + 4 * 64, E), (A + 4 * 129, E), (A + 4 * 192, E), (D, A), (D, A + 4),
                                   (A, A + 4 * 63), (A, A), (A - 4 * 63, A + 4 * 64)])
@pytest.mark.parametrize("heads_first", [False, True])
def test_qk_refuses_overlap_inside_packed_heads(qo, ko, heads_first):
    """Query, key and value of each head side by side (64 elements each, four heads, eight tokens)."""
    strides = (192, 8 * 192) if heads_first else (4 * 192, 192)
    f = [(p, *strides, 4) for p in (A, A + 4 * 64, qo, ko)]
    assert qk(q=f[0], k=f[1], qo=f[2], ko=f[3]) == EINVAL
