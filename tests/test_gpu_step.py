"""The training-step operators on the GPU against their 64-bit forms
(tests/_step.py), at sizes, strides, masks and values where they can go
wrong; gradients also against differences of the forward pass."""
import numpy as np
import pytest

from paper_2410_15526_amd import sdp4
from tests import _step as ref
from tests._gpu import say, torch

pytestmark = pytest.mark.gpu


def dt(name):
    return {"f32": torch().float32, "bf16": torch().bfloat16}[name]


def f64(t):
    return t.double().cpu().numpy()


def rng(*key):
    return torch().Generator(device="cuda").manual_seed(hash(tuple(key)) % (1 << 31))


def normal(g, *shape, dtype="f32", scale=1.0):
    t = torch()
    return (t.randn(*shape, device="cuda", generator=g) * scale).to(dt(dtype))


def strided(x, gap, lead=1):
    """The same matrix as a part of a wider one, at an odd offset; what lies around it is NaN."""
    t = torch()
    buf = t.full((x.shape[0], x.shape[1] + gap), float("nan"), dtype=x.dtype, device="cuda")
    v = buf[:, lead:lead + x.shape[1]]
    v.copy_(x)
    return buf, v


def scratch(n):
    return torch().full((max(n, 16),), 0xFF, dtype=torch().uint8, device="cuda")   # NaN wherever it is read as floats


def close(got, want, bound, what):
    got = f64(got) if not isinstance(got, np.ndarray) else got
    assert got.shape == want.shape, (what, got.shape, want.shape)
    same = (np.isnan(got) & np.isnan(want)) | (got == want)
    with np.errstate(invalid="ignore"):
        bad = ~(same | (np.abs(got - want) <= bound))
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError((what, "at", i, got[i], want[i], float(np.asarray(bound)[i] if np.ndim(bound) else bound),
                              int(bad.sum())))


# ---------------------------------------------------------------------------
# dropout
# ---------------------------------------------------------------------------
SHAPES = [(1, 1), (1, 7), (3, 8), (1, 768), (5, 63), (17, 64), (2, 129), (33, 1000), (64, 2048), (257, 515), (9, 4097),
          (1030, 40)]


@pytest.mark.parametrize("x_dtype,y_dtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_dropout_add(rows, cols, x_dtype, y_dtype):
    t = torch()
    say("dropout_add", rows, cols, x_dtype, y_dtype)
    g = rng(rows, cols, 1)
    x, b, r = normal(g, rows, cols, dtype=x_dtype), normal(g, cols, dtype=x_dtype), normal(g, rows, cols, dtype=y_dtype)
    for p, bias, res, offset in ((0.1, b, r, 0), (0.5, None, r, 8 * ((1 << 40) + 3)), (0.9, b, None, 1 << 35), (0.3, None, None, 8)):
        y = t.full((rows, cols), float("nan"), dtype=dt(y_dtype), device="cuda")
        sdp4.sdp4_dropout_add(x, bias, res, p, 0xFEDCBA9876543210, offset, y)
        want, bound = ref.dropout_add(f64(x), None if bias is None else f64(bias), None if res is None else f64(res), p,
                                      0xFEDCBA9876543210, offset, y_dtype)
        close(y, want, bound, ("y", p))


@pytest.mark.parametrize("x_dtype,y_dtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("rows,cols", SHAPES + [(4099, 96)])
def test_dropout_add_grad(rows, cols, x_dtype, y_dtype):
    t = torch()
    say("dropout_add_grad", rows, cols, x_dtype, y_dtype)
    dy = normal(rng(rows, cols, 2), rows, cols, dtype=y_dtype)
    for p, with_bias in ((0.1, True), (0.0, True), (0.25, False)):
        dx = t.full((rows, cols), float("nan"), dtype=dt(x_dtype), device="cuda")
        db = t.full((cols,), float("nan"), device="cuda") if with_bias else None
        ws = scratch(sdp4.sdp4_dropout_grad_workspace(rows, cols)) if with_bias else None
        sdp4.sdp4_dropout_add_grad(dy, p, 7, 16, dx, db, ws)
        (want, bound), (wb, bb) = ref.dropout_grad(f64(dy), p, 7, 16, x_dtype)
        close(dx, want, bound, ("dx", p))
        if with_bias:
            close(db, wb, bb, ("dbias", p))


def test_dropout_strides_in_place_and_surroundings():
    t = torch()
    g = rng(3)
    for dtype in ("f32", "bf16"):
        x, r = normal(g, 37, 203, dtype=dtype), normal(g, 37, 203, dtype=dtype)
        b = normal(g, 203, dtype=dtype)
        want, bound = ref.dropout_add(f64(x), f64(b), f64(r), 0.2, 5, 64, dtype)
        xb, xs = strided(x, 6)
        rb, rs = strided(r, 10, 3)
        yb, ys = strided(t.zeros_like(x), 4)
        sdp4.sdp4_dropout_add(xs, b, rs, 0.2, 5, 64, ys)
        close(ys, want, bound, "strided")
        assert bool(t.isnan(yb[:, :1]).all()) and bool(t.isnan(yb[:, 204:]).all())
        sdp4.sdp4_dropout_add(xs, b, rs, 0.2, 5, 64, rs)                  # into the residual
        close(rs, want, bound, "in place")
        sdp4.sdp4_dropout_add(xs, b, r, 0.2, 5, 64, xs)                   # into the input
        close(xs, want, bound, "in place of x")
        both = t.cat([x, r], 1)                                           # two halves of the same rows
        sdp4.sdp4_dropout_add(both[:, :203], b, r, 0.2, 5, 64, both[:, 203:])
        close(both[:, 203:], want, bound, "beside the input")
        (wd, bd), (wb, bb) = ref.dropout_grad(f64(r), 0.2, 5, 64, dtype)
        db, ws = t.empty(203, device="cuda"), scratch(sdp4.sdp4_dropout_grad_workspace(37, 203))
        rb, rs = strided(r, 10, 3)
        sdp4.sdp4_dropout_add_grad(rs, 0.2, 5, 64, rs, db, ws)
        close(rs, wd, bd, "dx in place")
        close(db, wb, bb, "dbias")


def test_dropout_edges():
    t = torch()
    x = t.full((4, 40), float("inf"), device="cuda")
    x[1] = float("nan")
    r = normal(rng(4), 4, 40)
    y = t.empty_like(x)
    sdp4.sdp4_dropout_add(x, None, r, 1.0, 1, 0, y)                       # all dropped, whatever it holds
    assert t.equal(y, r)
    keep, _ = ref.keep_mask(4, 40, 0.5, 9, 0)
    sdp4.sdp4_dropout_add(x, None, r, 0.5, 9, 0, y)
    got = f64(y)
    assert np.array_equal(got[~keep], f64(r)[~keep]) and not np.isfinite(got[keep]).any()
    sdp4.sdp4_dropout_add(r, None, None, 0.0, 1, 0, y)
    assert t.equal(y, r)
    e = t.empty(0, 40, device="cuda")
    sdp4.sdp4_dropout_add(e, None, None, 0.5, 1, 0, e)
    db = t.full((40,), 3.0, device="cuda")
    sdp4.sdp4_dropout_add_grad(e, 0.5, 1, 0, e, db, None)
    assert bool((db == 0).all())                                          # the sum of no rows


def test_dropout_pieces_and_rate():
    """Pieces with matching offsets draw the one call's mask; the kept share and the mean are what p says."""
    t = torch()
    x = t.ones(512, 1021, device="cuda")
    y, z = t.empty_like(x), t.empty_like(x)
    sdp4.sdp4_dropout_add(x, None, None, 0.1, 42, 0, y)
    for a, b in ((0, 100), (100, 101), (101, 512)):
        sdp4.sdp4_dropout_add(x[a:b], None, None, 0.1, 42, a * 1024, z[a:b])
    assert t.equal(y, z)
    n, kept = y.numel(), int((y > 0).sum())
    assert abs(kept - 0.9 * n) < 6 * np.sqrt(0.09 * n)
    sdp4.sdp4_dropout_add(x, None, None, 0.1, 43, 0, z)
    assert abs(int(((z > 0) & (y > 0)).sum()) - 0.81 * n) < 6 * np.sqrt(0.81 * 0.19 * n)


# ---------------------------------------------------------------------------
# token log probabilities
# ---------------------------------------------------------------------------
def check_logprob(x, targets, k, vocab=None, dtype="f32"):
    t = torch()
    rows, vocab = x.shape[0], vocab or x.shape[1]
    lp, ls, en = (t.full((rows,), 7.0, device="cuda") for _ in range(3))
    tl, ti = t.full((rows, k), 7.0, device="cuda"), t.full((rows, k), 7, dtype=t.int64, device="cuda")
    ws = scratch(sdp4.sdp4_token_logprob_workspace(rows, vocab, k))
    sdp4.sdp4_token_logprob(x, targets, k, lp, ls, en, tl, ti, ws, vocab=vocab)
    xs, tg = f64(x[:, :vocab]), targets.cpu().numpy()
    wl, we, wn = ref.token_stats(xs, tg)
    bl, be, bn = ref.stats_bounds(xs, wl, wn)
    close(ls, we, be, "lse")
    close(lp, wl, bl, "logp")
    close(en, wn, bn, "entropy")
    if k:
        ids = ref.top(xs, k)
        assert np.array_equal(ti.cpu().numpy(), ids), ("ids", np.argwhere(ti.cpu().numpy() != ids)[:4])
        want = np.take_along_axis(ref.log_probs(xs), ids, 1)
        close(tl, want, np.stack([ref.stats_bounds(xs, want[:, i], wn)[0] for i in range(k)], 1), "top")
    return lp, ls, en


VOCABS = [1, 2, 3, 7, 8, 9, 63, 65, 255, 512, 513, 1000, 4096, 4097, 5003, 16385, 50001, 131072]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", VOCABS)
def test_token_logprob(vocab, dtype):
    t = torch()
    for rows in (1, 5, 300) if vocab < 20000 else (1, 67):
        say("token_logprob", rows, vocab, dtype)
        g = rng(rows, vocab, 5)
        x = normal(g, rows, vocab, dtype=dtype, scale=3.0)
        tg = t.randint(-1, vocab, (rows,), device="cuda", generator=g)
        for k in sorted({0, 1, min(5, vocab), min(32, vocab)}):
            check_logprob(x, tg, k, dtype=dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_token_logprob_many_rows(dtype):
    t = torch()
    for rows, vocab in ((4100, 777), (2500, 9001)):
        say("token_logprob", rows, vocab, dtype)
        g = rng(rows, vocab, 6)
        x = normal(g, rows, vocab, dtype=dtype, scale=3.0)
        check_logprob(x, t.randint(-1, vocab, (rows,), device="cuda", generator=g), 7, dtype=dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_token_logprob_padding_and_strides(dtype):
    t = torch()
    for rows, vocab in ((3, 100), (40, 5003), (2, 70001)):
        g = rng(rows, vocab, 7)
        buf, x = strided(normal(g, rows, vocab, dtype=dtype, scale=2.0), 13)
        tg = t.randint(0, vocab, (rows,), device="cuda", generator=g)
        check_logprob(x, tg, 4, dtype=dtype)
        check_logprob(buf[:, 1:], tg, 4, vocab=vocab, dtype=dtype)         # NaN in the padding


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [40, 600, 5003, 40009])
def test_token_logprob_masks_and_ties(vocab, dtype):
    """Rows of one value, few allowed tokens, a type's lowest value, sorted logits, large values on few lanes."""
    t = torch()
    g = rng(vocab, 8)
    low = t.finfo(dt(dtype)).min
    rows = 12
    x = normal(g, rows, vocab, dtype=dtype, scale=2.0)
    x[0] = 0.0
    x[1] = float("-inf")
    x[2] = low
    x[3, 3:] = float("-inf")
    x[4, 1:-1] = low
    x[5] = x[5].sort().values
    x[6] = x[6].sort(descending=True).values
    x[7] = (t.arange(vocab, device="cuda") % 3).to(x.dtype)
    x[8, ::2] = float("-inf")
    x[9] = -0.0
    x[9, vocab // 2:] = 0.0
    col = t.arange(vocab, device="cuda")                        # the largest elements all on three lanes of a wave
    x[10] = t.where((col // (8 if dtype == "bf16" else 4)) % 64 < 3, x[10].abs() + 20, x[10])
    x[11] = low
    x[11, vocab - 1] = float("-inf")
    tg = t.randint(0, vocab, (rows,), device="cuda", generator=g)
    tg[3], tg[4], tg[11] = 1, 0, 0
    for k in (0, 1, 5, 32):
        check_logprob(x, tg, k, dtype=dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [500, 9000])
def test_token_logprob_nan_and_inf(vocab, dtype):
    t = torch()
    g = rng(vocab, 9)
    x = normal(g, 6, vocab, dtype=dtype)
    x[1, vocab - 1] = float("nan")
    x[2, 3] = float("inf")
    x[3, :] = float("nan")
    tg = t.zeros(6, dtype=t.int64, device="cuda")
    tg[4], tg[5] = vocab, -5                                    # a mistake, and none
    lp, ls, en = (t.zeros(6, device="cuda") for _ in range(3))
    tl, ti = t.zeros(6, 3, device="cuda"), t.zeros(6, 3, dtype=t.int64, device="cuda")
    ws = scratch(sdp4.sdp4_token_logprob_workspace(6, vocab, 3))
    sdp4.sdp4_token_logprob(x, tg, 3, lp, ls, en, tl, ti, ws)
    bad = np.array([False, True, True, True, False, False])
    for a in (ls, en, tl[:, 0], tl[:, 2]):
        assert np.array_equal(np.isnan(f64(a)), bad)
    assert np.array_equal(np.isnan(f64(lp)), bad | (np.arange(6) == 4)) and float(lp[5]) == 0
    assert bool((ti[1:4] == -1).all()) and bool((ti[4:] >= 0).all())
    d, e = t.zeros_like(x), t.zeros_like(x)
    gl, ge = t.ones(6, device="cuda"), t.ones(6, device="cuda")
    for ent in (None, ge):
        sdp4.sdp4_token_logprob_grad(x, tg, ls, en, gl, ent, None, d)
        lp2, ls2, en2 = (t.zeros(6, device="cuda") for _ in range(3))
        sdp4.sdp4_token_loss(x, tg, gl, ent, None, lp2, ls2, en2, e, ws)
        for out in (d, e):
            assert np.array_equal(np.isnan(f64(out)).all(1), bad | (np.arange(6) == 4))
            assert np.array_equal(np.isnan(f64(out)).any(1), bad | (np.arange(6) == 4))


def bound_of_lse(vocab, dtype, xs, tn, ent, gn, pad):
    """Rows beyond what one block holds take lse from memory: their p has the rounding of lse too."""
    if vocab + pad <= (131072 if dtype == "bf16" else 65536):
        return 0.0
    return ref.token_grad(xs, tn, ent, *gn, vocab + pad, dtype)[1]


def grads_for(g, rows, which):
    t = torch()
    mk = lambda: normal(g, rows, scale=0.5)  # noqa: E731
    return tuple(mk() if w else None for w in which)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", VOCABS + [140001])
def test_token_grad_and_loss(vocab, dtype):
    t = torch()
    for rows, pad, which in ((1, 0, (1, 1, 1)), (7, 5, (1, 0, 0)), (66, 64, (1, 1, 0)), (3, 1, (0, 0, 1))):
        say("token_grad", rows, vocab, dtype, pad, which)
        g = rng(rows, vocab, 10)
        x = normal(g, rows, vocab, dtype=dtype, scale=3.0)
        tg = t.randint(-1, vocab, (rows,), device="cuda", generator=g)
        gs = grads_for(g, rows, which)
        xs, tn, gn = f64(x), tg.cpu().numpy(), [None if a is None else f64(a) for a in gs]
        _, lse, ent = ref.token_stats(xs, tn)
        l32, e32 = (t.from_numpy(a).float().cuda() for a in (lse, ent))
        want, bound = ref.token_grad(xs, tn, ent, *gn, vocab + pad, dtype)
        d = t.full((rows, vocab + pad), float("nan"), dtype=dt(dtype), device="cuda")
        sdp4.sdp4_token_logprob_grad(x, tg, l32, e32, *gs, d)
        close(d, want, bound, "dlogits")
        want, bound = ref.token_grad(xs, tn, ent, *gn, vocab + pad, dtype, lse_given=False)
        d = t.full((rows, vocab + pad), float("nan"), dtype=dt(dtype), device="cuda")
        lp, ls, en = (t.full((rows,), 7.0, device="cuda") for _ in range(3))
        ws = scratch(sdp4.sdp4_token_logprob_workspace(rows, vocab))
        sdp4.sdp4_token_loss(x, tg, *gs, lp, ls, en, d, ws)
        wl, we, wn = ref.token_stats(xs, tn)
        bl, be, bn = ref.stats_bounds(xs, wl, wn)
        close(ls, we, be, "lse")
        close(lp, wl, bl, "logp")
        close(en, wn, bn, "entropy")
        close(d, want, bound + 2 * bound_of_lse(vocab, dtype, xs, tn, ent, gn, pad), "dlogits of the loss")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [9, 700, 20003])
def test_token_grad_in_place_strided_and_masked(vocab, dtype):
    t = torch()
    g = rng(vocab, 11)
    rows, pad = 8, 6
    x = normal(g, rows, vocab, dtype=dtype, scale=2.0)
    x[1] = float("-inf")
    x[2] = t.finfo(x.dtype).min
    x[3, 1:] = float("-inf")
    tg = t.randint(0, vocab, (rows,), device="cuda", generator=g)
    tg[1], tg[3], tg[5] = 0, 0, -100
    gs = grads_for(g, rows, (1, 1, 1))
    xs, tn, gn = f64(x), tg.cpu().numpy(), [f64(a) for a in gs]
    _, lse, ent = ref.token_stats(xs, tn)
    l32, e32 = (t.from_numpy(a).float().cuda() for a in (lse, ent))
    for loss in (False, True):
        want, bound = ref.token_grad(xs, tn, ent, *gn, vocab + pad, dtype, lse_given=not loss)
        if loss:
            bound = bound + 2 * bound_of_lse(vocab, dtype, xs, tn, ent, gn, pad)
        # a given logsumexp of row 2, the lowest value itself, holds no log vocab
        rows_checked = list(range(rows)) if loss else [0, 1, 3, 4, 5, 6, 7]
        buf, xs_ = strided(x, pad + 3)
        d = buf[:, 1:1 + vocab + pad]
        if loss:
            o = [t.empty(rows, device="cuda") for _ in range(3)]
            sdp4.sdp4_token_loss(xs_, tg, *gs, *o, d, scratch(sdp4.sdp4_token_logprob_workspace(rows, vocab)))
        else:
            sdp4.sdp4_token_logprob_grad(xs_, tg, l32, e32, *gs, d)
        close(d[rows_checked], want[rows_checked], bound[rows_checked], ("in place", loss))
        assert bool(t.isfinite(d).all())
        assert bool(t.isnan(buf[:, 0]).all()) and bool(t.isnan(buf[:, -2:]).all())


def test_token_gradient_against_differences():
    """sum(a logp + b entropy + c lse) by central differences of the forward pass along random directions: steps of
    2^-5, float32 values of magnitude 10 off by 1e-6 each, third derivatives below 1."""
    t = torch()
    rows, vocab, h = 6, 301, 2.0 ** -5
    g = rng(12)
    x = normal(g, rows, vocab, scale=1.5)
    tg = t.randint(0, vocab, (rows,), device="cuda", generator=g)
    gs = grads_for(g, rows, (1, 1, 1))
    ws = scratch(sdp4.sdp4_token_logprob_workspace(rows, vocab))

    def value(z):
        o = [t.empty(rows, device="cuda") for _ in range(3)]
        sdp4.sdp4_token_logprob(z, tg, 0, *o, workspace=ws)
        lp, ls, en = o
        return f64(gs[0]) * f64(lp) + f64(gs[1]) * f64(en) + f64(gs[2]) * f64(ls)
    o = [t.empty(rows, device="cuda") for _ in range(3)]
    d = t.empty_like(x)
    sdp4.sdp4_token_loss(x, tg, *gs, *o, d, ws)
    for i in range(4):
        v = normal(g, rows, vocab)
        v /= v.norm(dim=1, keepdim=True)
        num = (value(x + h * v) - value(x - h * v)) / (2 * h)
        ana = (f64(d) * f64(v)).sum(1)
        assert np.all(np.abs(num - ana) <= 2e-3 * (1 + np.abs(ana))), (num, ana)


def test_token_rows_beyond_32_bits():
    """Rows more than 2^31 elements apart."""
    t = torch()
    stride, vocab = (1 << 30) + 5, 3001
    buf = t.empty(2 * stride + vocab + 8, dtype=t.bfloat16, device="cuda")
    x = t.as_strided(buf, (3, vocab), (stride, 1))
    small = normal(rng(13), 3, vocab, dtype="bf16", scale=2.0)
    x.copy_(small)
    tg = t.tensor([5, 0, vocab - 1], device="cuda")
    check_logprob(x, tg, 5, dtype="bf16")
    outs = []
    for z in (x, small):
        o = [t.empty(3, device="cuda") for _ in range(3)]
        d = z if z is x else t.empty_like(z)
        sdp4.sdp4_token_loss(z, tg, -t.ones(3, device="cuda"), None, None, *o, d,
                             scratch(sdp4.sdp4_token_logprob_workspace(3, vocab)))
        outs.append(d.clone())
    assert t.equal(*outs)
    y = t.as_strided(buf, (3, 1001), (stride, 1))
    a = normal(rng(14), 3, 1001, dtype="bf16")
    y.copy_(a)
    z = t.empty_like(a)
    sdp4.sdp4_dropout_add(a, None, None, 0.3, 1, 0, z)
    sdp4.sdp4_dropout_add(y, None, None, 0.3, 1, 0, y)
    assert t.equal(y, z)


# ---------------------------------------------------------------------------
# norm and rotation
# ---------------------------------------------------------------------------
def table_for(rows, rot, scale=1.0):
    t = torch()
    inv = 10000.0 ** (-t.arange(rot // 2, dtype=t.float64, device="cuda") / max(rot // 2, 1))
    tab = t.empty(rows, rot, device="cuda")
    sdp4.sdp4_rope_table(inv, tab, 0, scale)
    return tab


def test_rope_table():
    t = torch()
    inv = (t.rand(24, dtype=t.float64, device="cuda", generator=rng(20))).contiguous()
    tab = t.empty(100, 48, device="cuda")
    for start, scale in ((0, 1.0), (1 << 20, 0.7)):
        sdp4.sdp4_rope_table(inv, tab, start, scale)
        ang = (start + np.arange(100))[:, None] * inv.cpu().numpy()
        want = scale * np.concatenate([np.cos(ang), np.sin(ang)], 1)
        close(tab, want, ref.U * np.abs(want) + 1e-8, "table")   # an angle of 10^6 in float64 is good to 1e-10


QK = [(1, 1, 1, 2, 2), (3, 2, 1, 1, 0), (5, 3, 2, 64, 64), (7, 40, 8, 128, 128), (33, 4, 4, 128, 64), (9, 5, 1, 80, 80),
      (9, 12, 12, 80, 40), (4, 3, 3, 96, 48), (17, 2, 2, 256, 256), (3, 2, 1, 66, 66), (5, 2, 2, 67, 10), (2, 3, 1, 512, 512),
      (2, 2, 2, 511, 510), (6, 7, 1, 100, 60), (130, 1, 1, 128, 0), (3, 2, 2, 300, 100), (11, 3, 0, 72, 24)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("tokens,hq,hk,dim,rot", QK)
def test_qk_norm_rope(tokens, hq, hk, dim, rot, inter, dtype):
    t = torch()
    say("qk_norm_rope", tokens, hq, hk, dim, rot, inter, dtype)
    g = rng(tokens, hq, dim, 21)
    qkv = normal(g, tokens, hq + 2 * hk + 1, dim, dtype=dtype, scale=2.0)        # packed: strided views
    q, k = qkv[:, :hq], (qkv[:, hq:hq + hk] if hk else None)
    qw, kw = normal(g, dim, dtype=dtype), (normal(g, dim, dtype=dtype) if hk else None)
    tab = table_for(50, rot, 1.1) if rot else None
    pos = t.randint(0, 50, (tokens,), device="cuda", generator=g)
    for eps, weights, positions in ((1e-5, True, pos), (1e-6, False, None if tokens <= 50 else pos), (None, False, pos)):
        a, b = (qw, kw) if weights else (None, None)
        qo = t.full((tokens, hq, dim), float("nan"), dtype=dt(dtype), device="cuda")
        ko = t.full((hk, tokens, dim), float("nan"), dtype=dt(dtype), device="cuda").transpose(0, 1) if hk else None
        sdp4.sdp4_qk_norm_rope(q, k, a, b, eps, tab, positions, qo, ko, interleaved=inter)
        pn = np.arange(tokens) if positions is None else pos.cpu().numpy()
        for x, w, y in ((q, a, qo), (k, b, ko)):
            if x is None:
                continue
            want, bound = ref.qk(f64(x), None if w is None else f64(w), eps, None if tab is None else f64(tab), pn, inter,
                                 dtype)
            close(y, want, bound, ("y", eps))
        # backward
        gq = normal(g, tokens, hq, dim, dtype=dtype)
        gk = normal(g, hk, tokens, dim, dtype=dtype).transpose(0, 1) if hk else None
        dq, dk = t.full_like(qo, float("nan")), (t.full_like(ko, float("nan")) if hk else None)
        dqw = t.full((dim,), float("nan"), device="cuda") if weights else None
        dkw = t.full((dim,), float("nan"), device="cuda") if weights and hk else None
        ws = scratch(sdp4.sdp4_qk_grad_workspace(tokens, hq, hk, dim)) if weights else None
        norm = eps is not None
        sdp4.sdp4_qk_norm_rope_grad(gq, gk, q if norm else None, k if norm else None, a, b, eps, tab, positions, dq, dk, dqw,
                                    dkw, ws, interleaved=inter)
        for gy, x, w, d, dw in ((gq, q, a, dq, dqw), (gk, k, b, dk, dkw)):
            if gy is None:
                continue
            (wx, bx), ww = ref.qk_grad(f64(gy), f64(x), None if w is None else f64(w), eps,
                                       None if tab is None else f64(tab), pn, inter, dtype)
            close(d, wx, bx, ("dx", eps))
            if dw is not None:
                close(dw, *ww, "dw")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_qk_in_place_and_many_tokens(dtype):
    t = torch()
    tokens, hq, hk, dim = 3001, 10, 2, 64
    say("qk in place", dtype)
    g = rng(22)
    qkv = normal(g, tokens, hq + 2 * hk, dim, dtype=dtype)
    keep = qkv.clone()
    qw, kw, tab = normal(g, dim, dtype=dtype), normal(g, dim, dtype=dtype), table_for(tokens, dim)
    q, k = qkv[:, :hq], qkv[:, hq:hq + hk]
    want = [ref.qk(f64(x), f64(w), 1e-6, f64(tab), np.arange(tokens), False, dtype) for x, w in ((q, qw), (k, kw))]
    sdp4.sdp4_qk_norm_rope(q, k, qw, kw, 1e-6, tab, None, q, k)
    close(q, *want[0], "q")
    close(k, *want[1], "k")
    assert t.equal(qkv[:, hq + hk:], keep[:, hq + hk:])                          # values untouched
    d = normal(g, tokens, hq + 2 * hk, dim, dtype=dtype)
    dv = d[:, hq + hk:].clone()
    wants = [ref.qk_grad(f64(y), f64(x), f64(w), 1e-6, f64(tab), np.arange(tokens), False, dtype)
             for y, x, w in ((d[:, :hq], keep[:, :hq], qw), (d[:, hq:hq + hk], keep[:, hq:hq + hk], kw))]
    dw = [t.empty(dim, device="cuda") for _ in range(2)]
    ws = scratch(sdp4.sdp4_qk_grad_workspace(tokens, hq, hk, dim))
    sdp4.sdp4_qk_norm_rope_grad(d[:, :hq], d[:, hq:hq + hk], keep[:, :hq], keep[:, hq:hq + hk], qw, kw, 1e-6, tab, None,
                                d[:, :hq], d[:, hq:hq + hk], *dw, ws)
    for x, w, ((wx, bx), ww) in ((d[:, :hq], dw[0], wants[0]), (d[:, hq:hq + hk], dw[1], wants[1])):
        close(x, wx, bx, "dx")
        close(w, *ww, "dw")
    assert t.equal(d[:, hq + hk:], dv)


def test_qk_edges():
    t = torch()
    g = rng(23)
    x = normal(g, 5, 2, 16)
    x[1] = 0.0                                                                   # a head of zeros: r = eps^-1/2
    x[2, 0, 3] = float("inf")
    tab = table_for(4, 8)
    pos = t.tensor([0, 3, 1, 4, -1], device="cuda")                              # two rows that the table does not have
    y = t.empty_like(x)
    sdp4.sdp4_qk_norm_rope(x, None, None, None, 1e-6, tab, pos, y, None)
    got = f64(y)
    assert (got[1] == 0).all() and np.isfinite(got[0]).all()
    assert np.isnan(got[3:, :, :8]).all() and np.isfinite(got[3:, :, 8:]).all()
    sdp4.sdp4_qk_norm_rope(x, None, None, None, None, tab, t.zeros_like(pos), y, None)   # no norm: inf stays where it is
    assert int(t.isnan(y).sum()) <= 2 and bool(t.isfinite(y[2, 0, 8:]).all())
    e = t.empty(0, 2, 16, device="cuda")
    sdp4.sdp4_qk_norm_rope(e, e, None, None, 1e-6, tab, None, e, e)
    w, dw = t.ones(16, device="cuda"), t.full((16,), 3.0, device="cuda")
    sdp4.sdp4_qk_norm_rope_grad(e, None, e, None, w, None, 1e-6, tab, None, e, None, dw, None, None)
    assert bool((dw == 0).all())


def test_qk_gradient_against_differences():
    """sum(c y) by central differences of the forward pass along random directions (steps of 2^-5 of unit directions;
    curvature of a norm of 40 elements of size 1 below 1)."""
    t = torch()
    g = rng(24)
    tokens, heads, dim, h = 6, 3, 40, 2.0 ** -5
    x, w, c = normal(g, tokens, heads, dim), 1 + normal(g, dim, scale=0.2), normal(g, tokens, heads, dim)
    tab = table_for(tokens, 24)

    def value(z, weight):
        y = t.empty_like(z)
        sdp4.sdp4_qk_norm_rope(z, None, weight, None, 1e-6, tab, None, y, None, interleaved=True)
        return (f64(y) * f64(c)).sum()
    dx, dw = t.empty_like(x), t.empty_like(w)
    sdp4.sdp4_qk_norm_rope_grad(c, None, x, None, w, None, 1e-6, tab, None, dx, None, dw, None,
                                scratch(sdp4.sdp4_qk_grad_workspace(tokens, heads, 0, dim)), interleaved=True)
    for _ in range(4):
        v, u = normal(g, tokens, heads, dim), normal(g, dim)
        v, u = v / v.norm(), u / u.norm()
        for num, ana in (((value(x + h * v, w) - value(x - h * v, w)) / (2 * h), (f64(dx) * f64(v)).sum()),
                         ((value(x, w + h * u) - value(x, w - h * u)) / (2 * h), (f64(dw) * f64(u)).sum())):
            assert abs(num - ana) <= 5e-3 * (1 + abs(ana)), (num, ana)


# ---------------------------------------------------------------------------
# inside a program
# ---------------------------------------------------------------------------
def one_of_each(seed):
    """Inputs, outputs and a function that runs every operator into them."""
    t = torch()
    g = rng(seed, 30)
    rows, cols, vocab = 130, 768, 5003
    x, b, r = normal(g, rows, cols, dtype="bf16"), normal(g, cols, dtype="bf16"), normal(g, rows, cols, dtype="bf16")
    z = normal(g, rows, vocab, dtype="bf16", scale=2.0)
    tg = t.randint(0, vocab, (rows,), device="cuda", generator=g)
    gl = normal(g, rows)
    q, w, tab = normal(g, rows, 12, 64, dtype="bf16"), normal(g, 64, dtype="bf16"), table_for(rows, 64)
    e = lambda *s, d=t.float32: t.zeros(*s, dtype=d, device="cuda")  # noqa: E731
    outs = dict(y=e(rows, cols, d=t.bfloat16), dx=e(rows, cols, d=t.bfloat16), db=e(cols), lp=e(rows), ls=e(rows), en=e(rows),
                tl=e(rows, 5), ti=e(rows, 5, d=t.int64), dz=e(rows, vocab, d=t.bfloat16), lp2=e(rows), ls2=e(rows), en2=e(rows),
                dz2=e(rows, vocab, d=t.bfloat16), qo=e(rows, 12, 64, d=t.bfloat16), dq=e(rows, 12, 64, d=t.bfloat16), dw=e(64))
    ws = [scratch(n) for n in (sdp4.sdp4_dropout_grad_workspace(rows, cols), sdp4.sdp4_token_logprob_workspace(rows, vocab, 5),
                               sdp4.sdp4_qk_grad_workspace(rows, 12, 0, 64))]
    o = outs

    def run(stream=None):
        sdp4.sdp4_dropout_add(x, b, r, 0.1, seed, 0, o["y"], stream=stream)
        sdp4.sdp4_dropout_add_grad(r, 0.1, seed, 0, o["dx"], o["db"], ws[0], stream=stream)
        sdp4.sdp4_token_logprob(z, tg, 5, o["lp"], o["ls"], o["en"], o["tl"], o["ti"], ws[1], stream=stream)
        sdp4.sdp4_token_logprob_grad(z, tg, o["ls"], o["en"], gl, gl, gl, o["dz"], stream=stream)
        sdp4.sdp4_token_loss(z, tg, gl, None, None, o["lp2"], o["ls2"], o["en2"], o["dz2"], ws[1], stream=stream)
        sdp4.sdp4_qk_norm_rope(q, None, w, None, 1e-6, tab, None, o["qo"], None, stream=stream)
        sdp4.sdp4_qk_norm_rope_grad(q, None, q, None, w, None, 1e-6, tab, None, o["dq"], None, o["dw"], None, ws[2],
                                    stream=stream)
    return run, outs


def test_step_operators_replayed_from_a_hip_graph():
    t = torch()
    run, outs = one_of_each(1)
    run()
    t.cuda.synchronize()
    want = {n: v.clone() for n, v in outs.items()}
    s = t.cuda.Stream()
    s.wait_stream(t.cuda.current_stream())
    graph = t.cuda.CUDAGraph()
    with t.cuda.stream(s):
        with t.cuda.graph(graph, stream=s):
            run()
    t.cuda.current_stream().wait_stream(s)
    junk = t.randn(1 << 20, device="cuda")
    for i in range(4):
        for v in outs.values():
            v.fill_(3)
        t.cuda.synchronize()
        graph.replay()
        junk.mul_(1.0001)
        t.cuda.synchronize()
        for n, v in outs.items():
            assert t.equal(v, want[n]), (n, i)


def test_step_operators_on_other_streams_and_on_the_general_path(monkeypatch):
    """The same bits from a side stream, from two streams at once, and without the native marshalling."""
    t = torch()
    runs = [one_of_each(i) for i in (1, 2)]
    want = []
    for run, outs in runs:
        run()
        t.cuda.synchronize()
        want.append({n: v.clone() for n, v in outs.items()})

    def check(what):
        t.cuda.synchronize()
        for (_, outs), w in zip(runs, want):
            for n, v in outs.items():
                assert t.equal(v, w[n]), (what, n)
                v.zero_()
        t.cuda.synchronize()
    check("eager")
    streams = [t.cuda.Stream(), t.cuda.Stream()]
    for (run, _), s in zip(runs, streams):
        run(stream=s)
    check("two streams")
    for (run, _), s in zip(runs, streams):
        with t.cuda.stream(s):
            run()
    check("current streams")
    monkeypatch.setattr(sdp4, "_fast", None)
    for run, _ in runs:
        run()
    check("general path")


def test_step_bindings_refuse_what_does_not_fit():
    t = torch()
    e = lambda *s, d=t.float32: t.zeros(*s, dtype=d, device="cuda")  # noqa: E731
    x = e(4, 16)
    for call in (
            lambda: sdp4.sdp4_dropout_add(x, None, None, 0.1, 1, 0, e(4, 15)),
            lambda: sdp4.sdp4_dropout_add(x, e(15), None, 0.1, 1, 0, x),
            lambda: sdp4.sdp4_dropout_add(x, e(16, d=t.bfloat16), None, 0.1, 1, 0, x),
            lambda: sdp4.sdp4_dropout_add(x, None, e(4, 16, d=t.bfloat16), 0.1, 1, 0, x),
            lambda: sdp4.sdp4_dropout_add(x.cpu(), None, None, 0.1, 1, 0, x),
            lambda: sdp4.sdp4_dropout_add(x.half(), None, None, 0.1, 1, 0, x),
            lambda: sdp4.sdp4_dropout_add(e(16, 4).t(), None, None, 0.1, 1, 0, x),
            lambda: sdp4.sdp4_dropout_add_grad(x, 0.1, 1, 0, x, e(15), e(4096)),
            lambda: sdp4.sdp4_token_logprob(x, e(4), 0, e(4), e(4), e(4)),
            lambda: sdp4.sdp4_token_logprob(x, None, 2, None, e(4), e(4), e(4, 3), e(4, 2, d=t.int64)),
            lambda: sdp4.sdp4_token_logprob(x, None, 2, None, e(4), e(4)),
            lambda: sdp4.sdp4_token_logprob(x, None, 0, None, e(5), e(4)),
            lambda: sdp4.sdp4_token_logprob(x, None, 0, None, e(4), e(4), vocab=17),
            lambda: sdp4.sdp4_token_logprob_grad(x, None, e(4), None, None, None, e(4), e(4, 15)),
            lambda: sdp4.sdp4_token_logprob_grad(x, None, None, None, None, None, e(4), x),
            lambda: sdp4.sdp4_token_loss(x, None, None, None, e(4), None, e(4), None, x),
            lambda: sdp4.sdp4_qk_norm_rope(e(2, 3, 8), e(2, 3, 8), None, None, 1e-6, None, None, e(2, 3, 8), None),
            lambda: sdp4.sdp4_qk_norm_rope(e(2, 3, 8), e(3, 3, 8), None, None, 1e-6, None, None, e(2, 3, 8), e(3, 3, 8)),
            lambda: sdp4.sdp4_qk_norm_rope(e(2, 3, 8), None, e(7), None, 1e-6, None, None, e(2, 3, 8), None),
            lambda: sdp4.sdp4_qk_norm_rope(e(2, 3, 8), None, None, None, 1e-6, e(4, 8, d=t.float64), None, e(2, 3, 8), None),
            lambda: sdp4.sdp4_qk_norm_rope(e(2, 3, 8), None, None, None, 1e-6, None, e(3, d=t.int64), e(2, 3, 8), None),
            lambda: sdp4.sdp4_qk_norm_rope(e(2, 3, 8), None, None, None, 1e-6, None, None, e(2, 3, 9), None),
            lambda: sdp4.sdp4_rope_table(e(4), e(2, 8))):
        with pytest.raises(ValueError):
            call()
    for call in (
            lambda: sdp4.sdp4_dropout_add(x, None, None, 1.5, 1, 0, x),
            lambda: sdp4.sdp4_dropout_add(x, None, None, 0.5, 1, 4, x),
            lambda: sdp4.sdp4_dropout_add(e(8, 16)[:4], None, None, 0.5, 1, 0, e(8, 16)[:4]) or sdp4.sdp4_dropout_add(
                (b := e(8, 16))[:4], None, None, 0.5, 1, 0, b[1:5]),
            lambda: sdp4.sdp4_dropout_add_grad(x, 0.1, 1, 0, x, e(16), e(1)),
            lambda: sdp4.sdp4_dropout_add_grad(x, 0.1, 1, 0, x, e(16), None),
            lambda: sdp4.sdp4_token_logprob(x, None, 17, None, None, None, e(4, 17), e(4, 17, d=t.int64)),
            lambda: sdp4.sdp4_token_logprob(x, None, 0, e(4), None, None),
            lambda: sdp4.sdp4_token_logprob_grad(x, None, e(4), None, e(4), None, None, x),
            lambda: sdp4.sdp4_qk_norm_rope(e(2, 3, 8), None, e(8), None, None, None, None, e(2, 3, 8), None),
            lambda: sdp4.sdp4_qk_norm_rope(e(2, 3, 8), None, None, None, -1.0, None, None, e(2, 3, 8), None),
            lambda: sdp4.sdp4_qk_norm_rope(e(2, 3, 8), None, None, None, 1e-6, e(4, 3), None, e(2, 3, 8), None),
            lambda: sdp4.sdp4_qk_norm_rope(e(2, 3, 8), None, None, None, 1e-6, e(4, 10), None, e(2, 3, 8), None)):
        with pytest.raises(sdp4.Sdp4Error):
            call()
