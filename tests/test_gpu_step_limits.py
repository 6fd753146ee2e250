"""The training-step operators on the GPU where values, lengths or layouts go
to the limits of what the library's header allows, against 64-bit forms."""
import numpy as np
import pytest

from paper_2410_15526_amd import sdp4
from tests import _step as ref
from tests._gpu import say, torch
from tests.test_gpu_step import check_logprob, close, dt, f64, normal, scratch, table_for

pytestmark = pytest.mark.gpu


def rng(seed):
    return torch().Generator(device="cuda").manual_seed(seed)


def empties(rows, n=3):
    return [torch().full((rows,), 7.0, device="cuda") for _ in range(n)]


# ---------------------------------------------------------------------------
# logits of large magnitude
# ---------------------------------------------------------------------------
def grad_from(x, targets, lse, ent, g_logp, g_ent, g_lse, dtype):
    """(dlogits, bound) from a given float32 logsumexp: p = exp(x - lse), whatever these sum up to.  t = (x - lse) log2 e is
    off by at most 3 U of itself (difference, log2 e, product) and once more U where its share in the entropy's term is
    taken; the exponential by 2 U; the factors and their sum by 8 U of their magnitudes; bfloat16 by its final rounding."""
    d = x - lse[:, None]
    p = np.exp(d)
    dd = np.where(p > 0, d, 0.0)
    z = np.zeros(len(x))
    gl, ga, ge = (z if g is None else g for g in (g_lse, g_logp, g_ent))
    ga = np.where(targets < 0, 0.0, ga)
    v = p * ((gl - ga)[:, None] - ge[:, None] * (dd + ent[:, None]))
    mag = p * ((np.abs(gl) + np.abs(ga) + np.abs(ge * ent))[:, None] + np.abs(ge[:, None] * dd))
    bound = mag * ref.U * (4 * np.abs(dd) + 12)
    hit = np.nonzero(targets >= 0)[0]
    v[hit, targets[hit]] += ga[hit]
    bound[hit, targets[hit]] += 2 * ref.U * np.abs(ga[hit])
    return v, bound + ref.rounding(dtype) * np.abs(v) + 1000 * ref.TINY


LARGE = [1e5, 3e6, -2e8, 1.3e9, 5e9, -1e10, 1e20, -1e30, 1e38, -1e38]


def large_rows(g, vocab, dtype):
    """Rows of one large value; a large value among ordinary ones; half a row of masks at -1e30; ordinary rows."""
    t = torch()
    x = normal(g, 2 * len(LARGE) + 4, vocab, dtype=dtype, scale=2.0)
    for i, v in enumerate(LARGE):
        x[i] = v
        x[len(LARGE) + i, vocab // 2] = v
    x[-4, ::2] = -1e30
    x[-3, :vocab // 2] = -1e10
    x[-2] = x[-2] + 1e6
    tg = t.randint(0, vocab, (len(x),), device="cuda", generator=g)
    tg[2], tg[-1] = -100, vocab // 2
    return x, tg


@pytest.mark.parametrize("entropy", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [9, 700, 20003, 140001])
def test_token_gradients_of_large_logits(vocab, dtype, entropy):
    t = torch()
    say("large logits", vocab, dtype, entropy)
    g = rng(100 + vocab)
    x, tg = large_rows(g, vocab, dtype)
    rows = len(x)
    gs = [normal(g, rows, scale=0.5), normal(g, rows, scale=0.5) if entropy else None, normal(g, rows, scale=0.5)]
    xs, tn, gn = f64(x), tg.cpu().numpy(), [None if a is None else f64(a) for a in gs]
    logp, lse, ent = ref.token_stats(xs, tn)
    l32, e32 = (t.from_numpy(a).float().cuda() for a in (lse, ent))
    d = t.full((rows, vocab), float("nan"), dtype=dt(dtype), device="cuda")
    sdp4.sdp4_token_logprob_grad(x, tg, l32, e32, *gs, d)
    want, bound = grad_from(xs, tn, f64(l32), f64(e32), *gn, dtype)
    close(d, want, bound, "dlogits")
    d = t.full((rows, vocab), float("nan"), dtype=dt(dtype), device="cuda")
    lp, ls, en = empties(rows)
    sdp4.sdp4_token_loss(x, tg, *gs, lp, ls, en, d, scratch(sdp4.sdp4_token_logprob_workspace(rows, vocab)))
    bl, be, bn = ref.stats_bounds(xs, logp, ent)
    close(ls, lse, be, "lse")
    close(lp, logp, bl, "logp")
    close(en, ent, bn, "entropy")
    if vocab > (131072 if dtype == "bf16" else 65536):     # two launches: p from the rounded logsumexp
        want, bound = grad_from(xs, tn, f64(ls), f64(en), *gn, dtype)
    else:
        want, bound = ref.token_grad(xs, tn, ent, *gn, vocab, dtype, lse_given=False)
    close(d, want, bound, "dlogits of the loss")


def test_gradient_of_a_row_that_is_left_out():
    """No upstream gradient and no target: zeros, whatever finite values the row holds."""
    t = torch()
    for dtype in ("f32", "bf16"):
        x = t.tensor([[-1e10], [-1e30], [7e9], [1e38]], device="cuda").expand(4, 640).to(dt(dtype)).contiguous()
        tg, z = t.full((4,), -100, device="cuda"), t.zeros(4, device="cuda")
        d = t.full_like(x, float("nan"))
        sdp4.sdp4_token_loss(x, tg, z, z, z, *empties(4), d, scratch(sdp4.sdp4_token_logprob_workspace(4, 640)))
        assert bool((d == 0).all()), dtype


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(40, 250), (2100, 1000), (40, 20003)])
def test_statistics_of_large_logits(rows, vocab, dtype):
    """Rows of equal logits: lse = x + log vocab, entropy log vocab, each logp -log vocab, as for small ones.  The sum of n
    ones is off by (its 64 additions in a lane at most, 6 over the lanes and those over slices, the exponent's constants 4)
    U; the logarithm and its factor by 4 U of itself."""
    t = torch()
    x = t.logspace(2, 38, rows, device="cuda", dtype=t.float64)
    x[1::2] *= -1
    x = x.to(dt(dtype))[:, None].expand(rows, vocab).contiguous()
    tg = t.arange(rows, device="cuda") % vocab
    b = ref.U * (64 + 6 + 16 + 4 + 4 * np.log(vocab))
    d = t.empty_like(x)
    for loss in (False, True):
        lp, ls, en = empties(rows)
        ws = scratch(sdp4.sdp4_token_logprob_workspace(rows, vocab))
        if loss:
            sdp4.sdp4_token_loss(x, tg, None, None, None, lp, ls, en, d, ws)
        else:
            sdp4.sdp4_token_logprob(x, tg, 0, lp, ls, en, workspace=ws)
        close(lp, np.full(rows, -np.log(vocab)), b, ("logp", loss))
        close(en, np.full(rows, np.log(vocab)), b, ("entropy", loss))
        x0 = f64(x[:, 0])
        close(ls, x0 + np.log(vocab), b + 2 * ref.U * np.abs(x0), ("lse", loss))


# ---------------------------------------------------------------------------
# confident rows
# ---------------------------------------------------------------------------
def peaked(g, rows, vocab, dtype):
    """Logits around 0 with one that stands 0 to 40 above them, anywhere in the row; targets there."""
    t = torch()
    x = normal(g, rows, vocab, dtype="f32", scale=0.3)
    tg = t.randint(0, vocab, (rows,), device="cuda", generator=g)
    high = t.linspace(0, 40, rows, device="cuda")
    x.scatter_(1, tg[:, None], high[:, None])
    return x.to(dt(dtype)), tg


PEAKED = [(2100, 320), (2100, 1000), (2100, 4096), (300, 9001), (64, 70001)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", PEAKED)
def test_log_probabilities_are_not_positive(rows, vocab, dtype):
    t = torch()
    say("signs", rows, vocab, dtype)
    x, tg = peaked(rng(vocab), rows, vocab, dtype)
    for k in (0, 3):
        lp, ls, en = empties(rows)
        tl, ti = t.full((rows, k), 7.0, device="cuda"), t.zeros(rows, k, dtype=t.int64, device="cuda")
        sdp4.sdp4_token_logprob(x, tg, k, lp, ls, en, tl, ti, scratch(sdp4.sdp4_token_logprob_workspace(rows, vocab, k)))
        assert float(lp.max()) <= 0 and float(en.min()) >= 0
        assert not k or float(tl.max()) <= 0
    lp, ls, en = empties(rows)
    sdp4.sdp4_token_loss(x, tg, None, None, None, lp, ls, en, t.empty_like(x),
                         scratch(sdp4.sdp4_token_logprob_workspace(rows, vocab)))
    assert float(lp.max()) <= 0 and float(en.min()) >= 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", PEAKED)
def test_confident_rows_keep_their_precision(rows, vocab, dtype):
    """Errors relative to -logp and to the entropy H, wherever in its row the largest logit stands.

    With sums of 2^t relative to a reference whose mean exponent (weighted by probability) is at most 4, the weighted |t|
    is at most 4 + 2 H / ln 2 and the sum's logarithm at most 4 ln 2 + H.  A sum is then off by U times (a lane's additions +
    6 over the lanes + the joins' 16 + 4 for exponential and constants + 2 ln 2 |t|), logp by that and 3 U (-logp + 2 H +
    4 ln 2); the entropy twice by the sums' error, its second sum in proportion to |t|."""
    t = torch()
    say("confident rows", rows, vocab, dtype)
    x, tg = peaked(rng(vocab), rows, vocab, dtype)
    xs, tn = f64(x), tg.cpu().numpy()
    logp, lse, ent = ref.token_stats(xs, tn)
    slices = -(-vocab // 4096)
    adds = min(64, -(-vocab // 64)) + 6 + (16 if slices > 1 else 0) + 4
    rel = ref.U * (adds + 8 * np.log(2) + 4 * ent)
    b_logp = rel + 3 * ref.U * (-logp + 2 * ent + 4 * np.log(2))
    b_ent = rel + ref.U * (adds + 4) * (4 * np.log(2) + 2 * ent) + 3 * ref.U * (2 * ent + 4 * np.log(2))
    for loss in (False, True):
        lp, ls, en = empties(rows)
        ws = scratch(sdp4.sdp4_token_logprob_workspace(rows, vocab))
        if loss:
            sdp4.sdp4_token_loss(x, tg, None, None, None, lp, ls, en, t.empty_like(x), ws)
        else:
            sdp4.sdp4_token_logprob(x, tg, 0, lp, ls, en, workspace=ws)
        print("logp", np.abs(f64(lp) - logp).max(), "entropy", np.abs(f64(en) - ent).max(), flush=True)
        close(lp, logp, b_logp, ("logp", loss))
        close(en, ent, b_ent, ("entropy", loss))
        close(ls, lse, b_logp + 2 * ref.U * np.abs(lse), ("lse", loss))


@pytest.mark.parametrize("vocab", [700, 4096, 9001])
def test_a_workspace_serves_shorter_batches(vocab):
    """A buffer for the whole batch does for its last, shorter part."""
    t = torch()
    for k in (0, 3):
        x = normal(rng(5), 2500, vocab, dtype="bf16")
        ws = t.empty(sdp4.sdp4_token_logprob_workspace(2500, vocab, k), dtype=t.uint8, device="cuda")
        for rows in (2500, 513, 100, 1):
            tl, ti = t.empty(rows, k, device="cuda"), t.empty(rows, k, dtype=t.int64, device="cuda")
            sdp4.sdp4_token_logprob(x[:rows], None, k, None, *empties(rows, 2), tl, ti, ws)
            if k == 0:
                sdp4.sdp4_token_loss(x[:rows], None, None, None, None, None, *empties(rows, 2), t.empty_like(x[:rows]), ws)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,heads", [(1, 3), (5, 1), (7, 4)])
@pytest.mark.parametrize("heads_first", [False, True])
def test_qk_inside_heads_of_query_key_and_value(tokens, heads, heads_first, dtype):
    """A projection that packs each head's query, key and value side by side: strides of three heads.  In place and
    with both gradients in one array of that layout."""
    t = torch()
    g = rng(6)
    dim = 64
    shape = (heads, tokens, 3, dim) if heads_first else (tokens, heads, 3, dim)

    def parts(a):
        a = a.transpose(0, 1) if heads_first else a
        return a[:, :, 0], a[:, :, 1], a[:, :, 2]
    qkv, grads = normal(g, *shape, dtype=dtype), normal(g, *shape, dtype=dtype)
    qw, kw, tab = normal(g, dim, dtype=dtype), normal(g, dim, dtype=dtype), table_for(tokens, dim)
    (q, k, v), (gq, gk, gv) = parts(qkv), parts(grads)
    at = np.arange(tokens)
    q0, k0, v0, gv0 = q.clone(), k.clone(), v.clone(), gv.clone()
    want = [ref.qk(f64(x), f64(w), 1e-6, f64(tab), at, False, dtype) for x, w in ((q0, qw), (k0, kw))]
    wg = [ref.qk_grad(f64(y), f64(x), f64(w), 1e-6, f64(tab), at, False, dtype) for y, x, w in ((gq, q0, qw), (gk, k0, kw))]
    sdp4.sdp4_qk_norm_rope(q, k, qw, kw, 1e-6, tab, None, q, k)
    close(q, *want[0], "q")
    close(k, *want[1], "k")
    assert t.equal(v, v0)
    dw = [t.empty(dim, device="cuda") for _ in range(2)]
    sdp4.sdp4_qk_norm_rope_grad(gq, gk, q0, k0, qw, kw, 1e-6, tab, None, gq, gk, *dw,
                                scratch(sdp4.sdp4_qk_grad_workspace(tokens, heads, heads, dim)))
    for x, w, ((wx, bx), ww) in ((gq, dw[0], wg[0]), (gk, dw[1], wg[1])):
        close(x, wx, bx, "dx")
        close(w, *ww, "dw")
    assert t.equal(gv, gv0)


# ---------------------------------------------------------------------------
# forms of their own for long rows and many rows
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [262145, 300007, 1 << 20])
def test_rows_of_more_than_64_slices(vocab, dtype):
    """The longest rows, whose parts a wave joins in several rounds: ordinary, ties, masks, a peak at the end, NaN."""
    t = torch()
    say("long rows", vocab, dtype)
    x = normal(rng(vocab), 7, vocab, dtype=dtype, scale=3.0)
    x[1] = (t.arange(vocab, device="cuda") % 5).to(x.dtype)
    x[2] = float("-inf")
    x[2, vocab - 2:] = 1.0
    x[3, :-5] = t.finfo(x.dtype).min
    x[4, -1] = 90.0
    x[5] = 0.0
    tg = t.tensor([5, 4, vocab - 1, vocab - 3, vocab - 1, 0, 1], device="cuda")
    for k in (0, 1, 8, 9, 32):
        check_logprob(x, tg, k, dtype=dtype)
    x[0, vocab - 1] = float("nan")
    lp, ls, en = empties(7)
    tl, ti = t.zeros(7, 9, device="cuda"), t.zeros(7, 9, dtype=t.int64, device="cuda")
    sdp4.sdp4_token_logprob(x, tg, 9, lp, ls, en, tl, ti, scratch(sdp4.sdp4_token_logprob_workspace(7, vocab, 9)))
    assert bool(t.isnan(tl[0]).all()) and bool((ti[0] == -1).all()) and not bool(t.isnan(tl[1:]).any())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_loss_of_rows_of_more_than_64_slices(dtype):
    t = torch()
    vocab = 300007
    x = normal(rng(8), 3, vocab, dtype=dtype, scale=3.0)
    tg = t.tensor([0, vocab - 1, -1], device="cuda")
    gs = [normal(rng(9), 3, scale=0.5) for _ in range(3)]
    xs, tn, gn = f64(x), tg.cpu().numpy(), [f64(a) for a in gs]
    logp, lse, ent = ref.token_stats(xs, tn)
    d, (lp, ls, en) = t.full_like(x, float("nan")), empties(3)
    sdp4.sdp4_token_loss(x, tg, *gs, lp, ls, en, d, scratch(sdp4.sdp4_token_logprob_workspace(3, vocab)))
    for got, want, b, what in zip((lp, ls, en), (logp, lse, ent), ref.stats_bounds(xs, logp, ent), ("logp", "lse", "entropy")):
        close(got, want, b, what)
    want, bound = grad_from(xs, tn, f64(ls), f64(en), *gn, dtype)
    close(d, want, bound, "dlogits")


@pytest.mark.parametrize("x_dtype,y_dtype", [("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("rows,cols", [(6203, 5120), (6203, 5119), (21001, 515)])
def test_dropout_gradient_of_many_rows(rows, cols, x_dtype, y_dtype):
    """Several batches of rows for each block, in place where the types are one: the loop over whole batches, the one at
    the edges, and what both do to the generator's position."""
    t = torch()
    say("dropout gradient", rows, cols, x_dtype, y_dtype)
    dy = normal(rng(rows + cols), rows, cols, dtype=y_dtype)
    (want, bound), (wb, bb) = ref.dropout_grad(f64(dy), 0.1, 11, 24, x_dtype)
    dx = dy if x_dtype == y_dtype else t.full((rows, cols), float("nan"), dtype=dt(x_dtype), device="cuda")
    db = t.full((cols,), float("nan"), device="cuda")
    sdp4.sdp4_dropout_add_grad(dy, 0.1, 11, 24, dx, db, scratch(sdp4.sdp4_dropout_grad_workspace(rows, cols)))
    close(dx, want, bound, "dx")
    close(db, wb, bb, "dbias")


@pytest.mark.parametrize("x_dtype,y_dtype", [("f32", "bf16")])
@pytest.mark.parametrize("rows,cols", [(1, 7), (17, 64), (257, 515), (9, 4097), (4099, 96)])
def test_dropout_gradient_from_bfloat16_to_float32(rows, cols, x_dtype, y_dtype):
    t = torch()
    dy = normal(rng(rows), rows, cols, dtype=y_dtype)
    (want, bound), (wb, bb) = ref.dropout_grad(f64(dy), 0.25, 7, 16, x_dtype)
    dx, db = t.full((rows, cols), float("nan"), dtype=dt(x_dtype), device="cuda"), t.full((cols,), float("nan"), device="cuda")
    sdp4.sdp4_dropout_add_grad(dy, 0.25, 7, 16, dx, db, scratch(sdp4.sdp4_dropout_grad_workspace(rows, cols)))
    close(dx, want, bound, "dx")
    close(db, wb, bb, "dbias")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,hq,hk,dim,rot,inter", [(4001, 11, 3, 64, 64, False), (2003, 40, 8, 128, 64, True),
                                                        (3001, 7, 7, 67, 10, False)])
def test_qk_gradient_with_several_heads_a_lane_group(tokens, hq, hk, dim, rot, inter, dtype):
    """Numbers of heads that do not divide the step from one of a group's heads to its next."""
    t = torch()
    say("qk gradient", tokens, hq, hk, dim, rot, inter, dtype)
    g = rng(tokens)
    q, k = normal(g, tokens, hq, dim, dtype=dtype), normal(g, tokens, hk, dim, dtype=dtype)
    gq, gk = normal(g, tokens, hq, dim, dtype=dtype), normal(g, hk, tokens, dim, dtype=dtype).transpose(0, 1)
    qw, kw, tab = normal(g, dim, dtype=dtype), normal(g, dim, dtype=dtype), table_for(tokens, rot)
    want = [ref.qk_grad(f64(y), f64(x), f64(w), 1e-6, f64(tab), np.arange(tokens), inter, dtype)
            for y, x, w in ((gq, q, qw), (gk, k, kw))]
    dq, dk = t.full_like(q, float("nan")), t.full_like(k, float("nan"))
    dw = [t.full((dim,), float("nan"), device="cuda") for _ in range(2)]
    sdp4.sdp4_qk_norm_rope_grad(gq, gk, q, k, qw, kw, 1e-6, tab, None, dq, dk, *dw,
                                scratch(sdp4.sdp4_qk_grad_workspace(tokens, hq, hk, dim)), interleaved=inter)
    for x, w, ((wx, bx), ww) in ((dq, dw[0], want[0]), (dk, dw[1], want[1])):
        close(x, wx, bx, "dx")
        close(w, *ww, "dw")
