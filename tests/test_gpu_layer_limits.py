"""Attention, block norms, the embedding and the decoder on them at the limits
of their types, sizes and layouts."""
import numpy as np
import pytest

from tests import _layer as ref
from tests._gpu import say, torch
from tests.test_gpu_step import close, dt, f64

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------
# the decoder
# ---------------------------------------------------------------------------
def test_decoder_attention_is_float32(monkeypatch):
    """What the decoder's attention returns and its gradients are within the float32 bounds, with one rounding to bfloat16 at
    the end: no probability is rounded on the way."""
    torch()
    from paper_2410_15526_amd import sdp4
    from paper_2410_15526_amd.decoder import Config, Decoder, sequences
    calls = {"sdp4_attention": [], "sdp4_attention_grad": []}
    for name, made in calls.items():
        def watched(*args, made=made, plain=getattr(sdp4, name)):
            plain(*args)
            made.append([f64(x.detach()) if hasattr(x, "detach") else x for x in args])
        monkeypatch.setattr(sdp4, name, watched)
    model = Decoder(Config(batch=3), seed=4)
    tokens, targets = sequences(model.cfg, 3, 0)
    model.backward(tokens, targets, p=0.0)
    forward, backward = calls["sdp4_attention"], calls["sdp4_attention_grad"]
    assert len(forward) == len(backward) == model.cfg.layers
    lengths, last = [model.cfg.seq] * 3, lambda want, bound: bound + ref.V * np.abs(want)  # noqa: E731
    for q, k, v, scale, _, out, lse in forward:
        (want, bound), _ = ref.attention(q, k, v, lengths, scale, "f32")
        close(out, want, last(want, bound), "out")
    for dout, q, k, v, out, lse, scale, _, *grads, _ in backward:
        wants = ref.attention_grad(dout, q, k, v, out, lse, lengths, scale, "f32")
        for got, (want, bound), name in zip(grads, wants, ("dq", "dk", "dv")):
            close(got, want, last(want, bound), name)


# ---------------------------------------------------------------------------
# the embedding's gradient over more rows than one call takes
# ---------------------------------------------------------------------------
def table_gradient(ids, table, dout, scale):
    from paper_2410_15526_amd import autograd
    leaf = table.detach().requires_grad_()
    autograd.embedding(ids, leaf, scale, dout.dtype).backward(dout)
    return leaf.grad


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_embedding_gradient_in_several_calls(dtype, monkeypatch):
    """Rows of a few more calls than one, holes among them; the sums are float32 over the calls and rounded once."""
    t = torch()
    from paper_2410_15526_amd import sdp4
    g = t.Generator(device="cuda").manual_seed(5)
    ids = t.randint(-2, 45, (1000,), device="cuda", generator=g)
    table, dout = (t.randn(n, 37, device="cuda", generator=g).to(dt(dtype)) for n in (41, 1000))
    want = ref.embedding_grad(ids.cpu().numpy(), f64(dout), 0.5, 41, None, dtype)
    size = ref.embedding_grad(ids.cpu().numpy(), np.abs(f64(dout)), 0.5, 41, None, dtype)[0]
    rows, plain = [], sdp4.sdp4_embedding_grad

    def watched(ids, dout, *args, **kw):
        rows.append(len(ids))
        plain(ids, dout, *args, **kw)

    monkeypatch.setattr(sdp4, "sdp4_embedding_grad", watched)
    for limit in (1000, 999, 300, 1):
        say("embedding gradient", dtype, limit)
        monkeypatch.setattr(sdp4, "MAX_GRAD_TOKENS", limit)
        rows.clear()
        got = table_gradient(ids, table, dout, 0.5)
        calls = -(-1000 // limit)                            # one more rounding of a sum in each
        assert got.dtype == table.dtype and len(rows) == calls and max(rows) <= limit and sum(rows) == 1000
        close(got, want[0], want[1] + (calls - 1) * ref.U * size, limit)


def test_embedding_gradient_beyond_one_call():
    t = torch()
    from paper_2410_15526_amd import sdp4
    rows = sdp4.MAX_GRAD_TOKENS + 3
    say("embedding gradient", rows)
    g = t.Generator(device="cuda").manual_seed(6)
    ids = t.randint(0, 1000, (rows,), device="cuda", generator=g)
    table, dout = (t.randn(n, 4, device="cuda", generator=g) for n in (1000, rows))
    got = table_gradient(ids, table, dout, 1.0)
    close(got, *ref.embedding_grad(ids.cpu().numpy(), f64(dout), 1.0, 1000, None, "f32"), "gradient")


@pytest.mark.parametrize("rows", [8193, 8200, 10240, 32768, 32769, 131072, 131073, 140001])
def test_embedding_gradient_over_merged_runs(rows):
    """Numbers of rows around those at which another pass of merges begins; tokens of few rows, of many and of none."""
    t = torch()
    from paper_2410_15526_amd import sdp4
    g = t.Generator(device="cuda").manual_seed(rows)
    ids = (5000 * t.rand(rows, device="cuda", generator=g) ** 3).long()
    ids[::5], ids[1::1000] = 77, -1
    dout = t.randn(rows, 9, device="cuda", generator=g)
    d = t.full((5000, 9), float("nan"), device="cuda")
    work = t.full((sdp4.sdp4_embedding_grad_workspace(rows, 5000, 9),), 0xFF, dtype=t.uint8, device="cuda")
    sdp4.sdp4_embedding_grad(ids, dout, 1.0, d, work)
    close(d, *ref.embedding_grad(ids.cpu().numpy(), f64(dout), 1.0, 5000, None, "f32"), rows)



# ---------------------------------------------------------------------------
# more tiles of keys than are sorted
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,rows", [("bf16", 33100), ("f32", 16700)])
def test_attention_of_more_tiles_than_are_sorted(dtype, rows):
    """Tiles of 128 and 64 keys, 256 of them sorted at most: many sequences, one of them long."""
    from tests.test_gpu_layer import Case
    say("attention of many tiles", dtype, rows)
    r = np.random.default_rng(rows)
    lengths = []
    while sum(lengths) < rows:
        lengths.append(int(r.integers(0, 250)) if len(lengths) != 40 else 1500)
    Case(62, lengths, 11, 2, 1, 64, dtype, lead=3).check()



# ---------------------------------------------------------------------------
# an infinity in the first elements of a head that does not fill its columns
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [8, 40, 48, 72, 80, 104, 136, 160, 200, 248])
def test_attention_key_of_score_minus_infinity(dim, dtype):
    """A key whose first element makes its scores -inf weighs nothing, and rows that see no other come out as zeros, however the
    heads are laid out."""
    t = torch()
    from tests.test_gpu_layer import Case
    lengths, inf = [50, 41], float("inf")
    results = []
    for layout in ("dense", "odd"):
        say("attention of an infinite key", dim, dtype, layout)
        c = Case(60, lengths, 0, 4, 2, dim, dtype, layout=layout)
        c.q[:, :, 0] = c.q[:, :, 0].abs() + 0.5
        for at in (0, 17, 50, 51, 90):                       # the first of a sequence: row `at` sees no other key
            c.k[at, :, 0] = -inf
        results.append([x.clone() for x in c.forward()] + [x.clone() for x in c.backward()])
    (out, lse, *_), q, k, v = results[0], f64(c.q), f64(c.k), f64(c.v)
    assert bool((out[[0, 50, 51]] == 0).all()) and bool(t.isneginf(lse[:, [0, 50, 51]]).all())
    keep = np.isfinite(k[:, 0, 0])
    k0 = np.where(keep[:, None, None], k, 0.0)
    for a, b in ((0, 50), (50, 91)):
        for h in range(4):
            s = c.scale * q[a:b, h] @ k0[a:b, h // 2].T
            seen = np.tril(np.ones(s.shape, bool)) & keep[a:b]
            rows = seen.any(1)
            s = np.where(seen, s, -np.inf)[rows]
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            val = v[a:b, h // 2]
            want, size = p @ val, p @ np.abs(val)
            # as for any other scores: dim + 2 half steps of a score's terms, 10 of the score, those of the sums, the result's
            err = (dim + 2) * ref.U * c.scale * (np.abs(q[a:b, h]) @ np.abs(k0[a:b, h // 2]).T).max() + \
                10 * ref.U * np.abs(np.where(np.isfinite(s), s, 0.0)).max() + 8 * ref.U
            low = ref.V * (1 + 2.0 ** -7) if dtype == "bf16" else 0.0
            close(f64(out)[a:b, h][rows], want, size * (2 * err + 80 * ref.U + low) + ref.rounding(dtype) * np.abs(want) + ref.TINY,
                  (a, h))
    for x, y, name in zip(*results, ("out", "lse", "dq", "dk", "dv")):
        assert t.equal(x.isnan(), y.isnan()) and t.equal(x.nan_to_num(), y.nan_to_num()), name


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [8, 40, 80, 104, 136, 200])
def test_attention_query_of_score_minus_infinity(dim, dtype):
    """A query whose scores are all -inf gives no weight to any value: dv is finite, and that of the other queries."""
    t = torch()
    from tests.test_gpu_layer import Case
    results = []
    for layout in ("dense", "odd"):
        say("attention of an infinite query", dim, dtype, layout)
        c = Case(61, [70], 0, 4, 2, dim, dtype, layout=layout)
        c.k[:, :, 0] = c.k[:, :, 0].abs() + 0.5
        c.q[33, :, 0] = -float("inf")
        out, lse = c.forward()
        assert bool((out[33] == 0).all()) and bool(t.isneginf(lse[:, 33]).all())
        results.append(c.backward()[2].clone())
    dout, q = f64(c.dout), f64(c.q)
    dout[33], q[33] = 0.0, 0.0
    finite = np.where(np.isfinite(f64(lse)), f64(lse), 0.0)
    want, bound = ref.attention_grad(dout, q, f64(c.k), f64(c.v), f64(out), finite, [70], c.scale, dtype)[2]
    close(results[0], want, bound, "dv")
    assert t.equal(*results)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [8, 40, 80, 104, 200])
def test_padded_heads_do_not_see_what_is_masked(dim, dtype):
    """Heads that do not fill their columns: other sequences, later rows and rows in no sequence, holding NaN or infinities."""
    from tests.test_gpu_layer import test_attention_does_not_see_what_is_masked
    for value in (float("nan"), float("inf"), -float("inf")):
        say("masked", dim, dtype, value)
        test_attention_does_not_see_what_is_masked(dim, value, dtype)



# ---------------------------------------------------------------------------
# block norms of two types, of which one result is used
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("general", [False, True])
def test_norm_of_a_stream_whose_next_input_is_not_used(general, monkeypatch):
    """A float32 stream beside bfloat16 weights, and a gradient by y alone."""
    t = torch()
    from paper_2410_15526_amd import autograd, sdp4
    if general:
        sdp4.lib()
        monkeypatch.setattr(sdp4, "_fast", None)
    x = t.randn(9, 50, device="cuda").requires_grad_()
    w = t.ones(50, dtype=t.bfloat16, device="cuda").requires_grad_()
    y, h = autograd.block_norm(None, x, w, residual_scale=2.0, dtype=t.bfloat16)
    assert y.dtype == t.float32 and h.dtype == t.bfloat16
    (3 * y).sum().backward()
    assert bool((x.grad == 6).all()) and bool((w.grad == 0).all())


@pytest.mark.parametrize("cols", [64, 1000, 4097])
def test_gradients_that_need_no_branch(cols):
    """The residual stream's gradient and the next norm's weight's, with and without the branch in hand."""
    t = torch()
    from tests.test_gpu_layer import Joint
    c = Joint(63, 300, cols, "bf16", "f32", "post")
    c.w2 = t.randn(cols, device="cuda").bfloat16()
    y = t.randn(300, cols, device="cuda")
    both = c.backward(y)
    from paper_2410_15526_amd import sdp4
    from tests.test_gpu_step import scratch
    p, w1, gate, b, r = c.head()
    dr, dw = t.full_like(y, float("nan")), t.full((cols,), float("nan"), device="cuda")
    sdp4.sdp4_block_norm_grad(c.dh, c.dy, None, y, p, w1, gate, b, r, 1e-6, c.w2, None, dr, None, dw, None,
                              scratch(sdp4.sdp4_block_norm_grad_workspace(300, cols)))
    assert t.equal(dr, both["dresidual"]) and t.equal(dw, both["dpre_weight"])



@pytest.mark.parametrize("x,y", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")])
@pytest.mark.parametrize("rows,cols", [(4101, 203), (4500, 8), (2100, 700), (1100, 1500), (520, 3001)])
def test_block_norm_gradients_of_more_rows_than_parts(rows, cols, x, y):
    """Blocks that walk several rows, at each number of blocks that the width of a row allows."""
    t = torch()
    from tests.test_gpu_layer import Joint
    for kind in ("full", "pre"):
        say("block norm rows", rows, cols, x, y, kind)
        c = Joint(64, rows, cols, x, y, kind)
        yo, ho = (t.full((rows, cols), float("nan"), dtype=dt(ty), device="cuda") for ty in (y, x))
        c.forward(c.branch, c.residual, yo, ho)
        got, want = c.backward(yo), c.want_grad(yo)
        for k, v in got.items():
            if v is not None:
                close(v, *want[k], (k, kind))
        again = c.backward(yo)
        assert all(v is None or t.equal(v, again[k]) for k, v in got.items())



# ---------------------------------------------------------------------------
# the decoder's sizes beyond those of the operators
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("hidden,heads,seq,batch", [(256, 64, 64, 2), (768, 2, 64, 2), (768, 2, 64, 1), (512, 2, 2176, 1), (256, 1, 64, 2)])
def test_decoder_with_heads_beyond_the_operators(hidden, heads, seq, batch):
    """Heads of 4 and of 384 elements, long sequences of heads of 256 and short ones: gradients against float32, to the 30
    roundings of the decoder's other sizes."""
    torch()
    from paper_2410_15526_amd.decoder import Config, Decoder, sequences
    from tests.test_gpu_decoder import plain_loss
    model = Decoder(Config(batch=batch, hidden=hidden, heads=heads, layers=1, seq=seq), seed=3)
    tokens, targets = sequences(model.cfg, batch, 0)
    loss = model.backward(tokens, targets, p=0.0)
    leaves = {k: v.detach().float().requires_grad_() for k, v in model.weights.items()}
    want = plain_loss(model, tokens, targets, leaves)
    want.backward()
    assert abs(float(loss) - float(want.detach())) < 0.02 * float(want.detach())
    for k, v in leaves.items():
        rel = float((model.grads[k] - v.grad).norm() / v.grad.norm())
        assert rel < 0.06, (k, rel)


def test_decoder_beyond_the_widest_norm():
    """More columns than a block norm takes, no layers: the embedding, a norm and the loss."""
    torch()
    from paper_2410_15526_amd import sdp4
    from paper_2410_15526_amd.decoder import Config, Decoder, sequences
    from tests.test_gpu_decoder import plain_loss
    model = Decoder(Config(vocab=60, width=64, batch=2, hidden=sdp4.MAX_HIDDEN + 256, heads=64, layers=0), seed=3)
    tokens, targets = sequences(model.cfg, 2, 0)
    model.backward(tokens, targets, p=0.0)
    leaves = {k: v.detach().float().requires_grad_() for k, v in model.weights.items()}
    plain_loss(model, tokens, targets, leaves).backward()
    got, want = model.grads["embed"], leaves["embed"].grad
    assert float((got - want).norm() / want.norm()) < 0.06
