"""Attention, block norms and the embedding on the GPU against their 64-bit
forms (tests/_layer.py), at sizes, layouts, masks and values where they can go
wrong; gradients also against differences of the forward pass."""
import zlib

import numpy as np
import pytest

from paper_2410_15526_amd import sdp4
from tests import _layer as ref
from tests._gpu import say, torch
from tests.test_gpu_step import close, dt, f64, normal, scratch

pytestmark = pytest.mark.gpu
NAN = float("nan")


def rng(*key):
    """The same numbers in every run."""
    return torch().Generator(device="cuda").manual_seed(zlib.crc32(repr(key).encode()))


def offsets_of(lengths, lead=0):
    t = torch()
    return t.tensor(np.concatenate([[0], np.cumsum(lengths)]) + lead, dtype=t.int64, device="cuda")


def heads_like(tokens, heads, dim, dtype, layout, fill=NAN):
    """[tokens, heads, dim] inside a larger array of `fill`: (array, view)."""
    t = torch()
    if layout == "dense":
        buf = t.full((tokens, heads, dim), fill, dtype=dt(dtype), device="cuda")
        return buf, buf
    if layout == "odd":                      # odd strides and an odd start
        buf = t.full((tokens, heads * (dim + 3) + 5), fill, dtype=dt(dtype), device="cuda")
        return buf, buf[:, 1:1 + heads * (dim + 3)].unflatten(1, (heads, dim + 3))[:, :, :dim]
    buf = t.full((heads, tokens + 1, dim), fill, dtype=dt(dtype), device="cuda")    # head by head
    return buf, buf[:, 1:].transpose(0, 1)


def put(x, dtype, layout="dense"):
    buf, v = heads_like(*x.shape, dtype, layout)
    v.copy_(x)
    return v


class Case:
    def __init__(self, seed, lengths, tail, hq, hk, dim, dtype, lead=0, layout="dense", sharp=1.5):
        g = rng(seed, sum(lengths), tail, hq, hk, dim, dtype)
        n = lead + sum(lengths) + tail
        self.lengths, self.lead, self.n, self.dtype, self.scale = lengths, lead, n, dtype, dim ** -0.5
        self.q, self.k, self.v = (put(normal(g, n, h, dim, dtype=dtype, scale=s), dtype, layout)
                                  for h, s in ((hq, sharp), (hk, sharp), (hk, 1.0)))
        self.dout = put(normal(g, n, hq, dim, dtype=dtype), dtype, layout)
        self.offsets = offsets_of(lengths, lead)
        self.layout = layout

    def forward(self, offsets=True):
        t = torch()
        self.out_buf, self.out = heads_like(self.n, self.q.shape[1], self.q.shape[2], self.dtype, self.layout)
        self.lse = t.full((self.q.shape[1], self.n), NAN, device="cuda")
        sdp4.sdp4_attention(self.q, self.k, self.v, self.scale, self.offsets if offsets else None, self.out, self.lse)
        return self.out, self.lse

    def backward(self, offsets=True):
        pairs = [heads_like(self.n, x.shape[1], x.shape[2], self.dtype, self.layout) for x in (self.q, self.k, self.v)]
        self.bufs, grads = [p[0] for p in pairs], [p[1] for p in pairs]
        work = scratch(sdp4.sdp4_attention_grad_workspace(self.n, self.q.shape[1], self.k.shape[1], self.q.shape[2]))
        sdp4.sdp4_attention_grad(self.dout, self.q, self.k, self.v, self.out, self.lse, self.scale,
                                 self.offsets if offsets else None, *grads, work)
        return grads

    def check(self):
        cut = slice(self.lead, None)
        q, k, v = (f64(x)[cut] for x in (self.q, self.k, self.v))
        out, lse = self.forward()
        (wo, bo), (wl, bl) = ref.attention(q, k, v, self.lengths, self.scale, self.dtype)
        close(f64(out)[cut], wo, bo, "out")
        close(f64(lse)[:, cut], wl, bl, "lse")
        assert np.isnan(f64(out)[:self.lead]).all() and np.isnan(f64(lse)[:, :self.lead]).all()     # left as they were
        grads = self.backward()
        want = ref.attention_grad(f64(self.dout)[cut], q, k, v, np.nan_to_num(f64(out)[cut]), np.nan_to_num(f64(lse)[:, cut]),
                                  self.lengths, self.scale, self.dtype)
        for got, (w, b), name in zip(grads, want, ("dq", "dk", "dv")):
            close(f64(got)[cut], w, b, name)
            assert np.isnan(f64(got)[:self.lead]).all()


LENGTHS = [([1], 0), ([2], 1), ([31, 1, 0, 33], 0), ([64], 0), ([65, 63], 5), ([1] * 70, 3), ([130, 0, 0, 7, 200], 0), ([300], 40),
           ([0], 4), ([5, 0, 129, 1, 1, 250, 64], 19)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hk,dim", [(2, 2, 64), (6, 2, 128), (3, 1, 80), (4, 4, 96), (2, 1, 256)])
@pytest.mark.parametrize("lengths,tail", LENGTHS)
def test_attention(lengths, tail, hq, hk, dim, dtype):
    say("attention", lengths, tail, hq, hk, dim, dtype)
    Case(1, lengths, tail, hq, hk, dim, dtype).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [8, 9, 13, 31, 33, 63, 72, 79, 97, 120, 127, 129, 160, 192, 201, 255])
def test_attention_head_sizes(dim, dtype):
    say("attention dim", dim, dtype)
    Case(2, [40, 101, 3], 2, 4, 2, dim, dtype).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["odd", "heads"])
@pytest.mark.parametrize("dim", [64, 77, 128])
def test_attention_layouts(dim, layout, dtype):
    """Odd strides, head by head, rows before the first sequence; what lies around the outputs stays."""
    t = torch()
    say("attention layout", dim, layout, dtype)
    c = Case(3, [33, 90, 1], 6, 4, 2, dim, dtype, lead=5, layout=layout)
    c.check()
    for buf, view in [(c.out_buf, c.out)] + list(zip(c.bufs, (c.q, c.k, c.v))):
        assert int((~t.isnan(buf)).sum()) == sum(c.lengths) * view.shape[1] * dim


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_of_long_sequences(dtype):
    say("attention long", dtype)
    Case(4, [1500, 700], 0, 5, 1, 64, dtype, sharp=2.0).check()
    t = torch()
    c = Case(5, [777], 0, 2, 2, 128, dtype)                  # one sequence: with offsets and without
    a = [x.clone() for x in c.forward()] + [x.clone() for x in c.backward()]
    b = [x.clone() for x in c.forward(False)] + [x.clone() for x in c.backward(False)]
    assert all(t.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hk,dim,layout", [(4, 2, 40, "dense"), (2, 2, 77, "odd"), (3, 1, 128, "heads"), (2, 1, 250, "dense")])
def test_attention_gradient_in_pieces(hq, hk, dim, layout, dtype):
    """Few blocks and long walks: several blocks share one, some of them with nothing to do."""
    t = torch()
    say("attention pieces", hq, hk, dim, layout, dtype)
    lengths = [1, 900, 0, 3, 1100, 64]
    c = Case(10, lengths, 7, hq, hk, dim, dtype, lead=2, layout=layout)
    c.check()
    clean = [x.clone() for x in c.backward()]
    for buf, view in zip(c.bufs, (c.q, c.k, c.v)):
        assert int((~t.isnan(buf)).sum()) == sum(lengths) * view.shape[1] * dim
    for x, y in zip(clean, c.backward()):                    # the same bits again
        assert t.equal(x[2:-7], y[2:-7])
    at = 2 + 1 + 900 + 3 + 600                               # one value of the second long sequence, and what no row sees
    for x in (c.q, c.k, c.v, c.dout):
        x[at, :, dim // 2] = NAN
        x[:2], x[-7:] = NAN, float("inf")
    c.forward()
    spoilt = [x.clone() for x in c.backward()]
    first, last = at - 600, 2 + sum(lengths) - 64            # its sequence
    for x, y in zip(clean, spoilt):
        assert t.equal(x[2:first], y[2:first]) and t.equal(x[last:-7], y[last:-7])
        assert bool(t.isnan(y[at]).all())
    assert t.equal(clean[0][first:at], spoilt[0][first:at]) and bool(t.isnan(spoilt[0][at:last]).all())
    assert all(bool(t.isnan(y[first:at]).all()) for y in spoilt[1:])


@pytest.mark.parametrize("count", [255, 256, 257, 1000, 5000])
def test_attention_of_many_sequences(count):
    r = np.random.default_rng(count)
    lengths = [int(n) for n in r.integers(0, 4, count)]
    lengths[count // 2] = 150
    say("attention sequences", count)
    Case(6, lengths, 9, 1, 1, 64, "bf16").check()


def test_attention_gradient_against_differences():
    t = torch()
    c = Case(7, [20, 1, 41], 0, 4, 2, 16, "f32")
    c.forward()
    grads = c.backward()
    g = rng(8)
    for i, name in enumerate(("q", "k", "v")):
        x = getattr(c, name)
        way = normal(g, *x.shape)
        keep, eps, ends = x.clone(), 1e-2, []
        for s in (1, -1):
            x.copy_(keep + s * eps * way)
            ends.append(float((c.forward()[0].double() * c.dout.double()).sum()))
        x.copy_(keep)
        got, want = float((grads[i].double() * way.double()).sum()), (ends[0] - ends[1]) / (2 * eps)
        # third derivatives, eps^2 / 6 of a sum of order of the gradient, and float32 outputs divided by 2 eps
        scale = float((grads[i].double() ** 2).sum()) ** 0.5 * float((way.double() ** 2).sum()) ** 0.5
        noise = c.out.numel() ** 0.5 * 40 * 2.0 ** -24 * 10 / eps
        assert abs(got - want) < 1e-3 * scale + noise, (name, got, want)
    assert bool(t.isfinite(grads[0]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_attention_does_not_see_what_is_masked(dim, value, dtype):
    """Other sequences, later rows and rows in no sequence, holding NaN or infinities: not one bit of the others changes."""
    t = torch()
    lengths = [37, 50, 20]
    clean = Case(9, lengths, 30, 4, 2, dim, dtype)
    dirty = Case(9, lengths, 30, 4, 2, dim, dtype)
    at = 37 + 25                                             # row 25 of the second sequence
    for x in (dirty.q, dirty.k, dirty.v, dirty.dout):
        x[at, :, dim // 2] = value
        x[107:] = value
    for c in (clean, dirty):
        c.forward(), setattr(c, "grads", c.backward())
    same = lambda a, b: t.equal(a, b)  # noqa: E731
    for rows in (slice(0, at), slice(87, 107)):              # forward: all rows before it, and the other sequences
        assert same(clean.out[rows], dirty.out[rows]) and same(clean.lse[:, rows], dirty.lse[:, rows])
        assert same(clean.grads[0][rows], dirty.grads[0][rows])
    for i in (1, 2):                                         # keys and values: rows behind it, and the other sequences
        for rows in (slice(0, 37), slice(at + 1, 107)):
            if rows.start == 0:
                assert same(clean.grads[i][rows], dirty.grads[i][rows])
        assert same(clean.grads[i][87:107], dirty.grads[i][87:107])
    assert bool(t.isnan(dirty.out[107:]).all())              # still what the array was filled with
    assert not bool(t.isfinite(dirty.out[at].float()).all())
    if value != value:
        assert bool(t.isnan(dirty.out[at:87].float()).any(-1).all())
    # a later query's NaN alone leaves the gradients of the keys behind it alone
    late = Case(9, lengths, 30, 4, 2, dim, dtype)
    late.q[at, :, 0] = value
    late.dout[at, :, 1] = value
    late.forward()
    g = late.backward()
    for i in (1, 2):
        assert same(clean.grads[i][at + 1:107], g[i][at + 1:107]) and not bool(t.isfinite(g[i][at].float()).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_of_extreme_scores(dtype):
    t = torch()
    for big in (1e3, 1e5, 1e9, 1e15, 1e18):                  # scores of about big^2: one key takes a row
        c = Case(10, [90], 0, 2, 2, 64, dtype)
        c.q.mul_(big), c.k.mul_(1 if big > 1e9 else big)
        out, lse = c.forward()
        s = np.einsum("nhd,mhd->hnm", f64(c.q), f64(c.k)) * c.scale
        s[:, ~np.tril(np.ones((90, 90), bool))] = -np.inf
        best = s.argmax(2)
        second = np.sort(s, 2)[:, :, -2]
        # a product of 64 terms is off by 66 half steps of the sum of their magnitudes, which a score that cancels stays far below
        mag = np.einsum("nhd,mhd->hnm", np.abs(f64(c.q)), np.abs(f64(c.k))) * c.scale
        err = 70 * 2.0 ** -24 * np.where(np.isfinite(s), mag, 0).max(2)
        clear = s.max(2) - second > 40 + 20 * err            # rows that one key decides, whatever the roundings
        assert clear.sum() > 60
        v, o = f64(c.v), f64(out)
        for h in range(2):
            rows = np.nonzero(clear[h])[0]
            close(o[rows, h], v[best[h, rows], h], 2.0 ** -20 * np.abs(v[best[h, rows], h]) + 1e-12, ("out", big))
        assert np.isfinite(o).all() and bool(t.isfinite(lse).all())
        assert (np.abs(f64(lse) - s.max(2)) <= err * 4 + 5).all()
        assert all(bool(t.isfinite(g.float()).all()) for g in c.backward()), big
    c = Case(11, [70], 0, 2, 2, 64, dtype)                   # products beyond float32: -inf scores, and none but those
    c.q.fill_(1e30), c.k.fill_(-1e30)
    out, lse = c.forward()
    assert bool((out == 0).all()) and bool(t.isneginf(lse).all())
    dq, dk, dv = c.backward()
    assert bool((dv == 0).all())
    c.k.fill_(1e30)
    assert bool(t.isnan(c.forward()[0].float()).all())
    c = Case(12, [50], 0, 2, 2, 64, dtype)                   # equal scores, also the type's lowest value
    for fill in (0.0, float(t.finfo(dt(dtype)).min) / 1e4):
        c.q.fill_(0.0), c.k.fill_(fill)
        out, _ = c.forward()
        want = np.cumsum(f64(c.v), 0) / np.arange(1, 51)[:, None, None]
        low = 2.0 ** -8 * 1.01 if dtype == "bf16" else 0.0
        mag = np.cumsum(np.abs(f64(c.v)), 0) / np.arange(1, 51)[:, None, None]
        close(out, want, mag * (80 * 2.0 ** -24 + 2 * low), "means")


def test_attention_with_wrong_offsets_stays_inside():
    """Offsets that fall or leave the batch: wrong rows, nothing outside the arrays."""
    t = torch()
    for bad in ([0, 50, 20, 100], [-7, 30, 100], [0, 500], [90, 40, 0], [5, 5, 5, 5], [200, 300], [0, 1 << 40], [-(1 << 40), 60]):
        say("offsets", bad)
        c = Case(13, [100], 0, 2, 1, 64, "bf16", layout="odd")
        c.offsets = t.tensor(bad, dtype=t.int64, device="cuda")
        c.forward(), c.backward()
        t.cuda.synchronize()
        for buf in [c.out_buf] + c.bufs:
            heads = 2 if buf.shape[1] > 80 else 1
            around = t.ones_like(buf, dtype=t.bool)
            around[:, 1:1 + heads * 67].unflatten(1, (heads, 67))[:, :, :64] = False
            assert bool(t.isnan(buf[around]).all())


def test_attention_offsets_beyond_32_bits():
    """Heads whose elements lie more than 2^31 elements apart."""
    t = torch()
    n, hk, dim = 130, 2, 64
    g = rng(14)
    step = (1 << 25) + 8                                     # 130 rows: 4.4e9 elements
    big = t.empty(n * step, dtype=t.bfloat16, device="cuda")
    c = Case(15, [70, 60], 0, 4, hk, dim, "bf16")
    far = big.as_strided((n, hk, dim), (step, dim, 1))
    far.copy_(normal(g, n, hk, dim, dtype="bf16"))
    want = [Case.forward(c)]
    c.k = far.contiguous()
    want = [x.clone() for x in c.forward()] + [x.clone() for x in c.backward()]
    c.k = far
    got = [x.clone() for x in c.forward()] + [x.clone() for x in c.backward()]
    assert all(t.equal(a, b) for a, b in zip(want, got))


# ---------------------------------------------------------------------------
# block norms
# ---------------------------------------------------------------------------
COLS = [1, 3, 4, 7, 8, 9, 64, 255, 257, 500, 513, 768, 1000, 1025, 2048, 2050, 4097, 5120, 6145, 8192, 8200, 12291, 16384]
KINDS = ["full", "post", "pre", "plain", "gate"]


class Joint:
    def __init__(self, seed, rows, cols, x, y, kind):
        t = torch()
        g = rng(seed, rows, cols, x, y, kind)
        self.x, self.y_type, self.rows, self.cols = x, y, rows, cols
        self.branch = None if kind == "pre" else normal(g, rows, cols, dtype=x)
        self.residual = normal(g, rows, cols, dtype=y, scale=2.0)
        self.post = None if kind in ("pre", "plain") else 1e-5
        self.w1 = normal(g, cols, dtype=x) if kind in ("full", "post", "plain") else None
        self.w2 = normal(g, cols, dtype=x) if kind in ("full", "pre") else None
        self.gate = t.rand(rows, device="cuda", generator=g) if kind in ("full", "gate") else None
        self.scales = (1.0, 1.0) if kind == "plain" else (0.3, -1.7)
        self.dh, self.dy = normal(g, rows, cols, dtype=x), normal(g, rows, cols, dtype=y)

    def head(self):
        b, r = self.scales
        return [self.post, self.w1, self.gate, b, r]

    def forward(self, branch, residual, y, h):
        p, w1, gate, b, r = self.head()
        sdp4.sdp4_block_norm(branch, residual, p, w1, gate, b, r, y, 1e-6, self.w2, h)

    def numbers(self):
        n = lambda v: None if v is None else f64(v)  # noqa: E731
        return n(self.branch), n(self.residual), n(self.w1), n(self.gate), n(self.w2)

    def want(self):
        b, r, w1, gate, w2 = self.numbers()
        return ref.block_norm(b, r, self.post, w1, gate, *self.scales, 1e-6, w2, self.x, self.y_type)

    def want_grad(self, y, dh=True, dy=True):
        b, _, w1, gate, w2 = self.numbers()
        return ref.block_norm_grad(f64(self.dh) if dh else None, f64(self.dy) if dy else None, b, f64(y) if dh else None, self.post,
                                   w1, gate, *self.scales, 1e-6, w2, self.x, self.y_type)

    def backward(self, y, dh=True, dy=True, db=None, dr=None):
        t = torch()
        e = lambda n: t.full((n,), NAN, device="cuda")  # noqa: E731
        db = t.full((self.rows, self.cols), NAN, dtype=dt(self.x), device="cuda") if db is None else db
        dr = t.full((self.rows, self.cols), NAN, dtype=dt(self.y_type), device="cuda") if dr is None else dr
        dw1 = e(self.cols) if self.w1 is not None and self.branch is not None else None
        dw2 = e(self.cols) if self.w2 is not None and dh else None
        dg = e(self.rows) if self.gate is not None else None
        p, w1, gate, b, r = self.head()
        sdp4.sdp4_block_norm_grad(self.dh if dh else None, self.dy if dy else None, self.branch, y if dh else None, p, w1, gate, b, r,
                                  1e-6, self.w2, db, dr, dw1, dw2, dg, scratch(sdp4.sdp4_block_norm_grad_workspace(self.rows, self.cols)))
        return dict(dbranch=db, dresidual=dr, dpost_weight=dw1, dpre_weight=dw2, dgate=dg)


@pytest.mark.parametrize("x,y", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("cols", COLS)
def test_block_norm(cols, x, y):
    t = torch()
    for kind in KINDS:
        for rows in (1, 5, 67):
            say("block_norm", rows, cols, x, y, kind)
            c = Joint(20, rows, cols, x, y, kind)
            yo = t.full((rows, cols), NAN, dtype=dt(y), device="cuda")
            ho = t.full((rows, cols), NAN, dtype=dt(x), device="cuda")
            c.forward(c.branch, c.residual, yo, ho)
            (wy, by), (wh, bh) = c.want()
            close(yo, wy, by, ("y", kind))
            close(ho, wh, bh, ("h", kind))
            if kind == "pre" and rows > 1:
                h2 = t.full_like(ho, NAN)
                c.forward(None, c.residual, None, h2)        # y not wanted
                assert t.equal(h2, ho)
            for dh, dy in ((True, True), (True, False), (False, True)):
                got, want = c.backward(yo, dh, dy), c.want_grad(yo, dh, dy)
                for k, v in got.items():
                    if v is not None:
                        close(v, *want[k], (k, kind, dh, dy))


@pytest.mark.parametrize("x,y", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
def test_block_norm_many_rows_strides_and_in_place(x, y):
    t = torch()
    say("block_norm strides", x, y)
    c = Joint(21, 1301, 203, x, y, "full")
    (wy, by), (wh, bh) = c.want()

    def inside(v, gap, lead=1):
        buf = t.full((v.shape[0], v.shape[1] + gap), NAN, dtype=v.dtype, device="cuda")
        part = buf[:, lead:lead + v.shape[1]]
        part.copy_(v)
        return buf, part

    _, b = inside(c.branch, 3)
    _, r = inside(c.residual, 9, 5)
    ybuf, yo = inside(t.zeros_like(c.residual), 2)
    hbuf, ho = inside(t.zeros_like(c.branch), 6, 3)
    c.forward(b, r, yo, ho)
    close(yo, wy, by, "y")
    close(ho, wh, bh, "h")
    for buf, lead, gap in ((ybuf, 1, 2), (hbuf, 3, 6)):
        assert bool(t.isnan(buf[:, :lead]).all()) and bool(t.isnan(buf[:, lead + 203:]).all())
    y0 = yo.clone()
    c.forward(b, r, r, b)                                    # into the inputs
    assert t.equal(r, y0) and t.equal(b, ho)
    want = c.want_grad(y0)
    plain = c.backward(y0)
    for k, v in plain.items():
        close(v, *want[k], k)
    dh, dy = c.dh.clone(), c.dy.clone()
    again = c.backward(y0, db=c.dh, dr=c.dy)                 # into the gradients that came
    assert all(t.equal(again[k], plain[k]) for k in plain)
    c.dh, c.dy = dh, dy
    keep = c.branch.clone()
    again = c.backward(y0, db=c.branch, dr=y0)               # into what the forward pass left
    assert all(t.equal(again[k], plain[k]) for k in plain)
    c.branch = keep


def test_block_norm_against_differences():
    t = torch()
    c = Joint(22, 6, 40, "f32", "f32", "full")
    yo, ho = t.empty_like(c.residual), t.empty_like(c.residual)
    c.forward(c.branch, c.residual, yo, ho)
    grads = c.backward(yo)
    g = rng(23)
    for name, x in (("dbranch", c.branch), ("dresidual", c.residual), ("dpost_weight", c.w1), ("dpre_weight", c.w2), ("dgate", c.gate)):
        way, keep, ends, eps = normal(g, *x.shape), x.clone(), [], 1e-2
        for s in (1, -1):
            x.copy_(keep + s * eps * way)
            y2, h2 = t.empty_like(yo), t.empty_like(ho)
            c.forward(c.branch, c.residual, y2, h2)
            ends.append(float((h2.double() * c.dh.double()).sum() + (y2.double() * c.dy.double()).sum()))
        x.copy_(keep)
        got, want = float((grads[name].double() * way.double()).sum()), (ends[0] - ends[1]) / (2 * eps)
        size = float((grads[name].double() ** 2).sum()) ** 0.5 * float((way.double() ** 2).sum()) ** 0.5
        assert abs(got - want) < 2e-3 * size + 1e-3, (name, got, want)


def test_block_norm_edges():
    t = torch()
    x = t.zeros(3, 100, device="cuda")
    x[1] = 1e-30
    y, h = t.empty_like(x), t.empty_like(x)
    sdp4.sdp4_block_norm(x, None, 1e-6, None, None, 1.0, 1.0, y, 1e-6, None, h)     # rows of zeros: zeros
    assert bool((y[0] == 0).all()) and bool((h[0] == 0).all()) and bool(t.isfinite(h).all())
    x[2, 7] = NAN
    sdp4.sdp4_block_norm(x, x, 1e-6, None, None, 1.0, 1.0, y, 1e-6, None, h)
    assert bool(t.isnan(h[2]).all()) and bool(t.isfinite(h[:2]).all())             # rows stand alone
    e = t.empty(0, 100, device="cuda")
    sdp4.sdp4_block_norm(e, e, None, None, None, 1.0, 1.0, e, 1e-6, None, e)
    d1, d2 = t.full((100,), 3.0, device="cuda"), t.full((100,), 3.0, device="cuda")
    w = t.ones(100, device="cuda")
    sdp4.sdp4_block_norm_grad(e, e, e, e, 1e-6, w, None, 1.0, 1.0, 1e-6, w, e, e, d1, d2)
    assert bool((d1 == 0).all()) and bool((d2 == 0).all())                         # empty sums


# ---------------------------------------------------------------------------
# embedding
# ---------------------------------------------------------------------------
def tokens_of(g, rows, vocab, kind):
    t = torch()
    if kind == "one":
        return t.full((rows,), vocab // 2, dtype=t.int64, device="cuda")
    ids = t.randint(0, vocab, (rows,), device="cuda", generator=g)
    if kind == "skewed":
        ids = (vocab * t.rand(rows, device="cuda", generator=g) ** 6).long()
    if kind == "holes":
        ids[::3] = -1
        ids[1::7] = vocab + 5
        ids[2::11] = -(1 << 40)
        ids[4::13] = 1 << 40
    return ids


@pytest.mark.parametrize("x,y", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("rows,vocab,cols,kind", [
    (1, 1, 1, "any"), (7, 3, 5, "holes"), (31, 40, 64, "any"), (33, 11, 7, "skewed"), (64, 9, 130, "one"), (65, 2, 513, "one"),
    (100, 5000, 36, "any"), (128, 1, 96, "one"), (300, 12, 257, "holes"), (1000, 77, 100, "skewed"), (2047, 503, 765, "holes"),
    (8191, 900, 9, "skewed"), (8192, 31, 24, "one"), (8193, 1000, 24, "any"), (20001, 50, 17, "skewed"), (20001, 40000, 8, "holes"),
    (40000, 7, 12, "one"), (129, 600, 5120, "skewed")])
def test_embedding(rows, vocab, cols, kind, x, y):
    t = torch()
    say("embedding", rows, vocab, cols, kind, x, y)
    g = rng(rows, vocab, cols, kind, x, y)
    ids = tokens_of(g, rows, vocab, kind)
    table, dout, before = normal(g, vocab, cols, dtype=x), normal(g, rows, cols, dtype=x), normal(g, vocab, cols, dtype=y)
    out = t.full((rows, cols), NAN, dtype=dt(y), device="cuda")
    sdp4.sdp4_embedding(ids, table, 1.5, out)
    n = ids.cpu().numpy()
    close(out, *ref.embedding(n, f64(table), 1.5, y), "rows")
    work = scratch(sdp4.sdp4_embedding_grad_workspace(rows, vocab, cols))
    d = t.full((vocab, cols), NAN, dtype=dt(y), device="cuda")
    sdp4.sdp4_embedding_grad(ids, dout, 1.5, d, work)
    close(d, *ref.embedding_grad(n, f64(dout), 1.5, vocab, None, y), "gradient")
    first = d.clone()
    work.fill_(0x7F)
    sdp4.sdp4_embedding_grad(ids, dout, 1.5, d, work)
    assert t.equal(first, d)
    d = before.clone()
    sdp4.sdp4_embedding_grad(ids, dout, 1.5, d, work, accumulate=True)
    close(d, *ref.embedding_grad(n, f64(dout), 1.5, vocab, f64(before), y), "added")
    untouched = np.setdiff1d(np.arange(vocab), n)
    assert t.equal(d[untouched], before[untouched])          # rows of no token: not a bit


def test_embedding_strides_and_edges():
    t = torch()
    g = rng(30)
    ids = tokens_of(g, 500, 41, "holes")
    table = t.full((41, 110), NAN, device="cuda")
    table[:, 3:104] = normal(g, 41, 101)
    out = t.full((500, 120), NAN, device="cuda")
    sdp4.sdp4_embedding(ids, table[:, 3:104], -0.5, out[:, 7:108])
    close(out[:, 7:108], *ref.embedding(ids.cpu().numpy(), f64(table[:, 3:104]), -0.5, "f32"), "rows")
    assert bool(t.isnan(out[:, :7]).all()) and bool(t.isnan(out[:, 108:]).all())
    dout = out[:, 7:108].nan_to_num(0.0)
    wide = t.full((500, 103), NAN, device="cuda")
    wide[:, 1:102] = dout
    d = t.full((41, 109), NAN, device="cuda")
    sdp4.sdp4_embedding_grad(ids, wide[:, 1:102], 2.0, d[:, 5:106], scratch(sdp4.sdp4_embedding_grad_workspace(500, 41, 101)))
    close(d[:, 5:106], *ref.embedding_grad(ids.cpu().numpy(), f64(dout), 2.0, 41, None, "f32"), "gradient")
    assert bool(t.isnan(d[:, :5]).all()) and bool(t.isnan(d[:, 106:]).all())
    none = t.empty(0, dtype=t.int64, device="cuda")
    sdp4.sdp4_embedding(none, table, 1.0, t.empty(0, 110, device="cuda"))
    d.fill_(3.0)
    sdp4.sdp4_embedding_grad(none, t.empty(0, 109, device="cuda"), 1.0, d, scratch(sdp4.sdp4_embedding_grad_workspace(0, 41, 109)))
    assert bool((d == 0).all())
    d.fill_(3.0)
    sdp4.sdp4_embedding_grad(none, t.empty(0, 109, device="cuda"), 1.0, d, None, accumulate=True)
    assert bool((d == 3).all())


def test_embedding_of_a_large_table():
    """A table and a gradient of more than 2^31 elements: the last rows."""
    t = torch()
    vocab, cols = (1 << 20), 2056
    table = t.empty(vocab, cols, dtype=t.bfloat16, device="cuda")
    g = rng(31)
    ids = t.tensor([vocab - 1, 0, vocab - 1, vocab - 2], device="cuda")
    table[ids] = normal(g, 4, cols, dtype="bf16")
    out = t.empty(4, cols, dtype=t.bfloat16, device="cuda")
    sdp4.sdp4_embedding(ids, table, 1.0, out)
    assert t.equal(out, table[ids])
    dout = normal(g, 4, cols, dtype="bf16")
    table.fill_(NAN)
    sdp4.sdp4_embedding_grad(ids, dout, 1.0, table, scratch(sdp4.sdp4_embedding_grad_workspace(4, vocab, cols)))
    want = (dout[0].float() + dout[2].float()).bfloat16()
    assert t.equal(table[vocab - 1], want) and t.equal(table[vocab - 2], dout[3]) and t.equal(table[0], dout[1])
    assert bool((table[1:vocab - 2] == 0).all())


# ---------------------------------------------------------------------------
# together, captured, on other streams, through the general path
# ---------------------------------------------------------------------------
def a_layer(seed, dtype="bf16"):
    """A layer's passes, forward and backward, as a program with its own buffers calls them; returns (call, outputs)."""
    t = torch()
    g = rng(seed, dtype)
    n, hq, hk, d, vocab = 300, 6, 2, 64, 1000
    cols = hq * d
    e = lambda *s, ty=dt(dtype): t.zeros(*s, dtype=ty, device="cuda")  # noqa: E731
    s = dict(ids=t.randint(-1, vocab, (n,), device="cuda", generator=g), table=normal(g, vocab, cols, dtype=dtype),
             qkv=normal(g, n, hq + 2 * hk, d, dtype=dtype), w1=normal(g, cols, dtype=dtype), w2=normal(g, cols, dtype=dtype),
             gate=t.rand(n, device="cuda", generator=g), dh=normal(g, n, cols, dtype=dtype), off=offsets_of([100, 0, 150, 50]))
    q, k, v = s["qkv"][:, :hq], s["qkv"][:, hq:hq + hk], s["qkv"][:, hq + hk:]
    x, out, lse, y, h = e(n, cols), e(n, hq, d), e(hq, n, ty=t.float32), e(n, cols), e(n, cols)
    db, dr, dqkv = e(n, cols), e(n, cols), e(n, hq + 2 * hk, d)
    dw1, dw2, dg, dt_ = e(cols, ty=t.float32), e(cols, ty=t.float32), e(n, ty=t.float32), e(vocab, cols, ty=t.float32)
    works = [scratch(f) for f in (sdp4.sdp4_attention_grad_workspace(n, hq, hk, d), sdp4.sdp4_block_norm_grad_workspace(n, cols),
                                  sdp4.sdp4_embedding_grad_workspace(n, vocab, cols))]

    def call(stream=None):
        kw = {} if stream is None else dict(stream=stream)
        sdp4.sdp4_embedding(s["ids"], s["table"], 2.0, x, **kw)
        sdp4.sdp4_attention(q, k, v, 0.125, s["off"], out, lse, **kw)
        sdp4.sdp4_block_norm(out.view(n, cols), x, 1e-6, s["w1"], s["gate"], 0.5, 1.5, y, 1e-6, s["w2"], h, **kw)
        sdp4.sdp4_block_norm_grad(s["dh"], None, out.view(n, cols), y, 1e-6, s["w1"], s["gate"], 0.5, 1.5, 1e-6, s["w2"], db, dr, dw1,
                                  dw2, dg, works[1], **kw)
        sdp4.sdp4_attention_grad(db.view(n, hq, d), q, k, v, out, lse, 0.125, s["off"], dqkv[:, :hq], dqkv[:, hq:hq + hk],
                                 dqkv[:, hq + hk:], works[0], **kw)
        sdp4.sdp4_embedding_grad(s["ids"], dr, 2.0, dt_, works[2], **kw)

    return call, [x, out, lse, y, h, db, dr, dqkv, dw1, dw2, dg, dt_], s


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_layer_from_a_hip_graph(dtype):
    t = torch()
    call, outs, s = a_layer(40, dtype)
    call()
    t.cuda.synchronize()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        call()
    for i in range(4):
        for o in outs:
            o.fill_(0)
        s["ids"].copy_(s["ids"].roll(1)), s["qkv"].mul_(1.01), s["off"][2].add_(1)
        graph.replay()
        t.cuda.synchronize()
        got = [o.clone() for o in outs]
        for o in outs:
            o.fill_(0)
        call()                                               # the program's own eager work between replays
        t.cuda.synchronize()
        assert all(t.equal(a, b) for a, b in zip(got, outs)), i


def test_layers_on_other_streams_and_on_the_general_path(monkeypatch):
    t = torch()
    made = [a_layer(41), a_layer(42), a_layer(43, "f32")]
    for call, _, _ in made:
        call()
    t.cuda.synchronize()
    want = [[o.clone() for o in outs] for _, outs, _ in made]
    for _, outs, _ in made:
        for o in outs:
            o.fill_(0)
    t.cuda.synchronize()
    streams = [t.cuda.Stream() for _ in made]
    for _ in range(3):
        for (call, _, _), st in zip(made, streams):
            call(st)
    t.cuda.synchronize()
    assert all(t.equal(a, b) for w, (_, outs, _) in zip(want, made) for a, b in zip(w, outs))
    for _, outs, _ in made:
        for o in outs:
            o.fill_(0)
    t.cuda.synchronize()
    monkeypatch.setattr(sdp4, "_fast", None)
    for (call, _, _), st in zip(made, streams):
        with t.cuda.stream(st):
            call()
    t.cuda.synchronize()
    assert all(t.equal(a, b) for w, (_, outs, _) in zip(want, made) for a, b in zip(w, outs))


def test_layer_bindings_refuse_what_does_not_fit():
    t = torch()
    x, h = t.zeros(6, 64, device="cuda"), t.zeros(6, 2, 32, device="cuda")
    ids, off, lse = t.zeros(6, dtype=t.int64, device="cuda"), offsets_of([6]), t.zeros(2, 6, device="cuda")
    w = t.ones(64, device="cuda")
    work = scratch(1 << 20)
    o = t.zeros_like(h)
    bad = [
        lambda: sdp4.sdp4_attention(h, h[:5], h, 1.0, off, o, lse), lambda: sdp4.sdp4_attention(h, h, h[:, :1], 1.0, off, o, lse),
        lambda: sdp4.sdp4_attention(h, h, h, 1.0, off.int(), o, lse), lambda: sdp4.sdp4_attention(h, h, h, 1.0, off, o, lse.T),
        lambda: sdp4.sdp4_attention(h, h, h, 1.0, off, o.bfloat16(), lse), lambda: sdp4.sdp4_attention(h, h, h.cpu(), 1.0, off, o, lse),
        lambda: sdp4.sdp4_attention(h, h, h, 1.0, off[:0], o, lse), lambda: sdp4.sdp4_attention(h, h, h, 1.0, off.cpu(), o, lse),
        lambda: sdp4.sdp4_attention_grad(h, h, h, h, h, None, 1.0, off, o, o.clone(), o.clone(), work),
        lambda: sdp4.sdp4_attention_grad(h, h, h, h, h, lse, 1.0, off, o, o.clone()[:, :1], o.clone(), work),
        lambda: sdp4.sdp4_block_norm(x, x[:5], None, None, None, 1.0, 1.0, x, 1e-6, None, None),
        lambda: sdp4.sdp4_block_norm(x, x, None, w[:5], None, 1.0, 1.0, x, 1e-6, None, None),
        lambda: sdp4.sdp4_block_norm(x, x.bfloat16(), None, None, None, 1.0, 1.0, x, 1e-6, None, None),
        lambda: sdp4.sdp4_block_norm(x, x, None, None, w[:6].double(), 1.0, 1.0, x, 1e-6, None, None),
        lambda: sdp4.sdp4_block_norm(None, None, None, None, None, 1.0, 1.0, None, 1e-6, None, None),
        lambda: sdp4.sdp4_block_norm_grad(x, None, x, x, 1e-6, w, None, 1.0, 1.0, 1e-6, w, x.clone(), None, w.bfloat16(), None, None, work),
        lambda: sdp4.sdp4_embedding(ids.int(), x, 1.0, x.clone()), lambda: sdp4.sdp4_embedding(ids[:5], x, 1.0, x.clone()),
        lambda: sdp4.sdp4_embedding(ids, x, 1.0, t.zeros(6, 63, device="cuda")), lambda: sdp4.sdp4_embedding(None, x, 1.0, x.clone()),
        lambda: sdp4.sdp4_embedding_grad(ids, x.half(), 1.0, x.clone(), work),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
        print(i, flush=True)
    for f in (lambda: sdp4.sdp4_attention(h, h, h, 1.0, off, h, lse), lambda: sdp4.sdp4_attention(h, h, h, 0.0, off, o, lse),
              lambda: sdp4.sdp4_attention_grad(h, h, h, h, h, lse, 1.0, off, o, t.zeros_like(h), t.zeros_like(h), None),
              lambda: sdp4.sdp4_block_norm(x, x, -1.0, None, None, 1.0, 1.0, x, 1e-6, None, None),
              lambda: sdp4.sdp4_embedding_grad(ids, x, 1.0, x, work), lambda: sdp4.sdp4_embedding_grad(ids, x, 1.0, x.clone(), None)):
        with pytest.raises(sdp4.Sdp4Error):
            f()
