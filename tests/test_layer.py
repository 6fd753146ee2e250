"""Attention, block norms and the embedding without a GPU: the 64-bit forms the
GPU tests compare with, and the library's refusals (these calls never launch)."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2410_15526_amd import sdp4
from tests import _layer as ref

OK, EINVAL, EALIGN = 0, 1, 2
A = 0x7F0000000000          # made-up device addresses (never dereferenced)
B, D, E, F, G, H, I, J, W = (A + (i << 36) for i in range(1, 10))


def test_plain_attention_agrees_with_torch():
    torch = pytest.importorskip("torch")
    r = np.random.default_rng(1)
    lengths, n = [3, 0, 7, 1], 13
    q, k, v, do = (r.standard_normal((n, h, 8)) for h in (4, 2, 2, 4))
    z = [torch.tensor(x, requires_grad=True) for x in (q, k, v)]
    seq = np.repeat(np.arange(4), lengths)
    seen = torch.tensor((seq[:, None] == seq[None, :]) & (np.arange(11)[:, None] >= np.arange(11)[None, :]))
    outs, lses = [], []
    for h in range(4):
        s = (z[0][:11, h] @ z[1][:11, h // 2].T * 0.3).masked_fill(~seen, -math.inf)
        lses.append(torch.logsumexp(s, 1))
        outs.append(torch.softmax(s, 1) @ z[2][:11, h // 2])
    o = torch.stack(outs, 1)
    (want, _), (lse, _) = ref.attention(q, k, v, lengths, 0.3, "f32")
    assert np.allclose(want[:11], o.detach().numpy(), rtol=1e-12) and np.isnan(want[11:]).all()
    assert np.allclose(lse[:, :11], torch.stack(lses).detach().numpy(), rtol=1e-12)
    (o * torch.tensor(do[:11])).sum().backward()
    for (got, _), t in zip(ref.attention_grad(do, q, k, v, want, lse, lengths, 0.3, "f32"), z):
        assert np.allclose(got[:11], t.grad.numpy()[:11], rtol=1e-9, atol=1e-12) and np.isnan(got[11:]).all()


@pytest.mark.parametrize("post", [1e-5, None])
def test_plain_block_norm_agrees_with_torch(post):
    torch = pytest.importorskip("torch")
    r = np.random.default_rng(2)
    b, x, dh, dy = (r.standard_normal((5, 12)) for _ in range(4))
    w1, w2, gate = r.standard_normal(12), r.standard_normal(12), r.standard_normal(5)
    zb, zx, z1, z2, zg = (torch.tensor(t, requires_grad=True) for t in (b, x, w1, w2, gate))
    u = (zb * torch.rsqrt((zb ** 2).mean(1, keepdim=True) + post) if post else zb) * z1
    y = 0.7 * zx + 1.3 * zg[:, None] * u
    h = y * torch.rsqrt((y ** 2).mean(1, keepdim=True) + 1e-4) * z2
    (wy, _), (wh, _) = ref.block_norm(b, x, post, w1, gate, 1.3, 0.7, 1e-4, w2, "f32", "f32")
    assert np.allclose(wy, y.detach().numpy(), rtol=1e-12) and np.allclose(wh, h.detach().numpy(), rtol=1e-12)
    ((h * torch.tensor(dh)).sum() + (y * torch.tensor(dy)).sum()).backward()
    got = ref.block_norm_grad(dh, dy, b, wy, post, w1, gate, 1.3, 0.7, 1e-4, w2, "f32", "f32")
    for name, t in (("dbranch", zb), ("dresidual", zx), ("dpost_weight", z1), ("dpre_weight", z2), ("dgate", zg)):
        assert np.allclose(got[name][0], t.grad.numpy(), rtol=1e-9, atol=1e-12), name


# ---------------------------------------------------------------------------
# refusals
# ---------------------------------------------------------------------------
def addr(h):
    return None if h is None else C.addressof(h)


def heads(h):
    return None if h is None else sdp4.Heads(*h)


def prm(dt=0, dim=64, scale=0.125, offsets=W, sequences=3):
    return sdp4.AttentionParams(dt, dim, scale, offsets, sequences)


def attention(q=(A, 512, 64, 4), k=(B, 512, 64, 2), v=(D, 512, 64, 2), out=(E, 256, 64, 4), lse=F, tokens=8, **kw):
    hs, p = [heads(h) for h in (q, k, v, out)], prm(**kw)
    return sdp4.lib().sdp4_attention(*(addr(h) for h in hs[:3]), C.addressof(p), tokens, addr(hs[3]), lse, None)


@pytest.mark.cpu_only
@pytest.mark.parametrize("kw,want", [
    (dict(dt=2), EINVAL), (dict(dim=7), EINVAL), (dict(dim=257), EINVAL), (dict(scale=0.0), EINVAL), (dict(scale=-1.0), EINVAL),
    (dict(scale=math.inf), EINVAL), (dict(scale=math.nan), EINVAL), (dict(scale=2.0 ** -41), EINVAL), (dict(scale=2.0 ** 41), EINVAL),
    (dict(sequences=-1), EINVAL), (dict(sequences=1 << 31), EINVAL),
    (dict(offsets=W + 4), EALIGN), (dict(tokens=-1), EINVAL), (dict(tokens=(1 << 30) + 1), EINVAL), (dict(q=None), EINVAL),
    (dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(out=None), EINVAL), (dict(q=(None, 512, 64, 4)), EINVAL),
    (dict(k=(B, 512, 64, 3), v=(D, 512, 64, 3)), EINVAL), (dict(v=(D, 512, 64, 4)), EINVAL), (dict(out=(E, 256, 64, 3)), EINVAL),
    (dict(k=(B, 512, 64, 0), v=(D, 512, 64, 0)), EINVAL), (dict(k=(B, 1024, 64, 8), v=(D, 1024, 64, 8)), EINVAL),
    (dict(q=(A + 2, 512, 64, 4)), EALIGN), (dict(out=(E + 1, 256, 64, 4)), EALIGN), (dict(lse=F + 2), EALIGN),
    (dict(q=(A, 512, 63, 4)), EINVAL), (dict(k=(B, 0, 64, 2)), EINVAL), (dict(out=(A, 512, 64, 4)), EINVAL),
    (dict(out=(B, 256, 64, 4)), EINVAL), (dict(out=(D + 64, 256, 64, 4)), EINVAL), (dict(lse=A), EINVAL), (dict(lse=B), EINVAL),
    (dict(lse=E), EINVAL), (dict(lse=W), EINVAL), (dict(out=(W, 256, 64, 4)), EINVAL), (dict(tokens=0), OK),
    (dict(tokens=0, q=(None, 0, 0, 4)), OK),
])
def test_attention_refusals(kw, want):
    assert attention(**kw) == want


def attention_grad(dout=(A, 256, 64, 4), q=(B, 512, 64, 4), k=(B + 4 * 256, 512, 64, 2), v=(B + 4 * 384, 512, 64, 2),
                   out=(D, 256, 64, 4), lse=E, dq=(F, 512, 64, 4), dk=(F + 4 * 256, 512, 64, 2), dv=(F + 4 * 384, 512, 64, 2), ws=G,
                   nb=1 << 20, tokens=8, **kw):
    hs, p = [heads(h) for h in (dout, q, k, v, out, dq, dk, dv)], prm(**kw)
    a = [addr(h) for h in hs]
    return sdp4.lib().sdp4_attention_grad(*a[:5], lse, C.addressof(p), tokens, *a[5:], ws, nb, None)


@pytest.mark.cpu_only
@pytest.mark.parametrize("kw,want", [
    (dict(dt=9), EINVAL), (dict(dim=4), EINVAL), (dict(scale=math.nan), EINVAL), (dict(dout=None), EINVAL), (dict(out=None), EINVAL),
    (dict(dq=None), EINVAL), (dict(dk=None), EINVAL), (dict(dv=None), EINVAL), (dict(lse=None), EINVAL), (dict(lse=E + 1), EALIGN),
    (dict(dout=(A, 256, 64, 2)), EINVAL), (dict(dk=(F + 4 * 256, 512, 64, 1)), EINVAL), (dict(ws=None), EINVAL),
    (dict(nb=8 * 4 * 4 - 1), EINVAL), (dict(ws=G + 8), EALIGN), (dict(dq=(B, 512, 64, 4)), EINVAL), (dict(dq=(A, 256, 64, 4)), EINVAL),
    (dict(dk=(F + 4 * 64, 512, 64, 2)), EINVAL), (dict(dv=(F + 4 * 256, 512, 64, 2)), EINVAL), (dict(ws=A), EINVAL),
    (dict(ws=D), EINVAL), (dict(ws=F), EINVAL), (dict(ws=E), EINVAL), (dict(ws=W), EINVAL), (dict(dq=(D, 256, 64, 4)), EINVAL),
    (dict(dq=(E, 256, 64, 4)), EINVAL), (dict(dq=(F + 2, 512, 64, 4)), EALIGN), (dict(tokens=0), OK),
])
def test_attention_grad_refusals(kw, want):
    assert attention_grad(**kw) == want


def block_prm(xt=0, yt=0, post=1, e1=1e-6, e2=1e-6, w1=I, w2=I + 4096, gate=I + 8192, bs=1.0, rs=1.0):
    return sdp4.BlockParams(xt, yt, post, e1, e2, w1, w2, gate, bs, rs)


def block(b=A, b_s=64, r=B, r_s=64, rows=4, cols=64, y=D, y_s=64, h=E, h_s=64, **kw):
    p = block_prm(**kw)
    return sdp4.lib().sdp4_block_norm(b, b_s, r, r_s, rows, cols, C.addressof(p), y, y_s, h, h_s, None)


@pytest.mark.cpu_only
@pytest.mark.parametrize("kw,want", [
    (dict(xt=2), EINVAL), (dict(yt=-1), EINVAL), (dict(rows=-1), EINVAL), (dict(cols=-1), EINVAL), (dict(cols=16385), EINVAL),
    (dict(e1=-1.0), EINVAL), (dict(e2=math.nan), EINVAL), (dict(e1=math.inf), EINVAL), (dict(bs=math.inf), EINVAL),
    (dict(rs=math.nan), EINVAL), (dict(b_s=63), EINVAL), (dict(r_s=1), EINVAL), (dict(y_s=0), EINVAL), (dict(h_s=-64), EINVAL),
    (dict(b=None, r=None), EINVAL), (dict(y=None, h=None), EINVAL), (dict(b=None), EINVAL), (dict(b=None, post=0), EINVAL),
    (dict(b=None, post=0, w1=None), EINVAL), (dict(b=A + 2), EALIGN), (dict(y=D + 1), EALIGN), (dict(w1=I + 2), EALIGN),
    (dict(gate=I + 8194), EALIGN), (dict(y=A + 4), EINVAL), (dict(h=B + 8), EINVAL), (dict(h=D), EINVAL), (dict(y=I), EINVAL),
    (dict(h=I + 4096), EINVAL), (dict(y=I + 8192), EINVAL), (dict(y=A, xt=0, yt=1, r=None), EINVAL), (dict(rows=0), OK),
    (dict(cols=0, b=None, r=None, y=None, h=None), OK),
])
def test_block_norm_refusals(kw, want):
    assert block(**kw) == want


def block_grad(dh=A, dy=B, b=D, y=E, s=64, rows=4, cols=64, db=F, dr=G, dw1=H, dw2=H + 4096, dg=H + 8192, ws=J, nb=1 << 20, **kw):
    p = block_prm(**kw)
    return sdp4.lib().sdp4_block_norm_grad(dh, s, dy, s, b, s, y, s, rows, cols, C.addressof(p), db, s, dr, s, dw1, dw2, dg, ws, nb,
                                           None)


@pytest.mark.cpu_only
@pytest.mark.parametrize("kw,want", [
    (dict(xt=5), EINVAL), (dict(s=32), EINVAL), (dict(dh=None, dy=None), EINVAL), (dict(y=None), EINVAL), (dict(dh=None), EINVAL),
    (dict(w1=None), EINVAL), (dict(w2=None), EINVAL), (dict(gate=None), EINVAL), (dict(b=None), EINVAL),
    (dict(b=None, dw1=None, dg=None), EINVAL), (dict(b=None, dw1=None, post=0), EINVAL),
    (dict(db=None, dr=None, dw1=None, dw2=None, dg=None), EINVAL), (dict(ws=None), EINVAL), (dict(nb=100), EINVAL),
    (dict(ws=J + 4), EALIGN), (dict(dh=A + 2), EALIGN), (dict(dw1=H + 2), EALIGN), (dict(db=A + 8), EINVAL), (dict(dr=F), EINVAL),
    (dict(db=I), EINVAL), (dict(dr=H), EINVAL), (dict(dw1=A), EINVAL), (dict(dw2=H + 4), EINVAL), (dict(ws=E), EINVAL),
    (dict(ws=H), EINVAL), (dict(dg=I + 8192), EINVAL), (dict(cols=0), EINVAL), (dict(cols=0, dg=None), OK),
    (dict(rows=0, dw1=None, dw2=None), OK), (dict(rows=0, dw2=H + 16), EINVAL),
])
def test_block_norm_grad_refusals(kw, want):
    assert block_grad(**kw) == want


def embed(t=A, rows=4, tab=B, tt=0, ts=64, vocab=100, cols=64, scale=1.0, out=D, ot=0, os_=64):
    return sdp4.lib().sdp4_embedding(t, rows, tab, tt, ts, vocab, cols, scale, out, ot, os_, None)


@pytest.mark.cpu_only
@pytest.mark.parametrize("kw,want", [
    (dict(tt=2), EINVAL), (dict(ot=3), EINVAL), (dict(rows=-1), EINVAL), (dict(vocab=0), EINVAL), (dict(vocab=(1 << 20) + 1), EINVAL),
    (dict(scale=math.inf), EINVAL), (dict(scale=math.nan), EINVAL), (dict(ts=63), EINVAL), (dict(os_=1), EINVAL), (dict(t=None), EINVAL),
    (dict(tab=None), EINVAL), (dict(out=None), EINVAL), (dict(t=A + 4), EALIGN), (dict(tab=B + 2), EALIGN), (dict(out=D + 3), EALIGN),
    (dict(out=B), EINVAL), (dict(out=A), EINVAL), (dict(rows=0), OK), (dict(cols=0, tab=None, out=None), OK),
])
def test_embedding_refusals(kw, want):
    assert embed(**kw) == want


def embed_grad(t=A, rows=4, d=B, dt=0, ds=64, vocab=100, cols=64, scale=1.0, acc=0, tab=D, tt=0, ts=64, ws=W, nb=1 << 20):
    return sdp4.lib().sdp4_embedding_grad(t, rows, d, dt, ds, vocab, cols, scale, acc, tab, tt, ts, ws, nb, None)


@pytest.mark.cpu_only
@pytest.mark.parametrize("kw,want", [
    (dict(tt=2), EINVAL), (dict(dt=3), EINVAL), (dict(rows=-1), EINVAL), (dict(vocab=0), EINVAL), (dict(scale=math.nan), EINVAL),
    (dict(rows=(1 << 21) + 1, nb=1 << 40), EINVAL), (dict(ds=60), EINVAL), (dict(ts=60), EINVAL), (dict(t=None), EINVAL), (dict(d=None), EINVAL), (dict(tab=None), EINVAL),
    (dict(t=A + 4), EALIGN), (dict(d=B + 2), EALIGN), (dict(tab=D + 2), EALIGN), (dict(ws=None), EINVAL), (dict(nb=16), EINVAL),
    (dict(ws=W + 8), EALIGN), (dict(tab=B), EINVAL), (dict(tab=A), EINVAL), (dict(ws=A), EINVAL), (dict(ws=B), EINVAL),
    (dict(ws=D), EINVAL), (dict(rows=0, acc=1), OK), (dict(cols=0), OK),
])
def test_embedding_grad_refusals(kw, want):
    assert embed_grad(**kw) == want


@pytest.mark.cpu_only
def test_workspace_helpers():
    L = sdp4.lib()
    f = L.sdp4_attention_grad_workspace
    assert f(-1, 4, 2, 64) == -1 and f(8, 4, 3, 64) == -1 and f(8, 2, 4, 64) == -1 and f(8, 4, 2, 7) == -1 and f(8, 4, 2, 257) == -1
    assert f(0, 4, 2, 64) >= 0 and f(8192, 40, 8, 128) >= 8192 * 40 * 4
    f = L.sdp4_block_norm_grad_workspace
    assert f(-1, 8) == -1 and f(8, 16385) == -1 and f(0, 8) == 0 and f(8192, 5120) > 0
    f = L.sdp4_embedding_grad_workspace
    assert f(-1, 10, 8) == -1 and f(8, 0, 8) == -1 and f(8, (1 << 20) + 1, 8) == -1 and f(8, 10, -1) == -1 and f(0, 10, 8) > 0


@pytest.mark.cpu_only
def test_workspaces_serve_fewer_rows():
    L = sdp4.lib()
    rows = [*range(0, 300), *range(300, 20000, 37), 8191, 8192, 8193, 1 << 20]
    for f in (lambda n: L.sdp4_embedding_grad_workspace(n, 1000, 77), lambda n: L.sdp4_block_norm_grad_workspace(n, 77),
              lambda n: L.sdp4_attention_grad_workspace(n, 12, 4, 80)):
        sizes = [f(n) for n in sorted(rows)]
        assert sizes == sorted(sizes)


def test_inline_assembly_names_the_registers_that_it_writes():
    """m0 says where in LDS a load goes: it is an operand, so that the compiler knows, and no statement sets it by itself."""
    import glob
    import os
    import re
    root = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2410_15526_amd")
    loads = 0
    for path in sorted(glob.glob(os.path.join(root, "csrc*", "*.h*"))):
        with open(path) as f:
            for text in re.findall(r"\basm\b(?:\s+volatile)?\s*\((.*?)\)\s*;", f.read(), re.S):
                assert not re.search(r"s_\w+\s+m0\b", text), (path, text)
                if re.search(r"_lds_|\blds\b", text):
                    loads += 1
                    assert '"{m0}"(' in text, (path, text)
    assert loads > 0


@pytest.fixture(scope="module")
def shares(tmp_path_factory):
    """csrc_step/shares.hpp, compiled for the host."""
    import os
    import subprocess
    root = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2410_15526_amd", "csrc_step")
    folder = tmp_path_factory.mktemp("shares")
    (folder / "shares.cpp").write_text("""
#include "shares.hpp"
#include <vector>
extern "C" int64_t blocks(int64_t items) { return sdp4::shared_blocks(items); }
extern "C" void deal(int64_t blocks, int64_t items, int64_t *out)
{
    for (int64_t b = 0; b < blocks; ++b)
        out[b] = sdp4::shared_item(b, items);
}
extern "C" void places(int per_head, int64_t units, int64_t *out)
{
    for (int64_t x = 0; x < units; ++x)
        out[x] = sdp4::dealt_place(x, per_head, units);
}
""")
    lib = str(folder / "shares.so")
    subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", root, str(folder / "shares.cpp"), "-o", lib], check=True)
    L = C.CDLL(lib)
    L.blocks.restype, L.blocks.argtypes, L.deal.argtypes = C.c_int64, [C.c_int64], [C.c_int64, C.c_int64, C.c_void_p]
    L.places.argtypes = [C.c_int, C.c_int64, C.c_void_p]
    return L


def dealt(shares, blocks, items):
    out = np.empty(blocks, np.int64)
    shares.deal(blocks, items, out.ctypes.data)
    return out


@pytest.mark.parametrize("items", [1, 7, 8, 9, 63, 1000, (1 << 22) - 8, (1 << 22) + 1, (1 << 22) + 4096])
def test_every_work_item_is_dealt_once(items, shares):
    """Grids of more than 2^22 blocks are rounded up to whole rows of 2^22: the blocks of the rest have nothing to do."""
    n = shares.blocks(items)
    grid = n if n <= 1 << 22 else -(-n >> 22) << 22
    got = dealt(shares, grid, items)
    assert np.array_equal(np.sort(got[got < items]), np.arange(items)) and got.min() >= 0


@pytest.mark.parametrize("heads", [1, 2, 3, 4, 5, 7, 8, 9, 12, 16, 40])
@pytest.mark.parametrize("per_head", [1, 2, 5, 16, 29, 64, 100, 256, 2048])
def test_sorted_walks_are_dealt_evenly(heads, per_head, shares):
    """Each head's places once, and no share with more than its number of mean walks and two of the longest: of whole heads it
    has all, of the one that begins and the one that ends in it an even sample."""
    units = heads * per_head
    place = np.empty(units, np.int64)
    shares.places(per_head, units, place.ctypes.data)
    assert np.array_equal(np.sort(place.reshape(heads, per_head), 1), np.tile(np.arange(per_head), (heads, 1)))
    walks = np.sort(np.arange(per_head) % 16 + 1)[::-1].astype(float)          # sequences of 16 tiles
    for share in range(8):
        mine = place[share * -(-units // 8):(share + 1) * -(-units // 8)]
        assert walks[mine].sum() <= len(mine) * walks.mean() + 2 * walks.max()


def test_every_block_norm_of_the_library_is_reached():
    """A lane has as few accesses as eight waves leave: no kernel is built for more than the widest row asks for."""
    import re
    import subprocess
    names = subprocess.run(["nm", "-C", sdp4._LIB_PATH], capture_output=True, text=True, check=True).stdout
    found = set(re.findall(r"k_block_norm(?:_grad)?<(unsigned short|float), (unsigned short|float), (\d+), ", names))
    assert len(found) >= 16
    for x, y, accesses in found:
        elements = 8 if x == y == "unsigned short" else 4
        fewer = {1: 0, 2: 1, 3: 2, 4: 3, 8: 4}[int(accesses)]
        assert 64 * 8 * fewer * elements < sdp4.MAX_HIDDEN, (x, y, accesses)


@pytest.mark.cpu_only
def test_narrow_rows_fill_the_chip():
    """Sums of narrow rows' weight gradients over as many blocks as make eight waves on each of 256 compute units, of wide rows
    over 256 blocks: the workspace holds two sums of each."""
    f = sdp4.lib().sdp4_block_norm_grad_workspace
    for cols in (8, 64, 256, 512, 768, 1024, 1536, 2048, 3000, 5120, 16384):
        parts, waves = f(1 << 20, cols) // (8 * -(-cols // 8) * 8), -(-cols // 512)
        assert parts >= 256 and (parts * waves > 1024 or waves > 4), (cols, parts)
        assert parts == 256 or parts * waves <= 2048
        assert f(parts // 2, cols) == f(1 << 20, cols) // 2
