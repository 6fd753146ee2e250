// k_qk.hip -- RMS norm of every query and key head and the position
// rotation, in one pass, and the backward pass with the weights' gradients.
//
// For a head x of D elements at position p: r = 1 / sqrt(mean x^2 + eps),
// u = x r w, and every pair (a, b) among the first `rot` elements of u turns
// by the table's angle: a' = a c - b s, b' = b c + a s.  Backward: g is dy
// turned back, dw = sum g x r, dx = r (w g - x r mean(w g x r)).
//
// A head is the work of `lanes` neighbouring lanes (a power of two), each of
// which holds units of two chunks of W elements: the two members of W pairs
// in the half layout (chunks rot / 2 apart), chunks half of the elements apart
// in the interleaved layout and behind the rotated part.  So a rotation never
// crosses lanes, neighbouring lanes access neighbouring chunks, and a norm
// joins `lanes` lanes.
#include "step_device.hpp"

namespace sdp4 {

namespace {

// How heads are spread over lanes.
struct Layout {
    int dim, rot, half;   // half = rot / 2
    int rot_units, units; // units of two chunks: of the rotated part, of the head
    int lanes_log2;
    float inv_dim;
};

template <class T>
struct Side { // queries or keys
    const T *dy, *x;
    T *out;
    int64_t dy_token, dy_head, x_token, x_head, out_token, out_head;
    Divisor heads;
    uint32_t inv32;        // floor((2^32 - 1) / heads)
    int64_t items, blocks; // heads of all tokens, and the blocks that share them
    const T *weight;
    float *parts; // [blocks][dim] partial weight gradients
};

// One lane's unit of a head: where its two chunks lie, and which angles turn them.  Places that do not exist (`on`,
// `on_b`) name existing ones: they are read like the others and what is read is not used.
template <int W, bool INTER>
struct Unit {
    int a, b;      // first elements of the chunks
    bool on, on_b; // the unit exists; its second chunk does
    bool turn_a, turn_b;
    int angle_a, angle_b; // first angle of the chunk (in the half layout of both)
    SDP4_DEV Unit(const Layout &l, int u)
    {
        on = u < l.units;
        u = on ? u : 0;
        if constexpr (INTER && W > 1) {
            a = W * u, b = a + W * l.units;
            turn_a = a < l.rot, turn_b = b < l.rot;
            angle_a = turn_a ? a / 2 : 0, angle_b = turn_b ? b / 2 : 0;
        } else {
            const bool turned = u < l.rot_units;
            const int v = turned ? u : u - l.rot_units;
            a = turned ? (INTER ? 2 * u : W * u) : l.rot + W * v;
            b = turned ? (INTER ? a + 1 : a + l.half) : a + W * (l.units - l.rot_units);
            turn_a = turn_b = turned;
            angle_a = angle_b = turned ? W * u : 0;
        }
        on_b = on && b < l.dim;
        b = b < l.dim ? b : a;
        turn_b &= on_b;
    }
};

// W float32 table entries, which other lanes and blocks read again.
template <int W>
SDP4_DEV void load_kept(const float *p, float (&v)[W])
{
    constexpr int N = W > 4 ? 4 : W;
#pragma unroll
    for (int k = 0; k < W / N; ++k) {
        Raw<float, N> r;
        r.template load<false>(p + N * k);
        r.get(*reinterpret_cast<float(*)[N]>(v + N * k));
    }
}

// Two chunks of a lane's unit, as loaded and as values.
template <class T, int W>
struct RawTwo {
    Raw<T, W> a, b;
    template <bool NT, class U>
    SDP4_DEV void load(const T *head, const U &u)
    {
        a.template load<NT>(head + u.a);
        b.template load<NT>(head + u.b);
    }
};
template <int W>
struct Two {
    float a[W], b[W];
    template <class T>
    SDP4_DEV void get(const RawTwo<T, W> &r)
    {
        r.a.get(a);
        r.b.get(b);
    }
    SDP4_DEV void fill(float v)
    {
#pragma unroll
        for (int j = 0; j < W; ++j)
            a[j] = b[j] = v;
    }
    // what does not exist counts nothing in sums
    template <class U>
    SDP4_DEV void only(const U &u)
    {
        if (!u.on_b) {
#pragma unroll
            for (int j = 0; j < W; ++j)
                a[j] = u.on ? a[j] : 0.0f, b[j] = 0.0f;
        }
    }
    template <class T, class U>
    SDP4_DEV void store(T *head, const U &u) const
    {
        Raw<T, W> r;
        if (u.on) {
            r.put(a);
            r.store(head + u.a);
        }
        if (u.on_b) {
            r.put(b);
            r.store(head + u.b);
        }
    }
};

// Angles of a unit and their use.
template <int W, bool INTER>
struct Angles {
    // half layout (and W = 1): W cosines and sines for both chunks; interleaved: W / 2 of either for each chunk
    float c[W], s[W];
    SDP4_DEV void load(const Layout &l, const Unit<W, INTER> &u, const Rope &rope, int64_t position)
    {
        const bool known = position >= 0 && position < rope.rows;
        const float *row = rope.table + (known ? position : 0) * l.rot;
        if constexpr (INTER && W > 1) {
            constexpr int H = W / 2;
            float(&c0)[H] = *reinterpret_cast<float(*)[H]>(c), (&c1)[H] = *reinterpret_cast<float(*)[H]>(c + H);
            float(&s0)[H] = *reinterpret_cast<float(*)[H]>(s), (&s1)[H] = *reinterpret_cast<float(*)[H]>(s + H);
            load_kept<H>(row + u.angle_a, c0);
            load_kept<H>(row + l.half + u.angle_a, s0);
            load_kept<H>(row + u.angle_b, c1);
            load_kept<H>(row + l.half + u.angle_b, s1);
        } else {
            load_kept<W>(row + u.angle_a, c);
            load_kept<W>(row + l.half + u.angle_a, s);
        }
        if (!known) { // no such row: the result says so
#pragma unroll
            for (int j = 0; j < W; ++j)
                c[j] = s[j] = __builtin_nanf("");
        }
    }
    // BACK: by the opposite angle
    template <bool BACK>
    SDP4_DEV void turn(const Unit<W, INTER> &u, Two<W> &x) const
    {
        if (!u.turn_a)
            return;
        if constexpr (INTER && W > 1) {
#pragma unroll
            for (int j = 0; j < W / 2; ++j)
                one<BACK>(x.a[2 * j], x.a[2 * j + 1], c[j], s[j]);
            if (u.turn_b) { // only with turn_a: b lies behind a
#pragma unroll
                for (int j = 0; j < W / 2; ++j)
                    one<BACK>(x.b[2 * j], x.b[2 * j + 1], c[W / 2 + j], s[W / 2 + j]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < W; ++j)
                one<BACK>(x.a[j], x.b[j], c[j], s[j]);
        }
    }
    template <bool BACK>
    SDP4_DEV void all(Two<W> &x) const
    {
#pragma unroll
        for (int j = 0; j < W / (INTER && W > 1 ? 2 : 1); ++j) {
            if constexpr (INTER && W > 1) {
                one<BACK>(x.a[2 * j], x.a[2 * j + 1], c[j], s[j]);
                one<BACK>(x.b[2 * j], x.b[2 * j + 1], c[W / 2 + j], s[W / 2 + j]);
            } else {
                one<BACK>(x.a[j], x.b[j], c[j], s[j]);
            }
        }
    }
    template <bool BACK>
    SDP4_DEV static void one(float &a, float &b, float c, float s)
    {
        const float sn = BACK ? -s : s, x = a;
        a = __builtin_fmaf(x, c, -(b * sn));
        b = __builtin_fmaf(b, c, x * sn);
    }
};

SDP4_DEV int64_t position_of(const Rope &rope, int64_t token) { return rope.positions ? rope.positions[token] : token; }

// 1 / sqrt(v) to the last place but rounding: one Newton step on the estimate.
SDP4_DEV float rsqrt_of(float v)
{
    const float y = __builtin_amdgcn_rsqf(v);
    const float e = __builtin_fmaf(-v * y, y, 1.0f);
    const float z = __builtin_fmaf(0.5f * y, e, y);
    return e == e && __builtin_isfinite(y) ? z : y;
}

// Sum over the wave's groups of `lanes` lanes, lane by lane.
SDP4_DEV float sum_groups(float v, int lanes)
{
    if (lanes <= 1) v += xor_lane<1>(v);
    if (lanes <= 2) v += xor_lane<2>(v);
    if (lanes <= 4) v += xor_lane<4>(v);
    if (lanes <= 8) v += xor_lane<8>(v);
    if (lanes <= 16) v += xor_lane<16>(v);
    if (lanes <= 32) v += xor_lane<32>(v);
    return v;
}

// What a kernel knows beforehand.  The usual shapes are kernels of their own: 16-byte chunks, norm with weights, a known
// number of lanes and either every pair turned or, lane by lane, some.  What such a kernel need not ask (copies where
// optional turns and weights join, tests of the lane count) was a third of its vector instructions: backward of 8192 x 48
// bfloat16 heads of 128 59.9 -> 55.9 us (float32 111 -> 105), forward 36.0 -> 35.3, 8 tokens 4.14 -> 4.01.
enum Turn { kTurnAsked, kTurnAll, kTurnSome };
template <int W_, int NU_, bool INTER_, bool NORM_, int LL_ = -1, Turn TURN_ = kTurnAsked>
struct Known {
    static constexpr int W = W_, NU = NU_; // elements of a chunk, units of a lane
    static constexpr bool INTER = INTER_, NORM = NORM_;
    static constexpr int LL = LL_; // log2 of the lanes of a head, -1: asked
    static constexpr Turn TURN = TURN_;
    static constexpr bool WEIGHTS = LL >= 0; // given, otherwise asked
    SDP4_DEV static int lanes_log2(const Layout &l) { return LL >= 0 ? LL : l.lanes_log2; }
    SDP4_DEV static bool weights(const void *w) { return NORM && (WEIGHTS || w); }
    SDP4_DEV static bool turns(const Layout &l) { return TURN != kTurnAsked || l.rot; }
    template <bool BACK>
    SDP4_DEV static void turn(const Angles<W, INTER> &t, const Unit<W, INTER> &u, Two<W> &x)
    {
        if constexpr (TURN == kTurnAll) {
            t.template all<BACK>(x);
        } else if constexpr (TURN == kTurnSome) {
            Two<W> y = x;
            t.template all<BACK>(y);
#pragma unroll
            for (int j = 0; j < W; ++j)
                x.a[j] = u.turn_a ? y.a[j] : x.a[j], x.b[j] = u.turn_b ? y.b[j] : x.b[j];
        } else {
            t.template turn<BACK>(u, x);
        }
    }
};

// Forward: one head per group of lanes; the first blocks take the queries, the others the keys.  HBM bounds it: 205 MB
// (8192 x 48 bfloat16 heads of 128) in 35 us, 5.85 TB/s, float32 6.2, vector units half busy; table rows and weights come
// from the caches.
template <class T, class K>
__global__ __launch_bounds__(256) void k_qk(Layout l, Side<T> q, Side<T> k, float eps, Rope rope)
{
    constexpr int W = K::W, NU = K::NU;
    using U = Unit<W, K::INTER>;
    const int64_t wb = work_block();
    const bool keys = wb >= q.blocks;
    const Side<T> &s = keys ? k : q;
    const int ll = K::lanes_log2(l), lanes = 1 << ll, lane = threadIdx.x & (lanes - 1);
    // the block's first head, and from there the lane group's: below 2^9 + heads, so 32 bits do
    const int64_t first = (keys ? wb - q.blocks : wb) << (8 - ll);
    uint64_t head0;
    const int64_t token0 = (int64_t)divide((uint64_t)first, s.heads, head0);
    const uint32_t group = threadIdx.x >> ll;
    if (first + group >= s.items)
        return;
    uint32_t head = (uint32_t)head0 + group, ahead = __umulhi(head, s.inv32);
    head -= ahead * (uint32_t)s.heads.d;
    if (head >= (uint32_t)s.heads.d)
        head -= (uint32_t)s.heads.d, ++ahead;
    const int64_t token = token0 + ahead;
    const T *x = s.x + token0 * s.x_token + (uint64_t)ahead * (uint64_t)s.x_token + (uint64_t)head * (uint64_t)s.x_head;
    T *y = s.out + token0 * s.out_token + (uint64_t)ahead * (uint64_t)s.out_token + (uint64_t)head * (uint64_t)s.out_head;
    RawTwo<T, W> xr[NU], wr[NU];
    Two<W> v[NU], w[NU];
    Angles<W, K::INTER> turn[NU];
    const int64_t position = K::turns(l) ? position_of(rope, token) : 0;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
        const U u(l, lane + i * lanes);
        xr[i].template load<true>(x, u);
        if (K::weights(s.weight))
            wr[i].template load<false>(s.weight, u);
    }
    if (K::turns(l)) {
#pragma unroll
        for (int i = 0; i < NU; ++i)
            turn[i].load(l, U(l, lane + i * lanes), rope, position);
    }
#pragma unroll
    for (int i = 0; i < NU; ++i)
        v[i].get(xr[i]);
    if constexpr (K::NORM) {
        float sq = 0.0f;
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            v[i].only(U(l, lane + i * lanes));
#pragma unroll
            for (int j = 0; j < W; ++j) {
                sq = __builtin_fmaf(v[i].a[j], v[i].a[j], sq);
                sq = __builtin_fmaf(v[i].b[j], v[i].b[j], sq);
            }
        }
        const float r = rsqrt_of(__builtin_fmaf(sum_lanes(sq, lanes), l.inv_dim, eps));
#pragma unroll
        for (int i = 0; i < NU; ++i) {
#pragma unroll
            for (int j = 0; j < W; ++j)
                v[i].a[j] *= r, v[i].b[j] *= r;
            if (K::weights(s.weight)) {
                w[i].get(wr[i]);
#pragma unroll
                for (int j = 0; j < W; ++j)
                    v[i].a[j] *= w[i].a[j], v[i].b[j] *= w[i].b[j];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < NU; ++i) {
        const U u(l, lane + i * lanes);
        if (K::turns(l))
            K::template turn<false>(turn[i], u, v[i]);
        v[i].template store<T>(y, u);
    }
}

// Backward.  A block takes every blocks-th run of heads of its side; with DW it adds up the weights' gradient in
// registers, its lane groups and waves join at the end, and the block's sums go to the workspace.  The next head's loads
// are under way before the present one's stores: loads that follow stores wait for these.  8192 x 48 bfloat16 heads of 128:
// 306 MB in 51 us, 6.0 TB/s, and 4.5 for the sums over the blocks; without weight gradients 55.
template <class T, class K, bool DW>
__global__ __launch_bounds__(256) void k_qk_grad(Layout l, Side<T> q, Side<T> k, float eps, Rope rope)
{
    constexpr int W = K::W, NU = K::NU;
    using U = Unit<W, K::INTER>;
    __shared__ float lds[4][DW ? 2 * W : 1][kWave];
    const int64_t wb = work_block();
    const bool keys = wb >= q.blocks;
    const Side<T> &s = keys ? k : q;
    const int64_t block = keys ? wb - q.blocks : wb;
    const int ll = K::lanes_log2(l), lanes = 1 << ll, lane = threadIdx.x & (lanes - 1), group = threadIdx.x >> ll;
    const int groups = 256 >> ll;
    const uint32_t heads = (uint32_t)s.heads.d;
    // The lane group's heads are `step` apart: so many tokens and heads, where a carry makes one token more.
    uint64_t h0, hs;
    const int64_t step = s.blocks * groups;
    int64_t item = block * groups + group;
    int64_t token = (int64_t)divide((uint64_t)item, s.heads, h0);
    const int64_t token_step = (int64_t)divide((uint64_t)step, s.heads, hs);
    uint32_t head = (uint32_t)h0;
    const uint32_t head_step = (uint32_t)hs;
    const T *pdy = s.dy + token * s.dy_token + (int64_t)head * s.dy_head;
    const T *px = s.x + token * s.x_token + (int64_t)head * s.x_head;
    T *out = s.out + token * s.out_token + (int64_t)head * s.out_head, *next_out = out;
    const int64_t dy_step = token_step * s.dy_token + (int64_t)head_step * s.dy_head, dy_carry = s.dy_token - (int64_t)heads * s.dy_head;
    const int64_t x_step = token_step * s.x_token + (int64_t)head_step * s.x_head, x_carry = s.x_token - (int64_t)heads * s.x_head;
    const int64_t out_step = token_step * s.out_token + (int64_t)head_step * s.out_head, out_carry = s.out_token - (int64_t)heads * s.out_head;
    Two<W> dw[NU];
    RawTwo<T, W> dy[NU], x[NU], wr[NU];
#pragma unroll
    for (int i = 0; i < NU; ++i) {
        dw[i].fill(0.0f);
        if (K::weights(s.weight))
            wr[i].template load<false>(s.weight, U(l, lane + i * lanes));
    }
    int64_t position = 0;
    auto fetch = [&] {
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const U u(l, lane + i * lanes);
            dy[i].template load<true>(pdy, u);
            if constexpr (K::NORM)
                x[i].template load<true>(px, u);
        }
        if (K::turns(l))
            position = position_of(rope, token);
    };
    if (item < s.items)
        fetch();
    for (; item < s.items; item += step) {
        Two<W> g[NU], xv[NU];
        Angles<W, K::INTER> turn[NU];
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const U u(l, lane + i * lanes);
            g[i].get(dy[i]);
            g[i].only(u);
            if constexpr (K::NORM) {
                xv[i].get(x[i]);
                xv[i].only(u);
            }
            if (K::turns(l))
                turn[i].load(l, u, rope, position);
        }
        out = next_out;
        if (item + step < s.items) {
            const bool carry = head + head_step >= heads;
            head += head_step - (carry ? heads : 0u);
            token += token_step + carry;
            pdy += dy_step + (carry ? dy_carry : 0);
            px += x_step + (carry ? x_carry : 0);
            next_out += out_step + (carry ? out_carry : 0);
            fetch();
        }
        if (K::turns(l)) {
#pragma unroll
            for (int i = 0; i < NU; ++i)
                K::template turn<true>(turn[i], U(l, lane + i * lanes), g[i]);
        }
        if constexpr (K::NORM) {
            Two<W> gw[NU]; // w g
            float sq = 0.0f, dot = 0.0f;
#pragma unroll
            for (int i = 0; i < NU; ++i) {
                gw[i] = g[i];
                if (K::weights(s.weight)) {
                    Two<W> w;
                    w.get(wr[i]);
#pragma unroll
                    for (int j = 0; j < W; ++j)
                        gw[i].a[j] *= w.a[j], gw[i].b[j] *= w.b[j];
                }
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    sq = __builtin_fmaf(xv[i].a[j], xv[i].a[j], sq);
                    dot = __builtin_fmaf(gw[i].a[j], xv[i].a[j], dot);
                    sq = __builtin_fmaf(xv[i].b[j], xv[i].b[j], sq);
                    dot = __builtin_fmaf(gw[i].b[j], xv[i].b[j], dot);
                }
            }
            const float r = rsqrt_of(__builtin_fmaf(sum_lanes(sq, lanes), l.inv_dim, eps));
            const float m = -(sum_lanes(dot, lanes) * l.inv_dim) * r * r * r; // - mean(w g x r) r^2
#pragma unroll
            for (int i = 0; i < NU; ++i)
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    if constexpr (DW) {
                        dw[i].a[j] = __builtin_fmaf(g[i].a[j], xv[i].a[j] * r, dw[i].a[j]);
                        dw[i].b[j] = __builtin_fmaf(g[i].b[j], xv[i].b[j] * r, dw[i].b[j]);
                    }
                    g[i].a[j] = __builtin_fmaf(xv[i].a[j], m, gw[i].a[j] * r);
                    g[i].b[j] = __builtin_fmaf(xv[i].b[j], m, gw[i].b[j] * r);
                }
        }
#pragma unroll
        for (int i = 0; i < NU; ++i)
            g[i].template store<T>(out, U(l, lane + i * lanes));
    }
    if constexpr (DW) {
        if (!s.parts)
            return;
        const int wave = threadIdx.x / kWave;
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            if (i)
                __syncthreads();
#pragma unroll
            for (int j = 0; j < W; ++j) {
                dw[i].a[j] = sum_groups(dw[i].a[j], lanes), dw[i].b[j] = sum_groups(dw[i].b[j], lanes);
                if (lane_id() < lanes) {
                    lds[wave][2 * j][lane] = dw[i].a[j];
                    lds[wave][2 * j + 1][lane] = dw[i].b[j];
                }
            }
            __syncthreads();
            for (int o = threadIdx.x; o < 2 * W * lanes; o += 256) {
                const int which = o >> ll, ln = o & (lanes - 1);
                const U v(l, ln + i * lanes);
                const float sum = (lds[0][which][ln] + lds[1][which][ln]) + (lds[2][which][ln] + lds[3][which][ln]);
                const int at = (which & 1 ? v.b : v.a) + (which >> 1);
                if (which & 1 ? v.on_b : v.on)
                    s.parts[block * l.dim + at] = sum;
            }
        }
    }
}

__global__ __launch_bounds__(256) void k_rope_table(const double *inv_freq, int half, int64_t start, int64_t rows,
                                                    double scale, float *table)
{
    const int64_t i = work_block() * 256 + threadIdx.x;
    if (i >= rows * half)
        return;
    const int64_t row = i / half, j = i - row * half;
    double sn, cs;
    sincos((double)(start + row) * inv_freq[j], &sn, &cs);
    table[row * 2 * half + j] = (float)(cs * scale);
    table[row * 2 * half + half + j] = (float)(sn * scale);
}

// The widest chunk that cuts the rotated part and the rest evenly.
int chunk_width(int widest, int dim, const Rope &r)
{
    for (int w = widest; w > 1; w /= 2) {
        if (w == 2 || dim > 128 * w)
            continue;
        if (r.interleaved ? r.rot % w == 0 && dim % w == 0 : (r.rot / 2) % w == 0 && (dim - r.rot) % w == 0)
            return w;
    }
    return 1;
}

Layout layout_of(int dim, const Rope &r, int w, int &nu)
{
    Layout l{};
    l.dim = dim, l.rot = r.rot, l.half = r.rot / 2;
    l.inv_dim = 1.0f / (float)dim;
    if (r.interleaved && w > 1) {
        l.units = (dim / w + 1) / 2;
        l.rot_units = l.units;
    } else {
        l.rot_units = r.rot / 2 / w;
        l.units = l.rot_units + ((dim - r.rot) / w + 1) / 2;
    }
    while (l.lanes_log2 < 6 && (1 << l.lanes_log2) < l.units)
        ++l.lanes_log2;
    nu = l.units > 64 ? 4 : 1;
    return l;
}

template <class T>
Side<T> side_of(const Heads *dy, const Heads &x, const Heads &out, int64_t tokens, const void *weight)
{
    Side<T> s{};
    s.heads = Divisor((uint64_t)(out.heads > 0 ? out.heads : 1));
    s.inv32 = ~uint32_t(0) / (uint32_t)s.heads.d;
    s.items = tokens * out.heads;
    s.x = static_cast<const T *>(x.p), s.x_token = x.token_stride, s.x_head = x.head_stride;
    s.out = static_cast<T *>(out.p), s.out_token = out.token_stride, s.out_head = out.head_stride;
    if (dy)
        s.dy = static_cast<const T *>(dy->p), s.dy_token = dy->token_stride, s.dy_head = dy->head_stride;
    s.weight = static_cast<const T *>(weight);
    return s;
}

// Calls run(Known<...>) for the shape.
template <class T, class F>
int with_known(const Layout &l, int w, int nu, bool inter, const HeadNorm &norm, bool keys, F run)
{
    constexpr int CW = kChunk<T>;
    auto general = [&](auto wc, auto nc) {
        constexpr int W = decltype(wc)::value, NU = decltype(nc)::value;
        return inter ? (norm.on ? run(Known<W, NU, true, true>{}) : run(Known<W, NU, true, false>{}))
                     : (norm.on ? run(Known<W, NU, false, true>{}) : run(Known<W, NU, false, false>{}));
    };
    using std::integral_constant;
    if (w == CW && norm.on && norm.weight[0] && (norm.weight[1] || !keys) && l.rot > 0 && l.lanes_log2 >= 2 && l.lanes_log2 <= 5) {
        const bool all = l.rot == l.dim;
        auto at = [&](auto ll) {
            constexpr int LL = decltype(ll)::value;
            return inter ? (all ? run(Known<CW, 1, true, true, LL, kTurnAll>{}) : run(Known<CW, 1, true, true, LL, kTurnSome>{}))
                         : (all ? run(Known<CW, 1, false, true, LL, kTurnAll>{}) : run(Known<CW, 1, false, true, LL, kTurnSome>{}));
        };
        switch (l.lanes_log2) {
        case 2: return at(integral_constant<int, 2>{});
        case 3: return at(integral_constant<int, 3>{});
        case 4: return at(integral_constant<int, 4>{});
        default: return at(integral_constant<int, 5>{});
        }
    }
    if (w == CW)
        return general(integral_constant<int, CW>{}, integral_constant<int, 1>{});
    if constexpr (CW == 8)
        if (w == 4)
            return general(integral_constant<int, 4>{}, integral_constant<int, 1>{});
    return nu == 1 ? general(integral_constant<int, 1>{}, integral_constant<int, 1>{})
                   : general(integral_constant<int, 1>{}, integral_constant<int, 4>{});
}

// Blocks of the backward pass with weight gradients: about kGradBlocks for both sides, in proportion to their heads, each
// of which walks through the tokens with the others.  8192 x 48 heads of 128, bfloat16 / float32, blocks 576 / 768 / 960 /
// 1152: 61.3 / 56.7 / 58.1 / 67.8 us and 117.6 / 106.5 / 108.1 / 114.8; 768 are three to each of the 256 compute units.
constexpr int64_t kGradBlocks = 768;
int64_t grad_blocks(int64_t items, int64_t all, int groups)
{
    if (items == 0)
        return 0;
    const int64_t most = (items + groups - 1) / groups;
    const int64_t want = (kGradBlocks * items + all - 1) / all;
    return want < most ? want : most;
}

} // namespace

int64_t qk_grad_workspace(int64_t tokens, int q_heads, int k_heads, int dim)
{
    // as many blocks as any layout of such heads takes: 4 groups of lanes (of 64) in a block and more
    const int64_t qi = tokens * q_heads, ki = tokens * k_heads;
    if (qi + ki <= 0 || dim <= 0)
        return 0;
    return (grad_blocks(qi, qi + ki, 4) + grad_blocks(ki, qi + ki, 4)) * dim * (int64_t)sizeof(float);
}

int launch_qk(int dtype, const Heads (&x)[2], const Heads (&y)[2], int64_t tokens, int dim, const HeadNorm &norm,
              const Rope &rope, hipStream_t s)
{
    return with_type(dtype, [&](auto tag) {
        using T = decltype(tag);
        int nu;
        const int w = chunk_width(kChunk<T>, dim, rope);
        const Layout l = layout_of(dim, rope, w, nu);
        const int64_t groups = 256 >> l.lanes_log2;
        Side<T> q = side_of<T>(nullptr, x[0], y[0], tokens, norm.weight[0]);
        Side<T> k = side_of<T>(nullptr, x[1], y[1], tokens, norm.weight[1]);
        q.blocks = (q.items + groups - 1) / groups, k.blocks = (k.items + groups - 1) / groups;
        return with_known<T>(l, w, nu, rope.interleaved, norm, k.items > 0, [&](auto known) {
            return launch<4>(k_qk<T, decltype(known)>, q.blocks + k.blocks, kUncapped, s, l, q, k, norm.eps, rope);
        });
    });
}

int launch_qk_grad(int dtype, const Heads (&dy)[2], const Heads (&x)[2], const Heads (&dx)[2], int64_t tokens,
                   int dim, const HeadNorm &norm, const Rope &rope, float *const (&dw)[2], float *workspace,
                   hipStream_t s)
{
    const bool want_dw = dw[0] || dw[1];
    Side<float> sums[2]{};
    const int rc = with_type(dtype, [&](auto tag) {
        using T = decltype(tag);
        int nu;
        const int w = chunk_width(kChunk<T>, dim, rope);
        const Layout l = layout_of(dim, rope, w, nu);
        const int groups = 256 >> l.lanes_log2;
        Side<T> q = side_of<T>(&dy[0], x[0], dx[0], tokens, norm.weight[0]);
        Side<T> k = side_of<T>(&dy[1], x[1], dx[1], tokens, norm.weight[1]);
        const int64_t all = q.items + k.items;
        if (want_dw) {
            q.blocks = grad_blocks(q.items, all, groups), k.blocks = grad_blocks(k.items, all, groups);
            q.parts = dw[0] ? workspace : nullptr;
            k.parts = dw[1] ? workspace + q.blocks * dim : nullptr;
            sums[0].parts = q.parts, sums[0].blocks = q.blocks;
            sums[1].parts = k.parts, sums[1].blocks = k.blocks;
        } else { // nothing to add up: a block per group of heads
            q.blocks = (q.items + groups - 1) / groups, k.blocks = (k.items + groups - 1) / groups;
        }
        return with_known<T>(l, w, nu, rope.interleaved, norm, k.items > 0, [&](auto known) {
            using K = decltype(known);
            auto kernel = k_qk_grad<T, K, false>;
            if constexpr (K::NORM)
                if (want_dw)
                    kernel = k_qk_grad<T, K, true>;
            return launch<4>(kernel, q.blocks + k.blocks, kUncapped, s, l, q, k, norm.eps, rope);
        });
    });
    if (rc)
        return rc;
    if (sums[0].parts && sums[1].parts)
        return launch_sum_parts({{sums[0].parts, sums[0].blocks, dw[0]}, {sums[1].parts, sums[1].blocks, dw[1]}}, dim, dim, s);
    for (int i = 0; i < 2; ++i)
        if (sums[i].parts)
            return launch_sum_parts({{sums[i].parts, sums[i].blocks, dw[i]}, {}}, dim, dim, s);
    return 0;
}

int launch_rope_table(const double *inv_freq, int half, int64_t start, int64_t rows, double scale, float *table,
                      hipStream_t s)
{
    return launch<4>(k_rope_table, (rows * half + 255) / 256, kUncapped, s, inv_freq, half, start, rows, scale, table);
}

} // namespace sdp4
