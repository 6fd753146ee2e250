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
// in the half layout (chunks rot / 2 apart), neighbouring chunks in the
// interleaved layout and behind the rotated part.  So a rotation never
// crosses lanes, and a norm joins `lanes` lanes.
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
            a = 2 * W * u, b = a + W;
            turn_a = a < l.rot, turn_b = b < l.rot;
            angle_a = turn_a ? a / 2 : 0, angle_b = turn_b ? b / 2 : 0;
        } else {
            const bool turned = u < l.rot_units;
            const int v = turned ? u : u - l.rot_units;
            a = turned ? (INTER ? 2 * u : W * u) : l.rot + 2 * W * v;
            b = turned && !INTER ? a + l.half : a + W;
            turn_a = turn_b = turned;
            angle_a = angle_b = turned ? W * u : 0;
        }
        on_b = on && b < l.dim;
        b = b < l.dim ? b : a;
        turn_b &= on_b;
    }
};

// W elements at an element address.
template <class T, int W, bool NT>
SDP4_DEV void load_w(const T *p, float (&v)[W])
{
    if constexpr (W * sizeof(T) == 16) {
        unpack<T>(load_chunk<NT>(p), v);
    } else if constexpr (W * sizeof(T) == 8) {
        auto q = reinterpret_cast<const half_at<T> *>(p);
        const u32x2 c = NT ? (u32x2)__builtin_nontemporal_load(q) : (u32x2)*q;
        if constexpr (W == 2) {
            v[0] = __uint_as_float(c.x), v[1] = __uint_as_float(c.y);
        } else {
            v[0] = __uint_as_float(c.x << 16), v[1] = __uint_as_float(c.x & 0xFFFF0000u);
            v[2] = __uint_as_float(c.y << 16), v[3] = __uint_as_float(c.y & 0xFFFF0000u);
        }
    } else if constexpr (sizeof(T) == 4 && W % 4 == 0) {
#pragma unroll
        for (int k = 0; k < W / 4; ++k)
            unpack<T>(load_chunk<NT>(p + 4 * k), *reinterpret_cast<float(*)[4]>(v + 4 * k));
    } else {
#pragma unroll
        for (int j = 0; j < W; ++j)
            v[j] = to_f32<T>(p[j]);
    }
}
template <class T, int W>
SDP4_DEV void store_w(T *p, const float (&v)[W])
{
    if constexpr (W * sizeof(T) == 16)
        store_chunk<T>(p, pack<T>(v));
    else if constexpr (W * sizeof(T) == 8)
        store_half(p, v);
    else
#pragma unroll
        for (int j = 0; j < W; ++j)
            p[j] = from_f32<T>(v[j]);
}

// Two chunks of a lane's unit.
template <int W>
struct Two {
    float a[W], b[W];
    template <bool NT, class T, class U>
    SDP4_DEV void load(const T *head, const U &u)
    {
        load_w<T, W, NT>(head + u.a, a);
        load_w<T, W, NT>(head + u.b, b);
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
        if (u.on)
            store_w<T, W>(head + u.a, a);
        if (u.on_b)
            store_w<T, W>(head + u.b, b);
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
            load_w<float, H, false>(row + u.angle_a, c0);
            load_w<float, H, false>(row + l.half + u.angle_a, s0);
            load_w<float, H, false>(row + u.angle_b, c1);
            load_w<float, H, false>(row + l.half + u.angle_b, s1);
        } else {
            load_w<float, W, false>(row + u.angle_a, c);
            load_w<float, W, false>(row + l.half + u.angle_a, s);
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
            if (u.turn_b) {
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

// Forward: one head per group of lanes; the first blocks take the queries, the others the keys.
template <class T, int W, int NU, bool INTER, bool NORM>
__global__ __launch_bounds__(256) void k_qk(Layout l, Side<T> q, Side<T> k, float eps, Rope rope)
{
    const int64_t wb = work_block();
    const bool keys = wb >= q.blocks;
    const Side<T> &s = keys ? k : q;
    const int lanes = 1 << l.lanes_log2, lane = threadIdx.x & (lanes - 1);
    // the block's first head, and from there the lane group's: below 2^9 + heads, so 32 bits do
    const int64_t first = (keys ? wb - q.blocks : wb) << (8 - l.lanes_log2);
    uint64_t head0;
    const int64_t token0 = (int64_t)divide((uint64_t)first, s.heads, head0);
    const uint32_t group = threadIdx.x >> l.lanes_log2;
    if (first + group >= s.items)
        return;
    uint32_t head = (uint32_t)head0 + group, ahead = __umulhi(head, s.inv32);
    head -= ahead * (uint32_t)s.heads.d;
    if (head >= (uint32_t)s.heads.d)
        head -= (uint32_t)s.heads.d, ++ahead;
    const int64_t token = token0 + ahead;
    const T *x = s.x + token0 * s.x_token + (uint64_t)ahead * (uint64_t)s.x_token + (uint64_t)head * (uint64_t)s.x_head;
    T *y = s.out + token0 * s.out_token + (uint64_t)ahead * (uint64_t)s.out_token + (uint64_t)head * (uint64_t)s.out_head;
    Two<W> v[NU], w[NU];
    Angles<W, INTER> turn[NU];
    const int64_t position = l.rot ? position_of(rope, token) : 0;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
        const Unit<W, INTER> u(l, lane + i * lanes);
        v[i].template load<true>(x, u);
        if constexpr (NORM) {
            if (s.weight)
                w[i].template load<false>(s.weight, u);
        }
    }
    if (l.rot) {
#pragma unroll
        for (int i = 0; i < NU; ++i)
            turn[i].load(l, Unit<W, INTER>(l, lane + i * lanes), rope, position);
    }
    if constexpr (NORM) {
        float sq = 0.0f;
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            v[i].only(Unit<W, INTER>(l, lane + i * lanes));
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
            if (s.weight) {
#pragma unroll
                for (int j = 0; j < W; ++j)
                    v[i].a[j] *= w[i].a[j], v[i].b[j] *= w[i].b[j];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < NU; ++i) {
        const Unit<W, INTER> u(l, lane + i * lanes);
        if (l.rot)
            turn[i].template turn<false>(u, v[i]);
        v[i].store(y, u);
    }
}

// Backward.  A block takes every blocks-th run of heads of its side; with DW it adds up the weights' gradient in
// registers, its lane groups and waves join at the end, and the block's sums go to the workspace.  The next head's loads
// are under way before the present one's stores: loads that follow stores wait for these.
template <class T, int W, int NU, bool INTER, bool NORM, bool DW>
__global__ __launch_bounds__(256) void k_qk_grad(Layout l, Side<T> q, Side<T> k, float eps, Rope rope)
{
    __shared__ float lds[DW ? 256 * 2 * W : 1];
    const int64_t wb = work_block();
    const bool keys = wb >= q.blocks;
    const Side<T> &s = keys ? k : q;
    const int64_t block = keys ? wb - q.blocks : wb;
    const int lanes = 1 << l.lanes_log2, lane = threadIdx.x & (lanes - 1), group = threadIdx.x >> l.lanes_log2;
    const int groups = 256 >> l.lanes_log2;
    const uint32_t heads = (uint32_t)s.heads.d;
    // first head of the lane group, and the step to its next: tokens and heads, where a carry makes one token more
    uint64_t h0, hs;
    int64_t item = block * groups + group;
    const int64_t step = s.blocks * groups;
    int64_t token = (int64_t)divide((uint64_t)item, s.heads, h0);
    const int64_t token_step = (int64_t)divide((uint64_t)step, s.heads, hs);
    uint32_t head = (uint32_t)h0;
    const uint32_t head_step = (uint32_t)hs;
    Two<W> w[NU], dw[NU], dy[NU], x[NU];
#pragma unroll
    for (int i = 0; i < NU; ++i) {
        dw[i].fill(0.0f);
        if (NORM && s.weight)
            w[i].template load<false>(s.weight, Unit<W, INTER>(l, lane + i * lanes));
        else
            w[i].fill(1.0f);
    }
    int64_t position = 0;
    auto fetch = [&] {
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const Unit<W, INTER> u(l, lane + i * lanes);
            dy[i].template load<true>(s.dy + token * s.dy_token + (int64_t)head * s.dy_head, u);
            if constexpr (NORM)
                x[i].template load<true>(s.x + token * s.x_token + (int64_t)head * s.x_head, u);
        }
        if (l.rot)
            position = position_of(rope, token);
    };
    if (item < s.items)
        fetch();
    for (; item < s.items; item += step) {
        T *out = s.out + token * s.out_token + (int64_t)head * s.out_head;
        Two<W> g[NU], xv[NU];
        float sq = 0.0f, dot = 0.0f;
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const Unit<W, INTER> u(l, lane + i * lanes);
            g[i] = dy[i];
            g[i].only(u);
            if (l.rot) {
                Angles<W, INTER> t;
                t.load(l, u, rope, position);
                t.template turn<true>(u, g[i]);
            }
            if constexpr (NORM) {
                xv[i] = x[i];
                xv[i].only(u);
            }
        }
        if (DW || item + step < s.items) { // one head for each group of lanes otherwise
            token += token_step, head += head_step;
            if (head >= heads)
                head -= heads, ++token;
            if (item + step < s.items)
                fetch();
        }
        if constexpr (NORM) {
#pragma unroll
            for (int i = 0; i < NU; ++i)
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    sq = __builtin_fmaf(xv[i].a[j], xv[i].a[j], sq);
                    sq = __builtin_fmaf(xv[i].b[j], xv[i].b[j], sq);
                    dot = __builtin_fmaf(g[i].a[j] * w[i].a[j], xv[i].a[j], dot);
                    dot = __builtin_fmaf(g[i].b[j] * w[i].b[j], xv[i].b[j], dot);
                }
            const float r = rsqrt_of(__builtin_fmaf(sum_lanes(sq, lanes), l.inv_dim, eps));
            const float m = sum_lanes(dot, lanes) * l.inv_dim * r * r; // mean(w g x r) r
#pragma unroll
            for (int i = 0; i < NU; ++i)
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    if constexpr (DW) {
                        dw[i].a[j] = __builtin_fmaf(g[i].a[j], xv[i].a[j] * r, dw[i].a[j]);
                        dw[i].b[j] = __builtin_fmaf(g[i].b[j], xv[i].b[j] * r, dw[i].b[j]);
                    }
                    g[i].a[j] = r * __builtin_fmaf(-xv[i].a[j], m, g[i].a[j] * w[i].a[j]);
                    g[i].b[j] = r * __builtin_fmaf(-xv[i].b[j], m, g[i].b[j] * w[i].b[j]);
                }
        }
#pragma unroll
        for (int i = 0; i < NU; ++i)
            g[i].store(out, Unit<W, INTER>(l, lane + i * lanes));
    }
    if constexpr (DW) {
        if (!s.parts)
            return;
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            if (i)
                __syncthreads();
#pragma unroll
            for (int j = 0; j < W; ++j) {
                lds[(2 * j) * 256 + threadIdx.x] = dw[i].a[j];
                lds[(2 * j + 1) * 256 + threadIdx.x] = dw[i].b[j];
            }
            __syncthreads();
            // group 0's lanes hold the units: the threads of the block share out their 2 W sums
            for (int o = threadIdx.x; o < 2 * W * lanes; o += 256) {
                const int which = o >> l.lanes_log2, ln = o & (lanes - 1);
                const Unit<W, INTER> v(l, ln + i * lanes);
                float sum = 0.0f;
                for (int g = 0; g < groups; ++g)
                    sum += lds[which * 256 + (g << l.lanes_log2) + ln];
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

// Calls run(W, NU, INTER) as compile-time constants.
template <class T, class F>
int with_layout(int w, int nu, bool inter, F run)
{
    auto at = [&](auto wc, auto nc) {
        return inter ? run(wc, nc, std::true_type{}) : run(wc, nc, std::false_type{});
    };
    using std::integral_constant;
    if constexpr (sizeof(T) == 2)
        if (w == 8)
            return at(integral_constant<int, 8>{}, integral_constant<int, 1>{});
    if (w == 4)
        return at(integral_constant<int, 4>{}, integral_constant<int, 1>{});
    return nu == 1 ? at(integral_constant<int, 1>{}, integral_constant<int, 1>{})
                   : at(integral_constant<int, 1>{}, integral_constant<int, 4>{});
}

// Blocks of the backward pass of either side: about kGradBlocks for both, in proportion to their heads.
constexpr int64_t kGradBlocks = 2048;
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
    // as many blocks as any layout of such heads takes: groups of 4 (64 lanes) and more
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
        return with_layout<T>(w, nu, rope.interleaved, [&](auto wc, auto nc, auto inter) {
            constexpr int W = decltype(wc)::value, NU = decltype(nc)::value;
            constexpr bool I = decltype(inter)::value;
            auto kernel = norm.on ? k_qk<T, W, NU, I, true> : k_qk<T, W, NU, I, false>;
            return launch<4>(kernel, q.blocks + k.blocks, kUncapped, s, l, q, k, norm.eps, rope);
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
        return with_layout<T>(w, nu, rope.interleaved, [&](auto wc, auto nc, auto inter) {
            constexpr int W = decltype(wc)::value, NU = decltype(nc)::value;
            constexpr bool I = decltype(inter)::value;
            auto kernel = want_dw   ? k_qk_grad<T, W, NU, I, true, true>
                          : norm.on ? k_qk_grad<T, W, NU, I, true, false>
                                    : k_qk_grad<T, W, NU, I, false, false>;
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
