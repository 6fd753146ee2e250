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
    int64_t items, blocks; // heads of all tokens, and the blocks that share them
    const T *weight;
    float *parts; // [blocks][dim] partial weight gradients
};

// One lane's unit of a head: where its two chunks lie, and which angles turn them.
template <int W, bool INTER>
struct Unit {
    int a, b;      // first elements of the chunks
    bool on, on_b; // the unit exists; its second chunk does
    bool turn_a, turn_b;
    int angle_a, angle_b; // first angle of the chunk (in the half layout of both)
    SDP4_DEV Unit(const Layout &l, int u)
    {
        on = u < l.units;
        if constexpr (INTER && W > 1) {
            a = 2 * W * u, b = a + W;
            turn_a = a < l.rot, turn_b = b < l.rot;
            angle_a = a / 2, angle_b = b / 2;
        } else {
            const bool turned = u < l.rot_units;
            const int v = turned ? u : u - l.rot_units;
            a = turned ? (INTER ? 2 * u : W * u) : l.rot + 2 * W * v;
            b = turned && !INTER ? a + l.half : a + W;
            turn_a = turn_b = turned;
            angle_a = angle_b = W * u;
        }
        on_b = on && b < l.dim;
        turn_a &= on, turn_b &= on_b;
    }
};

// W elements at an element address.
template <class T, int W>
SDP4_DEV void load_w(const T *p, float (&v)[W])
{
    if constexpr (W * sizeof(T) == 16) {
        unpack<T>(load_chunk<true>(p), v);
    } else if constexpr (W * sizeof(T) == 8) {
        const u32x2 c = __builtin_nontemporal_load(reinterpret_cast<const u32x2_b2 *>(p));
        v[0] = __uint_as_float(c.x << 16), v[1] = __uint_as_float(c.x & 0xFFFF0000u);
        v[2] = __uint_as_float(c.y << 16), v[3] = __uint_as_float(c.y & 0xFFFF0000u);
    } else {
#pragma unroll
        for (int j = 0; j < W; ++j)
            v[j] = to_f32<T>(p[j]);
    }
}
template <class T, int W>
SDP4_DEV void store_w(T *p, const float (&v)[W])
{
    if constexpr (W * sizeof(T) == 16) {
        store_chunk<T>(p, pack<T>(v));
    } else if constexpr (W * sizeof(T) == 8) {
        const u32x2 c = {bf16x2_rne(v[0], v[1]), bf16x2_rne(v[2], v[3])};
        __builtin_nontemporal_store((u32x2_b2)c, reinterpret_cast<u32x2_b2 *>(p));
    } else {
#pragma unroll
        for (int j = 0; j < W; ++j)
            p[j] = from_f32<T>(v[j]);
    }
}
// Table entries and weights, which other lanes and blocks read again.
template <int W>
SDP4_DEV void load_kept(const float *p, float (&v)[W])
{
    if constexpr (W % 4 == 0) {
#pragma unroll
        for (int k = 0; k < W / 4; ++k)
            unpack<float>(load_chunk<false>(p + 4 * k), *reinterpret_cast<float(*)[4]>(v + 4 * k));
    } else {
#pragma unroll
        for (int j = 0; j < W; ++j)
            v[j] = p[j];
    }
}
template <class T, int W>
SDP4_DEV void load_weight(const T *p, float (&v)[W])
{
#pragma unroll
    for (int j = 0; j < W; ++j)
        v[j] = to_f32<T>(p[j]);
}

// Angles of a unit and their use.  BACK: by the opposite angle.
template <int W, bool INTER>
struct Angles {
    // half layout (and W = 1): W cosines and sines for both chunks; interleaved: W / 2 of either for each chunk
    float c[W], s[W];
    SDP4_DEV void load(const Layout &l, const Unit<W, INTER> &u, const Rope &rope, int64_t token)
    {
#pragma unroll
        for (int j = 0; j < W; ++j)
            c[j] = 1.0f, s[j] = 0.0f;
        if (!u.turn_a)
            return;
        const int64_t p = rope.positions ? rope.positions[token] : token;
        if (p < 0 || p >= rope.rows) { // no such row: the result says so
#pragma unroll
            for (int j = 0; j < W; ++j)
                c[j] = s[j] = __builtin_nanf("");
            return;
        }
        const float *row = rope.table + p * l.rot;
        if constexpr (INTER && W > 1) {
            constexpr int H = W / 2;
            load_kept<H>(row + u.angle_a, *reinterpret_cast<float(*)[H]>(c));
            load_kept<H>(row + l.half + u.angle_a, *reinterpret_cast<float(*)[H]>(s));
            if (u.turn_b) {
                load_kept<H>(row + u.angle_b, *reinterpret_cast<float(*)[H]>(c + H));
                load_kept<H>(row + l.half + u.angle_b, *reinterpret_cast<float(*)[H]>(s + H));
            }
        } else {
            load_kept<W>(row + u.angle_a, c);
            load_kept<W>(row + l.half + u.angle_a, s);
        }
    }
    template <bool BACK>
    SDP4_DEV void turn(const Unit<W, INTER> &u, float (&a)[W], float (&b)[W]) const
    {
        if constexpr (INTER && W > 1) {
#pragma unroll
            for (int j = 0; j < W / 2; ++j) {
                one<BACK>(a[2 * j], a[2 * j + 1], c[j], s[j]);
                if (u.turn_b)
                    one<BACK>(b[2 * j], b[2 * j + 1], c[W / 2 + j], s[W / 2 + j]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < W; ++j)
                one<BACK>(a[j], b[j], c[j], s[j]);
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

// 1 / sqrt(v) to the last place but rounding: one Newton step on the estimate.
SDP4_DEV float rsqrt_of(float v)
{
    const float y = __builtin_amdgcn_rsqf(v);
    const float e = __builtin_fmaf(-v * y, y, 1.0f);
    const float z = __builtin_fmaf(0.5f * y, e, y);
    return e == e && __builtin_isfinite(y) ? z : y;
}

template <class T, int W>
SDP4_DEV void load_unit(const T *head, bool on, bool on_b, int a, int b, float (&va)[W], float (&vb)[W])
{
#pragma unroll
    for (int j = 0; j < W; ++j)
        va[j] = vb[j] = 0.0f;
    if (on)
        load_w<T, W>(head + a, va);
    if (on_b)
        load_w<T, W>(head + b, vb);
}

// Forward: one head per group of lanes; the first blocks take the queries, the others the keys.
template <class T, int W, int NU, bool INTER, bool NORM>
__global__ __launch_bounds__(256) void k_qk(Layout l, Side<T> q, Side<T> k, float eps, Rope rope)
{
    const int64_t wb = work_block();
    const bool keys = wb >= q.blocks;
    const Side<T> &s = keys ? k : q;
    const int lanes = 1 << l.lanes_log2, lane = threadIdx.x & (lanes - 1);
    const int64_t item = ((keys ? wb - q.blocks : wb) << (8 - l.lanes_log2)) + (threadIdx.x >> l.lanes_log2);
    if (item >= s.items)
        return;
    uint64_t head;
    const int64_t token = (int64_t)divide((uint64_t)item, s.heads, head);
    const T *x = s.x + token * s.x_token + (int64_t)head * s.x_head;
    T *y = s.out + token * s.out_token + (int64_t)head * s.out_head;
    float a[NU][W], b[NU][W];
#pragma unroll
    for (int i = 0; i < NU; ++i) {
        const Unit<W, INTER> u(l, lane + i * lanes);
        load_unit<T, W>(x, u.on, u.on_b, u.a, u.b, a[i], b[i]);
    }
    float r = 1.0f;
    if constexpr (NORM) {
        float sq = 0.0f;
#pragma unroll
        for (int i = 0; i < NU; ++i)
#pragma unroll
            for (int j = 0; j < W; ++j) {
                sq = __builtin_fmaf(a[i][j], a[i][j], sq);
                sq = __builtin_fmaf(b[i][j], b[i][j], sq);
            }
        r = rsqrt_of(__builtin_fmaf(sum_lanes(sq, lanes), l.inv_dim, eps));
    }
#pragma unroll
    for (int i = 0; i < NU; ++i) {
        const Unit<W, INTER> u(l, lane + i * lanes);
        if constexpr (NORM) {
            float wa[W], wb_[W];
#pragma unroll
            for (int j = 0; j < W; ++j)
                wa[j] = wb_[j] = 1.0f;
            if (s.weight) {
                if (u.on)
                    load_weight<T, W>(s.weight + u.a, wa);
                if (u.on_b)
                    load_weight<T, W>(s.weight + u.b, wb_);
            }
#pragma unroll
            for (int j = 0; j < W; ++j) {
                a[i][j] = a[i][j] * r * wa[j];
                b[i][j] = b[i][j] * r * wb_[j];
            }
        }
        if (u.turn_a) {
            Angles<W, INTER> t;
            t.load(l, u, rope, token);
            t.template turn<false>(u, a[i], b[i]);
        }
        if (u.on)
            store_w<T, W>(y + u.a, a[i]);
        if (u.on_b)
            store_w<T, W>(y + u.b, b[i]);
    }
}

// Backward.  Each block takes every blocks-th group of heads of its side and adds up the weights' gradient in
// registers; its lane groups and waves join at the end, and the block's sums go to the workspace.
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
    float wa[NU][W], wv[NU][W], da[NU][W] = {}, db[NU][W] = {};
#pragma unroll
    for (int i = 0; i < NU; ++i) {
        const Unit<W, INTER> u(l, lane + i * lanes);
#pragma unroll
        for (int j = 0; j < W; ++j)
            wa[i][j] = wv[i][j] = 1.0f;
        if (NORM && s.weight) {
            if (u.on)
                load_weight<T, W>(s.weight + u.a, wa[i]);
            if (u.on_b)
                load_weight<T, W>(s.weight + u.b, wv[i]);
        }
    }
    for (int64_t item = block * groups + group; item < s.items; item += s.blocks * groups) {
        uint64_t head;
        const int64_t token = (int64_t)divide((uint64_t)item, s.heads, head);
        const T *dy = s.dy + token * s.dy_token + (int64_t)head * s.dy_head;
        const T *x = NORM ? s.x + token * s.x_token + (int64_t)head * s.x_head : nullptr;
        T *dx = s.out + token * s.out_token + (int64_t)head * s.out_head;
        float ga[NU][W], gb[NU][W], xa[NU][W], xb[NU][W];
        float sq = 0.0f, dot = 0.0f;
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const Unit<W, INTER> u(l, lane + i * lanes);
            load_unit<T, W>(dy, u.on, u.on_b, u.a, u.b, ga[i], gb[i]);
            if constexpr (NORM)
                load_unit<T, W>(x, u.on, u.on_b, u.a, u.b, xa[i], xb[i]);
        }
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const Unit<W, INTER> u(l, lane + i * lanes);
            if (u.turn_a) {
                Angles<W, INTER> t;
                t.load(l, u, rope, token);
                t.template turn<true>(u, ga[i], gb[i]);
            }
            if constexpr (NORM) {
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    sq = __builtin_fmaf(xa[i][j], xa[i][j], sq);
                    sq = __builtin_fmaf(xb[i][j], xb[i][j], sq);
                    dot = __builtin_fmaf(ga[i][j] * wa[i][j], xa[i][j], dot);
                    dot = __builtin_fmaf(gb[i][j] * wv[i][j], xb[i][j], dot);
                }
            }
        }
        if constexpr (NORM) {
            const float r = rsqrt_of(__builtin_fmaf(sum_lanes(sq, lanes), l.inv_dim, eps));
            const float m = sum_lanes(dot, lanes) * l.inv_dim * r * r; // mean(w g x r) r
#pragma unroll
            for (int i = 0; i < NU; ++i)
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    if constexpr (DW) {
                        da[i][j] = __builtin_fmaf(ga[i][j], xa[i][j] * r, da[i][j]);
                        db[i][j] = __builtin_fmaf(gb[i][j], xb[i][j] * r, db[i][j]);
                    }
                    ga[i][j] = r * __builtin_fmaf(-xa[i][j], m, ga[i][j] * wa[i][j]);
                    gb[i][j] = r * __builtin_fmaf(-xb[i][j], m, gb[i][j] * wv[i][j]);
                }
        }
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const Unit<W, INTER> u(l, lane + i * lanes);
            if (u.on)
                store_w<T, W>(dx + u.a, ga[i]);
            if (u.on_b)
                store_w<T, W>(dx + u.b, gb[i]);
        }
    }
    if constexpr (DW) {
        if (!s.parts)
            return;
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const Unit<W, INTER> u(l, lane + i * lanes);
            if (i)
                __syncthreads();
#pragma unroll
            for (int j = 0; j < W; ++j) {
                lds[(2 * j) * 256 + threadIdx.x] = da[i][j];
                lds[(2 * j + 1) * 256 + threadIdx.x] = db[i][j];
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
constexpr int64_t kGradBlocks = 1024;
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
    for (int i = 0; i < 2; ++i)
        if (sums[i].parts) {
            const int e = launch_sum_parts(sums[i].parts, sums[i].blocks, dim, dim, dw[i], s);
            if (e)
                return e;
        }
    return 0;
}

int launch_rope_table(const double *inv_freq, int half, int64_t start, int64_t rows, double scale, float *table,
                      hipStream_t s)
{
    return launch<4>(k_rope_table, (rows * half + 255) / 256, kUncapped, s, inv_freq, half, start, rows, scale, table);
}

} // namespace sdp4
