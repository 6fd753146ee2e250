// k_block_norm.hip -- the joint of two blocks of a decoder in one pass over
// its rows: the norm behind a block, its gate and scale, the residual stream,
// and the norm in front of the next block; and the backward pass.
//
//      u = b r_b w_post,  r_b = (mean b^2 + eps)^-1/2 (or u = b w_post),
//      y = residual_scale x + branch_scale gate u,
//      h = y r_y w_pre,   r_y = (mean y^2 + eps)^-1/2.
// Backward, from dh and dy:
//      t = dy + r_y (dh w_pre - y r_y mean(dh w_pre y r_y)),  dx = residual_scale t,
//      s = branch_scale gate t w_post,  db = r_b (s - b r_b mean(s b r_b)),
//      dw_pre = sum dh y r_y, dw_post = sum branch_scale gate t b r_b over the
//      rows, dgate = branch_scale sum t u over the columns.
// A row stays in the registers of its waves between the sums: every array is
// read or written once, and HBM bounds both passes.
#include "step_device.hpp"

namespace sdp4 {

namespace {

// Sums over a block's waves, the same in every lane: lanes, then waves in order through LDS (two places in turn, so that one
// barrier a sum is enough).
constexpr int kMostWaves = 8;
template <int COUNT>
struct BlockSums {
    float (*lds)[COUNT][kMostWaves];
    int waves, turn = 0;
    SDP4_DEV BlockSums(float (*l)[COUNT][kMostWaves]) : lds(l), waves(blockDim.x / kWave)
    {
        for (int i = threadIdx.x; i < 2 * COUNT * kMostWaves; i += blockDim.x)
            (&lds[0][0][0])[i] = 0.0f; // of the waves that are not there
        __syncthreads();
    }
    SDP4_DEV void add(float (&v)[COUNT])
    {
#pragma unroll
        for (int i = 0; i < COUNT; ++i)
            v[i] = sum_lanes(v[i], kWave);
        if (waves == 1)
            return;
        if (lane_id() == 0) {
#pragma unroll
            for (int i = 0; i < COUNT; ++i)
                lds[turn][i][threadIdx.x / kWave] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            float w[kMostWaves];
#pragma unroll
            for (int j = 0; j < kMostWaves; ++j)
                w[j] = lds[turn][i][j];
#pragma unroll
            for (int n = kMostWaves / 2; n > 0; n /= 2)
#pragma unroll
                for (int j = 0; j < n; ++j)
                    w[j] += w[j + n];
            v[i] = w[0];
        }
        turn ^= 1;
    }
};

// Elements of a lane in one access: 16 bytes of the wider type.
template <class X, class Y>
constexpr int kJoint = sizeof(X) == 4 || sizeof(Y) == 4 ? 4 : 8;

// A lane's places in a row: C accesses of N elements.  WHOLE: the row is whole accesses, so that a place is in it or not;
// otherwise the last one is read and written as load_row, end_row and store_elems do.
template <int N, int C, bool WHOLE>
struct Places {
    int64_t cols;
    int at[C];
    SDP4_DEV explicit Places(int64_t n) : cols(n)
    {
#pragma unroll
        for (int i = 0; i < C; ++i)
            at[i] = N * (i * (int)blockDim.x + (int)threadIdx.x);
    }
    SDP4_DEV bool in(int i) const { return at[i] < (int)cols; }
    template <class T>
    SDP4_DEV void load(const T *row, Raw<T, N> (&r)[C]) const
    {
#pragma unroll
        for (int i = 0; i < C; ++i) {
            if constexpr (WHOLE)
                r[i].template load<true>(row + (uint32_t)(in(i) ? at[i] : 0));
            else
                load_row(row, at[i], cols, r[i]);
        }
    }
    template <class T>
    SDP4_DEV void load_kept(const T *row, Raw<T, N> (&r)[C]) const // of weights, which every row reads again
    {
#pragma unroll
        for (int i = 0; i < C; ++i) {
            if constexpr (WHOLE)
                r[i].template load<false>(row + (uint32_t)(in(i) ? at[i] : 0));
            else
                load_row(row, at[i], cols, r[i]);
        }
    }
    // What was loaded, moved to its places where the row ends inside an access, with zeros beyond the row.
    template <class T>
    SDP4_DEV void settle(Raw<T, N> (&r)[C]) const
    {
#pragma unroll
        for (int i = 0; i < C; ++i)
            if (at[i] + N > (int)cols) {
                float v[N];
                if constexpr (WHOLE) {
#pragma unroll
                    for (int j = 0; j < N; ++j)
                        v[j] = 0.0f;
                } else {
                    r[i].get(v);
                    end_row(at[i], cols, v);
                }
                r[i].put(v); // the same numbers: as they came
            }
    }
    template <class T>
    SDP4_DEV void weight(const Raw<T, N> (&r)[C], bool there, int i, float (&v)[N]) const
    {
        if (there) {
            r[i].get(v);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j)
                v[j] = 1.0f;
        }
    }
    template <class T>
    SDP4_DEV void store(T *row, int i, const float (&v)[N]) const
    {
        if constexpr (WHOLE) {
            if (in(i)) {
                Raw<T, N> r;
                r.put(v);
                r.store(row + (uint32_t)at[i]);
            }
        } else {
            store_elems(row + at[i], cols - at[i], v);
        }
    }
};

// A block for a row: as few accesses of a lane as eight waves allow and no more waves than that takes, so that a short row has few
// to wait for.  8192 x 5120 bfloat16 with both norms and a gate 58 us (5.8 TB/s; a block of fixed width, 69), one row of 768 2.6.
template <class X, class Y, int C, bool WHOLE>
__global__ __launch_bounds__(64 * kMostWaves) void k_block_norm(BlockNorm p, int64_t rows, int64_t cols, Rows<const X *> branch,
                                                                Rows<const Y *> res, Rows<Y *> y, Rows<X *> h)
{
    constexpr int N = kJoint<X, Y>;
    __shared__ __align__(16) float lds[2][1][kMostWaves];
    const int64_t row = work_block();
    if (row >= rows)
        return;
    const Places<N, C, WHOLE> at(cols);
    Raw<X, N> br[C], w1[C], w2[C];
    Raw<Y, N> rr[C];
    if (branch.p)
        at.load(branch.p + row * branch.stride, br);
    if (res.p)
        at.load(res.p + row * res.stride, rr);
    if (p.post_weight)
        at.load_kept(static_cast<const X *>(p.post_weight), w1);
    if (p.pre_weight)
        at.load_kept(static_cast<const X *>(p.pre_weight), w2);
    BlockSums<1> sums(lds);
    if (branch.p)
        at.settle(br);
    if (res.p)
        at.settle(rr);
    if (p.post_weight)
        at.settle(w1);
    if (p.pre_weight)
        at.settle(w2);
    float v[C][N];
    float by = p.branch_scale;
    if (p.gate)
        by *= p.gate[row];
    if (branch.p) {
        float s[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < C; ++i) {
            br[i].get(v[i]);
#pragma unroll
            for (int j = 0; j < N; ++j)
                s[0] = __builtin_fmaf(v[i][j], v[i][j], s[0]);
        }
        if (p.post_norm) {
            sums.add(s);
            by *= 1.0f / __builtin_sqrtf(s[0] / (float)cols + p.post_eps);
        }
#pragma unroll
        for (int i = 0; i < C; ++i) {
            float w[N];
            at.weight(w1, p.post_weight, i, w);
#pragma unroll
            for (int j = 0; j < N; ++j)
                v[i][j] = v[i][j] * w[j] * by;
        }
    } else {
#pragma unroll
        for (int i = 0; i < C; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j)
                v[i][j] = 0.0f;
    }
    if (res.p) {
#pragma unroll
        for (int i = 0; i < C; ++i) {
            float w[N];
            rr[i].get(w);
#pragma unroll
            for (int j = 0; j < N; ++j)
                v[i][j] = __builtin_fmaf(w[j], p.residual_scale, v[i][j]);
        }
    }
    if (y.p) {
#pragma unroll
        for (int i = 0; i < C; ++i)
            at.store(y.p + row * y.stride, i, v[i]);
    }
    if (h.p) {
        float s[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < C; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j)
                s[0] = __builtin_fmaf(v[i][j], v[i][j], s[0]);
        sums.add(s);
        const float r = 1.0f / __builtin_sqrtf(s[0] / (float)cols + p.pre_eps);
#pragma unroll
        for (int i = 0; i < C; ++i) {
            float w[N];
            at.weight(w2, p.pre_weight, i, w);
#pragma unroll
            for (int j = 0; j < N; ++j)
                v[i][j] = v[i][j] * r * w[j];
            at.store(h.p + row * h.stride, i, v[i]);
        }
    }
}

// Rows part, part + parts, ... of a block, so that the chip's blocks walk through memory together; the next row's loads are under
// way before the present one is stored.  The weight gradients of a block's rows go to the workspace, from where the sums over the
// parts are taken in order.  8192 x 5120 bfloat16, both norms and a gate: 96 us and 6 for the sums over the parts (six arrays:
// 5.2 TB/s); what is waited for is the row's one exchange of sums, with one or two blocks on a compute unit.  Rows of more than
// 8192 columns do not fit the registers: 4096 x 8192 82 us, x 12288 196 (bfloat16) and 808 (float32), x 16384 754.
// JOINT: the sums with the branch are wanted, for a post norm or the gate's gradient.
template <class X, class Y, int C, bool WHOLE, bool JOINT>
__global__ __launch_bounds__(64 * kMostWaves) void k_block_norm_grad(BlockNorm p, int64_t rows, int64_t cols, int64_t pitch, int parts,
                                                                     BlockNormGrad<X, Y> g)
{
    constexpr int N = kJoint<X, Y>;
    constexpr int SUMS = JOINT ? 6 : 2;
    __shared__ __align__(16) float lds[2][SUMS][kMostWaves];
    const int64_t part = work_block();
    if (part >= parts)
        return;
    const Places<N, C, WHOLE> at(cols);
    // a row as it lies in memory: half the registers of its values where it is bfloat16
    struct Row {
        Raw<X, N> dh[C], b[C];
        Raw<Y, N> dy[C], y[C];
        float gate;
    };
    auto fetch = [&](int64_t row, Row &r) {
        if (g.dh.p) {
            at.load(g.dh.p + row * g.dh.stride, r.dh);
            at.load(g.y.p + row * g.y.stride, r.y);
        }
        if (g.branch.p)
            at.load(g.branch.p + row * g.branch.stride, r.b);
        if (g.dy.p)
            at.load(g.dy.p + row * g.dy.stride, r.dy);
        r.gate = p.gate ? p.gate[row] : 1.0f;
    };
    Row now, next;
    fetch(part, now);
    Raw<X, N> w1[C], w2[C];
    if (p.post_weight)
        at.load_kept(static_cast<const X *>(p.post_weight), w1);
    if (p.pre_weight)
        at.load_kept(static_cast<const X *>(p.pre_weight), w2);
    BlockSums<SUMS> sums(lds);
    if (p.post_weight)
        at.settle(w1);
    if (p.pre_weight)
        at.settle(w2);
    float dpost[C][N] = {}, dpre[C][N] = {};
    const float over = 1.0f / (float)cols;
    for (int64_t row = part; row < rows; row += parts) {
        const float by = p.branch_scale * now.gate;
        if (g.dh.p)
            at.settle(now.dh), at.settle(now.y);
        if (g.dy.p)
            at.settle(now.dy);
        if (g.branch.p)
            at.settle(now.b);
        // One round of sums a row: of y^2, g y, b^2 with g = dh w_pre, and of dy u, g u, y u with u = b w_post, of which the sum
        // of t u is made.
        float s[SUMS] = {};
#pragma unroll
        for (int i = 0; i < C; ++i) {
            float v[N], y[N], b[N], w[N];
            if constexpr (JOINT) {
                now.b[i].get(b);
                at.weight(w1, p.post_weight, i, w);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    s[2] = __builtin_fmaf(b[j], b[j], s[2]);
                    b[j] *= w[j];
                }
                if (g.dy.p) {
                    now.dy[i].get(v);
#pragma unroll
                    for (int j = 0; j < N; ++j)
                        s[3] = __builtin_fmaf(v[j], b[j], s[3]);
                }
            }
            if (g.dh.p) {
                now.dh[i].get(v);
                now.y[i].get(y);
                at.weight(w2, p.pre_weight, i, w);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    v[j] *= w[j];
                    s[0] = __builtin_fmaf(y[j], y[j], s[0]);
                    s[1] = __builtin_fmaf(v[j], y[j], s[1]);
                }
                if constexpr (JOINT) {
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        s[4] = __builtin_fmaf(v[j], b[j], s[4]);
                        s[5] = __builtin_fmaf(y[j], b[j], s[5]);
                    }
                }
            }
        }
        if (row + parts < rows)
            fetch(row + parts, next);
        sums.add(s);
        const float ry = 1.0f / __builtin_sqrtf(s[0] * over + p.pre_eps);
        const float along = s[1] * over * ry * ry; // of y, by which g is shortened
        float rb = 1.0f, mean = 0.0f;
        if constexpr (JOINT) {
            const float tu = g.dh.p ? s[3] + ry * (s[4] - along * s[5]) : s[3];
            if (p.post_norm) {
                rb = 1.0f / __builtin_sqrtf(s[2] * over + p.post_eps);
                mean = by * tu * rb * rb * over;
            }
            if (g.dgate && threadIdx.x == 0)
                g.dgate[row] = p.branch_scale * rb * tu;
        }
#pragma unroll
        for (int i = 0; i < C; ++i) {
            float t[N], w[N], b[N];
            if (g.dh.p) {
                float y[N];
                now.dh[i].get(t);
                now.y[i].get(y);
                at.weight(w2, p.pre_weight, i, w);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    dpre[i][j] = __builtin_fmaf(t[j], y[j] * ry, dpre[i][j]);
                    t[j] = ry * (t[j] * w[j] - y[j] * along);
                }
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j)
                    t[j] = 0.0f;
            }
            if (g.dy.p) {
                float d[N];
                now.dy[i].get(d);
#pragma unroll
                for (int j = 0; j < N; ++j)
                    t[j] += d[j];
            }
            if (g.dres.p) {
                float o[N];
#pragma unroll
                for (int j = 0; j < N; ++j)
                    o[j] = t[j] * p.residual_scale;
                at.store(g.dres.p + row * g.dres.stride, i, o);
            }
            at.weight(w1, p.post_weight, i, w);
            if (g.branch.p) {
                now.b[i].get(b);
#pragma unroll
                for (int j = 0; j < N; ++j)
                    dpost[i][j] = __builtin_fmaf(t[j] * by, b[j] * rb, dpost[i][j]);
            }
            if (g.dbranch.p) {
#pragma unroll
                for (int j = 0; j < N; ++j)
                    t[j] *= w[j] * by;
                if (JOINT && p.post_norm) {
#pragma unroll
                    for (int j = 0; j < N; ++j)
                        t[j] = rb * (t[j] - b[j] * mean);
                }
                at.store(g.dbranch.p + row * g.dbranch.stride, i, t);
            }
        }
        now = next;
    }
#pragma unroll
    for (int i = 0; i < C; ++i)
        if (at.in(i)) { // the pitch is a multiple of 8
#pragma unroll
            for (int j = 0; j < N; j += 4) {
                if (g.post_parts)
                    store_elems(g.post_parts + part * pitch + at.at[i] + j, 4, *reinterpret_cast<const float(*)[4]>(&dpost[i][j]));
                if (g.pre_parts)
                    store_elems(g.pre_parts + part * pitch + at.at[i] + j, 4, *reinterpret_cast<const float(*)[4]>(&dpre[i][j]));
            }
        }
}

// As many parts as make eight waves on each compute unit where a lane takes eight elements of a row: a row of few waves leaves the
// others idle and waits for its own loads and sums.  256 / 512 / 1024 / 2048 parts, bfloat16 with both norms and their weights, us:
// 8192 x 256 43 / 27 / 19 / 19, 65536 x 256 298 / 165 / 85 / 64, 8192 x 768 52 / 36 / 27 / 34, 8192 x 2048 56 / 48 / 58 / 66,
// 8192 x 3000 67 / 72 / 83 / 104, 8192 x 5120 102 / 110 / 125 / 156: beyond these the partial sums of more
// parts cost more than their blocks gain.  Without weights 65536 x 64 175 / 94 / 50 / 32, 8192 x 5120 62 / 63 / 65 / 70.
constexpr int kWideRow = 512; // elements of a wave
int64_t pitch_of(int64_t cols) { return (cols + 7) / 8 * 8; }
int parts_of(int64_t rows, int64_t cols)
{
    const int64_t waves = (cols + kWideRow - 1) / kWideRow, most = 256 * (waves < 8 ? 8 / waves : 1);
    return (int)(rows < most ? rows : most);
}

// A body with the accesses of a lane (as few as eight waves leave) for rows of `cols` elements, N in an access, and whether they
// are whole.
template <int N, class F>
int with_shape(int64_t cols, F body)
{
    using std::integral_constant;
    const int64_t places = (cols + N - 1) / N;
    auto waves = [&](int c) { return (int)((places + 64 * c - 1) / (64 * c)); };
    auto with = [&](auto c) {
        return cols % N == 0 ? body(c, integral_constant<bool, true>{}, waves(c)) : body(c, integral_constant<bool, false>{}, waves(c));
    };
    constexpr int most = 64 * kMostWaves;
    if (places <= most)
        return with(integral_constant<int, 1>{});
    if (places <= 2 * most)
        return with(integral_constant<int, 2>{});
    if (places <= 3 * most)
        return with(integral_constant<int, 3>{});
    if constexpr (4 * most * N < SDP4_MAX_HIDDEN)
        if (places > 4 * most)
            return with(integral_constant<int, 8>{});
    return with(integral_constant<int, 4>{});
}

} // namespace

int64_t block_norm_grad_workspace(int64_t rows, int64_t cols)
{
    return rows <= 0 || cols <= 0 ? 0 : 2 * parts_of(rows, cols) * pitch_of(cols) * (int64_t)sizeof(float);
}

int launch_block_norm(int x_dtype, int y_dtype, const BlockNorm &p, int64_t rows, int64_t cols, Rows<const void *> branch,
                      Rows<const void *> residual, Rows<void *> y, Rows<void *> h, hipStream_t s)
{
    return with_type(x_dtype, [&](auto x_tag) {
        return with_type(y_dtype, [&](auto y_tag) {
            using X = decltype(x_tag);
            using Y = decltype(y_tag);
            constexpr int N = kJoint<X, Y>;
            return with_shape<N>(cols, [&](auto accesses, auto whole, int waves) {
                return launch_waves(waves, k_block_norm<X, Y, accesses, whole>, rows, kUncapped, s, p, rows, cols, typed<const X>(branch),
                                     typed<const Y>(residual), typed<Y>(y), typed<X>(h));
            });
        });
    });
}

int launch_block_norm_grad(int x_dtype, int y_dtype, const BlockNorm &p, int64_t rows, int64_t cols, const BlockNormArrays &a,
                           float *workspace, hipStream_t s)
{
    const int parts = parts_of(rows, cols);
    const int64_t pitch = pitch_of(cols);
    float *post = a.dpost_weight ? workspace : nullptr, *pre = a.dpre_weight ? workspace + (post ? parts * pitch : 0) : nullptr;
    const int rc = with_type(x_dtype, [&](auto x_tag) {
        return with_type(y_dtype, [&](auto y_tag) {
            using X = decltype(x_tag);
            using Y = decltype(y_tag);
            constexpr int N = kJoint<X, Y>;
            const BlockNormGrad<X, Y> g{typed<const X>(a.dh), typed<const Y>(a.dy), typed<const X>(a.branch), typed<const Y>(a.y),
                                        typed<X>(a.dbranch), typed<Y>(a.dresidual), a.dgate, post, pre};
            return with_shape<N>(cols, [&](auto accesses, auto whole, int waves) {
                auto kernel = (p.post_norm && a.branch.p) || a.dgate ? k_block_norm_grad<X, Y, accesses, whole, true>
                                                                     : k_block_norm_grad<X, Y, accesses, whole, false>;
                return launch_waves(waves, kernel, parts, kUncapped, s, p, rows, cols, pitch, parts, g);
            });
        });
    });
    if (rc || (!post && !pre))
        return rc;
    if (!post)
        return launch_sum_parts({{pre, parts, a.dpre_weight}, {}}, pitch, cols, s);
    return launch_sum_parts({{post, parts, a.dpost_weight}, {pre, parts, a.dpre_weight}}, pitch, cols, s);
}

} // namespace sdp4
