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
template <int WAVES, int COUNT>
struct BlockSums {
    float (*lds)[WAVES][COUNT];
    int turn = 0;
    SDP4_DEV void add(float (&v)[COUNT])
    {
#pragma unroll
        for (int i = 0; i < COUNT; ++i)
            v[i] = sum_lanes(v[i], kWave);
        if constexpr (WAVES > 1) {
            if (lane_id() == 0) {
#pragma unroll
                for (int i = 0; i < COUNT; ++i)
                    lds[turn][threadIdx.x / kWave][i] = v[i];
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < COUNT; ++i) {
                v[i] = 0.0f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w)
                    v[i] += lds[turn][w][i];
            }
            turn ^= 1;
        }
    }
};

// Elements of a lane in one access: 16 bytes of the wider type.
template <class X, class Y>
constexpr int kJoint = sizeof(X) == 4 || sizeof(Y) == 4 ? 4 : 8;

template <class T, int N, int C>
SDP4_DEV void fetch(const T *row, int64_t cols, const int (&c)[C], Raw<T, N> (&r)[C])
{
#pragma unroll
    for (int i = 0; i < C; ++i)
        load_row(row, c[i], cols, r[i]);
}
template <class T, int N>
SDP4_DEV void take(const Raw<T, N> &r, int c, int64_t cols, float (&v)[N])
{
    r.get(v);
    end_row(c, cols, v);
}
template <class T, int N>
SDP4_DEV void weight_at(const T *w, int c, int64_t cols, float (&v)[N])
{
    if (w) {
        load_row(w, c, cols, v);
        end_row(c, cols, v);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
            v[j] = 1.0f;
    }
}

// A block of WAVES waves for a row, C accesses of a lane.
template <class X, class Y, int WAVES, int C>
__global__ __launch_bounds__(64 * WAVES) void k_block_norm(BlockNorm p, int64_t rows, int64_t cols, Rows<const X *> branch,
                                                           Rows<const Y *> res, Rows<Y *> y, Rows<X *> h)
{
    constexpr int N = kJoint<X, Y>;
    __shared__ float lds[2][WAVES][1];
    BlockSums<WAVES, 1> sums{lds};
    const int64_t row = work_block();
    if (row >= rows)
        return;
    int c[C];
#pragma unroll
    for (int i = 0; i < C; ++i)
        c[i] = N * (i * 64 * WAVES + (int)threadIdx.x);
    Raw<X, N> br[C];
    Raw<Y, N> rr[C];
    if (branch.p)
        fetch(branch.p + row * branch.stride, cols, c, br);
    if (res.p)
        fetch(res.p + row * res.stride, cols, c, rr);
    float v[C][N];
    float by = p.branch_scale;
    if (p.gate)
        by *= p.gate[row];
    if (branch.p) {
        float s[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < C; ++i) {
            take(br[i], c[i], cols, v[i]);
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
            weight_at(static_cast<const X *>(p.post_weight), c[i], cols, w);
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
            take(rr[i], c[i], cols, w);
#pragma unroll
            for (int j = 0; j < N; ++j)
                v[i][j] = __builtin_fmaf(w[j], p.residual_scale, v[i][j]);
        }
    }
    if (y.p) {
#pragma unroll
        for (int i = 0; i < C; ++i)
            store_elems(y.p + row * y.stride + c[i], cols - c[i], v[i]);
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
            weight_at(static_cast<const X *>(p.pre_weight), c[i], cols, w);
#pragma unroll
            for (int j = 0; j < N; ++j)
                v[i][j] = v[i][j] * r * w[j];
            store_elems(h.p + row * h.stride + c[i], cols - c[i], v[i]);
        }
    }
}

// Rows part, part + parts, ... of a block; the weight gradients of its rows go to the workspace, from where the sums over the
// parts are taken in order.
template <class X, class Y, int WAVES, int C>
__global__ __launch_bounds__(64 * WAVES) void k_block_norm_grad(BlockNorm p, int64_t rows, int64_t cols, int64_t pitch, int parts,
                                                                BlockNormGrad<X, Y> g)
{
    constexpr int N = kJoint<X, Y>;
    __shared__ float lds[2][WAVES][3];
    BlockSums<WAVES, 3> sums{lds};
    const int64_t part = work_block();
    if (part >= parts)
        return;
    int c[C];
#pragma unroll
    for (int i = 0; i < C; ++i)
        c[i] = N * (i * 64 * WAVES + (int)threadIdx.x);
    float dpost[C][N] = {}, dpre[C][N] = {};
    for (int64_t row = part; row < rows; row += parts) {
        Raw<X, N> dhr[C], br[C];
        Raw<Y, N> dyr[C], yr[C];
        if (g.dh.p) {
            fetch(g.dh.p + row * g.dh.stride, cols, c, dhr);
            fetch(g.y.p + row * g.y.stride, cols, c, yr);
        }
        if (g.dy.p)
            fetch(g.dy.p + row * g.dy.stride, cols, c, dyr);
        if (g.branch.p)
            fetch(g.branch.p + row * g.branch.stride, cols, c, br);
        float t[C][N], b[C][N];
        float s[3] = {0.0f, 0.0f, 0.0f}; // y^2, dh w_pre y, b^2
#pragma unroll
        for (int i = 0; i < C; ++i) {
            if (g.dh.p) {
                float y[N], w[N];
                take(dhr[i], c[i], cols, t[i]);
                take(yr[i], c[i], cols, y);
                weight_at(static_cast<const X *>(p.pre_weight), c[i], cols, w);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    s[0] = __builtin_fmaf(y[j], y[j], s[0]);
                    s[1] = __builtin_fmaf(t[i][j] * w[j], y[j], s[1]);
                }
            }
            if (g.branch.p) {
                take(br[i], c[i], cols, b[i]);
#pragma unroll
                for (int j = 0; j < N; ++j)
                    s[2] = __builtin_fmaf(b[i][j], b[i][j], s[2]);
            }
        }
        sums.add(s);
        const float ry = 1.0f / __builtin_sqrtf(s[0] / (float)cols + p.pre_eps);
        const float along = s[1] / (float)cols * ry * ry;                     // of y, by which dh w_pre is shortened
        const float rb = p.post_norm ? 1.0f / __builtin_sqrtf(s[2] / (float)cols + p.post_eps) : 1.0f;
        const float gate = p.gate ? p.gate[row] : 1.0f, by = p.branch_scale * gate;
        float q[3] = {0.0f, 0.0f, 0.0f}; // t u / r_b, and nothing else
#pragma unroll
        for (int i = 0; i < C; ++i) {
            if (g.dh.p) {
                float y[N], w[N];
                take(yr[i], c[i], cols, y);
                weight_at(static_cast<const X *>(p.pre_weight), c[i], cols, w);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    dpre[i][j] = __builtin_fmaf(t[i][j], y[j] * ry, dpre[i][j]);
                    t[i][j] = ry * (t[i][j] * w[j] - y[j] * along);
                }
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j)
                    t[i][j] = 0.0f;
            }
            if (g.dy.p) {
                float d[N];
                take(dyr[i], c[i], cols, d);
#pragma unroll
                for (int j = 0; j < N; ++j)
                    t[i][j] += d[j];
            }
            if (g.dres.p) {
                float o[N];
#pragma unroll
                for (int j = 0; j < N; ++j)
                    o[j] = t[i][j] * p.residual_scale;
                store_elems(g.dres.p + row * g.dres.stride + c[i], cols - c[i], o);
            }
            float w[N];
            weight_at(static_cast<const X *>(p.post_weight), c[i], cols, w);
            if (g.branch.p) {
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    dpost[i][j] = __builtin_fmaf(t[i][j] * by, b[i][j] * rb, dpost[i][j]);
                    q[0] = __builtin_fmaf(t[i][j] * w[j], b[i][j], q[0]);
                }
            }
#pragma unroll
            for (int j = 0; j < N; ++j)
                t[i][j] *= w[j] * by;
        }
        float mean = 0.0f;
        if (p.post_norm || g.dgate) {
            sums.add(q);
            if (g.dgate && threadIdx.x == 0)
                g.dgate[row] = p.branch_scale * rb * q[0];
            mean = p.post_norm ? by * q[0] * rb * rb / (float)cols : 0.0f;
        }
        if (g.dbranch.p) {
#pragma unroll
            for (int i = 0; i < C; ++i) {
                if (p.post_norm) {
#pragma unroll
                    for (int j = 0; j < N; ++j)
                        t[i][j] = rb * (t[i][j] - b[i][j] * mean);
                }
                store_elems(g.dbranch.p + row * g.dbranch.stride + c[i], cols - c[i], t[i]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < C; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (c[i] + j < cols) {
                if (g.post_parts)
                    g.post_parts[part * pitch + c[i] + j] = dpost[i][j];
                if (g.pre_parts)
                    g.pre_parts[part * pitch + c[i] + j] = dpre[i][j];
            }
}

constexpr int kMostParts = 512;
int64_t pitch_of(int64_t cols) { return (cols + 7) / 8 * 8; }
int parts_of(int64_t rows) { return (int)(rows < kMostParts ? rows : kMostParts); }

// A body with the waves and accesses of rows of `places` accesses.
template <class F>
int with_shape(int64_t places, F body)
{
    using std::integral_constant;
    if (places <= 64)
        return body(integral_constant<int, 1>{}, integral_constant<int, 1>{});
    if (places <= 128)
        return body(integral_constant<int, 1>{}, integral_constant<int, 2>{});
    if (places <= 256)
        return body(integral_constant<int, 1>{}, integral_constant<int, 4>{});
    if (places <= 512)
        return body(integral_constant<int, 4>{}, integral_constant<int, 2>{});
    if (places <= 768)
        return body(integral_constant<int, 4>{}, integral_constant<int, 3>{});
    if (places <= 1024)
        return body(integral_constant<int, 4>{}, integral_constant<int, 4>{});
    if (places <= 2048)
        return body(integral_constant<int, 8>{}, integral_constant<int, 4>{});
    return body(integral_constant<int, 8>{}, integral_constant<int, 8>{});
}

} // namespace

int64_t block_norm_grad_workspace(int64_t rows, int64_t cols)
{
    return rows <= 0 || cols <= 0 ? 0 : 2 * parts_of(rows) * pitch_of(cols) * (int64_t)sizeof(float);
}

int launch_block_norm(int x_dtype, int y_dtype, const BlockNorm &p, int64_t rows, int64_t cols, Rows<const void *> branch,
                      Rows<const void *> residual, Rows<void *> y, Rows<void *> h, hipStream_t s)
{
    return with_type(x_dtype, [&](auto x_tag) {
        return with_type(y_dtype, [&](auto y_tag) {
            using X = decltype(x_tag);
            using Y = decltype(y_tag);
            constexpr int N = kJoint<X, Y>;
            return with_shape((cols + N - 1) / N, [&](auto waves, auto chunks) {
                return launch<waves>(k_block_norm<X, Y, waves, chunks>, rows, kUncapped, s, p, rows, cols, typed<const X>(branch),
                                     typed<const Y>(residual), typed<Y>(y), typed<X>(h));
            });
        });
    });
}

int launch_block_norm_grad(int x_dtype, int y_dtype, const BlockNorm &p, int64_t rows, int64_t cols, const BlockNormArrays &a,
                           float *workspace, hipStream_t s)
{
    const int parts = parts_of(rows);
    const int64_t pitch = pitch_of(cols);
    float *post = a.dpost_weight ? workspace : nullptr, *pre = a.dpre_weight ? workspace + (post ? parts * pitch : 0) : nullptr;
    const int rc = with_type(x_dtype, [&](auto x_tag) {
        return with_type(y_dtype, [&](auto y_tag) {
            using X = decltype(x_tag);
            using Y = decltype(y_tag);
            constexpr int N = kJoint<X, Y>;
            const BlockNormGrad<X, Y> g{typed<const X>(a.dh), typed<const Y>(a.dy), typed<const X>(a.branch), typed<const Y>(a.y),
                                        typed<X>(a.dbranch), typed<Y>(a.dresidual), a.dgate, post, pre};
            return with_shape((cols + N - 1) / N, [&](auto waves, auto chunks) {
                return launch<waves>(k_block_norm_grad<X, Y, waves, chunks>, parts, kUncapped, s, p, rows, cols, pitch, parts, g);
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
