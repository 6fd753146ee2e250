// k_dropout.hip -- bias, dropout and residual in one pass, its backward pass
// with the bias gradient, and the sum over partial column sums.
//
// y = residual + keep ? (x + bias) s : 0 with keep = h(e) >= T: h(e) is the
// 16-bit uniform that Philox4x32-10 gives element position e (device.hpp:
// one evaluation for eight elements), so the mask costs no memory and the
// backward pass draws it again.  Rows start at multiples of the width
// rounded up to 8, which keeps the eight elements of an evaluation in one
// row: they are the work of one lane.
#include "step_device.hpp"

namespace sdp4 {

namespace {

// Sets dropped elements to 0 and scales the others.  A select, not a product: what is dropped may be infinite or NaN.
SDP4_DEV void apply_mask(uint64_t seed, uint64_t block, uint32_t drop, float scale, float (&v)[8])
{
    uint32_t c[4] = {(uint32_t)block, (uint32_t)(block >> 32), 0u, 0u};
    philox4x32_10(c, (uint32_t)seed, (uint32_t)(seed >> 32));
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        v[2 * w] = (c[w] & 0xFFFFu) >= drop ? v[2 * w] * scale : 0.0f;
        v[2 * w + 1] = (c[w] >> 16) >= drop ? v[2 * w + 1] * scale : 0.0f;
    }
}

// Eight elements per lane, 256 lanes in a block, rows one after the other.
template <class In, class Out, bool BIAS, bool RES>
__global__ __launch_bounds__(256) void k_dropout_add(Dropout d, Divisor per_row, int64_t total, Rows<const In *> x,
                                                     const In *bias, Rows<const Out *> res, Rows<Out *> y)
{
    const int64_t t = work_block() * 256 + threadIdx.x;
    if (t >= total)
        return;
    uint64_t k;
    const int64_t r = (int64_t)divide((uint64_t)t, per_row, k);
    const int64_t c = 8 * (int64_t)k, valid = d.cols - c;
    float v[8], b[8], a[8];
    load_elems(x.p + r * x.stride + c, valid, v);
    if constexpr (BIAS)
        load_elems(bias + c, valid, b);
    if constexpr (RES)
        load_elems(res.p + r * res.stride + c, valid, a);
    if constexpr (BIAS) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            v[j] += b[j];
    }
    if (d.drop)
        apply_mask(d.seed, d.offset / 8 + (uint64_t)t, d.drop, d.scale, v);
    if constexpr (RES) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            v[j] += a[j];
    }
    store_elems(y.p + r * y.stride + c, valid, v);
}

// Backward with column sums.  A block takes `lx` neighbouring 8-element columns and a range of rows, 256 / lx rows
// at a time; a lane adds up its eight columns in registers, the block's rows join through LDS, and the sums of the
// row ranges go to the workspace, from where k_sum_parts adds them in order: no atomics, one result.
template <class In, class Out>
__global__ __launch_bounds__(256) void k_dropout_grad(Dropout d, int lx_log2, int64_t per_row, int64_t col_tiles,
                                                      int64_t rows_each, Rows<const In *> dy, Rows<Out *> dx,
                                                      float *parts)
{
    __shared__ float lds[256 * 8];
    const int lx = 1 << lx_log2, ly = 256 >> lx_log2;
    const uint32_t tile = (uint32_t)(work_block() % col_tiles);
    const int64_t part = work_block() / col_tiles;
    const int tx = threadIdx.x & (lx - 1), ty = threadIdx.x >> lx_log2;
    const int64_t k = (int64_t)tile * lx + tx, c = 8 * k, valid = d.cols - c;
    const int64_t end = (part + 1) * rows_each < d.rows ? (part + 1) * rows_each : d.rows;
    float acc[8] = {};
    if (k < per_row) {
        for (int64_t r = part * rows_each + ty; r < end; r += ly) {
            float v[8];
            load_elems(dy.p + r * dy.stride + c, valid, v);
            apply_mask(d.seed, d.offset / 8 + (uint64_t)(r * per_row + k), d.drop, d.scale, v);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                acc[j] += v[j];
            store_elems(dx.p + r * dx.stride + c, valid, v);
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        lds[j * 256 + threadIdx.x] = acc[j];
    __syncthreads();
    // column j of lane tx: sum over ty, by consecutive threads
    for (int o = threadIdx.x; o < 8 * lx; o += 256) {
        const int j = o & 7, l = o >> 3;
        float sum = 0.0f;
        for (int i = 0; i < ly; ++i)
            sum += lds[j * 256 + (i << lx_log2) + l];
        const int64_t col = 8 * ((int64_t)tile * lx) + o;
        if (col < 8 * per_row)
            parts[part * 8 * per_row + col] = sum;
    }
}

// 256 threads: CX columns by 256 / CX slices of the parts.
template <int CX>
__global__ __launch_bounds__(256) void k_sum_parts(const float *parts, int64_t nparts, int64_t pitch, int64_t cols,
                                                   float *out)
{
    __shared__ float lds[256];
    constexpr int SL = 256 / CX;
    const int64_t c = work_block() * CX + threadIdx.x % CX;
    const int sl = threadIdx.x / CX;
    float sum = 0.0f;
    if (c < cols) {
#pragma unroll 8
        for (int64_t i = sl; i < nparts; i += SL)
            sum += parts[i * pitch + c];
    }
    lds[threadIdx.x] = sum;
    __syncthreads();
    if (sl == 0 && c < cols) {
        float s = 0.0f;
        for (int i = 0; i < SL; ++i)
            s += lds[i * CX + threadIdx.x];
        out[c] = s;
    }
}

template <class T, class P>
Rows<T *> typed(Rows<P> r)
{
    return {static_cast<T *>(r.p), r.stride};
}

// The split of the backward pass: 8-element columns side by side in a block, and row ranges.
struct GradSplit {
    int lx_log2;
    int64_t per_row, col_tiles, rows_each, parts;
};
GradSplit grad_split(int64_t rows, int64_t cols)
{
    GradSplit g;
    g.per_row = (cols + 7) / 8;
    g.lx_log2 = 0;
    while (g.lx_log2 < 6 && (int64_t(1) << g.lx_log2) < g.per_row)
        ++g.lx_log2;
    g.col_tiles = (g.per_row + (1 << g.lx_log2) - 1) >> g.lx_log2;
    const int64_t step = 256 >> g.lx_log2;          // rows a block takes at a time
    int64_t want = (1024 + g.col_tiles - 1) / g.col_tiles;
    const int64_t most = (rows + 2 * step - 1) / (2 * step);
    want = want < most ? want : most;
    want = want < 1 ? 1 : want;
    g.rows_each = ((rows + want - 1) / want + step - 1) / step * step;
    g.parts = (rows + g.rows_each - 1) / g.rows_each;
    return g;
}

} // namespace

int64_t dropout_grad_workspace(int64_t rows, int64_t cols)
{
    if (rows <= 0 || cols <= 0)
        return 0;
    const GradSplit g = grad_split(rows, cols);
    return g.parts * g.per_row * 8 * (int64_t)sizeof(float);
}

int launch_dropout_add(const Dropout &d, int in, Rows<const void *> x, const void *bias, int out,
                       Rows<const void *> residual, Rows<void *> y, hipStream_t s)
{
    const int64_t per_row = (d.cols + 7) / 8, total = d.rows * per_row;
    return with_type(in, [&](auto in_tag) {
        return with_type(out, [&](auto out_tag) {
            using In = decltype(in_tag);
            using Out = decltype(out_tag);
            auto k = bias ? (residual.p ? k_dropout_add<In, Out, true, true> : k_dropout_add<In, Out, true, false>)
                          : (residual.p ? k_dropout_add<In, Out, false, true> : k_dropout_add<In, Out, false, false>);
            return launch<4>(k, (total + 255) / 256, kUncapped, s, d, Divisor((uint64_t)per_row), total,
                             typed<const In>(x), static_cast<const In *>(bias), typed<const Out>(residual),
                             typed<Out>(y));
        });
    });
}

int launch_dropout_grad(const Dropout &d, int in, Rows<const void *> dy, int out, Rows<void *> dx, float *dbias,
                        float *workspace, hipStream_t s)
{
    const GradSplit g = grad_split(d.rows, d.cols);
    const int rc = with_type(in, [&](auto in_tag) {
        return with_type(out, [&](auto out_tag) {
            using In = decltype(in_tag);
            using Out = decltype(out_tag);
            return launch<4>(k_dropout_grad<In, Out>, g.col_tiles * g.parts, kUncapped, s, d, g.lx_log2, g.per_row,
                             g.col_tiles, g.rows_each, typed<const In>(dy), typed<Out>(dx), workspace);
        });
    });
    return rc ? rc : launch_sum_parts(workspace, g.parts, 8 * g.per_row, d.cols, dbias, s);
}

int launch_sum_parts(const float *parts, int64_t nparts, int64_t pitch, int64_t cols, float *out, hipStream_t s)
{
    return launch<4>(k_sum_parts<16>, (cols + 15) / 16, kUncapped, s, parts, nparts, pitch, cols, out);
}

} // namespace sdp4
