// k_dropout.hip -- bias, dropout and residual in one pass, its backward pass
// with the bias gradient, and the sum over partial column sums.
//
// y = residual + keep ? (x + bias) s : 0 with keep = h(e) >= T: h(e) is the
// 16-bit uniform that Philox4x32-10 gives element position e (device.hpp:
// one evaluation for eight elements), so the mask costs no memory and the
// backward pass draws it again.  Rows start at multiples of the width
// rounded up to 8, which keeps the eight elements of an evaluation in one
// row: they are the work of one lane.
//
// HBM bounds all of it; the generator's 20 products for eight elements keep the vector units 40 % busy in the forward
// pass (p = 0, without them, takes the same time).
#include "step_device.hpp"

namespace sdp4 {

namespace {

// The generator's words for one block of eight elements.
SDP4_DEV void draw(const Dropout &d, uint64_t block, uint32_t (&c)[4])
{
    const uint64_t n = d.offset / 8 + block;
    c[0] = (uint32_t)n, c[1] = (uint32_t)(n >> 32), c[2] = c[3] = 0u;
    philox4x32_10(c, (uint32_t)d.seed, (uint32_t)(d.seed >> 32));
}

// Sets dropped elements to 0 and scales the others.  A select, not a product: what is dropped may be infinite or NaN.
template <int N>
SDP4_DEV void apply_mask(const uint32_t *words, uint32_t drop, float scale, float (&v)[N])
{
#pragma unroll
    for (int w = 0; w < N / 2; ++w) {
        v[2 * w] = (words[w] & 0xFFFFu) >= drop ? v[2 * w] * scale : 0.0f;
        v[2 * w + 1] = (words[w] >> 16) >= drop ? v[2 * w + 1] * scale : 0.0f;
    }
}

// A wave's 64 blocks of eight elements, as its lanes hold them: N elements per access and lane, neighbouring lanes at
// neighbouring addresses.  bfloat16 rows: a lane's eight elements are one 16-byte access.  With float32 on either side
// they would be two, 32 bytes apart between lanes: there a lane takes the same half (lane % 2) of blocks lane / 2 and
// 32 + lane / 2, evaluates the generator for one of them and swaps two words with its neighbour.
template <bool HALVES>
struct Lanes {
    static constexpr int N = HALVES ? 4 : 8, COUNT = HALVES ? 2 : 1;
    SDP4_DEV static int block(int i) { return HALVES ? 32 * i + lane_id() / 2 : lane_id(); }
    SDP4_DEV static int start() { return HALVES ? 4 * (lane_id() & 1) : 0; } // first element in the block
    SDP4_DEV static int mine() { return HALVES ? block(lane_id() & 1) : block(0); } // the block it evaluates
    // words of the lane's elements in access i, from the number of the block it evaluates
    SDP4_DEV static void draw(const Dropout &d, uint64_t block, uint32_t (&words)[COUNT][N / 2])
    {
        uint32_t c[4];
        sdp4::draw(d, block, c);
        if constexpr (HALVES) {
            const bool odd = lane_id() & 1;
            const uint32_t a = dpp_u32<kDppXor1>(odd ? c[0] : c[2]), b = dpp_u32<kDppXor1>(odd ? c[1] : c[3]);
            words[0][0] = odd ? a : c[0], words[0][1] = odd ? b : c[1];
            words[1][0] = odd ? c[2] : a, words[1][1] = odd ? c[3] : b;
        } else {
#pragma unroll
            for (int w = 0; w < 4; ++w)
                words[0][w] = c[w];
        }
    }
};

// 512 elements per wave, four waves in a block, rows one after the other: 8192 x 5120 bfloat16 40.7 us, 6.2 TB/s (float32
// 79, 6.4, and 105 in a form in which a lane read its 32 bytes together).  A wave whose blocks are all whole and in one
// row addresses them as a scalar base plus a lane offset; the others find each lane's row.
template <class In, class Out, bool BIAS, bool RES>
__global__ __launch_bounds__(256) void k_dropout_add(Dropout d, Divisor per_row, uint32_t inv32, int64_t total,
                                                     Rows<const In *> x, const In *bias, Rows<const Out *> res,
                                                     Rows<Out *> y)
{
    using L = Lanes<sizeof(In) == 4 || sizeof(Out) == 4>;
    constexpr int N = L::N, C = L::COUNT;
    const uint64_t first = (uint64_t)work_block() * 256 + uniform(threadIdx.x / kWave) * kWave;
    if (first >= (uint64_t)total)
        return;
    uint64_t k0;
    const uint64_t r0 = divide(first, per_row, k0);
    float v[C][N], b[C][N], a[C][N];
    uint32_t words[C][N / 2];
    auto finish = [&](int i) {
        if constexpr (BIAS) {
#pragma unroll
            for (int j = 0; j < N; ++j)
                v[i][j] += b[i][j];
        }
        if (d.drop)
            apply_mask(words[i], d.drop, d.scale, v[i]);
        if constexpr (RES) {
#pragma unroll
            for (int j = 0; j < N; ++j)
                v[i][j] += a[i][j];
        }
    };
    if ((int64_t)k0 + kWave <= d.cols / 8) {
        const In *xw = x.p + (int64_t)r0 * x.stride + 8 * k0, *bw = bias + 8 * k0;
        const Out *rw = res.p + (int64_t)r0 * res.stride + 8 * k0;
        Out *yw = y.p + (int64_t)r0 * y.stride + 8 * k0;
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const uint32_t at = 8 * L::block(i) + L::start();
            load_whole(xw + at, v[i]);
            if constexpr (RES)
                load_whole(rw + at, a[i]);
            if constexpr (BIAS)
                load_whole(bw + at, b[i]);
        }
        if (d.drop)
            L::draw(d, first + L::mine(), words);
#pragma unroll
        for (int i = 0; i < C; ++i) {
            finish(i);
            store_elems(yw + (8 * L::block(i) + L::start()), N, v[i]);
        }
        return;
    }
    const In *xw = x.p + (int64_t)r0 * x.stride;
    const Out *rw = res.p + (int64_t)r0 * res.stride;
    Out *yw = y.p + (int64_t)r0 * y.stride;
    const uint32_t left = (uint64_t)total - first < kWave ? (uint32_t)((uint64_t)total - first) : kWave; // blocks of the wave
    uint32_t ahead[C]; // rows from the wave's first
    int32_t c[C];
#pragma unroll
    for (int i = 0; i < C; ++i) {
        const uint32_t b0 = L::block(i);
        uint32_t k = (uint32_t)k0 + (b0 < left ? b0 : left - 1), q = __umulhi(k, inv32);
        k -= q * (uint32_t)per_row.d;
        if (k >= (uint32_t)per_row.d)
            k -= (uint32_t)per_row.d, ++q;
        ahead[i] = q, c[i] = (int32_t)(8 * k) + L::start();
        load_row(xw + (uint64_t)q * (uint64_t)x.stride, c[i], d.cols, v[i]);
        if constexpr (RES)
            load_row(rw + (uint64_t)q * (uint64_t)res.stride, c[i], d.cols, a[i]);
        if constexpr (BIAS)
            load_row(bias, c[i], d.cols, b[i]);
    }
    if (d.drop)
        L::draw(d, first + L::mine(), words);
#pragma unroll
    for (int i = 0; i < C; ++i) {
        end_row(c[i], d.cols, v[i]);
        if constexpr (RES)
            end_row(c[i], d.cols, a[i]);
        if constexpr (BIAS)
            end_row(c[i], d.cols, b[i]);
        finish(i);
        store_elems(yw + (uint64_t)ahead[i] * (uint64_t)y.stride + c[i], (uint32_t)L::block(i) < left ? d.cols - c[i] : 0, v[i]);
    }
}

// Backward with column sums.  A block takes 2^lx_log2 neighbouring 8-element columns and every parts-th batch of rows; a
// lane adds up its columns in registers, the block's lanes of one column join through LDS, and the blocks' sums go to the
// workspace, from where k_sum_parts adds them in order: no atomics, one result.
//
// Batches in turn rather than a range of rows for each block, so that the chip's accesses move through memory on one
// front.  The loop over whole batches has no test in it and steps its addresses, and it has the next batch's loads under
// way before it stores the present one, since loads that follow stores wait for these.  4095 x 2048 float32 12.2 us, 5.7
// TB/s with its partial sums, and 4.5 for the sums over the parts, which is a launch and one trip to memory; 8192 x 5120
// bfloat16 34.6 in all.
template <class In, class Out>
__global__ __launch_bounds__(256) void k_dropout_grad(Dropout d, int lx_log2, int64_t per_row, int64_t col_tiles,
                                                      int64_t nparts, Rows<const In *> dy, Rows<Out *> dx,
                                                      float *parts)
{
    constexpr bool H = sizeof(In) == 4 || sizeof(Out) == 4;
    using L = Lanes<H>;
    constexpr int N = L::N, C = L::COUNT, U = 4 / C; // U rows of a lane in a batch
    __shared__ float lds[256 * 8];
    const int lx = 1 << lx_log2, ly = 256 >> lx_log2;
    const int64_t part = work_block() / col_tiles, tile = work_block() - part * col_tiles;
    const int64_t batch = U * ly, stride = nparts * batch; // rows of a batch, and to the block's next
    // the block's 256 (column, row) places, 64 to a wave: place -> column place % lx, row place / lx
    const int wave = uniform(threadIdx.x / kWave) * kWave;
    const int64_t col0 = tile * lx;
    float acc[C][N] = {};
    int64_t r0 = part * batch;
    // the generator's block of the lane's first row, and the steps from row to row
    const int drawn = wave + L::mine();
    uint64_t block = (uint64_t)((r0 + (drawn >> lx_log2)) * per_row + col0 + (drawn & (lx - 1)));
    const uint64_t row_step = (uint64_t)(ly * per_row), batch_step = (uint64_t)(stride * per_row);
    if (8 * (col0 + lx) <= d.cols && r0 + batch <= d.rows) {
        const In *src[C];
        Out *dst[C];
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int place = wave + L::block(i);
            const int64_t c = 8 * (col0 + (place & (lx - 1))) + L::start(), r = r0 + (place >> lx_log2);
            src[i] = dy.p + r * dy.stride + c, dst[i] = dx.p + r * dx.stride + c;
        }
        const int64_t in_row = ly * dy.stride, out_row = ly * dx.stride, in_step = stride * dy.stride, out_step = stride * dx.stride;
        Raw<In, N> next[U][C];
        auto fetch = [&] {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < C; ++i)
                    next[u][i].template load<true>(src[i] + u * in_row);
#pragma unroll
            for (int i = 0; i < C; ++i)
                src[i] += in_step;
        };
        fetch();
        for (; r0 + batch <= d.rows; r0 += stride) {
            float v[U][C][N];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < C; ++i)
                    next[u][i].get(v[u][i]);
            if (r0 + stride + batch <= d.rows)
                fetch();
#pragma unroll
            for (int u = 0; u < U; ++u) {
                uint32_t words[C][N / 2] = {};
                if (d.drop)
                    L::draw(d, block + u * row_step, words);
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    apply_mask(words[i], d.drop, d.scale, v[u][i]);
#pragma unroll
                    for (int j = 0; j < N; ++j)
                        acc[i][j] += v[u][i][j];
                    Raw<Out, N> o;
                    o.put(v[u][i]);
                    o.store(dst[i] + u * out_row);
                }
            }
#pragma unroll
            for (int i = 0; i < C; ++i)
                dst[i] += out_step;
            block += batch_step;
        }
    }
    // Rows and columns that need looking after: the same loop with tests, places beyond the array reading others.  Batch after
    // batch in flight here too, since these blocks end last: 8192 x 5119 bfloat16 48.8 / 42.4 us, 4095 x 2047 float32 20.3 /
    // 17.9, 4095 x 2048 17.8 / 16.8.
    if (r0 < d.rows) {
        Raw<In, N> next[U][C];
        auto fetch = [&](int64_t from) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    const int place = wave + L::block(i);
                    const int64_t r = from + u * ly + (place >> lx_log2), k = col0 + (place & (lx - 1));
                    load_row(dy.p + (r < d.rows ? r : d.rows - 1) * dy.stride, k < per_row ? 8 * k + L::start() : 0, d.cols,
                             next[u][i]);
                }
        };
        fetch(r0);
#pragma unroll 1
        for (; r0 < d.rows; r0 += stride, block += batch_step) {
            float v[U][C][N];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < C; ++i)
                    next[u][i].get(v[u][i]);
            if (r0 + stride < d.rows)
                fetch(r0 + stride);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                uint32_t words[C][N / 2] = {};
                if (d.drop)
                    L::draw(d, block + u * row_step, words);
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    const int place = wave + L::block(i);
                    const int64_t r = r0 + u * ly + (place >> lx_log2), k = col0 + (place & (lx - 1)), c = 8 * k + L::start();
                    if (r < d.rows && k < per_row) {
                        end_row(c, d.cols, v[u][i]);
                        apply_mask(words[i], d.drop, d.scale, v[u][i]);
#pragma unroll
                        for (int j = 0; j < N; ++j)
                            acc[i][j] += v[u][i][j];
                        store_elems(dx.p + r * dx.stride + c, d.cols - c, v[u][i]);
                    }
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < C; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j)
            lds[(L::start() + j) * 256 + wave + L::block(i)] = acc[i][j];
    __syncthreads();
    for (int o = threadIdx.x; o < 8 * lx; o += 256) {
        const int j = o & 7, l = o >> 3;
        float sum = 0.0f;
        for (int i = 0; i < ly; ++i)
            sum += lds[j * 256 + (i << lx_log2) + l];
        if (8 * col0 + o < (nparts == 1 ? d.cols : 8 * per_row)) // one part: the sums themselves
            parts[part * 8 * per_row + 8 * col0 + o] = sum;
    }
}

// Sums over parts: a block of 8 waves takes 16 columns, 32 threads share the parts of each.  Few columns and many parts
// make this a matter of latency: a thread has 16 loads in flight, each an offset from one scalar base (64-bit products
// for the addresses took longer than the loads), and one barrier joins the waves.
constexpr int kSumColumns = 16, kSumThreads = 512, kSumShare = kSumThreads / kSumColumns;
template <class Offset> // uint32_t where the parts lie within 4 GB
__global__ __launch_bounds__(kSumThreads) void k_sum_parts(Parts first, Parts second, int64_t blocks_each, int64_t pitch, int64_t cols)
{
    __shared__ float lds[kSumThreads / kWave][kSumColumns];
    const int64_t wb = work_block();
    const Parts s = wb < blocks_each ? first : second;
    if (!s.out)
        return;
    const int col = threadIdx.x % kSumColumns, share = threadIdx.x / kSumColumns;
    const int64_t c0 = (wb < blocks_each ? wb : wb - blocks_each) * kSumColumns;
    const bool on = c0 + col < cols;
    const char *base = reinterpret_cast<const char *>(s.p + c0);
    const Offset step = (Offset)(kSumShare * sizeof(float)) * (Offset)pitch;
    Offset at = ((Offset)share * (Offset)pitch + (on ? col : 0)) * (Offset)sizeof(float);
    float sum = 0.0f;
    for (int i = share; i < (int)s.count; i += 16 * kSumShare) {
        float v[16];
        Offset o = at;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            v[j] = *reinterpret_cast<const float *>(base + o);
            o = i + (j + 1) * kSumShare < (int)s.count ? o + step : at; // beyond the last part: the first again, not used
        }
#pragma unroll
        for (int j = 0; j < 16; ++j)
            sum += i + j * kSumShare < (int)s.count ? v[j] : 0.0f;
        at += 16 * step;
    }
    sum += xor_lane<16>(sum);
    sum += xor_lane<32>(sum);
    if (lane_id() < kSumColumns)
        lds[threadIdx.x / kWave][col] = sum;
    __syncthreads();
    if (threadIdx.x < kSumColumns && on) {
        float total = 0.0f;
#pragma unroll
        for (int w = 0; w < kSumThreads / kWave; ++w)
            total += lds[w][col];
        s.out[c0 + col] = total;
    }
}

// The split of the backward pass: 8-element columns side by side in a block, and the blocks that share a column's rows --
// about kGradBlocks in all, with 8 rows of a lane for each.
struct GradSplit {
    int lx_log2;
    int64_t per_row, col_tiles, parts;
};
// 768 / 1024 / 1280 / 1536 blocks: 8192 x 5120 bfloat16 39.8 / 38.7 / 36.8 / 37.9 us, float32 70.6 / 68.1 / 63.3 / 66.5
// (4095 x 2048 float32, which has fewer batches than that, 17.9 / 18.7 / 18.7 / 18.6).
constexpr int64_t kGradBlocks = 1280;
GradSplit grad_split(int64_t rows, int64_t cols)
{
    GradSplit g;
    g.per_row = (cols + 7) / 8;
    g.lx_log2 = 0;
    while (g.lx_log2 < 6 && (int64_t(1) << g.lx_log2) < g.per_row)
        ++g.lx_log2;
    g.col_tiles = (g.per_row + (1 << g.lx_log2) - 1) >> g.lx_log2;
    const int64_t want = (kGradBlocks + g.col_tiles - 1) / g.col_tiles;
    const int64_t rows_each = 4 * (256 >> g.lx_log2), most = (rows + rows_each - 1) / rows_each;
    g.parts = want < most ? want : most;
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
            return launch<4>(k, (total + 255) / 256, kUncapped, s, d, Divisor((uint64_t)per_row),
                             ~uint32_t(0) / (uint32_t)per_row, total,
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
                             g.col_tiles, g.parts, typed<const In>(dy), typed<Out>(dx), g.parts == 1 ? dbias : workspace);
        });
    });
    return rc || g.parts == 1 ? rc : launch_sum_parts({{workspace, g.parts, dbias}, {}}, 8 * g.per_row, d.cols, s);
}

int launch_sum_parts(const Parts (&parts)[2], int64_t pitch, int64_t cols, hipStream_t s)
{
    const int64_t each = (cols + kSumColumns - 1) / kSumColumns;
    const int64_t most = parts[0].count > parts[1].count ? parts[0].count : parts[1].count;
    auto k = (most + 17 * kSumShare) * pitch < (int64_t(1) << 30) ? k_sum_parts<uint32_t> : k_sum_parts<uint64_t>;
    return launch<kSumThreads / kWave>(k, parts[1].out ? 2 * each : each, kUncapped, s, parts[0], parts[1], each, pitch, cols);
}

} // namespace sdp4
