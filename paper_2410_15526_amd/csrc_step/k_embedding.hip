// k_embedding.hip -- rows of a table by token, and the table's gradient.
//
// The gradient of a table row is the sum of the rows of dy whose token it is.
// To take it in one order whatever the timing, the rows are sorted by token:
//  1. one tile of up to kTile rows, or tiles of 2^kManyLog2: each row's place
//     in its tile counted against the whole tile (a comparison a pair: no
//     exchange between lanes, no passes);
//  2. with more than one tile, kWays of them merged at a time until one is
//     left: each row's place by binary searches in the others;
//  3. where each token's rows begin, by binary search, and the sums of runs of
//     kRun sorted rows of one token;
//  4. the table, every row written once: the sums, with whole runs from step
//     3, and zeros elsewhere.
// The rest is HBM's: dy is read once, the table written once.
#include "step_device.hpp"

#include <limits.h>

namespace sdp4 {

namespace {

template <class X, class Y>
constexpr int kEmbed = sizeof(X) == 4 || sizeof(Y) == 4 ? 4 : 8; // elements of a lane in one access

// A wave for 64 accesses of a row.  8192 x 5120 from a bfloat16 table of 50000 rows: 28 to 29 us, 5.8 to 6.0 TB/s.
template <class X, class Y>
__global__ __launch_bounds__(256) void k_embedding(Tokens t, int64_t cols, float scale, Divisor per_row, int64_t waves,
                                                   Rows<const X *> table, Rows<Y *> y)
{
    constexpr int N = kEmbed<X, Y>;
    const int64_t w = work_block() * 4 + uniform(threadIdx.x / kWave);
    if (w >= waves)
        return;
    uint64_t part;
    const int64_t row = (int64_t)divide((uint64_t)w, per_row, part);
    const int64_t c = N * ((int64_t)part * kWave + lane_id());
    const int64_t token = (int64_t)uniform((uint64_t)t.p[row]);
    float v[N];
    if (token >= 0 && token < t.vocab) {
        load_row(table.p + token * table.stride, c, cols, v);
        end_row(c, cols, v);
#pragma unroll
        for (int j = 0; j < N; ++j)
            v[j] *= scale;
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
            v[j] = token < 0 ? 0.0f : __builtin_nanf("");
    }
    store_elems(y.p + row * y.stride + c, cols - c, v);
}

// ---------------------------------------------------------------------------
// sorting
// ---------------------------------------------------------------------------
constexpr int kTileLog2 = 13, kTile = 1 << kTileLog2, kRun = 32;
// Rows of a tile where one is not enough, and runs merged at a time.  The whole gradient of 65536 / 524288 / 2^21 rows of 64
// columns, 1000 tokens, in us: 95 / 408 / 1546; runs of two 98 / 411 / 1500, of eight 101 / 421 / 1600, of 16 108 / 464 / 1709; eight
// with tiles of 1024 rows 105 / 414 / 1534, of 4096 110 / 495 / 1906; tiles of 8192, each row searched for in all others, 123 / 811
// / 4966.
constexpr int kManyLog2 = 11, kWaysLog2 = 2, kWays = 1 << kWaysLog2;
// A block places 32 rows, so that 8192 take all 256 compute units: 17 us, 8 for 2047 rows.  Bound by the comparisons, a pair each.
constexpr int kSortRows = 32, kSortThreads = 512, kShares = kSortThreads / kSortRows; // rows of a block; threads of a row

// Tokens without a row of the table sort behind all others.
SDP4_DEV uint32_t key_of(const Tokens &t, int64_t row)
{
    if (row >= t.rows)
        return ~0u;
    const int64_t v = t.p[row];
    return v < 0 || v >= t.vocab ? (uint32_t)t.vocab : (uint32_t)v;
}

__global__ __launch_bounds__(kSortThreads) void k_sort_tiles(Tokens t, int tile_log2, uint32_t *keys, uint32_t *order)
{
    __shared__ __align__(16) uint32_t all[kTile];
    __shared__ int below[kShares][kSortRows];
    const int64_t first = work_block() * kSortRows, base = first >> tile_log2 << tile_log2;
    if (first >= t.rows)
        return;
    const int size = 1 << tile_log2;
    for (int i = threadIdx.x; i < size; i += 4 * kSortThreads) {
        uint32_t k[4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
            k[u] = key_of(t, base + i + u * kSortThreads);
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (i + u * kSortThreads < size)
                all[i + u * kSortThreads] = k[u];
    }
    __syncthreads();
    const int mine = (int)(first - base), share = threadIdx.x / kSortRows, r = threadIdx.x % kSortRows;
    const uint32_t key = all[mine + r];
    // earlier rows come first where tokens are equal
    const int each = size / kShares, a = share * each, b = a + each;
    int count = 0;
    const int before = b < mine ? b : mine, after = a > mine + kSortRows ? a : mine + kSortRows;
#pragma unroll 8
    for (int j = a; j < before; j += 4) {
        const u32x4 k = *reinterpret_cast<const u32x4 *>(all + j);
        count += (k.x <= key) + (k.y <= key) + (k.z <= key) + (k.w <= key);
    }
#pragma unroll 8
    for (int j = after; j < b; j += 4) {
        const u32x4 k = *reinterpret_cast<const u32x4 *>(all + j);
        count += (k.x < key) + (k.y < key) + (k.z < key) + (k.w < key);
    }
    for (int j = a > mine ? a : mine; j < (b < mine + kSortRows ? b : mine + kSortRows); ++j)
        count += all[j] < key || (all[j] == key && j < mine + r);
    below[share][r] = count;
    __syncthreads();
    if (threadIdx.x < kSortRows && first + r < t.rows) {
        int place = 0;
#pragma unroll
        for (int i = 0; i < kShares; ++i)
            place += below[i][r];
        keys[base + place] = key, order[base + place] = (uint32_t)(first + r);
    }
}

// Numbers below `key` (or up to it) among n sorted ones.
template <bool EQUAL>
SDP4_DEV int64_t count_below(const uint32_t *keys, int64_t n, uint32_t key)
{
    int64_t a = 0;
    while (n > 0) {
        const int64_t half = n / 2;
        const uint32_t k = keys[a + half];
        if (EQUAL ? k <= key : k < key)
            a += half + 1, n -= half + 1;
        else
            n = half;
    }
    return a;
}

// kWays sorted runs of 2^run_log2 rows each become one: a row's place among the others' by a search in each of them.
__global__ __launch_bounds__(256) void k_merge_runs(int64_t rows, int run_log2, const uint32_t *keys, const uint32_t *order,
                                                    uint32_t *to_keys, uint32_t *to_order)
{
    const int64_t i = work_block() * 256 + threadIdx.x;
    if (i >= rows)
        return;
    const uint32_t key = keys[i];
    const int64_t mine = i >> run_log2, first = mine / kWays * kWays;
    int64_t place = (first << run_log2) + i - (mine << run_log2);
    for (int64_t run = first; run < first + kWays; ++run) {
        const int64_t at = run << run_log2, n = rows - at < (int64_t)1 << run_log2 ? rows - at : (int64_t)1 << run_log2;
        if (n <= 0)
            break;
        if (run < mine)
            place += count_below<true>(keys + at, n, key);
        else if (run > mine)
            place += count_below<false>(keys + at, n, key);
    }
    to_keys[place] = key, to_order[place] = order[i];
}

// ---------------------------------------------------------------------------
// sums
// ---------------------------------------------------------------------------
// Adds U rows of dy to v, in order: a wave, the same rows in all lanes, A accesses of each.  row(u) names them.
template <int U, class X, int N, int A, class F>
SDP4_DEV void add_batch(const Rows<const X *> &dy, F row, const int (&c)[A], int64_t cols, float (&v)[A][N])
{
    Raw<X, N> r[U][A];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const X *p = dy.p + (int64_t)uniform((uint32_t)row(u)) * dy.stride;
#pragma unroll
        for (int k = 0; k < A; ++k)
            load_row(p, c[k], cols, r[u][k]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int k = 0; k < A; ++k) {
            float w[N];
            r[u][k].get(w);
            end_row(c[k], cols, w);
#pragma unroll
            for (int j = 0; j < N; ++j)
                v[k][j] += w[j];
        }
}
// `count` rows: as many at a time as there are, up to U.
template <int U, class X, int N, int A, class F>
SDP4_DEV void add_rows(const Rows<const X *> &dy, int64_t count, F row, const int (&c)[A], int64_t cols, float (&v)[A][N])
{
    int64_t i = 0;
    for (; i + U <= count; i += U)
        add_batch<U>(dy, [&](int u) { return row(i + u); }, c, cols, v);
    if constexpr (U > 1)
        add_rows<U / 2>(dy, count - i, [&](int64_t u) { return row(i + u); }, c, cols, v);
}

template <int N>
SDP4_DEV void load_sums(const float *p, float (&v)[N])
{
#pragma unroll
    for (int j = 0; j < N; j += 4) {
        float w[4];
        load_whole(p + j, w);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[j + i] = w[i];
    }
}

// The first `token_blocks` blocks: where each token's rows begin.  The others: sums of whole runs, a wave for 64 accesses.
template <class X, int N>
__global__ __launch_bounds__(256) void k_runs(Tokens t, int64_t cols, Rows<const X *> dy, const uint32_t *keys, const uint32_t *order,
                                              int64_t token_blocks, uint32_t *starts, int64_t col_parts, int64_t pitch, float *runs)
{
    constexpr int SAMPLES = 1024; // every so many sorted tokens: most steps of a search are made in LDS
    __shared__ uint32_t samples[SAMPLES];
    const int64_t block = work_block();
    if (block < token_blocks) {
        const int64_t step = (t.rows + SAMPLES - 1) / SAMPLES;
#pragma unroll
        for (int i = 0; i < SAMPLES / 256; ++i) {
            const int k = i * 256 + threadIdx.x;
            samples[k] = k * step < t.rows ? keys[k * step] : ~0u;
        }
        __syncthreads();
        const int64_t v = block * 256 + threadIdx.x;
        if (v > t.vocab)
            return;
        const int64_t behind = count_below<false>(samples, SAMPLES, (uint32_t)v); // the first sample that is not below
        const int64_t from = behind ? (behind - 1) * step + 1 : 0, to = behind * step < t.rows ? behind * step : t.rows;
        starts[v] = (uint32_t)(from < to ? from + count_below<false>(keys + from, to - from, (uint32_t)v) : to);
        return;
    }
    const int64_t w = (block - token_blocks) * 4 + uniform(threadIdx.x / kWave), run = w / col_parts, part = w - run * col_parts;
    const int64_t a = run * kRun;
    if (a + kRun > t.rows || keys[a] != keys[a + kRun - 1] || keys[a] >= (uint32_t)t.vocab)
        return;
    const int place = N * ((int)part * kWave + lane_id()), c[1] = {place < cols ? place : 0};
    float v[1][N] = {};
    add_rows<8>(dy, kRun, [&](int64_t i) { return order[a + i]; }, c, cols, v);
    if (place < cols) {
#pragma unroll
        for (int j = 0; j < N; ++j)
            runs[run * pitch + place + j] = v[0][j];
    }
}

// Two kinds of blocks, evenly mixed (`sums` of `blocks` are of the first), so that the trips to memory of the one run beside the
// other's stores.  A wave of the first kind takes 64 or 128 accesses of the row of a sorted position: where a token's rows begin,
// their sum goes to the table (ADD: onto what it holds).  A wave of the second writes zeros, kZeros accesses of the
// table in order, where a row has no token.
//
// 8192 x 5120 bfloat16 into 50000 float32 rows, all launches: 234 us, of which zeros alone take 165 (a fill 156).  One kind of
// wave for a part of each table row 335, sums in front of all zeros 325, sums that look their rows up in three trips 305.
constexpr int kZeros = 4;
template <bool ADD>
constexpr int kWide = ADD ? 1 : 2;
template <class X, class Y, bool ADD>
__global__ __launch_bounds__(256) void k_table(Tokens t, int64_t cols, float scale, Rows<const X *> dy, const uint32_t *keys,
                                               const uint32_t *order, const uint32_t *starts, int64_t pitch, const float *runs,
                                               Divisor wide_parts, Divisor parts, int64_t sums, Divisor blocks, Rows<Y *> table)
{
    constexpr int N = kEmbed<X, Y>, W = kWide<ADD>, U = 8 / W; // U rows of W accesses under way
    const int64_t block = work_block();
    if (block >= (int64_t)blocks.d)
        return;
    uint64_t rest;
    const int64_t before = (int64_t)divide((uint64_t)block * (uint64_t)sums, blocks, rest); // blocks of the first kind so far
    const int wave = uniform(threadIdx.x / kWave);
    uint64_t part;
    if (rest + (uint64_t)sums < blocks.d) { // the next one counts as many
        if (ADD)
            return;
        const int64_t w = ((block - before) * 4 + wave) * kZeros;
        int64_t token[kZeros], place[kZeros];
        bool none[kZeros];
#pragma unroll
        for (int k = 0; k < kZeros; ++k) {
            token[k] = (int64_t)divide((uint64_t)(w + k), parts, part);
            place[k] = N * ((int64_t)part * kWave + lane_id());
            none[k] = false;
            if (token[k] < t.vocab)
                none[k] = starts[token[k]] == starts[token[k] + 1];
        }
        const float zeros[N] = {};
#pragma unroll
        for (int k = 0; k < kZeros; ++k)
            if (none[k])
                store_elems(table.p + token[k] * table.stride + place[k], cols - place[k], zeros);
        return;
    }
    const int64_t a = (int64_t)divide((uint64_t)(before * 4 + wave), wide_parts, part);
    if (a >= t.rows)
        return;
    // the next 64 sorted rows, a lane each: what most tokens need, in one trip to memory
    const int64_t mine = a + lane_id() < t.rows ? a + lane_id() : t.rows - 1;
    const uint32_t key = keys[mine], row_of = order[mine], last = keys[a > 0 ? a - 1 : 0];
    const uint32_t token = uniform(key);
    if (token >= (uint32_t)t.vocab || (a > 0 && uniform(last) == token))
        return;
    int place[W], c[W];
    float v[W][N] = {};
#pragma unroll
    for (int k = 0; k < W; ++k) {
        place[k] = N * (((int)part * W + k) * kWave + lane_id());
        c[k] = place[k] < cols ? place[k] : 0;
    }
    const uint64_t others = ~__ballot(key == token && a + lane_id() < t.rows);
    if (others) {
        add_rows<U>(dy, __builtin_ctzll(others), [&](int64_t i) { return __builtin_amdgcn_readlane(row_of, (int)i); }, c, cols, v);
    } else { // 64 rows or more: whole runs, and the rows before and behind them
        const int64_t b = uniform(starts[token + 1]), whole = (a + kRun - 1) / kRun, behind = b / kRun;
        add_rows<U>(dy, whole * kRun - a, [&](int64_t i) { return order[a + i]; }, c, cols, v);
        for (int64_t i = whole; i < behind; i += U) {
            float r[U][W][N];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int k = 0; k < W; ++k)
                    load_sums(runs + (i + u < behind ? i + u : behind - 1) * pitch + c[k], r[u][k]);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int k = 0; k < W; ++k)
#pragma unroll
                    for (int j = 0; j < N; ++j)
                        v[k][j] += i + u < behind ? r[u][k][j] : 0.0f;
        }
        add_rows<U>(dy, b - behind * kRun, [&](int64_t i) { return order[behind * kRun + i]; }, c, cols, v);
    }
    Y *row = table.p + (int64_t)token * table.stride;
#pragma unroll
    for (int k = 0; k < W; ++k) {
        if constexpr (ADD) {
            float held[N];
            load_row(row, c[k], cols, held);
            end_row(c[k], cols, held);
#pragma unroll
            for (int j = 0; j < N; ++j)
                v[k][j] = __builtin_fmaf(v[k][j], scale, held[j]);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j)
                v[k][j] *= scale;
        }
        store_elems(row + place[k], cols - place[k], v[k]);
    }
}

// The workspace: sorted tokens and rows, the same before the tiles are merged, starts, sums of runs.
struct Layout {
    int64_t keys, order, tile_keys, tile_order, starts, runs, bytes, pitch;
    Layout(int64_t rows, int64_t vocab, int64_t cols)
    {
        int64_t at = 0;
        auto take = [&](int64_t n) {
            const int64_t here = at;
            at += (4 * n + 15) / 16 * 16;
            return here;
        };
        const bool merged = rows > kTile;
        pitch = (cols + 7) / 8 * 8;
        keys = take(rows), order = take(rows);
        tile_keys = take(merged ? rows : 0), tile_order = take(merged ? rows : 0);
        starts = take(vocab + 1);
        runs = take(rows / kRun * pitch);
        bytes = at;
    }
};

} // namespace

int launch_embedding(const Tokens &t, int64_t cols, float scale, int in, Rows<const void *> table, int out, Rows<void *> y,
                     hipStream_t s)
{
    return with_type(in, [&](auto in_tag) {
        return with_type(out, [&](auto out_tag) {
            using X = decltype(in_tag);
            using Y = decltype(out_tag);
            constexpr int64_t width = kEmbed<X, Y> * kWave;
            const int64_t per_row = (cols + width - 1) / width, waves = t.rows * per_row;
            return launch<4>(k_embedding<X, Y>, (waves + 3) / 4, kUncapped, s, t, cols, scale, Divisor((uint64_t)per_row), waves,
                             typed<const X>(table), typed<Y>(y));
        });
    });
}

int64_t embedding_grad_workspace(int64_t rows, int64_t vocab, int64_t cols) { return Layout(rows, vocab, cols).bytes; }

int launch_embedding_grad(const Tokens &t, int64_t cols, float scale, bool accumulate, int in, Rows<const void *> dy, int out,
                          Rows<void *> dtable, void *workspace, hipStream_t s)
{
    const Layout l(t.rows, t.vocab, cols);
    char *base = static_cast<char *>(workspace);
    auto at = [&](int64_t offset) { return reinterpret_cast<uint32_t *>(base + offset); };
    const bool merged = t.rows > kTile;
    int tile_log2 = merged ? kManyLog2 : kTileLog2, passes = 0;
    while (!merged && tile_log2 > 6 && (1 << (tile_log2 - 1)) >= t.rows) // one tile: only as large as the rows take
        --tile_log2;
    while (merged && (int64_t)1 << (tile_log2 + passes * kWaysLog2) < t.rows)
        ++passes;
    int rc = 0;
    if (t.rows > 0) {
        uint32_t *keys[2] = {at(l.keys), at(l.tile_keys)}, *order[2] = {at(l.order), at(l.tile_order)}; // in turn, the first at the end
        rc = launch<kSortThreads / kWave>(k_sort_tiles, (t.rows + kSortRows - 1) / kSortRows, kUncapped, s, t, tile_log2,
                                          keys[passes % 2], order[passes % 2]);
        for (int p = passes; p > 0 && !rc; --p, tile_log2 += kWaysLog2)
            rc = launch<4>(k_merge_runs, (t.rows + 255) / 256, kUncapped, s, t.rows, tile_log2, keys[p % 2], order[p % 2],
                           keys[(p - 1) % 2], order[(p - 1) % 2]);
    }
    if (rc)
        return rc;
    return with_type(in, [&](auto in_tag) {
        return with_type(out, [&](auto out_tag) {
            using X = decltype(in_tag);
            using Y = decltype(out_tag);
            constexpr int N = kEmbed<X, Y>;
            const int64_t per_row = (cols + N * kWave - 1) / (N * kWave), token_blocks = (t.vocab + 256) / 256;
            const int64_t run_waves = t.rows / kRun * per_row;
            float *runs = reinterpret_cast<float *>(base + l.runs);
            int rc = launch<4>(k_runs<X, N>, token_blocks + (run_waves + 3) / 4, kUncapped, s, t, cols, typed<const X>(dy), at(l.keys),
                               at(l.order), token_blocks, at(l.starts), per_row, l.pitch, runs);
            if (rc)
                return rc;
            const int64_t each = accumulate ? kWide<true> : kWide<false>, wide = (per_row + each - 1) / each;
            const int64_t sums = (t.rows * wide + 3) / 4;
            const int64_t blocks = sums + (accumulate ? 0 : (t.vocab * per_row + 4 * kZeros - 1) / (4 * kZeros));
            if (blocks == 0)
                return 0;
            auto k = accumulate ? k_table<X, Y, true> : k_table<X, Y, false>;
            return launch<4>(k, blocks, kUncapped, s, t, cols, scale, typed<const X>(dy), at(l.keys), at(l.order), at(l.starts),
                             l.pitch, runs, Divisor((uint64_t)wide), Divisor((uint64_t)per_row), sums, Divisor((uint64_t)blocks),
                             typed<Y>(dtable));
        });
    });
}

} // namespace sdp4
