// attention.hpp -- device building blocks of the attention kernels: tiles of
// rows in LDS, matrix fragments, and which rows see which.
//
// Matrix instructions take 32 x 16 by 16 x 32 products.  Of an operand, lane l
// holds eight elements along the summed axis of one row (column) l % 32:
// places 8 h .. 8 h + 7 with h = l / 32.  Of the 32 x 32 result it holds
// column l % 32 and rows 8 a + 4 h + b, register 4 a + b.  float32 takes eight
// 32 x 32 x 2 products for the same fragments.
//
// Scores are computed transposed (rows: keys, columns: queries), so that a
// query's scores lie in two lanes, and the registers of a result, taken eight
// by eight, are an operand of the next product as they stand: the summed axis
// may be walked in any order that both operands share, here keys 8 a + 4 h + b
// of a step of 16 at place 4 a + b.
#pragma once

#include "shares.hpp"
#include "step_device.hpp"

#include <limits.h>

namespace sdp4 {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

// Eight elements of an operand.
template <class T>
struct Frag;
template <>
struct Frag<bf16_t> {
    bf16x8 v;
    SDP4_DEV void set(const float (&x)[8])
    {
        const u32x4 w{bf16x2_rne(x[0], x[1]), bf16x2_rne(x[2], x[3]), bf16x2_rne(x[4], x[5]), bf16x2_rne(x[6], x[7])};
        v = __builtin_bit_cast(bf16x8, w);
    }
    SDP4_DEV float get(int j) const { return (float)v[j]; }
};
template <>
struct Frag<float> {
    float v[8];
    SDP4_DEV void set(const float (&x)[8])
    {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            v[j] = x[j];
    }
    SDP4_DEV float get(int j) const { return v[j]; }
};

SDP4_DEV void mma(const Frag<bf16_t> &a, const Frag<bf16_t> &b, f32x16 &c)
{
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, c, 0, 0, 0);
}
SDP4_DEV void mma(const Frag<float> &a, const Frag<float> &b, f32x16 &c)
{
#pragma unroll
    for (int j = 0; j < 8; ++j)
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[j], b.v[j], c, 0, 0, 0);
}

// Eight elements of one row in global memory, from element e on; zeros from `dim` on.
template <class T>
SDP4_DEV void load_frag(const T *row, int e, int dim, Frag<T> &f)
{
    float x[8];
    if (e + 8 <= dim) {
        if constexpr (sizeof(T) == 2) {
            f.v = __builtin_bit_cast(bf16x8, load_chunk<false>(row + e));
            return;
        } else {
            const u32x4 a = load_chunk<false>(row + e), b = load_chunk<false>(row + e + 4);
            const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
            for (int j = 0; j < 8; ++j)
                x[j] = __uint_as_float(w[j]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            x[j] = e + j < dim ? to_f32<T>(row[e + j]) : 0.0f;
    }
    f.set(x);
}

// Heads of up to 32 * DB elements, as rows of LD elements in LDS.
//
// 16-byte chunk c of row r lies at chunk c ^ f(r), so that both kinds of reads spread over the banks: 16 lanes that read one
// chunk of 16 neighbouring rows (f takes 16 values, or eight for the rows of one parity where two rows fill the banks), and
// the transposing reads, where a group of 32 lanes takes four neighbouring chunks of four rows (f moves them apart by four).
template <class T, int DB>
struct HeadTile {
    static constexpr int D = 32 * DB, LD = D <= 64 ? 64 : D <= 128 ? 128 : 256, N = kChunk<T>;
    static constexpr int CHUNKS = LD / N, USED = D / N, ROW = LD * (int)sizeof(T), STEPS = 2 * DB;

    SDP4_DEV static int twist(int r)
    {
        return CHUNKS == 8 ? ((r >> 1) & 1) << 2 | ((r >> 2) & 3) : (r & 3) << 2 | ((r >> 2) & 3);
    }
    SDP4_DEV static int at(int r, int chunk) { return r * ROW + ((chunk ^ twist(r)) << 4); }

};

// Where in LDS a lane finds its parts of the operands: addresses that are computed once and follow the tiles by move(); an
// access adds a constant, which is the instruction's.  AT: bytes from where the addresses point to the tile.
template <class V>
SDP4_DEV V read_lds(uint32_t at)
{
    return *(__attribute__((address_space(3))) const V *)(uintptr_t)at;
}
SDP4_DEV uint32_t lds_address(const void *p) { return uniform((uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)p); }

template <class T, int DB>
struct Reader;

template <int DB>
struct Reader<bf16_t, DB> {
    using H = HeadTile<bf16_t, DB>;
    uint32_t in_row[H::STEPS], in_column[DB][2];
    SDP4_DEV explicit Reader(uint32_t base)
    {
        const int l = lane_id(), r = l & 31, h = l >> 5, i = l & 15;
#pragma unroll
        for (int s = 0; s < H::STEPS; ++s)
            in_row[s] = base + H::at(r, 2 * s + h);
        // a transposing read gives lane i of 16 element i of four rows, of which lane i points at a quarter of row i / 4
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int a = 0; a < 2; ++a)
                in_column[db][a] = base + H::at(8 * a + 4 * h + (i >> 2), 4 * db + 2 * ((l >> 4) & 1) + ((i & 3) >> 1)) + 8 * (i & 1);
    }
    SDP4_DEV void move(uint32_t by)
    {
#pragma unroll
        for (int s = 0; s < H::STEPS; ++s)
            in_row[s] += by;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int a = 0; a < 2; ++a)
                in_column[db][a] += by;
    }
    // Operand with rows r0 + l % 32, elements 16 s + ... along the sum.
    template <int AT>
    SDP4_DEV void rows(int r0, int s, Frag<bf16_t> &f) const
    {
        f.v = read_lds<bf16x8>(in_row[s] + (AT + r0 * H::ROW));
    }
    // Operand with the tile's elements 32 db + l % 32 as rows and its rows r0 + 8 a + 4 h + b along the sum.
    template <int AT>
    SDP4_DEV void columns(int r0, int db, Frag<bf16_t> &f) const
    {
        s16x4 v[2];
#pragma unroll
        for (int a = 0; a < 2; ++a)
            v[a] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) s16x4 *)(uintptr_t)(in_column[db][a] + (AT + r0 * H::ROW)));
        f.v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

template <int DB>
struct Reader<float, DB> {
    using H = HeadTile<float, DB>;
    uint32_t in_row[H::STEPS], in_column[8];
    SDP4_DEV explicit Reader(uint32_t base)
    {
        const int l = lane_id(), r = l & 31, h = l >> 5;
#pragma unroll
        for (int s = 0; s < H::STEPS; ++s)
            in_row[s] = base + H::at(r, 4 * s + 2 * h); // tiles begin at multiples of 32 bytes, for the other half (^ 16)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            in_column[j] = base + H::at(8 * (j >> 2) + 4 * h + (j & 3), r >> 2) + 4 * (r & 3);
    }
    SDP4_DEV void move(uint32_t by)
    {
#pragma unroll
        for (int s = 0; s < H::STEPS; ++s)
            in_row[s] += by;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            in_column[j] += by;
    }
    template <int AT>
    SDP4_DEV void rows(int r0, int s, Frag<float> &f) const
    {
        const u32x4 a = read_lds<u32x4>(in_row[s] + (AT + r0 * H::ROW)), b = read_lds<u32x4>((in_row[s] ^ 16) + (AT + r0 * H::ROW));
        const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int j = 0; j < 8; ++j)
            f.v[j] = __uint_as_float(w[j]);
    }
    template <int AT>
    SDP4_DEV void columns(int r0, int db, Frag<float> &f) const
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) // in_column is element block 0's place: block db lies eight chunks a block away, twisted by bit 3
            f.v[j] = read_lds<float>(in_column[j] + (AT + r0 * H::ROW + ((((8 * db) ^ ((j & 2) << 2)) - ((j & 2) << 2)) << 4)));
    }
};

// The rows of a tile that stays where it is.
template <class T, int DB>
struct RowReader {
    using H = HeadTile<T, DB>;
    uint32_t in_row[H::STEPS];
    SDP4_DEV explicit RowReader(uint32_t base)
    {
        const int r = lane_id() & 31, h = lane_id() >> 5;
#pragma unroll
        for (int s = 0; s < H::STEPS; ++s)
            in_row[s] = base + H::at(r, sizeof(T) == 2 ? 2 * s + h : 4 * s + 2 * h);
    }
    template <int AT>
    SDP4_DEV void rows(int s, Frag<T> &f) const
    {
        if constexpr (sizeof(T) == 2) {
            f.v = read_lds<bf16x8>(in_row[s] + AT);
        } else {
            const u32x4 a = read_lds<u32x4>(in_row[s] + AT), b = read_lds<u32x4>((in_row[s] ^ 16) + AT);
            const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
            for (int j = 0; j < 8; ++j)
                f.v[j] = __uint_as_float(w[j]);
        }
    }
};
// Puts a lane's fragment s of row l % 32 into a tile.
template <class T, int DB>
SDP4_DEV void put_row(char *tile, int s, const Frag<T> &f)
{
    using H = HeadTile<T, DB>;
    const int r = lane_id() & 31, h = lane_id() >> 5;
    if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<bf16x8 *>(tile + H::at(r, 2 * s + h)) = f.v;
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            *reinterpret_cast<u32x4 *>(tile + H::at(r, 4 * s + 2 * h + i)) =
                u32x4{__float_as_uint(f.v[4 * i]), __float_as_uint(f.v[4 * i + 1]), __float_as_uint(f.v[4 * i + 2]),
                      __float_as_uint(f.v[4 * i + 3])};
    }
}

// All but the N youngest loads of the wave have arrived.
template <int N>
SDP4_DEV void wait_loads()
{
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}

// A buffer of plain bytes from an address on, without a stride: offsets from kBufferBytes on lie outside and read zeros.
constexpr uint32_t kBufferBytes = 1u << 31, kBufferFormat = 0x00020000;

// Rows first .. first + ROWS - 1 of one head on their way from global memory to a tile: load() starts them; after wait_loads()
// and store() they are in the tile, for all waves from the next barrier on.  Rows from `limit` on hold other rows of the head: they are masked, and masked
// rows may hold anything.  Elements from `dim` on are zeros.
//
// Straight into LDS, past the registers, where every row begins on 16 bytes and holds whole chunks: an instruction moves 64
// chunks to 64 places in turn, so the lanes fetch what belongs at theirs.  A place beyond the head's elements gets zeros, as its
// offset lies outside the buffer: whatever stood there would meet zeros of the other operand, and 0 times an infinity is NaN.
template <class T, int DB, int ROWS, int WAVES, bool DIRECT>
struct TileLoad {
    using H = HeadTile<T, DB>;
    static constexpr int COUNT = ROWS * H::CHUNKS / (64 * WAVES);
    static_assert(COUNT * 64 * WAVES == ROWS * H::CHUNKS, "whole rounds");
    const char *head;
    int64_t pitch; // bytes from row to row
    uint32_t offset[COUNT], element[COUNT], row[COUNT];

    SDP4_DEV void begin(const T *h, int64_t stride, int dim)
    {
        head = reinterpret_cast<const char *>(h), pitch = stride * (int64_t)sizeof(T);
        const int wave = uniform(threadIdx.x / kWave);
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int id = (wave * COUNT + i) * 64 + lane_id(), r = id / H::CHUNKS, c = (id % H::CHUNKS) ^ H::twist(r);
            row[i] = r;
            element[i] = c * H::N < dim ? c * 16 : kBufferBytes;
            offset[i] = row[i] * (uint32_t)pitch + element[i];
        }
    }
    SDP4_DEV void move(const T *h) { head = reinterpret_cast<const char *>(h); }
    SDP4_DEV void load(char *tile, int first, int limit)
    {
        const uint64_t from = uniform((uint64_t)(head + first * pitch));
        const u32x4 base = {(uint32_t)from, (uint32_t)(from >> 32), kBufferBytes, kBufferFormat};
        const uint32_t at = lds_address(tile) + uniform(threadIdx.x / kWave) * (COUNT * 1024);
        if (first + ROWS <= limit) {
#pragma unroll
            for (int i = 0; i < COUNT; ++i)
                start(at + i * 1024, offset[i], base);
        } else {
#pragma unroll
            for (int i = 0; i < COUNT; ++i) {
                const uint32_t last = limit - first - 1;
                start(at + i * 1024, (row[i] < last ? row[i] : last) * (uint32_t)pitch + element[i], base);
            }
        }
    }
    // Where in LDS: register m0, which the compiler sets as the operand that it is, one wait state before the load.  No register
    // is written, so the compiler need not know that this is under way: wait_loads() sees to it.
    SDP4_DEV static void start(uint32_t at, uint32_t off, u32x4 base)
    {
        asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "{m0}"(at), "v"(off), "s"(base) : "memory");
    }
    SDP4_DEV void store(char *, int, int) const {}
};

// A lane's row of a result, times `by`: four elements at a time, which meet their neighbours in the L2 cache.  (Stores past the
// caches wrote 4.5 times the bytes: 8192 tokens, 40 heads of 128 bfloat16, 376 MB instead of 84, and 296 us instead of 275 among other calls.)
template <class T, int DB>
SDP4_DEV void store_row(T *row, int dim, const f32x16 (&o)[DB], float by)
{
    const int h = lane_id() >> 5;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            const int d = 32 * db + 8 * a + 4 * h;
            float w[4];
#pragma unroll
            for (int b = 0; b < 4; ++b)
                w[b] = o[db][4 * a + b] * by;
            Raw<T, 4> r;
            r.put(w);
            if (d + 4 <= dim) {
                if constexpr (sizeof(T) == 4)
                    *reinterpret_cast<u32x4_b4 *>(row + d) = r.v;
                else
                    *reinterpret_cast<u32x2_b2 *>(row + d) = r.v;
            } else {
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    if (d + b < dim)
                        row[d + b] = from_f32<T>(w[b]);
            }
        }
}

// A number for each lane from its own address into LDS, as TileLoad does.
SDP4_DEV void load_word(float *to, const float *from)
{
    const uint32_t at = lds_address(to);
    asm volatile("s_nop 0\n\tglobal_load_lds_dword %1, off" : : "{m0}"(at), "v"(from) : "memory");
}

// Through registers, for all other heads: a head's last chunk, where it is not whole, is read as the head's last whole one and
// shifted.
template <class T, int DB, int ROWS, int WAVES>
struct TileLoad<T, DB, ROWS, WAVES, false> {
    using H = HeadTile<T, DB>;
    static constexpr int THREADS = 64 * WAVES, CHUNKS = ROWS * H::USED, COUNT = (CHUNKS + THREADS - 1) / THREADS;
    u32x4 v[COUNT];
    const T *head;
    int64_t stride;
    int dim;

    SDP4_DEV void begin(const T *h, int64_t s, int d) { head = h, stride = s, dim = d; }
    SDP4_DEV void move(const T *h) { head = h; }
    SDP4_DEV void load(char *, int first, int limit)
    {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int place = i * THREADS + (int)threadIdx.x, id = place < CHUNKS ? place : 0;
            const int r = id / H::USED, e = (id - r * H::USED) * H::N, row = first + r < limit ? first + r : limit - 1;
            v[i] = load_chunk<false>(head + row * stride + (e + H::N <= dim ? e : dim - H::N));
        }
    }
    SDP4_DEV void store(char *tile, int, int) const
    {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int id = i * THREADS + (int)threadIdx.x, r = id / H::USED, e = (id - r * H::USED) * H::N;
            u32x4 w = v[i];
            if (dim % H::N)
                w = e + H::N <= dim ? w : shifted(w, e + H::N - dim);
            if (id < CHUNKS)
                *reinterpret_cast<u32x4 *>(tile + H::at(r, e / H::N)) = e < dim ? w : u32x4{0, 0, 0, 0};
        }
    }
    SDP4_DEV static u32x4 shifted(u32x4 w, int by) // by elements toward the first, with zeros behind; by >= N is not used
    {
        const int bits = 8 * sizeof(T) * (by & (H::N - 1));
        return __builtin_bit_cast(u32x4, __builtin_bit_cast(unsigned __int128, w) >> bits);
    }
};

// Heads whose rows can go straight into LDS: whole chunks at multiples of 16 bytes, 64 rows within 2 GB.
inline bool direct(const Heads &h, int dtype, int dim)
{
    const int64_t size = dtype == SDP4_BF16 ? 2 : 4;
    return reinterpret_cast<uintptr_t>(h.p) % 16 == 0 && dim * size % 16 == 0 && h.token_stride * size % 16 == 0 &&
           h.head_stride * size % 16 == 0 && 64 * h.token_stride * size < (int64_t(1) << 31);
}

// A fragment whose masked places must not reach the product: what is infinite or NaN becomes 0 and is noted in `found`
// (bit j: element j), since 0 times such a value would be NaN.
SDP4_DEV uint32_t scrub(Frag<bf16_t> &f)
{
    u32x4 w = __builtin_bit_cast(u32x4, f.v);
    uint32_t found = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const bool lo = (w[j] & 0x7F80u) == 0x7F80u, hi = (w[j] & 0x7F800000u) == 0x7F800000u;
        w[j] &= (lo ? 0u : 0xFFFFu) | (hi ? 0u : 0xFFFF0000u);
        found |= (lo ? 1u << (2 * j) : 0u) | (hi ? 2u << (2 * j) : 0u);
    }
    f.v = __builtin_bit_cast(bf16x8, w);
    return found;
}
SDP4_DEV uint32_t scrub(Frag<float> &f)
{
    uint32_t found = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const bool bad = (__float_as_uint(f.v[j]) & 0x7F800000u) == 0x7F800000u;
        f.v[j] = bad ? 0.0f : f.v[j];
        found |= bad ? 1u << j : 0u;
    }
    return found;
}
// The tile rows (bits) of the elements that scrub found in the fragment at r0 of a tile of up to 64 rows.
SDP4_DEV uint64_t tile_rows(uint32_t found, int r0)
{
    const int h = lane_id() >> 5;
    const uint64_t bits = (found & 0xFu) | (found & 0xF0u) << 4; // places 4 a + b -> rows 8 a + b
    return bits << (r0 + 4 * h);
}
SDP4_DEV uint64_t or_wave(uint64_t v)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t lo = __shfl_xor((uint32_t)v, d), hi = __shfl_xor((uint32_t)(v >> 32), d);
        v |= (uint64_t)hi << 32 | lo;
    }
    return v;
}

// The sequence of a row: `samples` (LDS, kSeqSamples numbers, filled by fill_samples) narrow the search to a few offsets.
constexpr int kSeqSamples = 256;
SDP4_DEV int64_t sample_step(const Sequences &s) { return (s.count + kSeqSamples) / kSeqSamples; } // of count + 1 offsets
template <int THREADS>
SDP4_DEV void fill_samples(const Sequences &s, int64_t *samples)
{
    if (!s.offsets)
        return;
    const int64_t step = sample_step(s);
    for (int i = threadIdx.x; i < kSeqSamples; i += THREADS)
        samples[i] = i * step <= s.count ? s.offsets[i * step] : INT64_MAX;
    __syncthreads();
}
struct Span {
    int first, end; // rows of the sequence
    bool on;        // false: the row is in none
};
// Whatever the offsets hold, 0 <= first <= row < end <= tokens.
SDP4_DEV Span span_of(const Sequences &s, const int64_t *samples, int row)
{
    Span r{0, s.tokens, row < s.tokens};
    if (!s.offsets || !r.on)
        return r;
    int lo = 0, hi = kSeqSamples; // the last sample <= row lies in [lo, hi), if there is one
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (samples[mid] <= row)
            lo = mid;
        else
            hi = mid;
    }
    if (samples[0] > row) {
        r.on = false;
        return r;
    }
    const int64_t step = sample_step(s);
    int64_t a = lo * step, b = a + step < s.count + 1 ? a + step : s.count + 1;
    while (b - a > 1) {
        const int64_t mid = (a + b) / 2;
        if (s.offsets[mid] <= row)
            a = mid;
        else
            b = mid;
    }
    if (a >= s.count) {
        r.on = false;
        return r;
    }
    const int64_t first = s.offsets[a], end = s.offsets[a + 1];
    r.first = first < 0 ? 0 : first > row ? row : (int)first;
    r.end = end <= row ? row + 1 : end > s.tokens ? s.tokens : (int)end;
    return r;
}

// Smallest and largest value over a wave, on the scalar unit.
SDP4_DEV int min_wave(int v)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_xor(v, d);
        v = o < v ? o : v;
    }
    return (int)uniform((uint32_t)v);
}
SDP4_DEV int max_wave(int v) { return -min_wave(-v); }

// Which of the tiles of ROWS keys is number `place` by the rows that follow up to its sequence's end, those with most first, so
// that no long walk begins when the others end; a head's places are dealt to the XCDs (dealt_place).  dk and dv of four sequences
// of 2048, heads of 128, 5 query heads to one of 1 / 2 / 4 / 8 / 12: the whole backward pass in 163 / 216 / 372 / 696 / 1101 us,
// in the order of memory 171 / 210 / 373 / 828 / 1137, by work in runs 194 / 269 / 434 / 713 / 1105.  Twelve sequences of 16384
// rows in all, 16 heads over 4: 824, 972, 911; one of 16384: 3995, 4674, 4696.  Each block looks for its tile first: where
// walks are short or blocks many, the order of memory is up to 6 % faster (40 sequences of 8192 rows, 8 heads over 1: 138 against
// 144; twelve of 16384, 16 heads of 64: 480 against 507).  By queries, of which a launch has more blocks, the forward pass took
// 251 us so and 237 in the order of memory.  More tiles than kMostOrdered are left in order, as their ends are a small part.
constexpr int kMostOrdered = 256;
SDP4_DEV bool by_work(const Sequences &s, int tiles) { return s.offsets && tiles <= kMostOrdered; }
template <int THREADS, int ROWS>
SDP4_DEV int ordered_tile(const Sequences &s, const int64_t *samples, int (&work)[kMostOrdered], int &found, int tiles, int place)
{
    for (int t = threadIdx.x; t < tiles; t += THREADS) {
        const int a = t * ROWS, b = a + ROWS < s.tokens ? a + ROWS - 1 : s.tokens - 1;
        const Span x = span_of(s, samples, a), y = span_of(s, samples, b);
        work[t] = (y.on ? y.end : x.on ? x.end : a) - a;
    }
    __syncthreads();
    for (int t = threadIdx.x; t < tiles; t += THREADS) {
        const int mine = work[t];
        int before = 0;
        for (int u = 0; u < tiles; ++u)
            before += work[u] > mine || (work[u] == mine && u < t);
        if (before == place)
            found = t;
    }
    __syncthreads();
    return (int)uniform((uint32_t)found);
}

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// From here on (octaves) a reference is subtracted from the scores before their product with c = scale log2(e), whose rounding
// would otherwise move exponents by more than the 2^-12 that it is here: as much as the rounding of such a score itself.
constexpr float kLargeScore = 4096.0f;

// The value of lane ^ 32, without a trip through LDS.
SDP4_DEV float other_half(float v)
{
    const uint32_t u = __float_as_uint(v);
    const auto both = __builtin_amdgcn_permlane32_swap(u, u, false, false); // (low, low) and (high, high)
    return __uint_as_float(lane_id() < 32 ? both[1] : both[0]);
}

SDP4_DEV float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

} // namespace sdp4
