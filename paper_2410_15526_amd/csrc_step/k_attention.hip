// k_attention.hip -- causal attention over packed sequences.
//
// Row i of a sequence that begins at row b sees keys b .. i of it:
//      s_ij = scale q_i . k_j,  lse_i = log sum_j exp(s_ij),
//      out_i = sum_j exp(s_ij - lse_i) v_j,
// in one pass over the keys with a running reference of the maximum and a
// running sum.  A block takes rows of the batch as they lie, whatever
// sequences they belong to, and masks what lies outside a row's own: many
// short sequences share a block.
#include "attention.hpp"

namespace sdp4 {

namespace {

// The order of COUNT matrix instructions with READS loads from LDS each: AHEAD of them loaded in front, then one
// instruction and the loads of a later one in turn.  The compiler's own order loads more in front and waits for it:
// four sequences of 2048, 40 heads of 128 over 8, take 234.0 us in its order and 230.3 in this one; one of 16384, 16
// heads over 4, 1448 and 1432.
template <int GROUP, int COUNT, int AHEAD, int READS>
SDP4_DEV void spread()
{
    constexpr int MATRIX = 0x8, VECTOR = 0x402, LDS = 0x100; // vector: with the exponentials
    __builtin_amdgcn_sched_group_barrier(LDS, READS * AHEAD, GROUP);
    if (GROUP) // the weights are made under the first loads of the values
        __builtin_amdgcn_sched_group_barrier(VECTOR, 200, GROUP);
#pragma unroll
    for (int i = 0; i < COUNT - AHEAD; ++i) {
        __builtin_amdgcn_sched_group_barrier(MATRIX, 1, GROUP);
        __builtin_amdgcn_sched_group_barrier(LDS, READS, GROUP);
    }
    __builtin_amdgcn_sched_group_barrier(MATRIX, AHEAD, GROUP);
}

// WAVES waves of 32 rows each, BN keys at a time, STAGES tiles in LDS.  The scores are computed transposed, keys by rows, so that
// a lane holds one row's: its maximum and sum need one exchange, and p is the second product's operand as it lies.
//
// Four sequences of 2048, 40 heads of 128 over 8, bfloat16: 220 to 248 us by card and inputs, 693 to 781 TFLOP/s of the pairs that
// rows see (a library product of 8192^3 reaches 1143); one sequence of 16384, 16 heads over 4: 1345 to 1420 us, 774 to 817, where
// four key heads over eight XCDs give every other one three times the work of the rest.  float32: the four 1528 us, 112 TFLOP/s.  Neither memory nor
// either kind of unit alone is the bound: two waves on a SIMD wait for their own scores, maxima and exponentials.  Two, since a
// row's results, queries and scores take 224 registers; eight waves on a tile in place of four took 280 us where this took 248,
// 64 keys a tile halve the barriers and exchanges of 32 (265 and 295), and more tiles ahead change nothing: loads are not
// waited for.
// Heads of more than 128 take one wave on a SIMD and 32 keys, as their registers allow: four of 2048, 8 heads of 256, 264 us in
// bfloat16 and 1124 in float32, which spills a few registers.
template <class T, int DB, int WAVES, int BN, int STAGES, int OCC, bool DIRECT>
__global__ __launch_bounds__(64 * WAVES, OCC) void k_attention(Attention at, Heads qh, Heads kh, Heads vh, Heads oh, float *lse,
                                                             int tiles, int64_t items)
{
    using H = HeadTile<T, DB>;
    constexpr int BM = 32 * WAVES, THREADS = 64 * WAVES, RB = BN / 32;
    constexpr int S = DIRECT ? STAGES : 2; // through registers there is one tile ahead
    constexpr int TILE = BN * H::ROW;
    __shared__ __align__(128) char tiles_lds[S][2][TILE]; // keys, values
    __shared__ int64_t samples[kSeqSamples];
    __shared__ int edges[WAVES][2];

    const int64_t item = shared_item(work_block(), items);
    if (item >= items)
        return;
    const int64_t per_head = (int64_t)tiles * at.group;
    const int kv = (int)(item / per_head);
    const int64_t rest = item - kv * per_head;
    const int tile = tiles - 1 - (int)(rest / at.group), head = kv * at.group + (int)(rest % at.group);

    const int wave = uniform(threadIdx.x / kWave), lane = lane_id(), h = lane >> 5;
    const int q0 = tile * BM + 32 * wave, row = q0 + (lane & 31);
    fill_samples<THREADS>(at.seq, samples);
    const Span span = span_of(at.seq, samples, row);
    const int start = span.on ? span.first : INT_MAX;
    const uint32_t seen = span.on ? row - start + 1 : 0; // keys of the row, from start on
    const int w_first = min_wave(start), w_last = max_wave(span.on ? row : -1); // keys that the wave's rows see
    const int w_full = max_wave(start);                                        // from here to q0 all of them see all
    if (lane == 0)
        edges[wave][0] = w_first, edges[wave][1] = w_last;
    __syncthreads();
    int first = INT_MAX, last = -1;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        first = edges[w][0] < first ? edges[w][0] : first;
        last = edges[w][1] > last ? edges[w][1] : last;
    }
    if (last < 0) // no row of the block is in a sequence
        return;
    first = (int)uniform((uint32_t)first), last = (int)uniform((uint32_t)last);

    const T *qrow = static_cast<const T *>(qh.p) + (int64_t)(row < at.seq.tokens ? row : at.seq.tokens - 1) * qh.token_stride +
                    head * qh.head_stride;
    Frag<T> q[H::STEPS];
#pragma unroll
    for (int s = 0; s < H::STEPS; ++s)
        load_frag(qrow, 16 * s + 8 * h, at.dim, q[s]);
    const T *kp = static_cast<const T *>(kh.p) + kv * kh.head_stride, *vp = static_cast<const T *>(vh.p) + kv * vh.head_stride;

    const float c = at.scale * kLog2e;
    float m = -__builtin_inff(), total = 0.0f; // reference (a score) and the lane's share of the sum
    bool poison = false;
    f32x16 o[DB] = {};

    TileLoad<T, DB, BN, WAVES, DIRECT> kl, vl;
    kl.begin(kp, kh.token_stride, at.dim);
    vl.begin(vp, vh.token_stride, at.dim);
    // CAREFUL: infinities and NaN in masked places are kept from the product, where 0 times them would be NaN
    auto walk = [&](auto careful) {
        constexpr bool CAREFUL = decltype(careful)::value;
        constexpr int PER = DIRECT ? kl.COUNT + vl.COUNT : 0;
        Reader<T, DB> read(lds_address(tiles_lds[S - 1])); // the tile before the first
#pragma unroll
        for (int i = 0; i < S - 1; ++i)
            if (first + i * BN <= last) {
                kl.load(tiles_lds[i][0], first + i * BN, last + 1);
                vl.load(tiles_lds[i][1], first + i * BN, last + 1);
            }
        int stage = 0, ahead = S - 1;
        for (int k0 = first; k0 <= last; k0 += BN) {
            if (k0 + (S - 2) * BN <= last)
                wait_loads<(S - 2) * PER>(); // of the tiles after this one
            else
                wait_loads<0>();
            kl.store(tiles_lds[stage][0], k0, last + 1);
            vl.store(tiles_lds[stage][1], k0, last + 1);
            __syncthreads();
            if (k0 + (S - 1) * BN <= last) {
                kl.load(tiles_lds[ahead][0], k0 + (S - 1) * BN, last + 1);
                vl.load(tiles_lds[ahead][1], k0 + (S - 1) * BN, last + 1);
            }
            read.move(stage ? 2 * TILE : -(S - 1) * 2 * TILE);
            stage = stage + 1 == S ? 0 : stage + 1, ahead = ahead + 1 == S ? 0 : ahead + 1;
            if (k0 > w_last || k0 + BN <= w_first)
                continue;
            const bool masked = !(k0 >= w_full && k0 + BN - 1 <= q0);

            f32x16 x[RB] = {};
#pragma unroll
            for (int s = 0; s < H::STEPS; ++s)
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) {
                    Frag<T> a;
                    read.template rows<0>(32 * rb, s, a);
                    mma(a, q[s], x[rb]);
                }
            if constexpr (sizeof(T) == 2)
                spread<0, H::STEPS * RB, 4, 1>();
            if (masked) {
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const uint32_t key = k0 + 32 * rb + 8 * (r >> 2) + 4 * h + (r & 3);
                        x[rb][r] = key - start < seen ? x[rb][r] : -__builtin_inff();
                    }
            }
            float top[4]; // four chains, here and in the sum: each step of one waits for the step before
#pragma unroll
            for (int i = 0; i < 16 * RB; ++i)
                top[i % 4] = i < 4 ? x[0][i] : fmaxf(top[i % 4], x[i / 16][i % 16]);
            float mx = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
            mx = fmaxf(mx, other_half(mx));
            // The reference is the largest score so far, so that a key which takes a row alone has p = 1, without a rounding.
            // Tiles that raise none of the wave's rows leave the results as they are.
            const bool up = mx > m;
            if (__any(up)) {
                const float to = up ? mx : m;
                const float from = m * c, ref = to * c; // as the exponents below take them
                const bool large = __builtin_fabsf(from) >= kLargeScore || __builtin_fabsf(ref) >= kLargeScore;
                const float by = up ? exp2_of(large ? (m - to) * c : from - ref) : 1.0f;
                m = to;
                total *= by;
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        o[db][r] *= by;
            }
            float ref = m == -__builtin_inff() ? 0.0f : m * c;
            const bool large = __builtin_fabsf(ref) >= kLargeScore;
            if (__any(large)) { // a product's rounding would move its exponent: subtract first
#pragma unroll
                for (int i = 0; i < 16 * RB; ++i)
                    x[i / 16][i % 16] -= large ? m : 0.0f;
                ref = large ? 0.0f : ref;
            }
            float part[4] = {};
            // bfloat16: the one rounding on the way to the second product, whose operands the matrix instructions take so.  One
            // sequence of 2048, heads of 128: out is off by 2.0e-3 of itself, its own rounding alone by 1.6e-3.  A second product
            // with what the rounding leaves would bring 1.6e-3, and takes 317 us where this takes 248 (four of 2048, 40 heads over
            // 8), 1828 for 1345 (one of 16384, 16 over 4).  float32 heads have none.
            Frag<T> p[2 * RB];
#pragma unroll
            for (int s = 0; s < 2 * RB; ++s) {
                float w[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    w[j] = exp2_of(__builtin_fmaf(x[s / 2][8 * (s % 2) + j], c, -ref));
                    part[j % 4] += w[j];
                }
                p[s].set(w);
            }
            total += (part[0] + part[1]) + (part[2] + part[3]);
            uint64_t found = 0;
#pragma unroll
            for (int s = 0; s < 2 * RB; ++s)
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    Frag<T> a;
                    read.template columns<TILE>(16 * s, db, a);
                    if (CAREFUL)
                        found |= tile_rows(scrub(a), 16 * s);
                    mma(a, p[s], o[db]);
                }
            if constexpr (sizeof(T) == 2 && !CAREFUL)
                spread<1, 2 * RB * DB, 2, 2>();
            if (CAREFUL && __any(found != 0)) {
                found = or_wave(found);
                for (int j = 0; j < BN; ++j)
                    poison |= (found >> j & 1) && (uint32_t)(k0 + j - start) < seen;
            }
        }
    };
    walk(std::false_type{});
    // NaN: some value that is not finite, perhaps one that no row of the wave may see
    bool bad = false;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            bad |= o[db][r] != o[db][r];
    if (__syncthreads_or(bad)) {
        m = -__builtin_inff(), total = 0.0f;
#pragma unroll
        for (int db = 0; db < DB; ++db)
            o[db] = f32x16{};
        walk(std::true_type{});
    }

    total += other_half(total);
    if (!span.on)
        return;
    // a row whose scores are all -inf: zeros
    const float inv = poison ? __builtin_nanf("") : total > 0.0f ? 1.0f / total : total == 0.0f ? 0.0f : total;
    store_row(static_cast<T *>(oh.p) + (int64_t)row * oh.token_stride + head * oh.head_stride, at.dim, o, inv);
    if (lse && h == 0) // a small reference was taken as the rounded product
        lse[(int64_t)head * at.seq.tokens + row] =
            total > 0.0f ? (__builtin_fabsf(m * c) < kLargeScore ? (m * c + __log2f(total)) * kLn2 : m * at.scale + __logf(total))
            : total == 0.0f ? -__builtin_inff() : total;
}

template <class T, int DB, int WAVES, int BN, int STAGES, int OCC>
int run(int dtype, const Attention &at, const Heads &q, const Heads &k, const Heads &v, const Heads &out, float *lse, hipStream_t s)
{
    const int tiles = (at.seq.tokens + 32 * WAVES - 1) / (32 * WAVES);
    const int64_t items = (int64_t)tiles * q.heads;
    auto kernel = direct(k, dtype, at.dim) && direct(v, dtype, at.dim) ? k_attention<T, DB, WAVES, BN, STAGES, OCC, true>
                                                                       : k_attention<T, DB, WAVES, BN, STAGES, OCC, false>;
    return launch<WAVES>(kernel, shared_blocks(items), kUncapped, s, at, q, k, v, out, lse, tiles, items);
}

} // namespace

int launch_attention(int dtype, const Attention &at, const Heads &q, const Heads &k, const Heads &v, const Heads &out,
                     float *lse, hipStream_t s)
{
    const int db = (at.dim + 31) / 32;
    if (dtype == SDP4_BF16) {
        if (db <= 2)
            return run<bf16_t, 2, 4, 64, 2, 2>(dtype, at, q, k, v, out, lse, s);
        if (db == 3)
            return run<bf16_t, 3, 4, 64, 2, 2>(dtype, at, q, k, v, out, lse, s);
        if (db == 4)
            return run<bf16_t, 4, 4, 64, 2, 2>(dtype, at, q, k, v, out, lse, s);
        return run<bf16_t, 8, 4, 32, 2, 1>(dtype, at, q, k, v, out, lse, s);
    }
    if (db <= 2)
        return run<float, 2, 4, 32, 2, 2>(dtype, at, q, k, v, out, lse, s);
    if (db == 3)
        return run<float, 3, 4, 32, 2, 2>(dtype, at, q, k, v, out, lse, s);
    if (db == 4)
        return run<float, 4, 4, 32, 2, 2>(dtype, at, q, k, v, out, lse, s);
    return run<float, 8, 4, 32, 2, 1>(dtype, at, q, k, v, out, lse, s);
}

} // namespace sdp4
