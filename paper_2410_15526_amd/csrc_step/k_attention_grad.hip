// k_attention_grad.hip -- gradients of causal attention over packed sequences.
//
// With p_ij = exp(s_ij - lse_i), dP_ij = dout_i . v_j, D_i = dout_i . out_i and
// dS_ij = p_ij (dP_ij - D_i):
//      dq_i = scale sum_j dS_ij k_j,  dk_j = scale sum_i dS_ij q_i,
//      dv_j = sum_i p_ij dout_i,
// the latter two summed over the query heads of a group.  Two launches: one
// walks the keys for each block of queries and leaves what a row's scores and
// dP need taken off for the other, which
// walks the queries of all heads of the group for each block of keys.  The
// scores are computed twice (seven products in place of five), which costs
// less than adding dq up over the blocks of keys: each result is summed in
// registers, in one order, and written once.  Where a batch makes few blocks,
// their walks are split, and a third launch sums the parts in their order.
#include "attention.hpp"

namespace sdp4 {

namespace {

// p of scores x, from exponents fma(x, c, add).  `hard`: some place is masked, where x and y may be anything, or some score is
// large, whose roundings may leave more than float32's exponents hold: p is at most 1.  Place r is row `first` + 8 (r / 4) +
// r % 4 of the other side, and `seen` rows from 0 on are seen.
SDP4_DEV void probabilities(f32x16 &x, f32x16 &y, float c, float add, bool hard, uint32_t first, uint32_t seen)
{
#pragma unroll
    for (int r = 0; r < 16; ++r)
        x[r] = __builtin_fmaf(x[r], c, add);
    if (hard) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const bool on = first + (8 * (r >> 2) + (r & 3)) < seen;
            x[r] = on ? x[r] > 0.0f ? 0.0f : x[r] : -__builtin_inff();
            y[r] = on ? y[r] : 0.0f;
        }
    }
#pragma unroll
    for (int r = 0; r < 16; ++r)
        x[r] = exp2_of(x[r]);
}

// p or dS as operands of the second products: with bfloat16 heads their one rounding, as in the forward pass (gradients are off by
// 2.4e-3 of themselves, with only their own rounding by 1.7e-3).
template <class T>
SDP4_DEV void operands(const f32x16 &x, Frag<T> (&f)[2])
{
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        float w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            w[j] = x[8 * s + j];
        f[s].set(w);
    }
}

// out += tile's columns times p, for 32 rows of the tile from r0 on.  CAREFUL: what is infinite or NaN stays out and is noted.
template <int AT, bool CAREFUL, class T, int DB>
SDP4_DEV void add_product(const Reader<T, DB> &read, int r0, const Frag<T> (&p)[2], f32x16 (&out)[DB], uint64_t &found)
{
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            Frag<T> a;
            read.template columns<AT>(r0 + 16 * s, db, a);
            if (CAREFUL)
                found |= tile_rows(scrub(a), r0 + 16 * s);
            mma(a, p[s], out[db]);
        }
}

// The walk of a block in `count` pieces, each by a block of its own, whose results go to memory and are summed by k_join_pieces.
struct Pieces {
    static constexpr int kMost = 8;
    int count;
    float *parts; // [count][tokens][heads][pitch]
    SDP4_DEV int64_t from(int piece, int64_t steps) const { return steps * piece / count; }
    static SDP4_DEV int pitch(int dim) { return (dim + 3) / 4 * 4; }
    SDP4_DEV float *row(int piece, const Attention &at, int64_t row, int head, int heads) const
    {
        return parts + (((int64_t)piece * at.seq.tokens + row) * heads + head) * pitch(at.dim);
    }
};

template <int DB>
SDP4_DEV bool has_nan(const f32x16 (&x)[DB])
{
    bool bad = false;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            bad |= x[db][r] != x[db][r];
    return bad;
}
template <int DB>
SDP4_DEV void clear(f32x16 (&x)[DB])
{
#pragma unroll
    for (int db = 0; db < DB; ++db)
        x[db] = f32x16{};
}

// Sums over the groups of waves, in their order, in group 0.
template <int WAVES, int GROUPS, int DB>
SDP4_DEV void join_groups(char *lds, int wave, int mine, f32x16 (&x)[DB])
{
#pragma unroll
    for (int g = 1; g < GROUPS; ++g) {
        f32x16 *part = reinterpret_cast<f32x16 *>(lds) + wave * DB * 64 + lane_id();
        __syncthreads();
        if (mine == g) {
#pragma unroll
            for (int db = 0; db < DB; ++db)
                part[db * 64] = x[db];
        }
        __syncthreads();
        if (mine == 0) {
#pragma unroll
            for (int db = 0; db < DB; ++db)
                x[db] += part[db * 64];
        }
    }
}

// Columns are queries, as in the forward pass, and the tiles are its tiles.  Four sequences of 2048, 40 heads of 128 over 8,
// bfloat16: 320 to 370 us by inputs in the last-level cache (three products: 700 to 800 TFLOP/s), 358 for 320 with eight waves a block.
template <class T, int DB, int WAVES, int BN, int STAGES, int OCC, bool DIRECT>
__global__ __launch_bounds__(64 * WAVES, OCC) void k_attention_dq(Attention at, Heads doh, Heads qh, Heads kh, Heads vh, Heads oh,
                                                                const float *lse, Heads dqh, float *delta, int tiles,
                                                                int64_t items, Pieces pieces)
{
    using H = HeadTile<T, DB>;
    constexpr int BM = 32 * WAVES, THREADS = 64 * WAVES, RB = BN / 32;
    constexpr int S = DIRECT ? STAGES : 2;
    constexpr int TILE = BN * H::ROW;
    __shared__ __align__(128) char tiles_lds[S][2][TILE]; // keys, values
    __shared__ int64_t samples[kSeqSamples];
    __shared__ int edges[WAVES][2];

    const int64_t unit = shared_item(work_block(), items * pieces.count);
    if (unit >= items * pieces.count)
        return;
    const int64_t item = unit / pieces.count;
    const int piece = (int)(unit - item * pieces.count);
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
    const int w_first = min_wave(start), w_last = max_wave(span.on ? row : -1), w_full = max_wave(start);
    if (lane == 0)
        edges[wave][0] = w_first, edges[wave][1] = w_last;
    __syncthreads();
    int first = INT_MAX, last = -1;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        first = edges[w][0] < first ? edges[w][0] : first;
        last = edges[w][1] > last ? edges[w][1] : last;
    }
    if (last < 0)
        return;
    first = (int)uniform((uint32_t)first), last = (int)uniform((uint32_t)last);
    const int steps = (last - first) / BN + 1, till = first + (int)pieces.from(piece + 1, steps) * BN - 1;
    first += (int)pieces.from(piece, steps) * BN;
    last = till < last ? till : last; // before first: nothing in this piece

    const int64_t at_row = row < at.seq.tokens ? row : at.seq.tokens - 1;
    const T *qrow = static_cast<const T *>(qh.p) + at_row * qh.token_stride + head * qh.head_stride;
    const T *drow = static_cast<const T *>(doh.p) + at_row * doh.token_stride + head * doh.head_stride;
    const T *orow = static_cast<const T *>(oh.p) + at_row * oh.token_stride + head * oh.head_stride;
    Frag<T> q[H::STEPS], g[H::STEPS];
    float along = 0.0f;
#pragma unroll
    for (int s = 0; s < H::STEPS; ++s) {
        Frag<T> o;
        load_frag(qrow, 16 * s + 8 * h, at.dim, q[s]);
        load_frag(drow, 16 * s + 8 * h, at.dim, g[s]);
        load_frag(orow, 16 * s + 8 * h, at.dim, o);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            along = __builtin_fmaf(g[s].get(j), o.get(j), along);
    }
    along += xor_lane<32>(along);
    const int64_t at_stat = (int64_t)head * at.seq.tokens + at_row;
    // What is added to scores and dP, for the other launch too: -lse / scale (-inf for a row without a finite score, so that its
    // p are 0) and -D.
    const float c = at.scale * kLog2e, row_lse = lse[at_stat];
    const float shift = row_lse == -__builtin_inff() ? row_lse : -row_lse * (1.0f / at.scale);
    if (h == 0 && span.on && piece == 0)
        delta[at_stat] = shift, delta[(int64_t)qh.heads * at.seq.tokens + at_stat] = -along;
    const bool large = __any(span.on && __builtin_fabsf(shift) * c >= kLargeScore);
    const T *kp = static_cast<const T *>(kh.p) + kv * kh.head_stride, *vp = static_cast<const T *>(vh.p) + kv * vh.head_stride;

    bool poison = false;
    f32x16 dq[DB] = {};
    TileLoad<T, DB, BN, WAVES, DIRECT> kl, vl;
    kl.begin(kp, kh.token_stride, at.dim);
    vl.begin(vp, vh.token_stride, at.dim);
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
            const bool hard = large || !(k0 >= w_full && k0 + BN - 1 <= q0);
            uint64_t found = 0;
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                f32x16 x = {}, y = {};
#pragma unroll
                for (int s = 0; s < H::STEPS; ++s) {
                    Frag<T> a, b;
                    read.template rows<0>(32 * rb, s, a);
                    read.template rows<TILE>(32 * rb, s, b);
                    mma(a, q[s], x);
                    mma(b, g[s], y);
                }
                probabilities(x, y, c, shift * c, hard, k0 + 32 * rb + 4 * h - start, seen);
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    x[r] *= y[r] - along;
                Frag<T> p[2];
                operands(x, p);
                add_product<0, CAREFUL>(read, 32 * rb, p, dq, found);
            }
            if (CAREFUL && __any(found != 0)) {
                found = or_wave(found);
                for (int j = 0; j < BN; ++j)
                    poison |= (found >> j & 1) && (uint32_t)(k0 + j - start) < seen;
            }
        }
    };
    walk(std::false_type{});
    if (__syncthreads_or(has_nan(dq))) { // some value is not finite, perhaps one that no row of the wave may see
        clear(dq);
        walk(std::true_type{});
    }
    if (!span.on)
        return;
    const float by = poison ? __builtin_nanf("") : at.scale;
    if (pieces.count > 1)
        store_row(pieces.row(piece, at, at_row, head, qh.heads), at.dim, dq, by);
    else
        store_row(static_cast<T *>(dqh.p) + at_row * dqh.token_stride + head * dqh.head_stride, at.dim, dq, by);
}

// Columns are keys here, and a block's waves split them (32 to a wave) and the queries (GROUPS groups of waves take a tile's rows
// in turn, their sums joined at the end in the order of the groups): two waves on a SIMD, whose results and operands have to fit
// 256 registers each, so keys and values stay in LDS.  HELD: in registers, for one wave on a SIMD.  PARTS: 1 dv, 2 dk, 3 both.
//
// The same heads: 404 to 488 us by inputs in the last-level cache (four products: 700 to 850 TFLOP/s), tiles with the longest walks
// first; the whole backward pass 665 to 747.  Both launches together took 960 us when this form came, 1213 with HELD and one wave
// on a SIMD, 1505 with launches of their own for dk and dv.  What bounds it: the fixed operands come out of LDS for each tile
// again, and the two waves wait for p and dS.
// float32 heads are HELD, as their operands are twice as large, with 64 keys a block, as a batch may have few: 1,871 rows, 12 heads
// of 80 over 4, both launches 565 us when this form came, 913 with one group of four waves for 128 keys; 242 now, in pieces.
// Four of 2048, 40 heads of 128 over 8 in float32, the whole pass: 5407 us.
template <class T, int DB, int WAVES, int GROUPS, int STAGES, int OCC, bool DIRECT, int PARTS, bool HELD>
__global__ __launch_bounds__(64 * WAVES * GROUPS, OCC) void k_attention_dkv(Attention at, Heads doh, Heads qh, Heads kh, Heads vh,
                                                                          Heads dkh, Heads dvh, const float *delta, int tiles,
                                                                          int64_t items, Pieces pieces)
{
    using H = HeadTile<T, DB>;
    constexpr int BK = 32 * WAVES, BQ = 32 * GROUPS, ALL = WAVES * GROUPS, S = DIRECT ? STAGES : 2;
    constexpr bool WITH_V = PARTS & 1, WITH_K = PARTS & 2;
    constexpr int TILE = BQ * H::ROW, KEYS = BK * H::ROW;
    struct Lds {
        char tiles[S][2][TILE]; // queries, gradients
        char keys[HELD ? 16 : KEYS], values[WITH_K && !HELD ? KEYS : 16];
    };
    constexpr int JOIN = GROUPS > 1 ? WAVES * 64 * 64 * DB : 0; // one group's dk or dv
    __shared__ __align__(128) char lds[sizeof(Lds) > JOIN ? sizeof(Lds) : JOIN];
    Lds &mem = *reinterpret_cast<Lds *>(lds);
    __shared__ __align__(16) float stats[S][ALL][64]; // what delta holds for 32 queries; each wave's own
    __shared__ int64_t samples[kSeqSamples];
    __shared__ int edges[ALL][2], work[kMostOrdered], found_tile;

    const int64_t unit = shared_item(work_block(), items * pieces.count);
    if (unit >= items * pieces.count)
        return;
    const int per_head = tiles * pieces.count, kv = (int)(unit / per_head);
    const bool sorted = by_work(at.seq, tiles);
    const int place = sorted ? dealt_place(unit, per_head, items * pieces.count) : (int)(unit - (int64_t)kv * per_head);
    const int piece = place % pieces.count;
    fill_samples<64 * ALL>(at.seq, samples);
    int tile = place / pieces.count;
    if (sorted)
        tile = ordered_tile<64 * ALL, BK>(at.seq, samples, work, found_tile, tiles, tile);

    const int all = uniform(threadIdx.x / kWave), wave = all % WAVES, mine = all / WAVES; // keys, and rows of a tile
    const int lane = lane_id(), h = lane >> 5;
    const int key = tile * BK + 32 * wave + (lane & 31);
    const Span span = span_of(at.seq, samples, key);
    const int end = span.on ? span.end : -1;
    const int w_first = min_wave(span.on ? key : INT_MAX), w_end = max_wave(end); // queries that see the wave's keys
    const int w_all = max_wave(span.on ? key : INT_MAX), w_until = min_wave(end); // those that see all of them
    if (lane == 0)
        edges[all][0] = w_first, edges[all][1] = w_end;
    __syncthreads();
    int first = INT_MAX, limit = -1;
#pragma unroll
    for (int w = 0; w < ALL; ++w) {
        first = edges[w][0] < first ? edges[w][0] : first;
        limit = edges[w][1] > limit ? edges[w][1] : limit;
    }
    if (limit < 0)
        return;
    first = (int)uniform((uint32_t)first), limit = (int)uniform((uint32_t)limit);

    const int64_t at_key = key < at.seq.tokens ? key : at.seq.tokens - 1;
    const T *krow = static_cast<const T *>(kh.p) + at_key * kh.token_stride + kv * kh.head_stride;
    const T *vrow = static_cast<const T *>(vh.p) + at_key * vh.token_stride + kv * vh.head_stride;
    Frag<T> k[HELD ? H::STEPS : 1], v[HELD && WITH_K ? H::STEPS : 1];
    if constexpr (HELD) {
#pragma unroll
        for (int s = 0; s < H::STEPS; ++s) {
            load_frag(krow, 16 * s + 8 * h, at.dim, k[s]);
            if constexpr (WITH_K)
                load_frag(vrow, 16 * s + 8 * h, at.dim, v[s]);
        }
    } else { // into the tiles, a part by each of the groups
#pragma unroll
        for (int s = 0; s < H::STEPS; ++s)
            if (s % GROUPS == mine) {
                Frag<T> f;
                load_frag(krow, 16 * s + 8 * h, at.dim, f);
                put_row<T, DB>(mem.keys + 32 * wave * H::ROW, s, f);
                if constexpr (WITH_K) {
                    load_frag(vrow, 16 * s + 8 * h, at.dim, f);
                    put_row<T, DB>(mem.values + 32 * wave * H::ROW, s, f);
                }
            }
    }
    const float c = at.scale * kLog2e;
    const int a_head = (limit - first + BQ - 1) / BQ; // steps over one query head
    const int64_t steps = (int64_t)a_head * at.group, begin = pieces.from(piece, steps), count = pieces.from(piece + 1, steps);
    const uint32_t seen = span.on ? end - key : 0; // queries that see the key, from its own on

    bool poison_k = false, poison_v = false;
    f32x16 dk[WITH_K ? DB : 1] = {}, dv[WITH_V ? DB : 1] = {};
    TileLoad<T, DB, BQ, ALL, DIRECT> ql, gl;
    ql.begin(nullptr, qh.token_stride, at.dim);
    gl.begin(nullptr, doh.token_stride, at.dim);
    auto walk = [&](auto careful) {
        constexpr bool CAREFUL = decltype(careful)::value;
        constexpr int PER = DIRECT ? ql.COUNT + gl.COUNT + 1 : 0;
        Reader<T, DB> read(lds_address(mem.tiles[S - 1]) + 32 * mine * H::ROW); // the tile before the first
        RowReader<T, DB> fixed(lds_address(mem.keys) + 32 * wave * H::ROW); // the values lie behind
        int nq = first + (int)(begin % a_head) * BQ, nhead = kv * at.group + (int)(begin / a_head); // of the next load
        auto fetch = [&](int to) {
            ql.move(static_cast<const T *>(qh.p) + nhead * qh.head_stride);
            gl.move(static_cast<const T *>(doh.p) + nhead * doh.head_stride);
            ql.load(mem.tiles[to][0], nq, limit);
            gl.load(mem.tiles[to][1], nq, limit);
            const int r = nq + 32 * mine + (lane & 31);
            load_word(stats[to][all], delta + ((int64_t)(lane < 32 ? nhead : nhead + qh.heads) * at.seq.tokens +
                                               (r < limit ? r : limit - 1)));
            nq += BQ;
            if (nq >= limit)
                nq = first, ++nhead;
        };
        int stage = 0, ahead = S - 1, q0 = nq + 32 * mine; // the wave's first row
#pragma unroll
        for (int i = 0; i < S - 1; ++i)
            if (begin + i < count)
                fetch(i);
        for (int64_t i = begin; i < count; ++i, q0 = q0 - 32 * mine + BQ < limit ? q0 + BQ : first + 32 * mine) {
            if (i + S - 2 < count)
                wait_loads<(S - 2) * PER>(); // of the tiles after this one
            else
                wait_loads<0>();
            ql.store(mem.tiles[stage][0], q0, limit);
            gl.store(mem.tiles[stage][1], q0, limit);
            __syncthreads();
            if (i + S - 1 < count)
                fetch(ahead);
            read.move(stage ? 2 * TILE : -(S - 1) * 2 * TILE);
            const float *stat = stats[stage][all];
            stage = stage + 1 == S ? 0 : stage + 1, ahead = ahead + 1 == S ? 0 : ahead + 1;
            if (q0 >= w_end || q0 + 32 <= w_first)
                continue;
            const bool hard = !(q0 >= w_all && q0 + 32 <= w_until) || __any(__builtin_fabsf(stat[lane & 31]) * c >= kLargeScore);
            f32x16 x, y = {}; // from -lse / scale and -D on
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                x[r] = stat[8 * (r >> 2) + 4 * h + (r & 3)];
                if constexpr (WITH_K)
                    y[r] = stat[32 + 8 * (r >> 2) + 4 * h + (r & 3)];
            }
#pragma unroll
            for (int s = 0; s < H::STEPS; ++s) {
                Frag<T> a, b;
                read.template rows<0>(0, s, a);
                if constexpr (HELD) {
                    mma(a, k[s], x);
                } else {
                    fixed.template rows<0>(s, b);
                    mma(a, b, x);
                }
                if constexpr (WITH_K) {
                    read.template rows<TILE>(0, s, a);
                    if constexpr (HELD) {
                        mma(a, v[s], y);
                    } else {
                        fixed.template rows<KEYS>(s, b);
                        mma(a, b, y);
                    }
                }
            }
            probabilities(x, y, c, 0.0f, hard, q0 + 4 * h - key, seen);
            uint64_t found_q = 0, found_g = 0;
            Frag<T> p[2];
            if constexpr (WITH_V) {
                operands(x, p);
                add_product<TILE, CAREFUL>(read, 0, p, dv, found_g);
            }
            if constexpr (WITH_K) {
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    x[r] *= y[r];
                operands(x, p);
                add_product<0, CAREFUL>(read, 0, p, dk, found_q);
            }
            if (CAREFUL && __any((found_q | found_g) != 0)) {
                found_q = or_wave(found_q), found_g = or_wave(found_g);
                for (int j = 0; j < 32; ++j) {
                    const bool sees = (uint32_t)(q0 + j - key) < seen;
                    poison_k |= (found_q >> j & 1) && sees;
                    poison_v |= (found_g >> j & 1) && sees;
                }
            }
        }
    };
    walk(std::false_type{});
    if (__syncthreads_or(has_nan(dk) || has_nan(dv))) { // some value is not finite, perhaps one that is masked
        clear(dk);
        clear(dv);
        walk(std::true_type{});
    }
    if (poison_k) // the row's first element tells the others, and is joined with the other groups'
        dk[0][0] = __builtin_nanf("");
    if (poison_v)
        dv[0][0] = __builtin_nanf("");
    if constexpr (WITH_K)
        join_groups<WAVES, GROUPS>(lds, wave, mine, dk);
    if constexpr (WITH_V)
        join_groups<WAVES, GROUPS>(lds, wave, mine, dv);
    if (!span.on || mine)
        return;
    if constexpr (WITH_K) {
        const float by = dk[0][0] == dk[0][0] ? at.scale : dk[0][0];
        if (pieces.count > 1)
            store_row(pieces.row(piece, at, at_key, kv, dkh.heads), at.dim, dk, by);
        else
            store_row(static_cast<T *>(dkh.p) + at_key * dkh.token_stride + kv * dkh.head_stride, at.dim, dk, by);
    }
    if constexpr (WITH_V) {
        const float by = dv[0][0] == dv[0][0] ? 1.0f : dv[0][0];
        if (pieces.count > 1) // behind those of dk
            store_row(pieces.row(pieces.count + piece, at, at_key, kv, dvh.heads), at.dim, dv, by);
        else
            store_row(static_cast<T *>(dvh.p) + at_key * dvh.token_stride + kv * dvh.head_stride, at.dim, dv, by);
    }
}

// The sums over the pieces, in their order: a thread for four elements of a head.
struct Joined {
    Heads to;
    const float *from; // [count][tokens][heads][pitch]
    int count;
};
struct Joins {
    Joined a[3];
    int slots; // heads of all of them
};
template <class T>
__global__ __launch_bounds__(256) void k_join_pieces(Attention at, Joins joins, int64_t threads)
{
    __shared__ int64_t samples[kSeqSamples];
    fill_samples<256>(at.seq, samples);
    const int64_t id = work_block() * 256 + threadIdx.x;
    if (id >= threads)
        return;
    const int places = Pieces::pitch(at.dim) / 4;
    const int64_t at_head = id / places, row = at_head / joins.slots;
    const int d = 4 * (int)(id - at_head * places);
    int head = (int)(at_head - row * joins.slots);
    Joined j = joins.a[0];
#pragma unroll
    for (int i = 1; i < 3; ++i)
        if (head >= j.to.heads)
            head -= j.to.heads, j = joins.a[i];
    if (!span_of(at.seq, samples, (int)row).on)
        return;
    const float *from = j.from + (row * j.to.heads + head) * Pieces::pitch(at.dim) + d;
    const int64_t step = (int64_t)at.seq.tokens * j.to.heads * Pieces::pitch(at.dim);
    float4 part[Pieces::kMost];
#pragma unroll
    for (int p = 0; p < Pieces::kMost; ++p)
        part[p] = p < j.count ? *reinterpret_cast<const float4 *>(from + p * step) : float4{};
    float4 sum = part[0];
#pragma unroll
    for (int p = 1; p < Pieces::kMost; ++p)
        if (p < j.count)
            sum.x += part[p].x, sum.y += part[p].y, sum.z += part[p].z, sum.w += part[p].w;
    const float w[4] = {sum.x, sum.y, sum.z, sum.w};
    T *to = static_cast<T *>(j.to.p) + row * j.to.token_stride + head * j.to.head_stride + d;
    store_elems(to, at.dim - d, w);
}

// As many pieces as make kPieceBlocks blocks, of four steps at least: where a batch has fewer blocks than the chip has room for, its
// longest walk would be the time.  1,871 rows of nine sequences, 12 float32 heads of 80 over 4 (dq and dkv, with the join's 12 us):
// 184 and 360 us whole, 111 and 159 for 512 blocks, 129 and 140 (join 17) for 1024, before walks were dealt to the XCDs.  The whole
// pass for 256 / 512 / 1024 blocks: that batch 380 / 244 / 276; bfloat16, one sequence of 4096, 8 heads of 128 over 2, 262 / 222 /
// 231; 3000 rows, 12 of 96 over 4, 221 / 184 / 181; two of 2048, 12 of 64, 124 / 124 / 139; four of 512, 8 of 64 over 2, 47 / 49 /
// 56; float32, one of 2048, 12 of 64, 423 / 408 / 346.  Four sequences of 2048, 40 heads of 128 over 8 in bfloat16 make 512 blocks
// by keys, and two pieces of each would add 38 us of partial sums.
constexpr int64_t kPieceBlocks = 512, kPieceRows = 128 * kPieceBlocks;
int pieces_of(int64_t blocks, int64_t steps)
{
    int64_t n = kPieceBlocks / blocks;
    n = n < steps / 4 ? n : steps / 4;
    return n < 2 ? 1 : n < Pieces::kMost ? (int)n : Pieces::kMost;
}
int64_t stat_floats(int64_t tokens, int q_heads) { return (2 * tokens * q_heads + 3) / 4 * 4; } // -lse / scale and -D of every row
// Of pieces for any number of tokens up to this one: a block has 128 rows at most.
int64_t piece_floats(int64_t tokens, int heads, int dim)
{
    const int64_t rows = Pieces::kMost * tokens * heads;
    return (rows < kPieceRows ? rows : kPieceRows) * ((dim + 3) / 4 * 4);
}

struct Grad {
    const Attention &at;
    const Heads &dout, &q, &k, &v, &out;
    const float *lse;
    const Heads &dq, &dk, &dv;
    float *delta, *parts_q, *parts_k;
    hipStream_t s;

    int dtype;
    int pieces_q = 1, pieces_k = 1;

    template <class T, int DB, int WAVES, int BN, int STAGES, int OCC>
    int queries()
    {
        const int tiles = (at.seq.tokens + 32 * WAVES - 1) / (32 * WAVES);
        const int64_t items = (int64_t)tiles * q.heads;
        pieces_q = pieces_of(items, (at.seq.tokens + BN - 1) / BN);
        auto kernel = direct(k, dtype, at.dim) && direct(v, dtype, at.dim) ? k_attention_dq<T, DB, WAVES, BN, STAGES, OCC, true>
                                                                           : k_attention_dq<T, DB, WAVES, BN, STAGES, OCC, false>;
        return launch<WAVES>(kernel, shared_blocks(items * pieces_q), kUncapped, s, at, dout, q, k, v, out, lse, dq, delta, tiles,
                             items, Pieces{pieces_q, parts_q});
    }
    template <class T, int DB, int WAVES, int GROUPS, int STAGES, int OCC, int PARTS = 3, bool HELD = false>
    int keys()
    {
        const int tiles = (at.seq.tokens + 32 * WAVES - 1) / (32 * WAVES);
        const int64_t items = (int64_t)tiles * k.heads;
        pieces_k = pieces_of(items, (int64_t)((at.seq.tokens + 32 * GROUPS - 1) / (32 * GROUPS)) * at.group);
        auto kernel = direct(q, dtype, at.dim) && direct(dout, dtype, at.dim)
                          ? k_attention_dkv<T, DB, WAVES, GROUPS, STAGES, OCC, true, PARTS, HELD>
                          : k_attention_dkv<T, DB, WAVES, GROUPS, STAGES, OCC, false, PARTS, HELD>;
        return launch<WAVES * GROUPS>(kernel, shared_blocks(items * pieces_k), kUncapped, s, at, dout, q, k, v, dk, dv, delta, tiles,
                                      items, Pieces{pieces_k, parts_k});
    }
    template <class T>
    int join() const
    {
        Joins joins{};
        int n = 0;
        if (pieces_q > 1)
            joins.a[n++] = {dq, parts_q, pieces_q};
        const int64_t pitch = (at.dim + 3) / 4 * 4;
        if (pieces_k > 1) {
            joins.a[n++] = {dk, parts_k, pieces_k};
            joins.a[n++] = {dv, parts_k + pieces_k * (int64_t)at.seq.tokens * k.heads * pitch, pieces_k};
        }
        for (const Joined &j : joins.a)
            joins.slots += j.to.heads;
        if (!joins.slots)
            return 0;
        const int64_t threads = (int64_t)at.seq.tokens * joins.slots * (pitch / 4);
        return launch<4>(k_join_pieces<T>, (threads + 255) / 256, kUncapped, s, at, joins, threads);
    }
    // The launches by heads of up to 128 elements, and of more, where both results and both operands would not fit the registers.
    template <class T>
    int all();
};

template <>
int Grad::all<bf16_t>()
{
    const int db = (at.dim + 31) / 32;
    int rc;
    if (db <= 2)
        return (rc = queries<bf16_t, 2, 4, 64, 2, 2>()) ? rc : keys<bf16_t, 2, 4, 2, 2, 2>();
    if (db == 3)
        return (rc = queries<bf16_t, 3, 4, 64, 2, 2>()) ? rc : keys<bf16_t, 3, 4, 2, 2, 2>();
    if (db == 4)
        return (rc = queries<bf16_t, 4, 4, 64, 2, 2>()) ? rc : keys<bf16_t, 4, 4, 2, 2, 2>();
    if ((rc = queries<bf16_t, 8, 4, 32, 2, 1>()) || (rc = keys<bf16_t, 8, 4, 1, 2, 1, 1, true>()))
        return rc;
    return keys<bf16_t, 8, 4, 1, 2, 1, 2, true>();
}
template <>
int Grad::all<float>()
{
    const int db = (at.dim + 31) / 32;
    int rc;
    if (db <= 2)
        return (rc = queries<float, 2, 4, 32, 2, 1>()) ? rc : keys<float, 2, 2, 2, 2, 1, 3, true>();
    if (db == 3)
        return (rc = queries<float, 3, 4, 32, 2, 1>()) ? rc : keys<float, 3, 2, 2, 2, 1, 3, true>();
    if (db == 4)
        return (rc = queries<float, 4, 4, 32, 2, 1>()) ? rc : keys<float, 4, 2, 2, 2, 1, 3, true>();
    if ((rc = queries<float, 8, 4, 32, 2, 1>()) || (rc = keys<float, 8, 4, 1, 2, 1, 1, true>()))
        return rc;
    return keys<float, 8, 4, 1, 2, 1, 2, true>();
}

} // namespace

int64_t attention_grad_workspace(int64_t tokens, int q_heads, int k_heads, int dim)
{
    return (stat_floats(tokens, q_heads) + piece_floats(tokens, q_heads, dim) + 2 * piece_floats(tokens, k_heads, dim)) *
           (int64_t)sizeof(float);
}

int launch_attention_grad(int dtype, const Attention &at, const Heads &dout, const Heads &q, const Heads &k, const Heads &v,
                          const Heads &out, const float *lse, const Heads &dq, const Heads &dk, const Heads &dv,
                          float *workspace, hipStream_t s)
{
    float *parts_q = workspace + stat_floats(at.seq.tokens, q.heads);
    float *parts_k = parts_q + piece_floats(at.seq.tokens, q.heads, at.dim);
    Grad g{at, dout, q, k, v, out, lse, dq, dk, dv, workspace, parts_q, parts_k, s, dtype};
    return with_type(dtype, [&](auto tag) {
        using T = decltype(tag);
        const int rc = g.all<T>();
        return rc ? rc : g.join<T>();
    });
}

} // namespace sdp4
