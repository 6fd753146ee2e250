// k_attention_grad.hip -- gradients of causal attention over packed sequences.
//
// With p_ij = exp(s_ij - lse_i), dP_ij = dout_i . v_j, D_i = dout_i . out_i and
// dS_ij = p_ij (dP_ij - D_i):
//      dq_i = scale sum_j dS_ij k_j,  dk_j = scale sum_i dS_ij q_i,
//      dv_j = sum_i p_ij dout_i,
// the latter two summed over the query heads of a group.  Two launches: one
// walks the keys for each block of queries and leaves D for the other, which
// walks the queries of all heads of the group for each block of keys.  The
// scores are computed twice (seven products in place of five), which costs
// less than adding dq up over the blocks of keys: each result is summed in
// registers, in one order, and written once.
#include "attention.hpp"

namespace sdp4 {

namespace {

// lse in octaves; +inf for a row without a finite score, so that its p are 0
SDP4_DEV float octaves(float lse) { return lse == -__builtin_inff() ? __builtin_inff() : lse * kLog2e; }

// p of scores x.  Of large scores the roundings of both sides may leave more than float32's exponents hold: p is at most 1
// there (`large`: for some row of the wave).
template <int N>
SDP4_DEV void probabilities(f32x16 &x, float c, const float (&l)[N], bool large)
{
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        float t = __builtin_fmaf(x[r], c, -l[r % N]);
        if (large)
            t = t > 0.0f && __builtin_fabsf(l[r % N]) >= kLargeScore ? 0.0f : t;
        x[r] = exp2_of(t);
    }
}

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
template <bool CAREFUL, class T, int DB>
SDP4_DEV void add_product(const Reader<T, DB> &read, const char *tile, int r0, const Frag<T> (&p)[2], f32x16 (&out)[DB], uint64_t &found)
{
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            Frag<T> a;
            read.columns(tile, r0 + 16 * s, db, a);
            if (CAREFUL)
                found |= tile_rows(scrub(a), r0 + 16 * s);
            mma(a, p[s], out[db]);
        }
}

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
            store_elems(row + d, (int64_t)dim - d, w);
        }
}

template <class T, int DB, int WAVES, int BN, int OCC, bool DIRECT>
__global__ __launch_bounds__(64 * WAVES, OCC) void k_attention_dq(Attention at, Heads doh, Heads qh, Heads kh, Heads vh, Heads oh,
                                                                const float *lse, Heads dqh, float *delta, int tiles,
                                                                int64_t items)
{
    using H = HeadTile<T, DB>;
    constexpr int BM = 32 * WAVES, THREADS = 64 * WAVES, RB = BN / 32;
    __shared__ __align__(16) char kt[2][BN * H::ROW];
    __shared__ __align__(16) char vt[2][BN * H::ROW];
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
    const int64_t stat = (int64_t)head * at.seq.tokens + at_row;
    if (h == 0 && span.on)
        delta[stat] = along;
    const float c = at.scale * kLog2e, l[1] = {octaves(lse[stat])};
    const bool large = __any(span.on && __builtin_fabsf(l[0]) >= kLargeScore);
    const T *kp = static_cast<const T *>(kh.p) + kv * kh.head_stride, *vp = static_cast<const T *>(vh.p) + kv * vh.head_stride;

    bool poison = false;
    f32x16 dq[DB] = {};
    const Reader<T, DB> read;
    TileLoad<T, DB, BN, WAVES, DIRECT> kl, vl;
    kl.begin(kp, kh.token_stride, at.dim);
    vl.begin(vp, vh.token_stride, at.dim);
    auto walk = [&](auto careful) {
        constexpr bool CAREFUL = decltype(careful)::value;
        kl.load(kt[0], first, last + 1);
        vl.load(vt[0], first, last + 1);
        int stage = 0;
        for (int k0 = first; k0 <= last; k0 += BN) {
            kl.store(kt[stage], k0, last + 1);
            vl.store(vt[stage], k0, last + 1);
            __syncthreads();
            if (k0 + BN <= last) {
                kl.load(kt[stage ^ 1], k0 + BN, last + 1);
                vl.load(vt[stage ^ 1], k0 + BN, last + 1);
            }
            const char *kb = kt[stage], *vb = vt[stage];
            stage ^= 1;
            if (k0 > w_last || k0 + BN <= w_first)
                continue;
            const bool masked = !(k0 >= w_full && k0 + BN - 1 <= q0);
            uint64_t found = 0;
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                f32x16 x = {}, y = {};
#pragma unroll
                for (int s = 0; s < H::STEPS; ++s) {
                    Frag<T> a, b;
                    read.rows(kb, 32 * rb, s, a);
                    read.rows(vb, 32 * rb, s, b);
                    mma(a, q[s], x);
                    mma(b, g[s], y);
                }
                probabilities(x, c, l, large);
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    x[r] *= y[r] - along;
                if (masked) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const uint32_t key = k0 + 32 * rb + 8 * (r >> 2) + 4 * h + (r & 3);
                        x[r] = key - start < seen ? x[r] : 0.0f;
                    }
                }
                Frag<T> p[2];
                operands(x, p);
                if (CAREFUL && masked)
                    add_product<true>(read, kb, 32 * rb, p, dq, found);
                else
                    add_product<false>(read, kb, 32 * rb, p, dq, found);
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
    if (span.on)
        store_row(static_cast<T *>(dqh.p) + at_row * dqh.token_stride + head * dqh.head_stride, at.dim, dq,
                  poison ? __builtin_nanf("") : at.scale);
}

// Columns are keys here: a lane's key and value stay in registers as operands.  PARTS: 1 dv, 2 dk, 3 both.
template <class T, int DB, int WAVES, int BQ, int OCC, bool DIRECT, int PARTS>
__global__ __launch_bounds__(64 * WAVES, OCC) void k_attention_dkv(Attention at, Heads doh, Heads qh, Heads kh, Heads vh,
                                                                 const float *lse, Heads dkh, Heads dvh, const float *delta,
                                                                 int tiles, int64_t items)
{
    using H = HeadTile<T, DB>;
    constexpr int BK = 32 * WAVES, THREADS = 64 * WAVES, RB = BQ / 32;
    constexpr bool WITH_V = PARTS & 1, WITH_K = PARTS & 2;
    __shared__ __align__(16) char qt[2][BQ * H::ROW];
    __shared__ __align__(16) char gt[2][BQ * H::ROW];
    __shared__ __align__(16) float lt[2][BQ], dt[2][BQ];
    __shared__ int64_t samples[kSeqSamples];
    __shared__ int edges[WAVES][2];

    const int64_t item = shared_item(work_block(), items);
    if (item >= items)
        return;
    const int kv = (int)(item / tiles), tile = (int)(item - (int64_t)kv * tiles);

    const int wave = uniform(threadIdx.x / kWave), lane = lane_id(), h = lane >> 5;
    const int key = tile * BK + 32 * wave + (lane & 31);
    fill_samples<THREADS>(at.seq, samples);
    const Span span = span_of(at.seq, samples, key);
    const int end = span.on ? span.end : -1;
    const int w_first = min_wave(span.on ? key : INT_MAX), w_end = max_wave(end); // queries that see the wave's keys
    const int w_all = max_wave(span.on ? key : INT_MAX), w_until = min_wave(end); // those that see all of them
    if (lane == 0)
        edges[wave][0] = w_first, edges[wave][1] = w_end;
    __syncthreads();
    int first = INT_MAX, limit = -1;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        first = edges[w][0] < first ? edges[w][0] : first;
        limit = edges[w][1] > limit ? edges[w][1] : limit;
    }
    if (limit < 0)
        return;
    first = (int)uniform((uint32_t)first), limit = (int)uniform((uint32_t)limit);

    const int64_t at_key = key < at.seq.tokens ? key : at.seq.tokens - 1;
    const T *krow = static_cast<const T *>(kh.p) + at_key * kh.token_stride + kv * kh.head_stride;
    const T *vrow = static_cast<const T *>(vh.p) + at_key * vh.token_stride + kv * vh.head_stride;
    Frag<T> k[H::STEPS], v[WITH_K ? H::STEPS : 1];
#pragma unroll
    for (int s = 0; s < H::STEPS; ++s) {
        load_frag(krow, 16 * s + 8 * h, at.dim, k[s]);
        if constexpr (WITH_K)
            load_frag(vrow, 16 * s + 8 * h, at.dim, v[s]);
    }
    const float c = at.scale * kLog2e;
    const int per_head = (limit - first + BQ - 1) / BQ;
    const int64_t count = (int64_t)per_head * at.group;

    bool poison_k = false, poison_v = false;
    f32x16 dk[WITH_K ? DB : 1] = {}, dv[WITH_V ? DB : 1] = {};
    const Reader<T, DB> read;
    TileLoad<T, DB, BQ, WAVES, DIRECT> ql, gl;
    ql.begin(nullptr, qh.token_stride, at.dim);
    gl.begin(nullptr, doh.token_stride, at.dim);
    const uint32_t seen = span.on ? end - key : 0; // queries that see the key, from its own on
    auto walk = [&](auto careful) {
        constexpr bool CAREFUL = decltype(careful)::value;
        float stat = 0.0f; // threads 0 .. BQ - 1: lse, the next BQ: D
        int nq = first, nhead = kv * at.group;
        auto fetch = [&](int stage) {
            ql.move(static_cast<const T *>(qh.p) + nhead * qh.head_stride);
            gl.move(static_cast<const T *>(doh.p) + nhead * doh.head_stride);
            ql.load(qt[stage], nq, limit);
            gl.load(gt[stage], nq, limit);
            if (threadIdx.x < 2 * BQ) {
                const int r = nq + (threadIdx.x & (BQ - 1));
                stat = (threadIdx.x < BQ ? lse : delta)[(int64_t)nhead * at.seq.tokens + (r < limit ? r : limit - 1)];
            }
        };
        fetch(0);
        int stage = 0;
        for (int64_t i = 0; i < count; ++i) {
            const int q0 = nq;
            ql.store(qt[stage], q0, limit);
            gl.store(gt[stage], q0, limit);
            if (threadIdx.x < BQ)
                lt[stage][threadIdx.x] = octaves(stat);
            else if (threadIdx.x < 2 * BQ)
                dt[stage][threadIdx.x - BQ] = stat;
            __syncthreads();
            nq += BQ;
            if (nq >= limit)
                nq = first, ++nhead;
            if (i + 1 < count)
                fetch(stage ^ 1);
            const char *qb = qt[stage], *gb = gt[stage];
            const float *lb = lt[stage], *db = dt[stage];
            stage ^= 1;
            if (q0 >= w_end || q0 + BQ <= w_first)
                continue;
            const bool masked = !(q0 >= w_all && q0 + BQ <= w_until);
            uint64_t found_q = 0, found_g = 0;
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                f32x16 x = {}, y = {};
#pragma unroll
                for (int s = 0; s < H::STEPS; ++s) {
                    Frag<T> a, b;
                    read.rows(qb, 32 * rb, s, a);
                    if constexpr (WITH_K)
                        read.rows(gb, 32 * rb, s, b);
                    mma(a, k[s], x);
                    if constexpr (WITH_K)
                        mma(b, v[s], y);
                }
                float l[16];
                bool large = false;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    l[r] = lb[32 * rb + 8 * (r >> 2) + 4 * h + (r & 3)];
                    large |= __builtin_fabsf(l[r]) >= kLargeScore;
                }
                probabilities(x, c, l, __any(large));
                if (masked) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const uint32_t q = q0 + 32 * rb + 8 * (r >> 2) + 4 * h + (r & 3);
                        x[r] = q - key < seen ? x[r] : 0.0f;
                    }
                }
                Frag<T> p[2];
                if constexpr (WITH_V) {
                    operands(x, p);
                    if (CAREFUL && masked)
                        add_product<true>(read, gb, 32 * rb, p, dv, found_g);
                    else
                        add_product<false>(read, gb, 32 * rb, p, dv, found_g);
                }
                if constexpr (WITH_K) {
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        x[r] *= y[r] - db[32 * rb + 8 * (r >> 2) + 4 * h + (r & 3)];
                    if (masked) { // y and D may be NaN in masked places
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const uint32_t q = q0 + 32 * rb + 8 * (r >> 2) + 4 * h + (r & 3);
                            x[r] = q - key < seen ? x[r] : 0.0f;
                        }
                    }
                    operands(x, p);
                    if (CAREFUL && masked)
                        add_product<true>(read, qb, 32 * rb, p, dk, found_q);
                    else
                        add_product<false>(read, qb, 32 * rb, p, dk, found_q);
                }
            }
            if (CAREFUL && __any((found_q | found_g) != 0)) {
                found_q = or_wave(found_q), found_g = or_wave(found_g);
                for (int j = 0; j < BQ; ++j) {
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
    if (!span.on)
        return;
    if constexpr (WITH_K)
        store_row(static_cast<T *>(dkh.p) + at_key * dkh.token_stride + kv * dkh.head_stride, at.dim, dk,
                  poison_k ? __builtin_nanf("") : at.scale);
    if constexpr (WITH_V)
        store_row(static_cast<T *>(dvh.p) + at_key * dvh.token_stride + kv * dvh.head_stride, at.dim, dv,
                  poison_v ? __builtin_nanf("") : 1.0f);
}

struct Grad {
    const Attention &at;
    const Heads &dout, &q, &k, &v, &out;
    const float *lse;
    const Heads &dq, &dk, &dv;
    float *delta;
    hipStream_t s;

    int dtype;

    template <class T, int DB, int WAVES, int BN, int OCC>
    int queries() const
    {
        const int tiles = (at.seq.tokens + 32 * WAVES - 1) / (32 * WAVES);
        const int64_t items = (int64_t)tiles * q.heads;
        auto kernel = direct(k, dtype, at.dim) && direct(v, dtype, at.dim) ? k_attention_dq<T, DB, WAVES, BN, OCC, true>
                                                                           : k_attention_dq<T, DB, WAVES, BN, OCC, false>;
        return launch<WAVES>(kernel, shared_blocks(items), kUncapped, s, at, dout, q, k, v, out, lse, dq, delta, tiles, items);
    }
    template <class T, int DB, int WAVES, int BQ, int OCC, int PARTS = 3>
    int keys() const
    {
        const int tiles = (at.seq.tokens + 32 * WAVES - 1) / (32 * WAVES);
        const int64_t items = (int64_t)tiles * k.heads;
        auto kernel = direct(q, dtype, at.dim) && direct(dout, dtype, at.dim) ? k_attention_dkv<T, DB, WAVES, BQ, OCC, true, PARTS>
                                                                             : k_attention_dkv<T, DB, WAVES, BQ, OCC, false, PARTS>;
        return launch<WAVES>(kernel, shared_blocks(items), kUncapped, s, at, dout, q, k, v, lse, dk, dv, delta, tiles, items);
    }
};

} // namespace

int64_t attention_grad_workspace(int64_t tokens, int q_heads, int, int)
{
    return (tokens * q_heads * (int64_t)sizeof(float) + 15) / 16 * 16;
}

int launch_attention_grad(int dtype, const Attention &at, const Heads &dout, const Heads &q, const Heads &k, const Heads &v,
                          const Heads &out, const float *lse, const Heads &dq, const Heads &dk, const Heads &dv,
                          float *workspace, hipStream_t s)
{
    const Grad g{at, dout, q, k, v, out, lse, dq, dk, dv, workspace, s, dtype};
    const int db = (at.dim + 31) / 32;
    int rc;
    if (dtype == SDP4_BF16) {
        if (db <= 2)
            return (rc = g.queries<bf16_t, 2, 4, 64, 2>()) ? rc : g.keys<bf16_t, 2, 4, 32, 2>();
        if (db == 3)
            return (rc = g.queries<bf16_t, 3, 4, 64, 2>()) ? rc : g.keys<bf16_t, 3, 4, 64, 1>();
        if (db == 4)
            return (rc = g.queries<bf16_t, 4, 4, 64, 2>()) ? rc : g.keys<bf16_t, 4, 4, 32, 1>();
        return (rc = g.queries<bf16_t, 8, 4, 32, 1>()) ? rc : g.keys<bf16_t, 8, 4, 32, 1>();
    }
    if (db <= 2)
        return (rc = g.queries<float, 2, 4, 32, 1>()) ? rc : g.keys<float, 2, 4, 32, 1>();
    if (db == 3)
        return (rc = g.queries<float, 3, 4, 32, 1>()) ? rc : g.keys<float, 3, 4, 32, 1>();
    if (db == 4)
        return (rc = g.queries<float, 4, 4, 32, 1>()) ? rc : g.keys<float, 4, 4, 32, 1>();
    if ((rc = g.queries<float, 8, 4, 32, 1>()) || (rc = g.keys<float, 8, 4, 32, 1, 1>()))
        return rc;
    return g.keys<float, 8, 4, 32, 1, 2>(); // both results and both operands would not fit the registers
}

} // namespace sdp4
