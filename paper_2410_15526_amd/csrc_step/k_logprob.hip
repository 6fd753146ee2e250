// k_logprob.hip -- log probabilities of given tokens with logsumexp, entropy
// and the largest alternatives; their gradient; both in one pass.
//
// For a row x of `vocab` logits, with m = max x and t_j = (x_j - m) log2 e:
//   S = sum 2^t_j, T = sum 2^t_j t_j,
//   lse = m + ln 2 log2 S, logp = x_target - lse, H = ln 2 (log2 S - T / S).
// A logit of -inf counts nothing; a row of nothing else has lse = logp = -inf
// and H = 0; a NaN or +inf makes lse, logp and H NaN.
//
// Forward: a wave takes a slice of a row into registers (up to 4096 logits),
// finds its maximum, then S and T, and leaves (m, S, T) and its largest
// elements in the workspace; a second launch joins the slices of each row,
// one wave per row.  A row of one slice is finished by its wave.
#include "step_device.hpp"

namespace sdp4 {

namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int kMaxSlices = 256;  // of a row
constexpr int kMaxTop = SDP4_MAX_TOP;
constexpr int kListed = 256;     // candidates a wave lists for the alternatives

// What a slice leaves of its row: S and T relative to m.
struct alignas(16) Slice {
    float m, S, T, unused;
};

// Order of the alternatives as one number: larger values first (-0 and +0 equal), then lower indexes.
SDP4_DEV uint32_t order_bits(float v)
{
    const uint32_t b = __float_as_uint(v + 0.0f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
SDP4_DEV float from_order_bits(uint32_t k)
{
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
SDP4_DEV uint64_t entry_of(float v, uint32_t index) { return (uint64_t)order_bits(v) << 32 | (0xFFFFFFFFu - index); }
SDP4_DEV uint32_t entry_index(uint64_t e) { return 0xFFFFFFFFu - (uint32_t)e; }
constexpr uint64_t kNoEntry = 0; // below every element

SDP4_DEV float exp2_of(float t) { return __builtin_amdgcn_exp2f(t); }
SDP4_DEV float log2_of(float s) { return __builtin_amdgcn_logf(s); }

// Calls body(exponent, delta) with t(x) = (x - ref) log2 e - lg: one fma, whose constant's rounding error the caller
// takes out again by `delta` (t is too large by it), or, for magnitudes whose product with log2 e overflows (rows of a
// type's lowest value), a subtraction and an fma.
template <class F>
SDP4_DEV void with_exponent(float ref, float lg, F body)
{
    if (__builtin_fabsf(ref) < 1e38f) {
        const float c = __builtin_fmaf(ref, kLog2e, lg);
        body([=](float x) { return __builtin_fmaf(x, kLog2e, -c); }, __builtin_fmaf(ref, kLog2e, -c) + lg);
    } else {
        body([=](float x) { return __builtin_fmaf(x - ref, kLog2e, -lg); }, 0.0f);
    }
}

// The outputs of one row from its whole statistics.
SDP4_DEV void finish_row(const TokenStats &out, int64_t row, int64_t vocab, float m, float S, float T, float target_x,
                         int64_t target)
{
    const float ln_s = kLn2 * log2_of(S);
    const bool empty = S == 0.0f;
    if (out.lse)
        out.lse[row] = empty ? -__builtin_inff() : m + ln_s;
    if (out.entropy)
        out.entropy[row] = empty ? 0.0f : fmaxf(ln_s - kLn2 * (T / S), 0.0f) + (S - S);
    if (out.logp) {
        float v = target < 0 ? 0.0f : __builtin_nanf("");
        if (target >= 0 && target < vocab)
            v = empty ? -__builtin_inff() : (target_x - m) - ln_s;
        out.logp[row] = v;
    }
}

// Chunks of a wave's slice: chunk i * 64 + lane of `count`, from chunk `first` of the row.  A row's last chunk, where
// it is not whole, is read from the row's last whole chunk of elements instead and what lies before it masked; all
// other places that hold nothing read a valid chunk too and are masked, so that no load waits for a test.
template <class T, int NC>
struct SliceRegs {
    static constexpr int W = kChunk<T>;
    u32x4 raw[NC];
    uint32_t lane;
    int64_t first, count, vocab;

    SDP4_DEV int64_t chunk_start(int i) const // element of the row at which the chunk's register begins
    {
        int64_t c = (int64_t)i * kWave + lane;
        c = first + (c < count ? c : count - 1);
        return c * W + W <= vocab ? c * W : vocab - W;
    }
    SDP4_DEV void load(const T *row, int64_t row_vocab, int64_t first_, int64_t count_)
    {
        lane = lane_id();
        first = first_, count = count_, vocab = row_vocab;
        if (vocab >= W) {
#pragma unroll
            for (int i = 0; i < NC; ++i)
                raw[i] = load_chunk<true>(row + chunk_start(i));
            const bool ragged = (first + count) * W > vocab;
#pragma unroll
            for (int i = 0; i < NC; ++i)
                if (ragged || (i + 1) * kWave > count)
                    mask(i);
        } else { // fewer elements than a chunk
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                float v[W];
#pragma unroll
                for (int j = 0; j < W; ++j)
                    v[j] = i == 0 && lane == 0 && j < vocab ? to_f32<T>(row[j]) : -__builtin_inff();
                raw[i] = pack<T>(v);
            }
        }
    }
    SDP4_DEV void mask(int i)
    {
        const int64_t c = (int64_t)i * kWave + lane;
        const int64_t skip = c < count ? (first + c) * W - chunk_start(i) : W; // elements that are not this chunk's
        float v[W];
        unpack<T>(raw[i], v);
#pragma unroll
        for (int j = 0; j < W; ++j)
            v[j] = j < skip ? -__builtin_inff() : v[j];
        raw[i] = pack<T>(v);
    }
    // element of the row that value j of chunk i is; at least vocab for none
    SDP4_DEV int64_t index(int i, int j) const
    {
        const int64_t c = (int64_t)i * kWave + lane;
        if (vocab < W)
            return c == 0 && j < vocab ? j : vocab;
        if (c >= count)
            return vocab;
        const int64_t e = chunk_start(i) + j;
        return e >= (first + c) * W ? e : vocab;
    }
};

// The `k` largest elements of a slice, best first, into list[0..k) (missing ones kNoEntry).
//
// Every lane's largest element is known (cm: by chunk).  At least k elements are as good as the k-th best of these 64,
// which a bisection over their bits finds by counting lanes; among lanes that tie there, a second one over the
// positions of their chunks.  What is as good as that, k elements and few more, is listed in LDS, and each listed
// element's place is the number of better ones.
template <class T, int NC>
SDP4_DEV void slice_top(const SliceRegs<T, NC> &r, const float (&cm)[NC], float lane_max, int k, uint64_t *lds,
                        uint32_t *lds_count, uint64_t *list)
{
    constexpr int W = kChunk<T>;
    const uint32_t lane = r.lane;
    const uint32_t key = order_bits(lane_max);
    uint32_t tau = 0;
    constexpr int kLowest = sizeof(T) == 2 ? 16 : 0; // bfloat16 values differ in their upper bits only
    const uint32_t probe = key >> kLowest;
#pragma unroll 1
    for (int b = 31 - kLowest; b >= 0; --b) {
        const uint32_t mid = tau | (1u << b);
        if (__builtin_popcountll(__ballot(probe >= mid)) >= k)
            tau = mid;
    }
    // lanes whose largest is tau, in the order of its first chunk
    const uint64_t ties = __ballot(probe == tau);
    const int above = __builtin_popcountll(__ballot(probe > tau));
    uint32_t last = ~0u; // position of the last chunk from which elements equal to tau are needed
    const float tau_value = from_order_bits(kLowest ? (tau << 16) | (tau & 0x8000u ? 0u : 0xFFFFu) : tau);
    if (above + __builtin_popcountll(ties) > k) {
        uint32_t pos = ~0u;
#pragma unroll
        for (int i = NC - 1; i >= 0; --i)
            if (probe == tau && cm[i] == lane_max)
                pos = (uint32_t)i * kWave + lane;
        last = 0;
#pragma unroll 1
        for (int b = 31 - __builtin_clz(NC * kWave); b >= 0; --b) { // the smallest position with enough at or before it
            const uint32_t mid = last + (1u << b) - 1;
            if (above + __builtin_popcountll(__ballot(pos <= mid)) < k)
                last = mid + 1;
        }
    }
    if (lane == 0)
        *lds_count = 0;
    wave_lds_sync();
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        if (!__ballot(cm[i] >= tau_value))
            continue;
        float v[W];
        unpack<T>(r.raw[i], v);
#pragma unroll
        for (int j = 0; j < W; ++j) {
            if (v[j] > tau_value || (v[j] == tau_value && (uint32_t)i * kWave + lane <= last)) {
                const int64_t e = r.index(i, j);
                if (e < r.vocab) {
                    const uint32_t slot = atomicAdd(lds_count, 1u);
                    if (slot < kListed)
                        lds[slot] = entry_of(v[j], (uint32_t)e);
                }
            }
        }
    }
    wave_lds_sync();
    const int listed = (int)uniform(*lds_count);
    if (listed <= kListed) {
        for (int a = (int)lane; a < (listed > k ? listed : k); a += kWave) {
            const uint64_t mine = a < listed ? lds[a] : kNoEntry;
            int rank = a < listed ? 0 : a;
            if (a < listed)
                for (int o = 0; o < listed; ++o)
                    rank += lds[o] > mine;
            if (rank < k)
                list[rank] = mine;
        }
    } else {
        // More than the list holds (a few lanes with most of the largest elements): best of the rest, k times.
        uint64_t before = ~uint64_t(0);
#pragma unroll 1
        for (int a = 0; a < k; ++a) {
            uint64_t best = kNoEntry;
#pragma unroll 1
            for (int i = 0; i < NC; ++i) {
                float v[W];
                u32x4 c = r.raw[0];
#pragma unroll
                for (int q = 1; q < NC; ++q)
                    c = i == q ? r.raw[q] : c;
                unpack<T>(c, v);
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    const int64_t e = r.index(i, j);
                    const uint64_t x = e < r.vocab ? entry_of(v[j], (uint32_t)e) : kNoEntry;
                    best = x < before && x > best ? x : best;
                }
            }
            for (int o = 1; o < kWave; o <<= 1) {
                const uint64_t other = __shfl_xor(best, o);
                best = other > best ? other : best;
            }
            if (lane == 0)
                list[a] = best;
            before = best;
        }
    }
    wave_lds_sync();
}

// S: 0 for a row without a finite logit, NaN for one with a NaN or +inf.
SDP4_DEV void write_top(const TokenStats &out, int64_t row, int i, uint64_t e, float m, float S)
{
    const bool bad = !(S - S == 0.0f);
    const float v = S == 0.0f ? -__builtin_inff() : (from_order_bits((uint32_t)(e >> 32)) - m) - kLn2 * log2_of(S);
    out.top_logp[row * out.top_k + i] = bad ? __builtin_nanf("") : v;
    out.top_ids[row * out.top_k + i] = bad ? -1 : (int64_t)entry_index(e);
}

// One slice per wave, four waves in a block.
template <class T, int NC, bool TOP>
__global__ __launch_bounds__(256) void k_logprob_slices(Rows<const T *> x, int64_t rows, int64_t vocab,
                                                        Divisor slices, int64_t chunks_each, TokenStats out,
                                                        Slice *stats, uint64_t *lists)
{
    constexpr int W = kChunk<T>;
    __shared__ uint64_t lds[TOP ? 4 * kListed : 1];
    __shared__ uint64_t direct[TOP ? 4 * kMaxTop : 1];
    __shared__ uint32_t lds_count[4];
    const uint32_t wave = uniform(threadIdx.x / kWave);
    const uint64_t w = (uint64_t)work_block() * 4 + wave;
    uint64_t slice;
    const int64_t row = (int64_t)divide(w, slices, slice);
    if (row >= rows)
        return;
    const T *p = x.p + row * x.stride;
    const int64_t chunks = (vocab + W - 1) / W, first = (int64_t)slice * chunks_each;
    const int64_t count = chunks - first < chunks_each ? chunks - first : chunks_each;
    SliceRegs<T, NC> r;
    r.load(p, vocab, first, count);

    float cm[NC], m = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        float v[W];
        unpack<T>(r.raw[i], v);
        cm[i] = v[0];
#pragma unroll
        for (int j = 1; j < W; ++j)
            cm[i] = fmaxf(cm[i], v[j]);
        m = fmaxf(m, cm[i]);
    }
    const float lane_max = m;
    m = max_wave(m);
    float S = 0.0f, T2 = 0.0f;
    const float ref = m == -__builtin_inff() ? 0.0f : m;
    with_exponent(ref, 0.0f, [&](auto exponent, float delta) {
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            float v[W];
            unpack<T>(r.raw[i], v);
#pragma unroll
            for (int j = 0; j < W; ++j) {
                const float t = exponent(v[j]), e = exp2_of(t);
                S += e;
                T2 = __builtin_fmaf(e, fmaxf(t, -1000.0f), T2); // 2^-1000 is 0: -inf counts nothing
            }
        }
        S = sum_lanes(S, kWave);
        T2 = sum_lanes(T2, kWave);
        const float f = exp2_of(-delta);
        T2 = f * __builtin_fmaf(-delta, S, T2);
        S *= f;
    });

    const bool whole_row = slices.d == 1;
    if constexpr (TOP) {
        uint64_t *list = whole_row ? direct + wave * kMaxTop : lists + (int64_t)w * out.top_k;
        slice_top<T, NC>(r, cm, lane_max, out.top_k, lds + wave * kListed, lds_count + wave, list);
        if (whole_row && (int)r.lane < out.top_k)
            write_top(out, row, r.lane, list[r.lane], m, S);
    }
    if (r.lane == 0) {
        if (whole_row) {
            const int64_t target = out.targets ? out.targets[row] : -1;
            finish_row(out, row, vocab, m, S, T2, target >= 0 && target < vocab ? to_f32<T>(p[target]) : 0.0f, target);
        } else {
            stats[w] = Slice{m, S, T2, 0.0f};
        }
    }
}

// Joins the slices of a row: one wave each.
template <class T>
__global__ __launch_bounds__(256) void k_logprob_join(Rows<const T *> x, int64_t rows, int64_t vocab, int slices,
                                                      TokenStats out, const Slice *stats, const uint64_t *lists)
{
    const uint32_t lane = lane_id();
    const int64_t row = work_block() * 4 + uniform(threadIdx.x / kWave);
    if (row >= rows)
        return;
    const int64_t target = out.targets ? out.targets[row] : -1;
    const float tx = target >= 0 && target < vocab ? to_f32<T>(x.p[row * x.stride + target]) : 0.0f;
    constexpr int N = kMaxSlices / kWave;
    Slice s[N];
    uint64_t head[N];
    int at[N];
    const uint64_t *mine = lists + row * slices * (int64_t)out.top_k;
    float m = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int sl = i * kWave + (int)lane;
        s[i] = Slice{-__builtin_inff(), 0.0f, 0.0f, 0.0f};
        head[i] = kNoEntry;
        at[i] = 0;
        if (sl < slices) {
            s[i] = stats[row * slices + sl];
            if (out.top_k)
                head[i] = mine[(int64_t)sl * out.top_k];
        }
        m = fmaxf(m, s[i].m);
    }
    m = max_wave(m);
    float S = 0.0f, T2 = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (s[i].S != 0.0f) { // a slice without a finite logit counts nothing
            const float d = (s[i].m - m) * kLog2e, f = exp2_of(d);
            S += s[i].S * f;
            T2 += f * (f == 0.0f ? 0.0f : __builtin_fmaf(s[i].S, d, s[i].T));
        }
    }
    S = sum_lanes(S, kWave);
    T2 = sum_lanes(T2, kWave);
    if (lane == 0)
        finish_row(out, row, vocab, m, S, T2, tx, target);
    if (out.top_k) {
#pragma unroll 1
        for (int a = 0; a < out.top_k; ++a) {
            uint64_t best = head[0];
#pragma unroll
            for (int i = 1; i < N; ++i)
                best = head[i] > best ? head[i] : best;
            for (int o = 1; o < kWave; o <<= 1) {
                const uint64_t other = __shfl_xor(best, o);
                best = other > best ? other : best;
            }
            if (lane == 0)
                write_top(out, row, a, best, m, S);
#pragma unroll
            for (int i = 0; i < N; ++i) { // entries differ: one lane moves on
                if (head[i] == best && best != kNoEntry) {
                    ++at[i];
                    head[i] = at[i] < out.top_k ? mine[(int64_t)(i * kWave + (int)lane) * out.top_k + at[i]] : kNoEntry;
                }
            }
        }
    }
}

// ---------------------------------------------------------------------------
// gradient
// ---------------------------------------------------------------------------
// dx_j = p_j (A + B t_j) + [j = target] g_logp with t_j = (x_j - lse) log2 e, p_j = 2^t_j,
// A = g_lse - g_logp - g_H H, B = -g_H ln 2.
struct RowGrad {
    float ref, A, B, hit; // ref: lse, or 0 for a row without a finite logit
    int64_t target;       // -1: none
};

SDP4_DEV RowGrad row_grad(float lse, float entropy, int64_t target, int64_t vocab, float g_logp, float g_entropy,
                          float g_lse)
{
    RowGrad r;
    const bool empty = lse == -__builtin_inff();
    r.hit = target >= 0 ? g_logp : 0.0f;
    if (target >= vocab)
        r.hit = __builtin_nanf(""); // no such token: the row's gradient says so
    r.A = g_lse - r.hit - g_entropy * entropy;
    r.B = -kLn2 * g_entropy;
    r.ref = empty ? 0.0f : lse;
    r.target = target >= 0 && target < vocab && !empty ? target : -1;
    if (empty && target < vocab)
        r.A = r.B = 0.0f;
    if (!(lse == lse))
        r.A = lse;
    return r;
}

// Gradient of the W elements of a chunk that starts at element e of the row; zeros from vocab on.
template <int W, bool ENT, class X>
SDP4_DEV void grad_chunk(const RowGrad &g, float A, X exponent, float delta, int64_t e, int64_t vocab, float (&v)[W])
{
#pragma unroll
    for (int j = 0; j < W; ++j) {
        const float t = exponent(v[j]), p = exp2_of(t);
        if constexpr (ENT)
            v[j] = p * __builtin_fmaf(g.B, fmaxf(t, -1000.0f) - delta, A);
        else
            v[j] = p * A;
    }
    const int64_t at = g.target - e;
    if (at >= 0 && at < W) {
#pragma unroll
        for (int j = 0; j < W; ++j)
            v[j] += at == j ? g.hit : 0.0f;
    }
    if (e + W > vocab) {
#pragma unroll
        for (int j = 0; j < W; ++j)
            v[j] = e + j < vocab ? v[j] : 0.0f;
    }
}

// A wave takes U * 64 chunks of one row.
template <class T, int U, bool ENT>
__global__ __launch_bounds__(256) void k_logprob_grad(Rows<const T *> x, int64_t rows, int64_t vocab,
                                                      const int64_t *targets, const float *lse, const float *entropy,
                                                      TokenGrads g, Rows<T *> dx, int64_t width, Divisor tiles)
{
    constexpr int W = kChunk<T>;
    const uint32_t wave = uniform(threadIdx.x / kWave), lane = lane_id();
    const uint64_t w = (uint64_t)work_block() * 4 + wave;
    uint64_t tile;
    const int64_t row = (int64_t)divide(w, tiles, tile);
    if (row >= rows)
        return;
    const T *p = x.p + row * x.stride;
    T *q = dx.p + row * dx.stride;
    const int64_t first = (int64_t)tile * (U * kWave) + lane;
    float v[U][W];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int64_t e = (first + i * kWave) * W;
        load_elems(p + e, vocab - e, v[i]);
    }
    const RowGrad rg = row_grad(lse[row], ENT ? entropy[row] : 0.0f, targets ? targets[row] : -1, vocab,
                                g.logp ? g.logp[row] : 0.0f, ENT ? g.entropy[row] : 0.0f, g.lse ? g.lse[row] : 0.0f);
    with_exponent(rg.ref, 0.0f, [&](auto exponent, float delta) {
        const float f = exp2_of(-delta);
        RowGrad s = rg;
        s.B *= f;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int64_t e = (first + i * kWave) * W;
            grad_chunk<W, ENT>(s, rg.A * f, exponent, delta, e, vocab, v[i]);
            store_elems(q + e, width - e, v[i]);
        }
    });
}

// The loss and its gradient: a block holds a whole row in registers, so the logits are read once.
template <class T, int WAVES, int NC, bool ENT>
__global__ __launch_bounds__(64 * WAVES) void k_token_loss(Rows<const T *> x, int64_t rows, int64_t vocab,
                                                           TokenStats out, TokenGrads g, Rows<T *> dx, int64_t width)
{
    constexpr int W = kChunk<T>, NT = kWave * WAVES;
    __shared__ float red[3][WAVES];
    const int64_t row = work_block();
    if (row >= rows)
        return;
    const uint32_t wave = threadIdx.x / kWave, lane = lane_id();
    const T *p = x.p + row * x.stride;
    T *q = dx.p + row * dx.stride;
    const int64_t target = out.targets ? out.targets[row] : -1;
    const float g_logp = g.logp ? g.logp[row] : 0.0f, g_ent = ENT ? g.entropy[row] : 0.0f,
                g_lse = g.lse ? g.lse[row] : 0.0f;
    float tx = target >= 0 && target < vocab ? to_f32<T>(p[target]) : 0.0f;
    u32x4 raw[NC];
    float m = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int64_t e = ((int64_t)i * NT + threadIdx.x) * W;
        float v[W];
        if (e + W <= vocab) {
            raw[i] = load_chunk<true>(p + e);
        } else {
            load_elems(p + e, vocab - e, v, -__builtin_inff());
            raw[i] = pack<T>(v);
        }
    }
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        float v[W];
        unpack<T>(raw[i], v);
#pragma unroll
        for (int j = 0; j < W; ++j)
            m = fmaxf(m, v[j]);
    }
    m = max_wave(m);
    if (lane == 0)
        red[0][wave] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WAVES; ++i)
        m = fmaxf(m, red[0][i]);
    float S = 0.0f, T2 = 0.0f;
    with_exponent(m == -__builtin_inff() ? 0.0f : m, 0.0f, [&](auto exponent, float delta) {
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            float v[W];
            unpack<T>(raw[i], v);
#pragma unroll
            for (int j = 0; j < W; ++j) {
                const float t = exponent(v[j]), e = exp2_of(t);
                S += e;
                T2 = __builtin_fmaf(e, fmaxf(t, -1000.0f), T2);
            }
        }
        S = sum_lanes(S, kWave);
        T2 = sum_lanes(T2, kWave);
        if (lane == 0)
            red[1][wave] = S, red[2][wave] = T2;
        __syncthreads();
        S = T2 = 0.0f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i)
            S += red[1][i], T2 += red[2][i];
        const float f = exp2_of(-delta);
        T2 = f * __builtin_fmaf(-delta, S, T2);
        S *= f;
    });
    if (threadIdx.x == 0)
        finish_row(out, row, vocab, m, S, T2, tx, target);
    const bool empty = S == 0.0f;
    const float ln_s = kLn2 * log2_of(S);
    const float lse = empty ? -__builtin_inff() : m + ln_s;
    const float ent = ENT ? (empty ? 0.0f : fmaxf(ln_s - kLn2 * (T2 / S), 0.0f) + (S - S)) : 0.0f;
    const RowGrad rg = row_grad(lse, ent, target, vocab, g_logp, g_ent, g_lse);
    // from m and log2 S rather than from their rounded sum
    with_exponent(empty ? 0.0f : m, empty ? 0.0f : log2_of(S), [&](auto exponent, float delta) {
        const float f = exp2_of(-delta);
        RowGrad s = rg;
        s.B *= f;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int64_t e = ((int64_t)i * NT + threadIdx.x) * W;
            if (e < width) {
                float v[W];
                unpack<T>(raw[i], v);
                grad_chunk<W, ENT>(s, rg.A * f, exponent, delta, e, vocab, v);
                store_elems(q + e, width - e, v);
            }
        }
    });
}

template <class T, class P>
Rows<T *> typed(Rows<P> r)
{
    return {static_cast<T *>(r.p), r.stride};
}

// How a row is cut into slices: NC chunks per lane, `slices` of `each` chunks.
struct Cut {
    int nc;
    int64_t slices, each;
};
Cut cut_rows(int64_t rows, int64_t vocab, int chunk, int most)
{
    const int64_t chunks = (vocab + chunk - 1) / chunk;
    int nc = 1;
    const auto slices = [&](int n) { return (chunks + 64 * n - 1) / (64 * n); };
    // the largest slices that still give 2048 waves, no more than kMaxSlices of them
    while (nc < most && slices(nc) > 1 && (slices(nc) > kMaxSlices || rows * slices(2 * nc) >= 2048))
        nc *= 2;
    const int64_t each = (chunks + slices(nc) - 1) / slices(nc);
    return {nc, (chunks + each - 1) / each, each};
}

template <class T>
constexpr int kMostChunks = sizeof(T) == 2 ? 8 : 16;

template <class T, bool TOP>
auto slice_kernel(int nc)
{
    if constexpr (kMostChunks<T> == 16)
        if (nc == 16)
            return k_logprob_slices<T, 16, TOP>;
    return nc == 1   ? k_logprob_slices<T, 1, TOP>
           : nc == 2 ? k_logprob_slices<T, 2, TOP>
           : nc == 4 ? k_logprob_slices<T, 4, TOP>
                     : k_logprob_slices<T, 8, TOP>;
}

template <class T>
int logprob(Rows<const void *> x, int64_t rows, int64_t vocab, const TokenStats &out, void *workspace, hipStream_t s)
{
    const Cut c = cut_rows(rows, vocab, kChunk<T>, kMostChunks<T>);
    Slice *stats = static_cast<Slice *>(workspace);
    uint64_t *lists = reinterpret_cast<uint64_t *>(stats + (c.slices > 1 ? rows * c.slices : 0));
    auto k = out.top_k ? slice_kernel<T, true>(c.nc) : slice_kernel<T, false>(c.nc);
    const int rc = launch<4>(k, (rows * c.slices + 3) / 4, kUncapped, s, typed<const T>(x), rows, vocab,
                             Divisor((uint64_t)c.slices), c.each, out, stats, lists);
    if (rc || c.slices == 1)
        return rc;
    return launch<4>(k_logprob_join<T>, (rows + 3) / 4, kUncapped, s, typed<const T>(x), rows, vocab, (int)c.slices,
                     out, stats, lists);
}

template <class T, bool ENT>
int logprob_grad(Rows<const void *> x, int64_t rows, int64_t vocab, const int64_t *targets, const float *lse,
                 const float *entropy, const TokenGrads &g, Rows<void *> dx, int64_t width, hipStream_t s)
{
    const int64_t chunks = (width + kChunk<T> - 1) / kChunk<T>;
    auto run = [&](auto k, int u) {
        const int64_t tiles = (chunks + 64 * u - 1) / (64 * u);
        return launch<4>(k, (rows * tiles + 3) / 4, kUncapped, s, typed<const T>(x), rows, vocab, targets, lse,
                         entropy, g, typed<T>(dx), width, Divisor((uint64_t)tiles));
    };
    return run(k_logprob_grad<T, 2, ENT>, 2);
}

template <class T, bool ENT>
int token_loss(Rows<const void *> x, int64_t rows, int64_t vocab, const TokenStats &out, const TokenGrads &g,
               Rows<void *> dx, int64_t width, void *workspace, hipStream_t s)
{
    const int64_t chunks = (width + kChunk<T> - 1) / kChunk<T>;
    auto run = [&](auto waves, auto nc) {
        constexpr int WV = decltype(waves)::value, NC = decltype(nc)::value;
        return launch<WV>(k_token_loss<T, WV, NC, ENT>, rows, kUncapped, s, typed<const T>(x), rows, vocab, out, g,
                          typed<T>(dx), width);
    };
    if (chunks <= 256)
        return run(std::integral_constant<int, 1>{}, std::integral_constant<int, 4>{});
    if (chunks <= 2048)
        return run(std::integral_constant<int, 4>{}, std::integral_constant<int, 8>{});
    if (chunks <= 8192)
        return run(std::integral_constant<int, 16>{}, std::integral_constant<int, 8>{});
    if (chunks <= 16384)
        return run(std::integral_constant<int, 16>{}, std::integral_constant<int, 16>{});
    const int rc = logprob<T>(x, rows, vocab, out, workspace, s);
    return rc ? rc : logprob_grad<T, ENT>(x, rows, vocab, out.targets, out.lse, out.entropy, g, dx, width, s);
}

} // namespace

int64_t token_logprob_workspace(int64_t rows, int64_t vocab, int top_k)
{
    if (rows <= 0 || vocab <= 0)
        return 0;
    int64_t most = 0;
    for (int two = 0; two < 2; ++two) { // either type
        const Cut c = two ? cut_rows(rows, vocab, kChunk<bf16_t>, kMostChunks<bf16_t>)
                          : cut_rows(rows, vocab, kChunk<float>, kMostChunks<float>);
        const int64_t n = c.slices > 1 ? rows * c.slices * (int64_t)(sizeof(Slice) + sizeof(uint64_t) * top_k) : 0;
        most = n > most ? n : most;
    }
    return most;
}

int launch_token_logprob(int dtype, Rows<const void *> x, int64_t rows, int64_t vocab, const TokenStats &out,
                         void *workspace, hipStream_t s)
{
    return with_type(dtype, [&](auto t) { return logprob<decltype(t)>(x, rows, vocab, out, workspace, s); });
}

int launch_token_logprob_grad(int dtype, Rows<const void *> x, int64_t rows, int64_t vocab, const int64_t *targets,
                              const float *lse, const float *entropy, const TokenGrads &g, Rows<void *> dx,
                              int64_t width, hipStream_t s)
{
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        return g.entropy ? logprob_grad<T, true>(x, rows, vocab, targets, lse, entropy, g, dx, width, s)
                         : logprob_grad<T, false>(x, rows, vocab, targets, lse, entropy, g, dx, width, s);
    });
}

int launch_token_loss(int dtype, Rows<const void *> x, int64_t rows, int64_t vocab, const TokenStats &out,
                      const TokenGrads &g, Rows<void *> dx, int64_t width, void *workspace, hipStream_t s)
{
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        return g.entropy ? token_loss<T, true>(x, rows, vocab, out, g, dx, width, workspace, s)
                         : token_loss<T, false>(x, rows, vocab, out, g, dx, width, workspace, s);
    });
}

} // namespace sdp4
