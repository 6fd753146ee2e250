// k_logprob.hip -- log probabilities of given tokens with logsumexp, entropy
// and the largest alternatives; their gradient; both in one pass.
//
// For a row x of `vocab` logits, with m = max x and t_j = (x_j - m) log2 e:
//   S = sum 2^t_j, T = sum 2^t_j t_j,
//   lse = m + ln 2 log2 S, logp = x_target - lse, H = ln 2 (log2 S - T / S).
// A logit of -inf counts nothing; a row of nothing else has lse = logp = -inf
// and H = 0; a NaN or +inf makes lse, logp and H NaN.
//
// Forward: a wave takes a slice of a row into registers (up to 4096 logits) and leaves S and T, relative to a logit of
// the slice, in the workspace; a second launch joins the slices of each row, one wave per row.  A row of one slice is
// finished by its wave.  For the alternatives each lane also leaves the largest of its 64 logits, and the second launch
// finds from these which few groups of 64 can hold the row's largest and reads only those again.
//
// What bounds it: with bfloat16 logits the vector units as much as HBM -- 3.5 T logits a second at the rate of reads
// leave 11 issue slots for each, of which the exponential alone takes 4.  So the sums run without a pass for the maximum:
// any logit of the slice serves as the reference, as long as the sum is finite at the end.
#include "step_device.hpp"

namespace sdp4 {

namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int kMaxSlices = 256;  // of a row
constexpr int kMaxTop = SDP4_MAX_TOP;

// What a slice leaves of its row: S and T relative to `ref`, and its largest logit.
struct alignas(16) Slice {
    float ref, S, T, top;
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

// A lane's largest logit in a slice and the position (of its chunk, in the slice) where it first stands.  Of bfloat16
// order bits the upper 16 tell everything.
template <class T>
struct GroupKey;
template <>
struct GroupKey<bf16_t> {
    using Word = uint32_t;
    static constexpr int kValueBits = 16;
    SDP4_DEV static Word make(uint32_t order, uint32_t pos) { return (order & 0xFFFF0000u) | pos; }
    SDP4_DEV static uint32_t value(Word k) { return k >> 16; }
    SDP4_DEV static uint32_t pos(Word k) { return k & 0xFFFFu; }
    SDP4_DEV static uint32_t order(uint32_t value) { return value << 16 | (value & 0x8000u ? 0u : 0xFFFFu); }
};
template <>
struct GroupKey<float> {
    using Word = uint64_t;
    static constexpr int kValueBits = 32;
    SDP4_DEV static Word make(uint32_t order, uint32_t pos) { return (Word)order << 32 | pos; }
    SDP4_DEV static uint32_t value(Word k) { return (uint32_t)(k >> 32); }
    SDP4_DEV static uint32_t pos(Word k) { return (uint32_t)k; }
    SDP4_DEV static uint32_t order(uint32_t value) { return value; }
};

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

// Largest of a lane's values; NaN counts nothing.
template <class T, int NC>
SDP4_DEV float chunk_max(const u32x4 &raw)
{
    float v[kChunk<T>], m;
    unpack<T>(raw, v);
    m = v[0];
#pragma unroll
    for (int j = 1; j < kChunk<T>; ++j)
        m = fmaxf(m, v[j]);
    return m;
}

// S and T of the wave's `rounds` chunks per lane, relative to the `ref` it chooses (uniform over the wave).
//
// The quick way (`whole`: every chunk holds logits only) takes the largest of the first round as reference, so that
// every logit is seen once.  Where that does not do -- a logit of -inf, whose 0 * -inf spoils T, a reference that is
// not finite or far below the largest (T / S would cancel against log S), a type's lowest value, NaN -- the sums show
// it, and the wave goes over its registers again with the true maximum and a lower bound on the exponent.
template <class T, int NC>
SDP4_DEV void slice_sums(const u32x4 (&raw)[NC], int rounds, bool whole, float &ref, float &S, float &T2)
{
    constexpr int W = kChunk<T>;
    if (whole) {
        ref = max_wave(chunk_max<T, NC>(raw[0]));
        const float c = ref * kLog2e;
        S = T2 = 0.0f;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            if (i < rounds) {
                float v[W];
                unpack<T>(raw[i], v);
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    const float t = __builtin_fmaf(v[j], kLog2e, -c), e = exp2_of(t);
                    S += e;
                    T2 = __builtin_fmaf(e, t, T2);
                }
            }
        }
        S = sum_lanes(S, kWave);
        T2 = sum_lanes(T2, kWave);
        const float delta = __builtin_fmaf(ref, kLog2e, -c), f = exp2_of(-delta); // the rounding of c, taken out
        T2 = f * __builtin_fmaf(-delta, S, T2);
        S *= f;
        if (uniform((uint32_t)(S > 0.0f && S < 0x1p24f && T2 - T2 == 0.0f && __builtin_fabsf(ref) < 1e38f)))
            return;
    }
    float m = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < NC; ++i)
        if (i < rounds)
            m = fmaxf(m, chunk_max<T, NC>(raw[i]));
    m = max_wave(m);
    ref = m == -__builtin_inff() ? 0.0f : m;
    S = T2 = 0.0f;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        if (i < rounds) {
            float v[W];
            unpack<T>(raw[i], v);
#pragma unroll
            for (int j = 0; j < W; ++j) {
                const float t = (v[j] - ref) * kLog2e, e = exp2_of(t);
                S += e;
                T2 = __builtin_fmaf(e, fmaxf(t, -1000.0f), T2); // 2^-1000 is 0
            }
        }
    }
    S = sum_lanes(S, kWave);
    T2 = sum_lanes(T2, kWave);
}

// Joins N sums that a lane holds with those of the other lanes: relative to the largest reference of those that count.
template <int N>
SDP4_DEV void join_sums(const Slice (&s)[N], float &ref, float &S, float &T2)
{
    ref = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (s[i].S != 0.0f) // a slice without a finite logit counts nothing
            ref = fmaxf(ref, s[i].ref);
    ref = max_wave(ref);
    S = T2 = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (s[i].S != 0.0f) {
            const float d = (s[i].ref - ref) * kLog2e, f = exp2_of(d);
            S += s[i].S * f;
            T2 += f * (f == 0.0f ? 0.0f : __builtin_fmaf(s[i].S, d, s[i].T));
        }
    }
    S = sum_lanes(S, kWave);
    T2 = sum_lanes(T2, kWave);
}

// One slice per wave, four waves in a block: round i of a wave is 64 neighbouring chunks.
template <class T, int NC, bool TOP>
__global__ __launch_bounds__(256) void k_logprob_slices(Rows<const T *> x, int64_t rows, int64_t vocab,
                                                        Divisor slices, TokenStats out, Slice *stats,
                                                        typename GroupKey<T>::Word *keys)
{
    constexpr int W = kChunk<T>;
    const uint32_t wave = uniform(threadIdx.x / kWave), lane = lane_id();
    const uint64_t w = (uint64_t)work_block() * 4 + wave;
    uint64_t slice;
    const int64_t row = (int64_t)divide(w, slices, slice);
    if (row >= rows)
        return;
    const T *p = x.p + row * x.stride;
    const int64_t first = (int64_t)slice * (NC * kWave * W); // element of the row
    const int left = (int)(vocab - first < NC * kWave * W ? vocab - first : NC * kWave * W);
    const int rounds = (left + kWave * W - 1) / (kWave * W);
    const bool whole = left == NC * kWave * W;
    u32x4 raw[NC];
    if (whole) {
#pragma unroll
        for (int i = 0; i < NC; ++i)
            raw[i] = load_chunk<true>(p + first + (uint32_t)((i * kWave + lane) * W));
    } else {
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            if (i < rounds) {
                float v[W];
                const int64_t e = first + (i * kWave + (int)lane) * W;
                load_row(p, e < vocab ? e : 0, vocab, v);
                end_row(e, vocab, v, -__builtin_inff());
                raw[i] = pack<T>(v);
            }
        }
    }
    float ref, S, T2;
    slice_sums<T, NC>(raw, rounds, whole, ref, S, T2);

    float top = -__builtin_inff();
    if constexpr (TOP) {
        float cm[NC];
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            cm[i] = i < rounds ? chunk_max<T, NC>(raw[i]) : -__builtin_inff();
            top = fmaxf(top, cm[i]);
        }
        uint32_t pos = lane;
#pragma unroll
        for (int i = NC - 1; i >= 0; --i)
            if (cm[i] == top)
                pos = (uint32_t)i * kWave + lane;
        keys[w * kWave + lane] = GroupKey<T>::make(order_bits(top), pos);
        top = max_wave(top);
    }
    if (lane == 0) {
        if (!TOP && slices.d == 1) {
            const int64_t target = out.targets ? out.targets[row] : -1;
            finish_row(out, row, vocab, ref, S, T2, target >= 0 && target < vocab ? to_f32<T>(p[target]) : 0.0f, target);
        } else {
            stats[w] = Slice{ref, S, T2, top};
        }
    }
}

// The statistics of a row's slices, joined.  Returns the largest of each of the lane's slices.
template <class T, int N>
SDP4_DEV void join_row(const Rows<const T *> &x, int64_t row, int64_t vocab, int slices, const TokenStats &out,
                       const Slice *stats, float &ref, float &S, uint32_t (&tops)[N])
{
    const int lane = lane_id();
    const int64_t target = out.targets ? out.targets[row] : -1;
    const float tx = target >= 0 && target < vocab ? to_f32<T>(x.p[row * x.stride + target]) : 0.0f;
    Slice s[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        s[i] = Slice{0.0f, 0.0f, 0.0f, 0.0f};
        if (i * kWave + lane < slices)
            s[i] = stats[row * slices + i * kWave + lane];
        tops[i] = i * kWave + lane < slices ? order_bits(s[i].top) : 0u;
    }
    float T2;
    join_sums<N>(s, ref, S, T2);
    if (lane == 0)
        finish_row(out, row, vocab, ref, S, T2, tx, target);
}

template <class T>
__global__ __launch_bounds__(256) void k_logprob_join(Rows<const T *> x, int64_t rows, int64_t vocab, int slices,
                                                      TokenStats out, const Slice *stats)
{
    const int64_t row = work_block() * 4 + uniform(threadIdx.x / kWave);
    if (row >= rows)
        return;
    float ref, S;
    uint32_t tops[kMaxSlices / kWave];
    join_row<T>(x, row, vocab, slices, out, stats, ref, S, tops);
}

// The largest v with at least k of the lanes' N values >= v; unless EXACT, the first v on the way with exactly k of them.
template <int BITS, bool EXACT, int N>
SDP4_DEV uint32_t kth_largest(const uint32_t (&value)[N], int used, int k)
{
    uint32_t v = 0;
#pragma unroll 1
    for (int b = BITS - 1; b >= 0; --b) {
        const uint32_t mid = v | 1u << b;
        int n = 0;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < used)
                n += __builtin_popcountll(__ballot(value[i] >= mid));
        if (n >= k)
            v = mid;
        if (!EXACT && n == k)
            break;
    }
    return v;
}

// Joins the slices and finds the alternatives: one wave per row and block, up to K alternatives.
//
// Call a lane's logits of one slice a group.  The row's k largest logits lie in the k groups with the best largest logit
// (larger first, then earlier): each of these has one that is at least as good as any logit outside of them.  The same
// holds one step up, for the k slices with the best largest logit, where there are so many.  A bisection over the bits
// of the values, counting lanes, finds the k-th best slice (or group, with fewer slices); the groups from there up, k
// and a few more, are listed in LDS, and a group's place is the number of better ones.  Of the k best groups' logits
// (read again, k * NC chunks) those at least as good as the last one's largest are ranked in the same way.
template <class T, int NC, int K>
__global__ __launch_bounds__(64) void k_logprob_join_top(Rows<const T *> x, int64_t rows, int64_t vocab, int slices,
                                                         TokenStats out, const Slice *stats,
                                                         const typename GroupKey<T>::Word *keys)
{
    using Key = GroupKey<T>;
    constexpr int W = kChunk<T>, N = kMaxSlices / kWave, VB = Key::kValueBits;
    __shared__ uint16_t chosen[K];         // slices
    __shared__ uint32_t groups[K];         // slice << 6 | lane of the k best
    __shared__ uint64_t list[K * kWave];   // groups, or logits of k groups
    __shared__ uint16_t where[K * kWave];  // of listed groups: place in `chosen` << 6 | lane
    __shared__ uint32_t listed;
    static_assert(NC * W <= kWave, "logits of a group");
    const int lane = lane_id(), k = out.top_k;
    const int64_t row = work_block();
    if (row >= rows)
        return;
    const uint64_t below = (uint64_t(1) << lane) - 1;
    if (lane == 0)
        listed = 0;
    float ref, S;
    uint32_t tops[N];
    join_row<T>(x, row, vocab, slices, out, stats, ref, S, tops);

    // slices whose groups count, in order
    int count = slices;
    uint32_t tau = 0; // groups below it do not count
    if (slices >= k) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            tops[i] >>= 32 - VB;
        tau = kth_largest<VB, true>(tops, (slices + kWave - 1) / kWave, k);
        int above = 0;
#pragma unroll
        for (int i = 0; i < N; ++i)
            above += __builtin_popcountll(__ballot(tops[i] > tau));
        int equal = k - above; // of those at tau the first so many
        count = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const bool tie = tops[i] == tau && i * kWave + lane < slices;
            const uint64_t eq = __ballot(tie);
            const bool take = tops[i] > tau || (tie && __builtin_popcountll(eq & below) < equal);
            equal -= __builtin_popcountll(eq);
            const uint64_t all = __ballot(take);
            if (take)
                chosen[count + __builtin_popcountll(all & below)] = (uint16_t)(i * kWave + lane);
            count += __builtin_popcountll(all);
        }
    } else if (lane < count) {
        chosen[lane] = (uint16_t)lane;
    }
    wave_lds_sync();

    uint32_t value[K], pos[K];
#pragma unroll
    for (int r = 0; r < K; ++r) {
        if (r < count) {
            const typename Key::Word w = keys[(row * slices + chosen[r]) * kWave + lane];
            value[r] = Key::value(w), pos[r] = Key::pos(w);
        }
    }
    if (slices < k)
        tau = kth_largest<VB, false>(value, count, k);
    int above = 0;
#pragma unroll
    for (int r = 0; r < K; ++r)
        if (r < count)
            above += __builtin_popcountll(__ballot(value[r] > tau));
    int equal = k - above, n = 0; // of the groups at tau the first `equal` may be needed: slices in order, positions in a slice
#pragma unroll
    for (int r = 0; r < K; ++r) {
        if (r < count) {
            const bool tie = value[r] == tau && equal > 0;
            const int ties = __builtin_popcountll(__ballot(tie));
            uint32_t limit = ~0u; // positions below it are taken
            if (ties > equal && equal > 0) {
                limit = 0;
#pragma unroll 1
                for (int b = 15; b >= 0; --b) {
                    const uint32_t mid = limit | 1u << b;
                    if (__builtin_popcountll(__ballot(tie && pos[r] < mid)) <= equal)
                        limit = mid;
                }
            }
            const bool tie_taken = tie && pos[r] < limit;
            equal -= __builtin_popcountll(__ballot(tie_taken));
            const bool take = value[r] > tau || tie_taken;
            const uint64_t all = __ballot(take);
            if (take) {
                const int at = n + __builtin_popcountll(all & below);
                list[at] = (uint64_t)value[r] << 32 | (uint32_t)~(r << 16 | pos[r]);
                where[at] = (uint16_t)(r << 6 | lane);
            }
            n += __builtin_popcountll(all);
        }
    }
    wave_lds_sync();
    // the k best of them, and the k-th: from its value on, and at its value up to its chunk, a logit counts
    uint64_t kth = 0;
    for (int a = lane; a < n; a += kWave) {
        const uint64_t mine = list[a];
        int rank = 0;
        for (int o = 0; o < n; ++o)
            rank += list[o] > mine;
        if (rank < k)
            groups[rank] = (uint32_t)chosen[where[a] >> 6] << 6 | (where[a] & 63u);
        if (rank == k - 1)
            kth = mine;
    }
    const uint64_t has = __ballot(kth != 0);
    const int found = n < k ? n : k;
    const int from = has ? __builtin_ctzll(has) : 0;
    const uint32_t kth_value = __builtin_amdgcn_readlane((uint32_t)(kth >> 32), from);
    const uint32_t kth_place = ~(uint32_t)__builtin_amdgcn_readlane((uint32_t)kth, from);
    const float least = from_order_bits(Key::order(kth_value));
    const int64_t last = has ? (int64_t)chosen[(kth_place >> 16) & (K - 1)] * (NC * kWave) + (kth_place & 0xFFFFu) : 0;
    wave_lds_sync();

    const T *p = x.p + row * x.stride;
    const int64_t chunks = (vocab + W - 1) / W;
    for (int c = lane; c < found * NC; c += kWave) {
        const uint32_t g = groups[c / NC];
        const int64_t chunk = (int64_t)(g >> 6) * (NC * kWave) + (c % NC) * kWave + (g & 63u);
        if (chunk >= chunks)
            continue;
        const int64_t e = chunk * W;
        float v[W];
        load_row(p, e, vocab, v);
        end_row(e, vocab, v, -__builtin_inff());
#pragma unroll
        for (int j = 0; j < W; ++j)
            if (e + j < vocab && (v[j] > least || (v[j] == least && chunk <= last)))
                list[atomicAdd(&listed, 1u)] = entry_of(v[j], (uint32_t)(e + j));
    }
    wave_lds_sync();
    n = (int)uniform(listed);
    const bool bad = !(S - S == 0.0f);
    for (int a = lane; a < (n > k ? n : k); a += kWave) {
        const uint64_t mine = a < n ? list[a] : 0;
        int rank = a;
        if (a < n) {
            rank = 0;
            for (int o = 0; o < n; ++o)
                rank += list[o] > mine;
        }
        if (rank < k) {
            const int64_t at = row * k + rank;
            const float v = S == 0.0f ? -__builtin_inff() : (from_order_bits((uint32_t)(mine >> 32)) - ref) - kLn2 * log2_of(S);
            out.top_logp[at] = bad ? __builtin_nanf("") : v;
            out.top_ids[at] = bad ? -1 : (int64_t)entry_index(mine);
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
    int target;           // -W or less: none
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
    r.target = target >= 0 && target < vocab && !empty ? (int)target : -1024;
    if (empty && target < vocab)
        r.A = r.B = 0.0f;
    if (!(lse == lse))
        r.A = lse;
    return r;
}

// Gradient of the W elements of a chunk that starts at element e of the row; zeros from vocab on (WHOLE: it ends before).
template <int W, bool ENT, bool WHOLE, class X>
SDP4_DEV void grad_chunk(const RowGrad &g, X exponent, float delta, int e, int vocab, float (&v)[W])
{
#pragma unroll
    for (int j = 0; j < W; ++j) {
        const float t = exponent(v[j]), p = exp2_of(t);
        if constexpr (ENT)
            v[j] = p * __builtin_fmaf(g.B, fmaxf(t, -1000.0f) - delta, g.A);
        else
            v[j] = p * g.A;
    }
    const uint32_t at = (uint32_t)(g.target - e);
    if (at < (uint32_t)W) {
#pragma unroll
        for (int j = 0; j < W; ++j)
            v[j] += at == (uint32_t)j ? g.hit : 0.0f;
    }
    if (!WHOLE && e + W > vocab) {
#pragma unroll
        for (int j = 0; j < W; ++j)
            v[j] = e + j < vocab ? v[j] : 0.0f;
    }
}

// A wave takes U * 64 chunks of one row.
template <class T, int U, bool ENT>
__global__ __launch_bounds__(256) void k_logprob_grad(Rows<const T *> x, int64_t rows, int64_t vocab64,
                                                      const int64_t *targets, const float *lse, const float *entropy,
                                                      TokenGrads g, Rows<T *> dx, int64_t width64, Divisor tiles)
{
    constexpr int W = kChunk<T>;
    const int vocab = (int)vocab64, width = (int)width64; // below 2^31 with the lanes beyond them
    const uint32_t wave = uniform(threadIdx.x / kWave);
    const uint64_t w = (uint64_t)work_block() * 4 + wave;
    uint64_t tile;
    const int64_t row = (int64_t)divide(w, tiles, tile);
    if (row >= rows)
        return;
    const T *p = x.p + row * x.stride;
    T *q = dx.p + row * dx.stride;
    const int64_t start = (int64_t)tile * (U * kWave * W);
    const bool whole = start + U * kWave * W <= vocab;
    const int64_t at = start + lane_id() * W;
    float v[U][W];
    if (whole) {
#pragma unroll
        for (int i = 0; i < U; ++i)
            load_whole(p + start + (uint32_t)(lane_id() * W + i * (kWave * W)), v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int64_t e = at + i * (kWave * W);
            load_row(p, e < vocab ? e : 0, vocab, v[i]);
            end_row(e, vocab, v[i]);
        }
    }
    const RowGrad rg = row_grad(lse[row], ENT ? entropy[row] : 0.0f, targets ? targets[row] : -1, vocab,
                                g.logp ? g.logp[row] : 0.0f, ENT ? g.entropy[row] : 0.0f, g.lse ? g.lse[row] : 0.0f);
    with_exponent(rg.ref, 0.0f, [&](auto exponent, float delta) {
        const float f = exp2_of(-delta);
        RowGrad s = rg;
        s.A *= f, s.B *= f;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int64_t e = at + i * (kWave * W);
            if (whole) {
                grad_chunk<W, ENT, true>(s, exponent, delta, (int)e, vocab, v[i]);
                store_elems(q + start + (uint32_t)(lane_id() * W + i * (kWave * W)), W, v[i]);
            } else if (e < width) {
                grad_chunk<W, ENT, false>(s, exponent, delta, (int)e, vocab, v[i]);
                store_elems(q + e, width - e, v[i]);
            }
        }
    });
}

// The loss and its gradient: a block holds a whole row in registers, so the logits are read once.  Each wave sums up its
// own part, the parts are joined through LDS, and with the row's statistics every lane turns what it holds into the
// gradient.
template <class T, int WAVES, int NC, bool ENT>
__global__ __launch_bounds__(64 * WAVES) void k_token_loss(Rows<const T *> x, int64_t rows, int64_t vocab64,
                                                           TokenStats out, TokenGrads g, Rows<T *> dx, int64_t width64)
{
    constexpr int W = kChunk<T>, STEP = kWave * WAVES * W;
    __shared__ Slice red[WAVES];
    const int64_t row = work_block();
    if (row >= rows)
        return;
    const int vocab = (int)vocab64, width = (int)width64; // below 2^20, and a row's registers
    const int wave = (int)uniform(threadIdx.x / kWave), lane = lane_id();
    const T *p = x.p + row * x.stride;
    T *q = dx.p + row * dx.stride;
    const int64_t target = out.targets ? out.targets[row] : -1;
    const float g_logp = g.logp ? g.logp[row] : 0.0f, g_ent = ENT ? g.entropy[row] : 0.0f,
                g_lse = g.lse ? g.lse[row] : 0.0f;
    const float tx = target >= 0 && target < vocab ? to_f32<T>(p[target]) : 0.0f;
    // round i of the wave: 64 chunks from element start + i * STEP on
    const int start = wave * (kWave * W), at = start + lane * W;
    const int rounds = start < vocab ? (vocab - start + STEP - 1) / STEP : 0;
    const int full = start + kWave * W <= vocab ? (vocab - start - kWave * W) / STEP + 1 : 0; // whole rounds
    u32x4 raw[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        if (i < full) {
            raw[i] = load_chunk<true>(p + (uint32_t)(at + i * STEP));
        } else if (i < rounds) {
            float v[W];
            const int e = at + i * STEP;
            load_row(p, e < vocab ? e : 0, vocab, v);
            end_row(e, vocab, v, -__builtin_inff());
            raw[i] = pack<T>(v);
        }
    }
    Slice s{0.0f, 0.0f, 0.0f, 0.0f};
    if (rounds)
        slice_sums<T, NC>(raw, rounds, full == rounds, s.ref, s.S, s.T);
    float ref = s.ref, S = s.S, T2 = s.T;
    if constexpr (WAVES > 1) {
        if (lane == 0)
            red[wave] = s;
        __syncthreads();
        Slice part[1] = {lane < WAVES ? red[lane] : Slice{0.0f, 0.0f, 0.0f, 0.0f}};
        join_sums<1>(part, ref, S, T2);
    }
    if (threadIdx.x == 0)
        finish_row(out, row, vocab, ref, S, T2, tx, target);
    const bool empty = S == 0.0f;
    const float lg = empty ? 0.0f : log2_of(S), ln_s = kLn2 * lg;
    const float lse = empty ? -__builtin_inff() : ref + ln_s;
    const float ent = ENT ? (empty ? 0.0f : fmaxf(ln_s - kLn2 * (T2 / S), 0.0f) + (S - S)) : 0.0f;
    const RowGrad rg = row_grad(lse, ent, target, vocab, g_logp, g_ent, g_lse);
    // from the reference and log2 S rather than from their rounded sum
    with_exponent(empty ? 0.0f : ref, lg, [&](auto exponent, float delta) {
        const float f = exp2_of(-delta);
        RowGrad s = rg;
        s.A *= f, s.B *= f;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int e = at + i * STEP;
            if (i < full) {
                float v[W];
                unpack<T>(raw[i], v);
                grad_chunk<W, ENT, true>(s, exponent, delta, e, vocab, v);
                store_chunk<T>(q + (uint32_t)e, pack<T>(v));
            } else if (e < width) {
                float v[W];
                unpack<T>(raw[i], v); // nothing of it counts from vocab on
                grad_chunk<W, ENT, false>(s, exponent, delta, e, vocab, v);
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

// How a row is cut into slices of 64 * nc chunks: the largest that still give 2048 waves, and no more than 64 if that
// can be.
struct Cut {
    int nc;
    int64_t slices;
};
template <class T>
Cut cut_rows(int64_t rows, int64_t vocab)
{
    constexpr int most = sizeof(T) == 2 ? 8 : 16; // 4096 logits
    const int64_t chunks = (vocab + kChunk<T> - 1) / kChunk<T>;
    const auto slices = [&](int n) { return (chunks + 64 * n - 1) / (64 * n); };
    int nc = 1;
    while (nc < most && slices(nc) > 1 && (slices(nc) > kWave || rows * slices(2 * nc) >= 2048))
        nc *= 2;
    return {nc, slices(nc)};
}
static_assert(kMaxSlices * 4096 >= SDP4_MAX_VOCAB, "slices of a row");

template <class T, class F>
int with_chunks(int nc, F run)
{
    using std::integral_constant;
    if constexpr (sizeof(T) == 4)
        if (nc == 16)
            return run(integral_constant<int, 16>{});
    return nc == 1   ? run(integral_constant<int, 1>{})
           : nc == 2 ? run(integral_constant<int, 2>{})
           : nc == 4 ? run(integral_constant<int, 4>{})
                     : run(integral_constant<int, 8>{});
}

template <class T>
int logprob(Rows<const void *> x, int64_t rows, int64_t vocab, const TokenStats &out, void *workspace, hipStream_t s)
{
    using Word = typename GroupKey<T>::Word;
    const Cut c = cut_rows<T>(rows, vocab);
    Slice *stats = static_cast<Slice *>(workspace);
    Word *keys = reinterpret_cast<Word *>(stats + rows * c.slices);
    return with_chunks<T>(c.nc, [&](auto chunks) {
        constexpr int NC = decltype(chunks)::value;
        auto k = out.top_k ? k_logprob_slices<T, NC, true> : k_logprob_slices<T, NC, false>;
        const int rc = launch<4>(k, (rows * c.slices + 3) / 4, kUncapped, s, typed<const T>(x), rows, vocab,
                                 Divisor((uint64_t)c.slices), out, stats, keys);
        if (rc || (c.slices == 1 && !out.top_k))
            return rc;
        if (out.top_k)
            return launch<1>(out.top_k <= 8 ? k_logprob_join_top<T, NC, 8> : k_logprob_join_top<T, NC, kMaxTop>, rows,
                             kUncapped, s, typed<const T>(x), rows, vocab, (int)c.slices, out, stats, keys);
        return launch<4>(k_logprob_join<T>, (rows + 3) / 4, kUncapped, s, typed<const T>(x), rows, vocab,
                         (int)c.slices, out, stats);
    });
}

template <class T>
int64_t workspace_of(int64_t rows, int64_t vocab, int top_k)
{
    const Cut c = cut_rows<T>(rows, vocab);
    if (c.slices == 1 && !top_k)
        return 0;
    return rows * c.slices * (int64_t)(sizeof(Slice) + (top_k ? kWave * sizeof(typename GroupKey<T>::Word) : 0));
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
    using std::integral_constant;
    if (chunks <= 256)
        return run(integral_constant<int, 1>{}, integral_constant<int, 4>{});
    if (chunks <= 1024)
        return run(integral_constant<int, 4>{}, integral_constant<int, 4>{});
    if (chunks <= 2048)
        return run(integral_constant<int, 4>{}, integral_constant<int, 8>{});
    if (chunks <= 4096)
        return run(integral_constant<int, 8>{}, integral_constant<int, 8>{});
    if (chunks <= 6656)
        return run(integral_constant<int, 8>{}, integral_constant<int, 13>{});
    if (chunks <= 8192)
        return run(integral_constant<int, 16>{}, integral_constant<int, 8>{});
    if (chunks <= 16384)
        return run(integral_constant<int, 16>{}, integral_constant<int, 16>{});
    const int rc = logprob<T>(x, rows, vocab, out, workspace, s);
    return rc ? rc : logprob_grad<T, ENT>(x, rows, vocab, out.targets, out.lse, out.entropy, g, dx, width, s);
}

} // namespace

int64_t token_logprob_workspace(int64_t rows, int64_t vocab, int top_k)
{
    if (rows <= 0 || vocab <= 0)
        return 0;
    const int64_t a = workspace_of<bf16_t>(rows, vocab, top_k), b = workspace_of<float>(rows, vocab, top_k);
    return a > b ? a : b; // for either type
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
