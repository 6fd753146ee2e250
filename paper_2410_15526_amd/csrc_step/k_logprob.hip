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
// finished by its wave, unless alternatives are wanted.  For these each lane also leaves the largest of its 64 logits, and the
// second launch finds from them which few groups of 64 can hold the row's largest and reads only those again.
//
// What bounds it: HBM (4096 x 50001 bfloat16 without alternatives 65 us, 6.3 TB/s, float32 122, 6.7), and with bfloat16
// nearly the vector units too: at the rate of reads 3.5 T logits a second leave 11 issue slots for each, and the kernel
// takes 10 where it looks for alternatives, 71 us.  So the sums run without a pass for the maximum (the form with one took
// 78 us without alternatives): a logit of the slice serves as the reference, as long as the likely ones are not far above it.
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

// A lane's largest logit in a slice (its order bits; of bfloat16 the upper 16 tell everything), the round `at` in which it
// first stands, and an upper bound of the largest logit of the lane's other rounds.
template <class T>
struct GroupKey {
    static constexpr int kValueBits = sizeof(T) == 2 ? 16 : 32, kRestBits = sizeof(T) == 2 ? 12 : 28;
    using Word = std::conditional_t<sizeof(T) == 2, uint32_t, uint64_t>;
    SDP4_DEV static Word make(float top, uint32_t at, float rest)
    {
        return (Word)(order_bits(top) >> (32 - kValueBits)) << kValueBits | (Word)(order_bits(rest) >> (32 - kRestBits)) << 4 | at;
    }
    SDP4_DEV static uint32_t value(Word k) { return (uint32_t)(k >> kValueBits); }
    SDP4_DEV static uint32_t at(Word k) { return (uint32_t)k & 15u; }
    // order bits that no other logit of the group exceeds
    SDP4_DEV static uint32_t rest(Word k)
    {
        const uint32_t r = (uint32_t)(k >> 4) << (32 - kRestBits);
        return r | ((1u << (32 - kRestBits)) - 1);
    }
    SDP4_DEV static uint32_t order(uint32_t value)
    {
        return sizeof(T) == 2 ? value << 16 | (value & 0x8000u ? 0u : 0xFFFFu) : value;
    }
};

SDP4_DEV float exp2_of(float t) { return __builtin_amdgcn_exp2f(t); }
SDP4_DEV float log2_of(float s) { return __builtin_amdgcn_logf(s); }

// Largest reference for t = (x - ref) log2 e as one fma x log2 e - c with c = ref log2 e rounded: every t is off by that
// rounding, at most 2^-4 up to here, which is known and taken out.  It grows with ref, past the exponents of float32 from 3e9
// on.  Larger references take a subtraction and a product, which loses nothing: what is near such a reference differs from it
// exactly, and the rest has no share.
constexpr float kOneFma = 0x1p20f;

// Calls body(exponent, delta) with t(x) = (x - ref) log2 e - lg: one fma, whose constant's rounding error the caller
// takes out again by `delta` (t is too large by it), or, for larger references, a subtraction and an fma.
template <class F>
SDP4_DEV void with_exponent(float ref, float lg, F body)
{
    if (__builtin_fabsf(ref) < kOneFma) {
        const float c = __builtin_fmaf(ref, kLog2e, lg);
        body([=](float x) { return __builtin_fmaf(x, kLog2e, -c); }, __builtin_fmaf(ref, kLog2e, -c) + lg);
    } else {
        body([=](float x) { return __builtin_fmaf(x - ref, kLog2e, -lg); }, 0.0f);
    }
}

// Log probability of logit x.  Its terms' roundings may leave that of a certain token above 0, and no caller expects that;
// NaN stays.
SDP4_DEV float log_prob(float x, float ref, float ln_s)
{
    const float v = (x - ref) - ln_s;
    return v > 0.0f ? 0.0f : v;
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
            v = empty ? -__builtin_inff() : log_prob(target_x, m, ln_s);
        out.logp[row] = v;
    }
}

// Largest of a lane's values; NaN counts nothing.
template <class T>
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

// A wave's part of a row in registers: `full` chunks of each lane that hold logits only, and where the row ends in the
// wave's next round, that round as `tail`, with -inf behind the end.
//
// `lead`: bfloat16 rows at an odd element address are read in chunks from one element earlier on, which start at whole
// words: a burst of 16-byte loads at half words takes the loss of 8192 x 50001 from 290 to 340 us.  Element -1 of the row
// (in the same word as element 0) is replaced by a copy of element 0, whose share the sums take out again.
template <class T, int NC>
struct Held {
    static constexpr int W = kChunk<T>;
    u32x4 raw[NC], tail;
    int full, lead;
    bool has_tail, copied; // copied: the first lane's first chunk begins with the copy

    SDP4_DEV static int lead_of(const T *row, int vocab)
    {
        return sizeof(T) == 2 && vocab >= kWave * W && ((uintptr_t)row & 2) ? 1 : 0;
    }
    // Round i is the 64 chunks from element start + i * STEP - lead of the row on; at most `most` rounds.
    template <int STEP>
    SDP4_DEV void load(const T *row, int start, int most, int vocab, int lead_ = 0)
    {
        const int lane = lane_id(), ends = vocab + lead_;
        lead = lead_;
        full = start + kWave * W <= ends ? (ends - start - kWave * W) / STEP + 1 : 0;
        full = full < most ? full : most;
        has_tail = full < most && start + full * STEP < ends;
        copied = lead > 0 && start == 0;
        const T *p = row - lead;
#pragma unroll
        for (int i = 0; i < NC; ++i)
            if (i < full)
                raw[i] = load_chunk<true>(p + (uint32_t)(start + i * STEP + lane * W));
        tail = u32x4{0u, 0u, 0u, 0u};
        if (has_tail) {
            float v[W];
            const int e = start + full * STEP + lane * W - lead;
            load_row(row, e < vocab ? e : 0, vocab, v);
            end_row(e, vocab, v, -__builtin_inff());
            tail = pack<T>(v);
        }
        if (copied && lane == 0)
            raw[0].x = (raw[0].x & 0xFFFF0000u) | raw[0].x >> 16;
    }
    SDP4_DEV bool any() const { return full > 0 || has_tail; }
    // the copied element's value, in the lane that holds it; elsewhere -inf
    SDP4_DEV float copy() const { return copied && lane_id() == 0 ? to_f32<bf16_t>((bf16_t)raw[0].x) : -__builtin_inff(); }
};

// Sums of one chunk relative to `ref`; -inf counts nothing (2^-1000 is 0).
template <class T>
SDP4_DEV void add_guarded(const u32x4 &raw, float ref, float &S, float &T2)
{
    float v[kChunk<T>];
    unpack<T>(raw, v);
#pragma unroll
    for (int j = 0; j < kChunk<T>; ++j) {
        const float t = (v[j] - ref) * kLog2e, e = exp2_of(t);
        S += e;
        T2 = __builtin_fmaf(e, fmaxf(t, -1000.0f), T2);
    }
}

// The share of one logit, taken out of the sums.
SDP4_DEV void take_out(float x, float ref, float &S, float &T2)
{
    const float t = (x - ref) * kLog2e, e = exp2_of(t);
    S -= e;
    T2 = __builtin_fmaf(-e, fmaxf(t, -1000.0f), T2);
}

// A lane's largest logit, the round it first stands in, and the largest of its other rounds.
struct LaneTop {
    float top, rest;
    uint32_t at;
    SDP4_DEV void add(float m, int round)
    {
        rest = fmaxf(rest, fminf(top, m));
        at = m > top ? (uint32_t)round : at;
        top = fmaxf(top, m);
    }
};

// S and T of what the wave holds, relative to the `ref` it chooses (uniform over the wave), and with TOP each lane's top.
//
// The quick way takes the largest of the first round as reference, so that every logit is seen once.  Where that does not
// do -- a logit of -inf, whose 0 * -inf spoils T, a reference that is large (its exponents carry the rounding of c) or not
// finite, a type's lowest value, NaN, or likely logits so far above the reference that T / S cancels against log S and log S
// against the target's logit -- the sums or the reference show it, and the wave goes over its registers again with the true
// maximum and a lower bound on the exponent.  T / S is the mean exponent: up to 4, the mean |t| is at most 4 + 2 H / ln 2,
// since a logit below the reference has |t| <= - log2 p, and log2 S at most 4 + H / ln 2, so four octaves are all that cancels.
// Worst errors over rows with one token 0 to 40 above 4096 others, logp and entropy: 2.3e-6 and 2.3e-6, the same for a limit of
// 1, which costs 1.5 % of 4096 x 50001 in bfloat16; with S < 2^24 alone, 24 octaves, 3.7e-6 and 2.6e-5.
template <bool TOP, class T, int NC>
SDP4_DEV void slice_sums(const Held<T, NC> &h, float &ref, float &S, float &T2, LaneTop &lt)
{
    constexpr int W = kChunk<T>;
    lt = LaneTop{-__builtin_inff(), -__builtin_inff(), 0u}; // where nothing is larger than -inf, the first round
    const float tail_max = h.has_tail ? chunk_max<T>(h.tail) : -__builtin_inff();
    ref = max_wave(h.full ? chunk_max<T>(h.raw[0]) : tail_max);
    const float c = ref * kLog2e;
    S = T2 = 0.0f;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        if (i < h.full) {
            float v[W];
            unpack<T>(h.raw[i], v);
            if constexpr (TOP) {
                float m = v[0];
#pragma unroll
                for (int j = 1; j < W; ++j)
                    m = fmaxf(m, v[j]);
                lt.add(m, i);
            }
#pragma unroll
            for (int j = 0; j < W; ++j) {
                const float t = __builtin_fmaf(v[j], kLog2e, -c), e = exp2_of(t);
                S += e;
                T2 = __builtin_fmaf(e, t, T2);
            }
        }
    }
    const float delta = __builtin_fmaf(ref, kLog2e, -c), f = exp2_of(-delta); // the rounding of c, taken out
    T2 = f * __builtin_fmaf(-delta, S, T2);
    S *= f;
    if (h.has_tail) {
        add_guarded<T>(h.tail, ref, S, T2);
        if constexpr (TOP)
            lt.add(tail_max, h.full);
    }
    if (h.copied)
        take_out(h.copy(), ref, S, T2);
    S = sum_lanes(S, kWave);
    T2 = sum_lanes(T2, kWave);
    if (uniform((uint32_t)(S > 0.0f && T2 <= 4.0f * S && T2 - T2 == 0.0f && __builtin_fabsf(ref) < kOneFma)))
        return;
    float m = tail_max;
#pragma unroll
    for (int i = 0; i < NC; ++i)
        if (i < h.full)
            m = fmaxf(m, chunk_max<T>(h.raw[i]));
    m = max_wave(m);
    ref = m == -__builtin_inff() ? 0.0f : m;
    S = T2 = 0.0f;
#pragma unroll
    for (int i = 0; i < NC; ++i)
        if (i < h.full)
            add_guarded<T>(h.raw[i], ref, S, T2);
    if (h.has_tail)
        add_guarded<T>(h.tail, ref, S, T2);
    if (h.copied)
        take_out(h.copy(), ref, S, T2);
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

// What a slice leaves: its sums and, with TOP, its largest logit and the lane's key.
template <bool TOP, class T, int NC>
SDP4_DEV Slice take_slice(const Held<T, NC> &h, typename GroupKey<T>::Word &key)
{
    float ref, S, T2;
    LaneTop lt;
    slice_sums<TOP>(h, ref, S, T2, lt);
    float top = -__builtin_inff();
    if constexpr (TOP) {
        key = GroupKey<T>::make(lt.top, lt.at, lt.rest);
        top = max_wave(lt.top);
    }
    return Slice{ref, S, T2, top};
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
    Held<T, NC> h;
    h.template load<kWave * W>(p, (int)slice * (NC * kWave * W), NC, (int)vocab);
    typename GroupKey<T>::Word key;
    const Slice s = take_slice<TOP>(h, key);
    if constexpr (TOP && sizeof(key) == 8) // 3 % of what a float32 slice moves: past the caches (4096 x 50001, 160 / 154 us)
        __builtin_nontemporal_store(key, keys + w * kWave + lane);
    else if constexpr (TOP)
        keys[w * kWave + lane] = key;
    if (lane == 0) {
        if (!TOP && slices.d == 1) {
            const int64_t target = out.targets ? out.targets[row] : -1;
            finish_row(out, row, vocab, s.ref, s.S, s.T, target >= 0 && target < vocab ? to_f32<T>(p[target]) : 0.0f, target);
        } else {
            stats[w] = s;
        }
    }
}

// What a wave reads of a row's slices, slice i * 64 + lane each, and of its target.
template <class T, int N>
struct RowSlices {
    Slice s[N];
    int64_t target;
    float target_x;
    SDP4_DEV void load(const T *p, int64_t row, int64_t vocab, int slices, const TokenStats &out, const Slice *stats)
    {
        const int lane = lane_id();
        target = out.targets ? out.targets[row] : -1;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            s[i] = Slice{0.0f, 0.0f, 0.0f, -__builtin_inff()};
            if (i * kWave + lane < slices)
                s[i] = stats[i * kWave + lane];
        }
        target_x = target >= 0 && target < vocab ? to_f32<T>(p[target]) : 0.0f;
    }
    SDP4_DEV void finish(int64_t row, int64_t vocab, const TokenStats &out, float &ref, float &S) const
    {
        float T2;
        join_sums<N>(s, ref, S, T2);
        if (lane_id() == 0)
            finish_row(out, row, vocab, ref, S, T2, target_x, target);
    }
};

template <class T, int N> // N * 64 slices or fewer
__global__ __launch_bounds__(256) void k_logprob_join(Rows<const T *> x, int64_t rows, int64_t vocab, int slices,
                                                      TokenStats out, const Slice *stats)
{
    const int64_t row = work_block() * 4 + uniform(threadIdx.x / kWave);
    if (row >= rows)
        return;
    RowSlices<T, N> r;
    float ref, S;
    r.load(x.p + row * x.stride, row, vocab, slices, out, stats + row * slices);
    r.finish(row, vocab, out, ref, S);
}

// The largest v in [low, high], which hold it, with at least k of the lanes' values >= v: value(i), i < used <= N.  Found
// bit by bit from the first in which low and high differ, counting lanes.
template <int N, class V>
SDP4_DEV uint32_t kth_largest(uint32_t low, uint32_t high, int used, int k, V value)
{
    if (low == high)
        return low;
    int b = 31 - __builtin_clz(low ^ high);
    uint32_t v = low & ~((2u << b) - 1);
#pragma unroll 1
    for (; b >= 0; --b) {
        const uint32_t mid = v | 1u << b;
        int n = 0;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < used)
                n += __builtin_popcountll(__ballot(value(i) >= mid));
        if (n >= k)
            v = mid;
    }
    return v;
}

SDP4_DEV uint32_t max_wave(uint32_t v)
{
    v = max(v, dpp_u32<kDppXor1>(v));
    v = max(v, dpp_u32<kDppXor2>(v));
    v = max(v, dpp_u32<kDppHalfMirror>(v));
    v = max(v, dpp_u32<kDppRor8>(v));
    v = max(v, (uint32_t)__builtin_amdgcn_ds_swizzle((int)v, (16 << 10) | 0x1F));
    v = max(v, (uint32_t)__builtin_amdgcn_ds_bpermute((lane_id() ^ 32) << 2, (int)v));
    return uniform(v);
}

// Joins the slices and finds the alternatives: one wave per row and block, up to K alternatives.
//
// Call a lane's logits of one slice a group.  The row's k largest logits lie in the k groups with the best largest logit
// (larger first, then earlier): each of these has one that is at least as good as any logit outside of them.  The same
// holds one step up, for the k slices with the best largest logit.  Of the k groups' logits (read
// again: of most groups one chunk, as what its others hold is known to be less) those at least as good as the k-th best
// group's largest, k and a few more, are listed in LDS, and each one's place is the number of better ones.
//
// A row is a chain of reads from memory (slices, keys, chunks) with some 560 dependent vector instructions of one wave
// between them: 8 us for few rows, 11 for 4096 with 5 alternatives.  (Alternatives chosen in the slices themselves and
// joined here took 118 us in all for 4096 x 50001 and k = 5, 186 for 20, against 82 and 95.  A block for each row with its
// waves as the slices saves this launch and loses more by waves that wait: 94, without alternatives 83 against 65.)
constexpr int kListed = 256;
template <class T, int NC, int K, int N>
__global__ __launch_bounds__(64) void k_logprob_join_top(Rows<const T *> x, int64_t rows, int64_t vocab, int slices,
                                                         TokenStats out, const Slice *stats,
                                                         const typename GroupKey<T>::Word *keys)
{
    using Key = GroupKey<T>;
    constexpr int W = kChunk<T>, VB = Key::kValueBits;
    __shared__ uint16_t chosen[K];     // slices
    __shared__ uint64_t groups[K];     // bound of all but one round, then slice << 16 | chunk of the slice with the largest
    __shared__ uint64_t list[kListed]; // logits
    __shared__ uint32_t reads[K * NC]; // chunks of the row
    const int lane = lane_id(), k = out.top_k;
    const int64_t row = work_block();
    if (row >= rows)
        return;
    const uint64_t below = (uint64_t(1) << lane) - 1;
    stats += row * slices;
    keys += row * slices * kWave;
    const T *p = x.p + row * x.stride;
    RowSlices<T, N> rs;
    rs.load(p, row, vocab, slices, out, stats);

    // slices whose groups count, in order; the best group's largest, and a bound that k groups reach
    uint32_t tops[N], high = 0, low = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        tops[i] = i * kWave + lane < slices ? order_bits(rs.s[i].top) >> (32 - VB) : 0u;
        high = max(high, tops[i]);
    }
    high = max_wave(high);
    int count = slices;
    if (slices >= k)
        low = kth_largest<N>(0, high, (slices + kWave - 1) / kWave, k, [&](int i) { return tops[i]; });
    {
        int equal = slices; // of those at `low` the first so many
        if (slices >= k) {
            equal = k;
#pragma unroll
            for (int i = 0; i < N; ++i)
                equal -= __builtin_popcountll(__ballot(tops[i] > low));
        }
        count = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const bool is = i * kWave + lane < slices, tie = is && (tops[i] == low || slices < k);
            const uint64_t eq = __ballot(tie);
            const bool take = (is && tops[i] > low) || (tie && __builtin_popcountll(eq & below) < equal);
            equal -= __builtin_popcountll(eq);
            const uint64_t all = __ballot(take);
            if (take)
                chosen[count + __builtin_popcountll(all & below)] = (uint16_t)(i * kWave + lane);
            count += __builtin_popcountll(all);
        }
    }
    wave_lds_sync();
    typename Key::Word key[K];
#pragma unroll
    for (int r = 0; r < K; ++r)
        if (r < count)
            key[r] = keys[(int)chosen[r] * kWave + lane];
    float ref, S;
    rs.finish(row, vocab, out, ref, S); // while the keys come

    // the k best groups: those above tau, and of those at tau the first -- slices in order, positions in a slice
    const uint32_t tau = kth_largest<K>(low, high, count, k, [&](int r) { return Key::value(key[r]); });
    int equal = k, found = 0;
#pragma unroll
    for (int r = 0; r < K; ++r)
        if (r < count)
            equal -= __builtin_popcountll(__ballot(Key::value(key[r]) > tau));
    int64_t last = -1; // chunk of the row up to which logits equal to tau count
#pragma unroll
    for (int r = 0; r < K; ++r) {
        if (r < count) {
            const bool tie = Key::value(key[r]) == tau;
            const uint32_t pos = Key::at(key[r]) * kWave + (uint32_t)lane;
            uint32_t limit = equal > 0 ? ~0u : 0u; // positions below it are taken
            if (equal > 0 && __builtin_popcountll(__ballot(tie)) > equal) {
                limit = 0;
#pragma unroll 1
                for (int b = 10; b >= 0; --b) { // NC * 64 positions
                    const uint32_t mid = limit | 1u << b;
                    if (__builtin_popcountll(__ballot(tie && pos < mid)) <= equal)
                        limit = mid;
                }
            }
            const bool tie_taken = tie && pos < limit, take = tie_taken || Key::value(key[r]) > tau;
            const uint64_t ties = __ballot(tie_taken), all = __ballot(take);
            const uint32_t slice = chosen[r];
            equal -= __builtin_popcountll(ties);
            if (take)
                groups[found + __builtin_popcountll(all & below)] = (uint64_t)Key::rest(key[r]) << 32 | slice << 16 | pos;
            found += __builtin_popcountll(all);
            if (ties)
                last = (int64_t)slice * (NC * kWave) + max_wave(tie_taken ? pos : 0u);
        }
    }
    wave_lds_sync();

    // chunks of these groups that reach the k-th best: most often one of each
    const uint32_t least_order = Key::order(tau), chunks = (uint32_t)((vocab + W - 1) / W);
    const float least = from_order_bits(least_order);
    int n_read = 0;
    for (int c0 = 0; c0 < found * NC; c0 += kWave) {
        const int c = c0 + lane;
        const uint64_t g = groups[c < found * NC ? c / NC : 0];
        const uint32_t place = (uint32_t)g & 0xFFFFu, chunk = ((uint32_t)g >> 16) * (NC * kWave) + (c % NC) * kWave + place % kWave;
        const bool wanted = c < found * NC && chunk < chunks && (c % NC == (int)(place / kWave) || (uint32_t)(g >> 32) >= least_order);
        const uint64_t all = __ballot(wanted);
        if (wanted)
            reads[n_read + __builtin_popcountll(all & below)] = chunk;
        n_read += __builtin_popcountll(all);
    }
    wave_lds_sync();
    // Their logits from the k-th best on, an element a lane.  Should the list not hold them (the largest logits crowd into
    // few groups), passes that count find the k-th best entry bit by bit, and the last one lists the k from there up.
    constexpr int F = 4; // loads in flight
    uint64_t kth = 0;
    int n, bit = 64;
#pragma unroll 1
    for (;;) {
        const uint64_t from = bit >= 0 && bit < 64 ? kth | uint64_t(1) << bit : kth;
        n = 0;
#pragma unroll 1
        for (int e0 = 0; e0 < n_read * W; e0 += F * kWave) {
            float v[F];
            uint32_t chunk[F], at[F];
#pragma unroll
            for (int f = 0; f < F; ++f) {
                const int e = e0 + f * kWave + lane;
                chunk[f] = reads[e < n_read * W ? e / W : 0];
                at[f] = e < n_read * W ? chunk[f] * W + e % W : (uint32_t)vocab;
                v[f] = to_f32<T>(p[at[f] < vocab ? at[f] : 0]);
            }
#pragma unroll
            for (int f = 0; f < F; ++f) {
                const uint64_t entry = entry_of(v[f], at[f]);
                const bool is = at[f] < vocab && (v[f] > least || (v[f] == least && (int64_t)chunk[f] <= last)) && entry >= from;
                const uint64_t all = __ballot(is);
                const int slot = n + __builtin_popcountll(all & below);
                if (is && slot < kListed)
                    list[slot] = entry;
                n += __builtin_popcountll(all);
            }
        }
        if (bit == 64) {
            if (n <= kListed)
                break;
        } else if (bit >= 0) {
            kth = n >= k ? from : kth;
        } else {
            break;
        }
        --bit;
    }
    wave_lds_sync();
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
            const float v = S == 0.0f ? -__builtin_inff() : log_prob(from_order_bits((uint32_t)(mine >> 32)), ref, kLn2 * log2_of(S));
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

// A wave takes U * 64 chunks of one row: 2048 x 32768 float32 with all three gradients 86 us, 6.2 TB/s, nearly a copy's rate.
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
    // bfloat16 rows at an odd element address from whole words on, like Held (4096 x 32767: 96.2 / 92.3 us, 50001: 135.8 /
    // 135.2); the element before the row is dropped
    const int lead = sizeof(T) == 2 && vocab >= U * kWave * W && ((uintptr_t)p & 2) ? 1 : 0;
    const int64_t start = (int64_t)tile * (U * kWave * W) - lead;
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
                if (i == 0 && e < 0) {
#pragma unroll
                    for (int j = 1; j < W; ++j)
                        q[j - 1] = from_f32<T>(v[i][j]);
                } else {
                    store_elems(q + start + (uint32_t)(lane_id() * W + i * (kWave * W)), W, v[i]);
                }
            } else if (e < width) {
                grad_chunk<W, ENT, false>(s, exponent, delta, (int)e, vocab, v[i]);
                store_elems(q + e, width - e, v[i]);
            }
        }
    });
}

// The loss and its gradient: a block holds a whole row in registers, so the logits are read once.  Each wave sums up its
// own part, the parts are joined through LDS, and with the row's statistics every lane turns what it holds into the
// gradient.  8192 x 50000 bfloat16 272 us, 6.0 TB/s, vector units 65 % busy.  Shapes, when they were chosen: 16 waves
// with 7 chunks a lane 279 us, 8 with 13 298, 4 with 25 306.
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
    const int lead = Held<T, NC>::lead_of(p, vocab);
    const int start = wave * (kWave * W), at = start + lane * W - lead;
    Held<T, NC> h;
    h.template load<STEP>(p, start, NC, vocab, lead);
    Slice s{0.0f, 0.0f, 0.0f, 0.0f};
    if (h.any()) {
        LaneTop unused;
        slice_sums<false>(h, s.ref, s.S, s.T, unused);
    }
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
            if (i < h.full) {
                const int e = at + i * STEP;
                float v[W];
                unpack<T>(h.raw[i], v);
                grad_chunk<W, ENT, true>(s, exponent, delta, e, vocab, v);
                if (i == 0 && e < 0) { // the copy
#pragma unroll
                    for (int j = 1; j < W; ++j)
                        q[j - 1] = from_f32<T>(v[j]);
                } else {
                    store_chunk<T>(q + e, pack<T>(v));
                }
            }
        }
#pragma unroll 1
        for (int e = at + h.full * STEP; e < width; e += STEP) { // the tail, and the padding behind it
            float v[W];
            unpack<T>(h.tail, v);
            grad_chunk<W, ENT, false>(s, exponent, delta, e, vocab, v);
            store_elems(q + e, width - e, v);
        }
    });
}

// How a row is cut into slices of 64 * nc chunks: the largest that still give 2048 waves, two to a SIMD, and no more than
// 64 if that can be, which the join reads in one go.  1024 and 4096 waves take the same time within 3 % for 4 to 2048 rows
// of 131072 and 32000.  Slices of 2048 logits at most instead of 4096: 4096 x 50001 with 5 alternatives 88 us against 81,
// float32 157 against 151.
constexpr int64_t kSliceWaves = 2048;
struct Cut {
    int nc;
    int64_t slices;
};
template <class T>
constexpr int kMostChunks = sizeof(T) == 2 ? 8 : 16; // 4096 logits
template <class T>
Cut cut_rows(int64_t rows, int64_t vocab)
{
    constexpr int most = kMostChunks<T>;
    const int64_t chunks = (vocab + kChunk<T> - 1) / kChunk<T>;
    const auto slices = [&](int n) { return (chunks + 64 * n - 1) / (64 * n); };
    int nc = 1;
    while (nc < most && slices(nc) > 1 && (slices(nc) > kWave || rows * slices(2 * nc) >= kSliceWaves))
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
        // The join holds keys for as many slices and alternatives as it is built for.  With 256 slices and 32 alternatives
        // for every call: 4 x 131072 with 8 13.4 us against 10.6, 8192 x 6000 with 5 45 against 34.
        constexpr int most = kMaxSlices / kWave;
        const bool few = c.slices <= kWave;
        if (out.top_k) {
            auto j = few ? (out.top_k <= 8 ? k_logprob_join_top<T, NC, 8, 1> : k_logprob_join_top<T, NC, kMaxTop, 1>)
                         : (out.top_k <= 8 ? k_logprob_join_top<T, NC, 8, most> : k_logprob_join_top<T, NC, kMaxTop, most>);
            return launch<1>(j, rows, kUncapped, s, typed<const T>(x), rows, vocab, (int)c.slices, out, stats, keys);
        }
        return launch<4>(few ? k_logprob_join<T, 1> : k_logprob_join<T, most>, (rows + 3) / 4, kUncapped, s,
                         typed<const T>(x), rows, vocab, (int)c.slices, out, stats);
    });
}

// Workspace of `rows` rows, or with `fewer` the most that they or any smaller number of them take: fewer rows are cut into
// more slices, so the largest need may be that of the last number of rows before larger slices.
template <class T>
int64_t workspace_of(int64_t rows, int64_t vocab, int top_k, bool fewer)
{
    const auto need = [&](int64_t r) {
        const Cut c = cut_rows<T>(r, vocab);
        return c.slices == 1 && !top_k ? 0 : r * c.slices;
    };
    int64_t most = need(rows);
    const int64_t chunks = (vocab + kChunk<T> - 1) / kChunk<T>;
    for (int nc = 2; fewer && nc <= kMostChunks<T>; nc *= 2) {
        const int64_t slices = (chunks + 64 * nc - 1) / (64 * nc), last = (kSliceWaves - 1) / slices;
        if (last > 0 && last < rows && need(last) > most)
            most = need(last);
    }
    return most * (int64_t)(sizeof(Slice) + (top_k ? kWave * sizeof(typename GroupKey<T>::Word) : 0));
}

// May some row start at an odd element address?
template <class T>
bool has_odd_rows(const Rows<const void *> &x, int64_t rows)
{
    return sizeof(T) == 2 && ((reinterpret_cast<uintptr_t>(x.p) & 2) || (rows > 1 && x.stride % 2));
}

template <class T, bool ENT>
int logprob_grad(Rows<const void *> x, int64_t rows, int64_t vocab, const int64_t *targets, const float *lse,
                 const float *entropy, const TokenGrads &g, Rows<void *> dx, int64_t width, hipStream_t s)
{
    const int64_t chunks = (width + has_odd_rows<T>(x, rows) + kChunk<T> - 1) / kChunk<T>; // and one element of lead
    constexpr int U = 2; // 1 / 2 / 4: 2048 x 32768 float32 86.6 / 86.3 / 88.8 us, 4096 x 32768 bfloat16 85.4 / 84.6 / 83.9
    const int64_t tiles = (chunks + 64 * U - 1) / (64 * U);
    return launch<4>(k_logprob_grad<T, U, ENT>, (rows * tiles + 3) / 4, kUncapped, s, typed<const T>(x), rows, vocab, targets,
                     lse, entropy, g, typed<T>(dx), width, Divisor((uint64_t)tiles));
}

template <class T, bool ENT>
int token_loss(Rows<const void *> x, int64_t rows, int64_t vocab, const TokenStats &out, const TokenGrads &g,
               Rows<void *> dx, int64_t width, void *workspace, hipStream_t s)
{
    const int64_t chunks = (width + has_odd_rows<T>(x, rows) + kChunk<T> - 1) / kChunk<T>; // and one element of lead
    auto run = [&](auto waves, auto nc) {
        constexpr int WV = decltype(waves)::value, NC = decltype(nc)::value;
        return launch<WV>(k_token_loss<T, WV, NC, ENT>, rows, kUncapped, s, typed<const T>(x), rows, vocab, out, g,
                          typed<T>(dx), width);
    };
    // The fewest waves, then the fewest chunks a lane, that hold the row; longer rows take two launches.  Those where one
    // would do: 8192 x 1000 14.9 us against 10.1, 4096 x 50000 bfloat16 198 against 150, 4096 x 131072 507 against 402,
    // float32 4096 x 50000 414 against 318.  (Few long rows leave units empty here, but a loss is taken of many:
    // 64 x 131072 15.7 against 17.7.)
    using std::integral_constant;
    if (chunks <= 256)
        return run(integral_constant<int, 1>{}, integral_constant<int, 4>{});
    if (chunks <= 1024)
        return run(integral_constant<int, 4>{}, integral_constant<int, 4>{});
    if (chunks <= 2048)
        return run(integral_constant<int, 8>{}, integral_constant<int, 4>{});
    if (chunks <= 4096)
        return run(integral_constant<int, 16>{}, integral_constant<int, 4>{});
    if (chunks <= 7168)
        return run(integral_constant<int, 16>{}, integral_constant<int, 7>{});
    if (chunks <= 10240)
        return run(integral_constant<int, 16>{}, integral_constant<int, 10>{});
    if (chunks <= 13312)
        return run(integral_constant<int, 16>{}, integral_constant<int, 13>{});
    if (chunks <= 16384)
        return run(integral_constant<int, 16>{}, integral_constant<int, 16>{});
    const int rc = logprob<T>(x, rows, vocab, out, workspace, s);
    return rc ? rc : logprob_grad<T, ENT>(x, rows, vocab, out.targets, out.lse, out.entropy, g, dx, width, s);
}

} // namespace

int64_t token_logprob_workspace(int64_t rows, int64_t vocab, int top_k, bool fewer)
{
    if (rows <= 0 || vocab <= 0)
        return 0;
    const int64_t a = workspace_of<bf16_t>(rows, vocab, top_k, fewer), b = workspace_of<float>(rows, vocab, top_k, fewer);
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
