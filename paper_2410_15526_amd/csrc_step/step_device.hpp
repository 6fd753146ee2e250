// step_device.hpp -- device building blocks of the training-step operators.
//
// Rows have any stride and any width, so a row may start at an address that
// is only as aligned as one element.  Global memory serves 16-byte accesses
// at any element address, and a wave that reads 64 neighbouring chunks
// touches one cache line more than from an aligned start: rows are read and
// written in whole 16-byte chunks wherever they begin.  A row's last chunk,
// where it is not whole, is read as the row's last whole chunk of elements and
// shifted, and written element by element.  (The loss and the gradient of log
// probabilities read bfloat16 rows at odd addresses from the word before.)
#pragma once

#include "device.hpp"
#include "step.hpp"

#include <type_traits>

namespace sdp4 {

using bf16_t = uint16_t; // bfloat16 bits

template <class T>
constexpr int kChunk = 16 / sizeof(T); // elements of a 16-byte chunk

// Work block of the launch.
SDP4_DEV int64_t work_block() { return (int64_t)blockIdx.y << kGridXLog2 | blockIdx.x; }

// Division by a number known on the host, exact for every dividend: the
// multiplication by floor((2^64 - 1) / d) is at most one short.
struct Divisor {
    uint64_t d, inv;
    Divisor() = default;
    explicit Divisor(uint64_t n) : d(n), inv(~uint64_t(0) / n) {}
};
SDP4_DEV uint64_t divide(uint64_t n, const Divisor &v, uint64_t &rest)
{
    uint64_t q = __umul64hi(n, v.inv);
    rest = n - q * v.d;
    if (rest >= v.d) {
        rest -= v.d;
        ++q;
    }
    return q;
}

// A value that is the same in all lanes of a wave, on the scalar unit.
SDP4_DEV uint32_t uniform(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }
SDP4_DEV uint64_t uniform(uint64_t v)
{
    return (uint64_t)uniform((uint32_t)(v >> 32)) << 32 | uniform((uint32_t)v);
}

template <class T>
SDP4_DEV float to_f32(T v)
{
    if constexpr (sizeof(T) == 4)
        return v;
    else
        return __uint_as_float((uint32_t)v << 16);
}

template <class T>
SDP4_DEV T from_f32(float v)
{
    if constexpr (sizeof(T) == 4)
        return v;
    else
        return (T)(bf16x2_rne(v, 0.0f) & 0xFFFFu);
}

// Vectors at element addresses.
typedef u32x4 u32x4_b2 __attribute__((aligned(2)));
typedef u32x4 u32x4_b4 __attribute__((aligned(4)));
typedef u32x2 u32x2_b2 __attribute__((aligned(2)));
typedef u32x2 u32x2_b4 __attribute__((aligned(4)));
template <class T>
using chunk_at = std::conditional_t<sizeof(T) == 4, u32x4_b4, u32x4_b2>;
template <class T>
using half_at = std::conditional_t<sizeof(T) == 4, u32x2_b4, u32x2_b2>;

// One chunk, streamed past the caches (NT) or kept in them.
template <bool NT, class T>
SDP4_DEV u32x4 load_chunk(const T *p)
{
    auto q = reinterpret_cast<const chunk_at<T> *>(p);
    if constexpr (NT)
        return __builtin_nontemporal_load(q);
    else
        return *q;
}

template <class T>
SDP4_DEV void store_chunk(T *p, u32x4 v)
{
    __builtin_nontemporal_store((chunk_at<T>)v, reinterpret_cast<chunk_at<T> *>(p));
}

template <class T>
SDP4_DEV void unpack(u32x4 c, float (&v)[kChunk<T>])
{
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 4) {
            v[j] = __uint_as_float(w[j]);
        } else {
            v[2 * j] = __uint_as_float(w[j] << 16);
            v[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
        }
    }
}

template <class T>
SDP4_DEV u32x4 pack(const float (&v)[kChunk<T>])
{
    if constexpr (sizeof(T) == 4)
        return u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    else
        return u32x4{bf16x2_rne(v[0], v[1]), bf16x2_rne(v[2], v[3]), bf16x2_rne(v[4], v[5]), bf16x2_rne(v[6], v[7])};
}

// N elements as they lie in memory: 16 or 8 bytes, or one element.  Loops that load ahead carry this form, since values
// that are unpacked are values that have been waited for.
template <class T, int N>
struct Raw {
    static constexpr int BYTES = N * sizeof(T);
    static_assert(BYTES == 16 || BYTES == 8 || N == 1, "accesses");
    using V = std::conditional_t<BYTES == 16, u32x4, std::conditional_t<BYTES == 8, u32x2, T>>;
    V v;
    template <bool NT>
    SDP4_DEV void load(const T *p)
    {
        if constexpr (BYTES == 16) {
            v = load_chunk<NT>(p);
        } else if constexpr (BYTES == 8) {
            auto q = reinterpret_cast<const half_at<T> *>(p);
            v = NT ? (u32x2)__builtin_nontemporal_load(q) : (u32x2)*q;
        } else {
            v = *p;
        }
    }
    SDP4_DEV void get(float (&o)[N]) const
    {
        if constexpr (N == 1) {
            o[0] = to_f32<T>(v);
        } else {
            uint32_t w[BYTES / 4];
            __builtin_memcpy(w, &v, BYTES);
#pragma unroll
            for (int j = 0; j < BYTES / 4; ++j) {
                if constexpr (sizeof(T) == 4) {
                    o[j] = __uint_as_float(w[j]);
                } else {
                    o[2 * j] = __uint_as_float(w[j] << 16);
                    o[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
                }
            }
        }
    }
    SDP4_DEV void put(const float (&o)[N])
    {
        if constexpr (N == 1) {
            v = from_f32<T>(o[0]);
        } else {
            uint32_t w[BYTES / 4];
#pragma unroll
            for (int j = 0; j < BYTES / 4; ++j)
                w[j] = sizeof(T) == 4 ? __float_as_uint(o[j]) : bf16x2_rne(o[2 * j * (sizeof(T) == 2)], o[(2 * j + 1) * (sizeof(T) == 2)]);
            __builtin_memcpy(&v, w, BYTES);
        }
    }
    SDP4_DEV void store(T *p) const
    {
        if constexpr (BYTES == 16)
            store_chunk<T>(p, v);
        else if constexpr (BYTES == 8)
            __builtin_nontemporal_store((half_at<T>)v, reinterpret_cast<half_at<T> *>(p));
        else
            *p = v;
    }
};

// N elements from element address p.
template <class T, int N>
SDP4_DEV void load_whole(const T *p, float (&v)[N])
{
    Raw<T, N> r;
    r.template load<true>(p);
    r.get(v);
}

// Elements c .. c + N - 1 of a row of `cols`, in two steps, so that the loads of several rows are in flight together:
// where the row ends before, load_row reads its last N elements instead (what another lane may be replacing there is
// not used) and end_row moves them to their places.  Places beyond the row get `fill`.
template <class T, int N>
SDP4_DEV void load_row(const T *row, int64_t c, int64_t cols, Raw<T, N> &r)
{
    if (cols >= N) {
        r.template load<true>(row + (c + N <= cols ? c : cols - N));
    } else {
        float v[N];
#pragma unroll
        for (int j = 0; j < N; ++j)
            v[j] = to_f32<T>(row[j < cols ? j : 0]);
        r.put(v);
    }
}
template <class T, int N>
SDP4_DEV void load_row(const T *row, int64_t c, int64_t cols, float (&v)[N])
{
    Raw<T, N> r;
    load_row(row, c, cols, r);
    r.get(v);
}
template <int N>
SDP4_DEV void end_row(int64_t c, int64_t cols, float (&v)[N], float fill = 0.0f)
{
    if (c + N <= cols)
        return;
    if (cols < N) { // load_row read from column 0, and c is 0 or beyond the row
#pragma unroll
        for (int j = 0; j < N; ++j)
            v[j] = c + j < cols ? v[j] : fill;
        return;
    }
    const int64_t by = c - (cols - N);
    const int s = by < N ? (int)by : N;
#pragma unroll
    for (int b = N; b >= 1; b /= 2) {
        const bool take = s & b;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float from = j + b < N ? v[j + b < N ? j + b : j] : fill;
            v[j] = take ? from : v[j];
        }
    }
}

template <class T, int N>
SDP4_DEV void store_elems(T *p, int64_t valid, const float (&v)[N])
{
    if (valid >= N) {
        Raw<T, N> r;
        r.put(v);
        r.store(p);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j < valid)
                p[j] = from_f32<T>(v[j]);
    }
}

// Sum and largest value over an aligned block of `lanes` lanes (a power of
// two), in every lane of it; always joined in the same order.
SDP4_DEV float sum_lanes(float v, int lanes)
{
    if (lanes > 1) v += dpp_f32<kDppXor1>(v);
    if (lanes > 2) v += dpp_f32<kDppXor2>(v);
    if (lanes > 4) v += dpp_f32<kDppHalfMirror>(v);
    if (lanes > 8) v += dpp_f32<kDppRor8>(v);
    if (lanes > 16) v += xor_lane<16>(v);
    if (lanes > 32) v += xor_lane<32>(v);
    return v;
}

SDP4_DEV float max_wave(float v)
{
    v = fmaxf(v, dpp_f32<kDppXor1>(v));
    v = fmaxf(v, dpp_f32<kDppXor2>(v));
    v = fmaxf(v, dpp_f32<kDppHalfMirror>(v));
    v = fmaxf(v, dpp_f32<kDppRor8>(v));
    v = fmaxf(v, xor_lane<16>(v));
    return fmaxf(v, xor_lane<32>(v));
}

template <class T, class P>
Rows<T *> typed(Rows<P> r)
{
    return {static_cast<T *>(r.p), r.stride};
}

// Two calls of a body, for the element types.
template <class F>
int with_type(int dtype, F body)
{
    return dtype == SDP4_BF16 ? body(bf16_t{}) : body(float{});
}

} // namespace sdp4
