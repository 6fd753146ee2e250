// abi_checks.hpp -- what the argument checks of the training-step operators'
// entry points share (abi_step.cpp, abi_layer.cpp).
#pragma once

#include "step.hpp"

#include <cstdint>
#include <initializer_list>

namespace sdp4 {
namespace checks {

inline bool aligned(const void *p, std::uintptr_t a) { return reinterpret_cast<std::uintptr_t>(p) % a == 0; }
inline bool valid_dtype(int t) { return t == SDP4_F32 || t == SDP4_BF16; }
inline int64_t size_of(int dtype) { return dtype == SDP4_BF16 ? 2 : 4; }
inline hipStream_t as_stream(void *s) { return static_cast<hipStream_t>(s); }

// a * b for non-negative numbers, kept within the element limit
inline bool product_fits(int64_t a, int64_t b) { return a == 0 || b <= SDP4_MAX_ELEMENTS / a; }

// An array as the memory it touches: `rows` rows of `width` bytes, `pitch` bytes apart.
struct Area {
    const void *p;
    int64_t rows, width, pitch;
    int64_t bytes() const { return rows > 0 && width > 0 ? (rows - 1) * pitch + width : 0; }
};
inline Area flat(const void *p, int64_t bytes) { return {p, 1, p ? bytes : 0, bytes}; }

// May the two share a byte?  Rows of one pitch are told apart even where the areas interleave.
inline bool overlap(const Area &a, const Area &b)
{
    if (!a.p || !b.p || a.bytes() == 0 || b.bytes() == 0)
        return false;
    const auto a0 = reinterpret_cast<std::uintptr_t>(a.p), b0 = reinterpret_cast<std::uintptr_t>(b.p);
    if (a0 + (std::uintptr_t)a.bytes() <= b0 || b0 + (std::uintptr_t)b.bytes() <= a0)
        return false;
    if (a.rows > 1 && b.rows > 1 && a.pitch == b.pitch) {
        const std::uintptr_t pitch = (std::uintptr_t)a.pitch;
        const std::uintptr_t d = b0 >= a0 ? (b0 - a0) % pitch : (pitch - (a0 - b0) % pitch) % pitch;
        if (d >= (std::uintptr_t)a.width && d + (std::uintptr_t)b.width <= pitch)
            return false;
    }
    return true;
}
inline bool same(const Area &a, const Area &b) { return a.p == b.p && a.width == b.width && (a.rows <= 1 || a.pitch == b.pitch); }

// An output against the inputs it may be (exactly) and those it must not touch.
inline bool clash(const Area &out, std::initializer_list<Area> may_be, std::initializer_list<Area> others)
{
    for (const Area &a : may_be)
        if (!same(out, a) && overlap(out, a))
            return true;
    for (const Area &a : others)
        if (overlap(out, a))
            return true;
    return false;
}

struct Matrix {
    const void *p;
    int dtype;
    int64_t stride;
    Area area(int64_t rows, int64_t cols) const
    {
        const int64_t s = size_of(dtype);
        return {p, p ? rows : 0, cols * s, stride * s};
    }
};
inline bool valid_matrix(const Matrix &m, int64_t rows, int64_t cols)
{
    return rows <= 1 ? true : m.stride >= cols && product_fits(rows, m.stride);
}
inline bool valid_shape(int64_t rows, int64_t cols) { return rows >= 0 && cols >= 0 && cols <= INT32_MAX - 7 && product_fits(rows, cols + 7); }

inline int check_workspace(const void *w, int64_t have, int64_t need)
{
    if (need == 0)
        return SDP4_OK;
    if (!w || have < need)
        return SDP4_EINVAL;
    return aligned(w, 16) ? SDP4_OK : SDP4_EALIGN;
}

// Heads as memory: rows of the longer stride.
inline Area area_of(const sdp4_heads &h, int64_t tokens, int dim, int dtype)
{
    const int64_t s = size_of(dtype);
    if (h.token_stride >= h.head_stride)
        return {h.data, tokens, ((h.heads - 1) * h.head_stride + dim) * s, h.token_stride * s};
    return {h.data, h.heads, ((tokens - 1) * h.token_stride + dim) * s, h.head_stride * s};
}
// May two sets of heads share a byte?  Sets with one inner stride that divides both outer ones (each head's query and key
// side by side) are told apart by where their heads lie within it, the others as rows.
inline bool heads_overlap(const sdp4_heads &a, const sdp4_heads &b, int64_t tokens, int dim, int dtype)
{
    if (!overlap(area_of(a, tokens, dim, dtype), area_of(b, tokens, dim, dtype)))
        return false;
    const auto inner = [](const sdp4_heads &h) { return h.token_stride < h.head_stride ? h.token_stride : h.head_stride; };
    const int64_t in = inner(a);
    if (in != inner(b) || a.token_stride % in || a.head_stride % in || b.token_stride % in || b.head_stride % in)
        return true;
    const auto a0 = reinterpret_cast<std::uintptr_t>(a.data), b0 = reinterpret_cast<std::uintptr_t>(b.data);
    const std::uintptr_t pitch = (std::uintptr_t)(in * size_of(dtype)), width = (std::uintptr_t)(dim * size_of(dtype));
    const std::uintptr_t d = b0 >= a0 ? (b0 - a0) % pitch : (pitch - (a0 - b0) % pitch) % pitch;
    return d < width || d + width > pitch;
}
inline bool same_heads(const sdp4_heads &a, const sdp4_heads &b, int64_t tokens)
{
    return a.data == b.data && (tokens <= 1 || a.token_stride == b.token_stride) &&
           (a.heads <= 1 || a.head_stride == b.head_stride);
}
inline bool valid_heads(const sdp4_heads &h, int64_t tokens, int dim)
{
    if (h.heads < 1 || h.heads > (1 << 20) || !product_fits(tokens, (int64_t)h.heads * dim))
        return false;
    if (h.token_stride < 0 || h.head_stride < 0 || !product_fits(tokens, h.token_stride) ||
        !product_fits(h.heads, h.head_stride))
        return false;
    if ((tokens > 1 && h.token_stride < dim) || (h.heads > 1 && h.head_stride < dim))
        return false;
    if (tokens <= 1 || h.heads <= 1)
        return true;
    return h.token_stride >= (h.heads - 1) * h.head_stride + dim || h.head_stride >= (tokens - 1) * h.token_stride + dim;
}
// Strides that nothing steps over count as the width.
inline sdp4_heads normal(sdp4_heads h, int64_t tokens, int dim)
{
    if (h.heads <= 1)
        h.head_stride = dim;
    if (tokens <= 1)
        h.token_stride = h.heads * h.head_stride;
    return h;
}

inline sdp4::Heads launch_heads(const sdp4_heads &h) { return {h.data, h.token_stride, h.head_stride, h.heads}; }

} // namespace checks
} // namespace sdp4
