// abi_layer.cpp -- the C ABI of attention, block norms and the embedding
// declared in include/sdp4.h: host-side argument checks, then the launches.
//
// Every check runs before any HIP call.
#include "abi_checks.hpp"

#include <cmath>

namespace {

using namespace sdp4::checks;

// ---------------------------------------------------------------------------
// attention
// ---------------------------------------------------------------------------
int check_attention(const sdp4_attention_params *p, int64_t tokens)
{
    if (!p || tokens < 0 || tokens > SDP4_MAX_TOKENS || !valid_dtype(p->dtype) || p->head_dim < SDP4_MIN_ATTENTION_DIM ||
        p->head_dim > SDP4_MAX_ATTENTION_DIM || !(p->scale >= 0x1p-40f && p->scale <= 0x1p40f) ||
        (p->offsets && (p->sequences < 0 || p->sequences > SDP4_MAX_TOKENS)))
        return SDP4_EINVAL;
    return aligned(p->offsets, 8) ? SDP4_OK : SDP4_EALIGN;
}

// One set of heads: valid, aligned, as the launchers take it.
int take(const sdp4_heads *h, int64_t tokens, const sdp4_attention_params &p, sdp4_heads &out)
{
    if (!h || !valid_heads(*h, tokens, p.head_dim) || !h->data)
        return SDP4_EINVAL;
    if (!aligned(h->data, size_of(p.dtype)))
        return SDP4_EALIGN;
    out = normal(*h, tokens, p.head_dim);
    return SDP4_OK;
}

sdp4::Attention attention_of(const sdp4_attention_params &p, int64_t tokens, int q_heads, int k_heads)
{
    return {{p.offsets, p.offsets ? p.sequences : 0, static_cast<int>(tokens)}, p.head_dim, q_heads / k_heads, p.scale};
}

Area offsets_area(const sdp4_attention_params &p) { return flat(p.offsets, p.offsets ? 8 * (p.sequences + 1) : 0); }

// Heads that are written against those that are read, each other, and flat arrays.
template <int OUTS, int INS>
bool heads_clash(const sdp4_heads (&outs)[OUTS], const sdp4_heads (&ins)[INS], std::initializer_list<Area> flats, int64_t tokens,
                 const sdp4_attention_params &p)
{
    for (int i = 0; i < OUTS; ++i) {
        for (const sdp4_heads &in : ins)
            if (heads_overlap(outs[i], in, tokens, p.head_dim, p.dtype))
                return true;
        for (int j = 0; j < i; ++j)
            if (heads_overlap(outs[i], outs[j], tokens, p.head_dim, p.dtype))
                return true;
        for (const Area &a : flats)
            if (overlap(area_of(outs[i], tokens, p.head_dim, p.dtype), a))
                return true;
    }
    return false;
}

// ---------------------------------------------------------------------------
// block norms
// ---------------------------------------------------------------------------
int check_block(const sdp4_block_params *p, int64_t rows, int64_t cols)
{
    if (!p || !valid_dtype(p->x_dtype) || !valid_dtype(p->y_dtype) || !valid_shape(rows, cols) || cols > SDP4_MAX_HIDDEN ||
        (p->post_norm && (!(p->post_eps >= 0.0f) || !std::isfinite(p->post_eps))) || !(p->pre_eps >= 0.0f) ||
        !std::isfinite(p->pre_eps) || !std::isfinite(p->branch_scale) || !std::isfinite(p->residual_scale))
        return SDP4_EINVAL;
    const int64_t s = size_of(p->x_dtype);
    return aligned(p->post_weight, s) && aligned(p->pre_weight, s) && aligned(p->gate, 4) ? SDP4_OK : SDP4_EALIGN;
}

sdp4::BlockNorm block_of(const sdp4_block_params &p)
{
    return {p.post_norm != 0, p.post_eps, p.pre_eps, p.post_weight, p.pre_weight, p.gate, p.branch_scale, p.residual_scale};
}

// ---------------------------------------------------------------------------
// embedding
// ---------------------------------------------------------------------------
bool valid_tokens(int64_t rows, int64_t vocab, int64_t cols, float scale)
{
    return valid_shape(rows, cols) && rows <= SDP4_MAX_TOKENS && vocab >= 1 && vocab <= SDP4_MAX_VOCAB &&
           valid_shape(vocab, cols) && std::isfinite(scale);
}

} // namespace

extern "C" {

int sdp4_attention(const sdp4_heads *q, const sdp4_heads *k, const sdp4_heads *v, const sdp4_attention_params *params,
                   int64_t tokens, const sdp4_heads *out, float *lse, void *stream)
{
    int rc = check_attention(params, tokens);
    if (rc != SDP4_OK)
        return rc;
    if (!q || !k || !v || !out)
        return SDP4_EINVAL;
    if (tokens == 0)
        return SDP4_OK;
    const sdp4_attention_params &p = *params;
    sdp4_heads in[3], o[1];
    if ((rc = take(q, tokens, p, in[0])) || (rc = take(k, tokens, p, in[1])) || (rc = take(v, tokens, p, in[2])) ||
        (rc = take(out, tokens, p, o[0])))
        return rc;
    if (in[1].heads != in[2].heads || o[0].heads != in[0].heads || in[0].heads % in[1].heads ||
        !product_fits(in[0].heads, 4 * tokens))
        return SDP4_EINVAL;
    if (!aligned(lse, 4))
        return SDP4_EALIGN;
    const Area l = flat(lse, 4 * tokens * in[0].heads), offsets = offsets_area(p);
    if (heads_clash(o, in, {l, offsets}, tokens, p) || overlap(l, offsets))
        return SDP4_EINVAL;
    for (const sdp4_heads &h : in)
        if (overlap(l, area_of(h, tokens, p.head_dim, p.dtype)))
            return SDP4_EINVAL;
    return sdp4::launch_attention(p.dtype, attention_of(p, tokens, in[0].heads, in[1].heads), launch_heads(in[0]),
                                  launch_heads(in[1]), launch_heads(in[2]), launch_heads(o[0]), lse, as_stream(stream));
}

int sdp4_attention_grad(const sdp4_heads *dout, const sdp4_heads *q, const sdp4_heads *k, const sdp4_heads *v,
                        const sdp4_heads *out, const float *lse, const sdp4_attention_params *params, int64_t tokens,
                        const sdp4_heads *dq, const sdp4_heads *dk, const sdp4_heads *dv, void *workspace,
                        int64_t workspace_bytes, void *stream)
{
    int rc = check_attention(params, tokens);
    if (rc != SDP4_OK)
        return rc;
    if (!dout || !q || !k || !v || !out || !dq || !dk || !dv)
        return SDP4_EINVAL;
    if (tokens == 0)
        return SDP4_OK;
    const sdp4_attention_params &p = *params;
    const sdp4_heads *reads[5] = {dout, q, k, v, out}, *writes[3] = {dq, dk, dv};
    sdp4_heads in[5], o[3];
    for (int i = 0; i < 5; ++i)
        if ((rc = take(reads[i], tokens, p, in[i])))
            return rc;
    for (int i = 0; i < 3; ++i)
        if ((rc = take(writes[i], tokens, p, o[i])))
            return rc;
    const int hq = in[1].heads, hk = in[2].heads;
    if (in[0].heads != hq || in[4].heads != hq || o[0].heads != hq || in[3].heads != hk || o[1].heads != hk ||
        o[2].heads != hk || hq % hk || !product_fits(hq, 4 * tokens) || !lse)
        return SDP4_EINVAL;
    if (!aligned(lse, 4))
        return SDP4_EALIGN;
    const int64_t need = sdp4::attention_grad_workspace(tokens, hq, hk, p.head_dim);
    rc = check_workspace(workspace, workspace_bytes, need);
    if (rc != SDP4_OK)
        return rc;
    const Area l = flat(lse, 4 * tokens * hq), offsets = offsets_area(p), work = flat(workspace, need);
    if (heads_clash(o, in, {l, offsets, work}, tokens, p) || overlap(work, l) || overlap(work, offsets))
        return SDP4_EINVAL;
    for (const sdp4_heads &h : in)
        if (overlap(work, area_of(h, tokens, p.head_dim, p.dtype)))
            return SDP4_EINVAL;
    return sdp4::launch_attention_grad(p.dtype, attention_of(p, tokens, hq, hk), launch_heads(in[0]), launch_heads(in[1]),
                                       launch_heads(in[2]), launch_heads(in[3]), launch_heads(in[4]), lse, launch_heads(o[0]),
                                       launch_heads(o[1]), launch_heads(o[2]), static_cast<float *>(workspace),
                                       as_stream(stream));
}

int64_t sdp4_attention_grad_workspace(int64_t tokens, int q_heads, int k_heads, int head_dim)
{
    if (tokens < 0 || tokens > SDP4_MAX_TOKENS || k_heads < 1 || q_heads < k_heads || q_heads > (1 << 20) || q_heads % k_heads ||
        head_dim < SDP4_MIN_ATTENTION_DIM || head_dim > SDP4_MAX_ATTENTION_DIM || !product_fits(q_heads, 4 * tokens))
        return -1;
    return sdp4::attention_grad_workspace(tokens, q_heads, k_heads, head_dim);
}

int sdp4_block_norm(const void *branch, int64_t branch_stride, const void *residual, int64_t residual_stride, int64_t rows,
                    int64_t cols, const sdp4_block_params *params, void *y, int64_t y_stride, void *h, int64_t h_stride,
                    void *stream)
{
    int rc = check_block(params, rows, cols);
    if (rc != SDP4_OK)
        return rc;
    const sdp4_block_params &p = *params;
    const Matrix mb{branch, p.x_dtype, branch_stride}, mr{residual, p.y_dtype, residual_stride}, my{y, p.y_dtype, y_stride},
        mh{h, p.x_dtype, h_stride};
    for (const Matrix &m : {mb, mr, my, mh})
        if (m.p && !valid_matrix(m, rows, cols))
            return SDP4_EINVAL;
    if (rows == 0 || cols == 0)
        return SDP4_OK;
    if ((!branch && !residual) || (!y && !h) || (!branch && (p.post_norm || p.post_weight || p.gate)))
        return SDP4_EINVAL;
    for (const Matrix &m : {mb, mr, my, mh})
        if (!aligned(m.p, size_of(m.dtype)))
            return SDP4_EALIGN;
    const int64_t s = size_of(p.x_dtype);
    const Area b = mb.area(rows, cols), r = mr.area(rows, cols), ay = my.area(rows, cols), ah = mh.area(rows, cols),
               w1 = flat(p.post_weight, s * cols), w2 = flat(p.pre_weight, s * cols), g = flat(p.gate, 4 * rows);
    if (clash(ay, {b, r}, {w1, w2, g, ah}) || clash(ah, {b, r}, {w1, w2, g}))
        return SDP4_EINVAL;
    return sdp4::launch_block_norm(p.x_dtype, p.y_dtype, block_of(p), rows, cols, {branch, branch_stride},
                                   {residual, residual_stride}, {y, y_stride}, {h, h_stride}, as_stream(stream));
}

int sdp4_block_norm_grad(const void *dh, int64_t dh_stride, const void *dy, int64_t dy_stride, const void *branch,
                         int64_t branch_stride, const void *y, int64_t y_stride, int64_t rows, int64_t cols,
                         const sdp4_block_params *params, void *dbranch, int64_t dbranch_stride, void *dresidual,
                         int64_t dresidual_stride, float *dpost_weight, float *dpre_weight, float *dgate, void *workspace,
                         int64_t workspace_bytes, void *stream)
{
    int rc = check_block(params, rows, cols);
    if (rc != SDP4_OK)
        return rc;
    const sdp4_block_params &p = *params;
    const Matrix mdh{dh, p.x_dtype, dh_stride}, mdy{dy, p.y_dtype, dy_stride}, mb{branch, p.x_dtype, branch_stride},
        my{y, p.y_dtype, y_stride}, mdb{dbranch, p.x_dtype, dbranch_stride}, mdr{dresidual, p.y_dtype, dresidual_stride};
    for (const Matrix &m : {mdh, mdy, mb, my, mdb, mdr})
        if (m.p && !valid_matrix(m, rows, cols))
            return SDP4_EINVAL;
    if ((dpost_weight && !p.post_weight) || (dpre_weight && !p.pre_weight) || (dgate && !p.gate))
        return SDP4_EINVAL;
    if (!aligned(dpost_weight, 4) || !aligned(dpre_weight, 4) || !aligned(dgate, 4))
        return SDP4_EALIGN;
    if (cols == 0 && !(dgate && rows > 0))
        return SDP4_OK;
    if (cols == 0)
        return SDP4_EINVAL; // a gate's gradient over no columns
    if (rows == 0) {        // empty sums
        if (!dpost_weight && !dpre_weight)
            return SDP4_OK;
        if (overlap(flat(dpost_weight, 4 * cols), flat(dpre_weight, 4 * cols)))
            return SDP4_EINVAL;
        return sdp4::launch_sum_parts({{nullptr, 0, dpost_weight}, {nullptr, 0, dpre_weight}}, cols, cols, as_stream(stream));
    }
    // dh needs y; a norm's gradient, its weight's and the gate's need the branch
    if ((!dh && !dy) || (dh && !y) || (dpre_weight && !dh) || (!dbranch && !dresidual && !dpost_weight && !dpre_weight && !dgate) ||
        (!branch && ((dbranch && p.post_norm) || dpost_weight || dgate)))
        return SDP4_EINVAL;
    for (const Matrix &m : {mdh, mdy, mb, my, mdb, mdr})
        if (!aligned(m.p, size_of(m.dtype)))
            return SDP4_EALIGN;
    const int64_t need = dpost_weight || dpre_weight ? sdp4::block_norm_grad_workspace(rows, cols) : 0;
    rc = check_workspace(workspace, workspace_bytes, need);
    if (rc != SDP4_OK)
        return rc;
    const int64_t s = size_of(p.x_dtype);
    const Area ins[4] = {mdh.area(rows, cols), mdy.area(rows, cols), mb.area(rows, cols), my.area(rows, cols)};
    const Area small[3] = {flat(p.post_weight, s * cols), flat(p.pre_weight, s * cols), flat(p.gate, 4 * rows)};
    const Area outs[2] = {mdb.area(rows, cols), mdr.area(rows, cols)};
    const Area sums[4] = {flat(dpost_weight, 4 * cols), flat(dpre_weight, 4 * cols), flat(dgate, 4 * rows),
                          flat(need ? workspace : nullptr, need)};
    for (int i = 0; i < 2; ++i)
        if (clash(outs[i], {ins[0], ins[1], ins[2], ins[3]}, {small[0], small[1], small[2], sums[0], sums[1], sums[2], sums[3]}))
            return SDP4_EINVAL;
    if (overlap(outs[0], outs[1]))
        return SDP4_EINVAL;
    for (int i = 0; i < 4; ++i) {
        if (clash(sums[i], {}, {ins[0], ins[1], ins[2], ins[3], small[0], small[1], small[2]}))
            return SDP4_EINVAL;
        for (int j = 0; j < i; ++j)
            if (overlap(sums[i], sums[j]))
                return SDP4_EINVAL;
    }
    return sdp4::launch_block_norm_grad(p.x_dtype, p.y_dtype, block_of(p), rows, cols,
                                        {{dh, dh_stride}, {dy, dy_stride}, {branch, branch_stride}, {dh ? y : nullptr, y_stride},
                                         {dbranch, dbranch_stride}, {dresidual, dresidual_stride}, dpost_weight, dpre_weight, dgate},
                                        static_cast<float *>(workspace), as_stream(stream));
}

int64_t sdp4_block_norm_grad_workspace(int64_t rows, int64_t cols)
{
    return valid_shape(rows, cols) && cols <= SDP4_MAX_HIDDEN ? sdp4::block_norm_grad_workspace(rows, cols) : -1;
}

int sdp4_embedding(const int64_t *tokens, int64_t rows, const void *table, int table_dtype, int64_t table_stride, int64_t vocab,
                   int64_t cols, float scale, void *out, int out_dtype, int64_t out_stride, void *stream)
{
    const Matrix t{table, table_dtype, table_stride}, o{out, out_dtype, out_stride};
    if (!valid_dtype(table_dtype) || !valid_dtype(out_dtype) || !valid_tokens(rows, vocab, cols, scale) ||
        !valid_matrix(t, vocab, cols) || !valid_matrix(o, rows, cols))
        return SDP4_EINVAL;
    if (rows == 0 || cols == 0)
        return SDP4_OK;
    if (!tokens || !table || !out)
        return SDP4_EINVAL;
    if (!aligned(tokens, 8) || !aligned(table, size_of(table_dtype)) || !aligned(out, size_of(out_dtype)))
        return SDP4_EALIGN;
    if (clash(o.area(rows, cols), {}, {t.area(vocab, cols), flat(tokens, 8 * rows)}))
        return SDP4_EINVAL;
    return sdp4::launch_embedding({tokens, rows, vocab}, cols, scale, table_dtype, {table, table_stride}, out_dtype,
                                  {out, out_stride}, as_stream(stream));
}

int sdp4_embedding_grad(const int64_t *tokens, int64_t rows, const void *dout, int dout_dtype, int64_t dout_stride, int64_t vocab,
                        int64_t cols, float scale, int accumulate, void *dtable, int dtable_dtype, int64_t dtable_stride,
                        void *workspace, int64_t workspace_bytes, void *stream)
{
    const Matrix d{dout, dout_dtype, dout_stride}, t{dtable, dtable_dtype, dtable_stride};
    if (!valid_dtype(dout_dtype) || !valid_dtype(dtable_dtype) || !valid_tokens(rows, vocab, cols, scale) ||
        rows > SDP4_MAX_GRAD_TOKENS ||
        !valid_matrix(d, rows, cols) || !valid_matrix(t, vocab, cols))
        return SDP4_EINVAL;
    if (cols == 0 || (rows == 0 && accumulate))
        return SDP4_OK;
    if (!dtable || (rows > 0 && (!tokens || !dout)))
        return SDP4_EINVAL;
    if (!aligned(tokens, 8) || !aligned(dout, size_of(dout_dtype)) || !aligned(dtable, size_of(dtable_dtype)))
        return SDP4_EALIGN;
    const int64_t need = sdp4::embedding_grad_workspace(rows, vocab, cols);
    const int rc = check_workspace(workspace, workspace_bytes, need);
    if (rc != SDP4_OK)
        return rc;
    const Area in = d.area(rows, cols), out = t.area(vocab, cols), ids = flat(tokens, 8 * rows), work = flat(workspace, need);
    if (clash(out, {}, {in, ids, work}) || clash(work, {}, {in, ids}))
        return SDP4_EINVAL;
    return sdp4::launch_embedding_grad({tokens, rows, vocab}, cols, scale, accumulate != 0, dout_dtype, {dout, dout_stride},
                                       dtable_dtype, {dtable, dtable_stride}, workspace, as_stream(stream));
}

int64_t sdp4_embedding_grad_workspace(int64_t rows, int64_t vocab, int64_t cols)
{
    return valid_tokens(rows, vocab, cols, 1.0f) && rows <= SDP4_MAX_GRAD_TOKENS
               ? sdp4::embedding_grad_workspace(rows, vocab, cols)
               : -1;
}

} // extern "C"
