// abi_step.cpp -- the C ABI of the training-step operators declared in
// include/sdp4.h: host-side argument checks, then the launches.
//
// Every check runs before any HIP call.
#include "abi_checks.hpp"

#include <cmath>

namespace {

using namespace sdp4::checks;

int check_dropout(int64_t rows, int64_t cols, float p, uint64_t seed, uint64_t offset, sdp4::Dropout &d)
{
    if (!valid_shape(rows, cols) || !(p >= 0.0f && p <= 1.0f))
        return SDP4_EINVAL;
    if (offset % 8)
        return SDP4_EALIGN;
    d.rows = rows, d.cols = cols, d.seed = seed, d.offset = offset;
    d.drop = static_cast<uint32_t>(std::nearbyint(static_cast<double>(p) * 65536.0));
    d.scale = d.drop < 65536 ? static_cast<float>(65536.0 / (65536.0 - d.drop)) : 0.0f;
    return SDP4_OK;
}

// What the three token entry points share.
int check_tokens(const Matrix &x, int64_t rows, int64_t vocab, const int64_t *targets)
{
    if (!valid_dtype(x.dtype) || !valid_shape(rows, vocab) || vocab < 1 || vocab > SDP4_MAX_VOCAB ||
        !valid_matrix(x, rows, vocab))
        return SDP4_EINVAL;
    if (rows == 0)
        return SDP4_OK;
    if (!x.p)
        return SDP4_EINVAL;
    return aligned(x.p, size_of(x.dtype)) && aligned(targets, 8) ? SDP4_OK : SDP4_EALIGN;
}

int check_gradient(const Matrix &x, int64_t rows, int64_t vocab, const int64_t *targets, const sdp4::TokenGrads &g,
                   const Matrix &dx, int64_t width)
{
    if (width < vocab || width > INT32_MAX - 7 || !valid_shape(rows, width) || !valid_matrix(dx, rows, width) || !dx.p ||
        (g.logp && !targets))
        return SDP4_EINVAL;
    if (!aligned(dx.p, size_of(dx.dtype)) || !aligned(g.logp, 4) || !aligned(g.entropy, 4) || !aligned(g.lse, 4))
        return SDP4_EALIGN;
    // in place: the same rows, whose padding the gradient may write
    const Area in = x.area(rows, vocab), out = dx.area(rows, width);
    const bool in_place = dx.p == x.p && (rows <= 1 || dx.stride == x.stride);
    if (!in_place && overlap(out, in))
        return SDP4_EINVAL;
    return clash(out, {}, {flat(targets, 8 * rows), flat(g.logp, 4 * rows), flat(g.entropy, 4 * rows),
                           flat(g.lse, 4 * rows)})
               ? SDP4_EINVAL
               : SDP4_OK;
}

int check_qk(const sdp4_qk_params *p, int64_t tokens)
{
    if (!p || tokens < 0 || tokens > SDP4_MAX_ELEMENTS || !valid_dtype(p->dtype) || p->head_dim < 1 ||
        p->head_dim > SDP4_MAX_HEAD_DIM || p->rot_dim < 0 || p->rot_dim > p->head_dim || p->rot_dim % 2 ||
        (p->rot_dim > 0 && (!p->table || p->table_rows < 1 || !product_fits(p->table_rows, p->rot_dim))) ||
        (p->norm ? !(p->eps >= 0.0f) || !std::isfinite(p->eps) : p->q_weight || p->k_weight))
        return SDP4_EINVAL;
    const int64_t s = size_of(p->dtype);
    if (!aligned(p->q_weight, s) || !aligned(p->k_weight, s) || !aligned(p->table, 4) || !aligned(p->positions, 8))
        return SDP4_EALIGN;
    return SDP4_OK;
}

// One set of heads: valid, aligned; as the launchers take it.
int take_heads(const sdp4_heads *h, int64_t tokens, const sdp4_qk_params &p, sdp4_heads &out)
{
    if (!valid_heads(*h, tokens, p.head_dim) || !h->data)
        return SDP4_EINVAL;
    if (!aligned(h->data, size_of(p.dtype)))
        return SDP4_EALIGN;
    out = normal(*h, tokens, p.head_dim);
    return SDP4_OK;
}

sdp4::HeadNorm norm_of(const sdp4_qk_params &p) { return {p.norm != 0, p.eps, {p.q_weight, p.k_weight}}; }
sdp4::Rope rope_of(const sdp4_qk_params &p)
{
    return {p.table, p.table_rows, p.rot_dim, p.interleaved != 0, p.positions};
}

} // namespace

extern "C" {

int sdp4_dropout_add(const void *x, int x_dtype, int64_t x_stride, const void *bias, const void *residual,
                     int64_t residual_stride, int64_t rows, int64_t cols, float p, uint64_t seed, uint64_t offset,
                     void *y, int y_dtype, int64_t y_stride, void *stream)
{
    sdp4::Dropout d;
    const Matrix mx{x, x_dtype, x_stride}, mr{residual, y_dtype, residual_stride}, my{y, y_dtype, y_stride};
    if (!valid_dtype(x_dtype) || !valid_dtype(y_dtype))
        return SDP4_EINVAL;
    const int rc = check_dropout(rows, cols, p, seed, offset, d);
    if (rc != SDP4_OK)
        return rc;
    if (!valid_matrix(mx, rows, cols) || !valid_matrix(my, rows, cols) || (residual && !valid_matrix(mr, rows, cols)))
        return SDP4_EINVAL;
    if (rows == 0 || cols == 0)
        return SDP4_OK;
    if (!x || !y)
        return SDP4_EINVAL;
    if (!aligned(x, size_of(x_dtype)) || !aligned(bias, size_of(x_dtype)) || !aligned(residual, size_of(y_dtype)) ||
        !aligned(y, size_of(y_dtype)))
        return SDP4_EALIGN;
    if (clash(my.area(rows, cols), {mx.area(rows, cols), mr.area(rows, cols)}, {flat(bias, cols * size_of(x_dtype))}))
        return SDP4_EINVAL;
    return sdp4::launch_dropout_add(d, x_dtype, {x, x_stride}, bias, y_dtype, {residual, residual_stride},
                                    {y, y_stride}, as_stream(stream));
}

int sdp4_dropout_add_grad(const void *dy, int y_dtype, int64_t dy_stride, int64_t rows, int64_t cols, float p,
                          uint64_t seed, uint64_t offset, void *dx, int x_dtype, int64_t dx_stride, float *dbias,
                          void *workspace, int64_t workspace_bytes, void *stream)
{
    sdp4::Dropout d;
    const Matrix mdy{dy, y_dtype, dy_stride}, mdx{dx, x_dtype, dx_stride};
    if (!valid_dtype(x_dtype) || !valid_dtype(y_dtype))
        return SDP4_EINVAL;
    int rc = check_dropout(rows, cols, p, seed, offset, d);
    if (rc != SDP4_OK)
        return rc;
    if (!valid_matrix(mdy, rows, cols) || !valid_matrix(mdx, rows, cols))
        return SDP4_EINVAL;
    if (cols == 0 || (rows == 0 && !dbias))
        return SDP4_OK;
    if (rows > 0 && (!dy || !dx))
        return SDP4_EINVAL;
    if (!aligned(dy, size_of(y_dtype)) || !aligned(dx, size_of(x_dtype)) || !aligned(dbias, 4))
        return SDP4_EALIGN;
    if (!dbias)
        return clash(mdx.area(rows, cols), {mdy.area(rows, cols)}, {})
                   ? SDP4_EINVAL
                   : sdp4::launch_dropout_add(d, y_dtype, {dy, dy_stride}, nullptr, x_dtype, {}, {dx, dx_stride},
                                              as_stream(stream));
    const int64_t need = sdp4::dropout_grad_workspace(rows, cols);
    rc = check_workspace(workspace, workspace_bytes, need);
    if (rc != SDP4_OK)
        return rc;
    const Area in = mdy.area(rows, cols), out = mdx.area(rows, cols), sums = flat(dbias, 4 * cols),
               work = flat(workspace, need);
    if (clash(out, {in}, {sums, work}) || clash(sums, {}, {in, work}) || overlap(work, in))
        return SDP4_EINVAL;
    if (rows == 0) // an empty sum
        return sdp4::launch_sum_parts({{nullptr, 0, dbias}, {}}, cols, cols, as_stream(stream));
    return sdp4::launch_dropout_grad(d, y_dtype, {dy, dy_stride}, x_dtype, {dx, dx_stride}, dbias,
                                     static_cast<float *>(workspace), as_stream(stream));
}

int64_t sdp4_dropout_grad_workspace(int64_t rows, int64_t cols)
{
    return valid_shape(rows, cols) ? sdp4::dropout_grad_workspace(rows, cols) : -1;
}

int sdp4_token_logprob(const void *logits, int dtype, int64_t stride, int64_t rows, int64_t vocab,
                       const int64_t *targets, int top_k, float *logp, float *lse, float *entropy, float *top_logp,
                       int64_t *top_ids, void *workspace, int64_t workspace_bytes, void *stream)
{
    const Matrix x{logits, dtype, stride};
    int rc = check_tokens(x, rows, vocab, targets);
    if (rc != SDP4_OK)
        return rc;
    if (top_k < 0 || top_k > SDP4_MAX_TOP || top_k > vocab || (logp && !targets))
        return SDP4_EINVAL;
    if (rows == 0)
        return SDP4_OK;
    if (top_k > 0 && (!top_logp || !top_ids))
        return SDP4_EINVAL;
    if (!aligned(logp, 4) || !aligned(lse, 4) || !aligned(entropy, 4) || !aligned(top_logp, 4) || !aligned(top_ids, 8))
        return SDP4_EALIGN;
    const int64_t need = sdp4::token_logprob_workspace(rows, vocab, top_k, false);
    rc = check_workspace(workspace, workspace_bytes, need);
    if (rc != SDP4_OK)
        return rc;
    const Area ins[2] = {x.area(rows, vocab), flat(targets, 8 * rows)};
    const Area outs[6] = {flat(logp, 4 * rows), flat(lse, 4 * rows), flat(entropy, 4 * rows),
                          flat(top_k ? top_logp : nullptr, 4 * rows * top_k),
                          flat(top_k ? top_ids : nullptr, 8 * rows * top_k), flat(need ? workspace : nullptr, need)};
    for (int i = 0; i < 6; ++i) {
        if (clash(outs[i], {}, {ins[0], ins[1]}))
            return SDP4_EINVAL;
        for (int j = 0; j < i; ++j)
            if (overlap(outs[i], outs[j]))
                return SDP4_EINVAL;
    }
    return sdp4::launch_token_logprob(dtype, {logits, stride}, rows, vocab,
                                      {targets, logp, lse, entropy, top_k, top_logp, top_ids}, workspace,
                                      as_stream(stream));
}

int64_t sdp4_token_logprob_workspace(int64_t rows, int64_t vocab, int top_k)
{
    if (!valid_shape(rows, vocab) || vocab < 1 || vocab > SDP4_MAX_VOCAB || top_k < 0 || top_k > SDP4_MAX_TOP)
        return -1;
    return sdp4::token_logprob_workspace(rows, vocab, top_k, true);
}

int sdp4_token_logprob_grad(const void *logits, int dtype, int64_t stride, int64_t rows, int64_t vocab,
                            const int64_t *targets, const float *lse, const float *entropy, const float *g_logp,
                            const float *g_entropy, const float *g_lse, void *dlogits, int64_t dlogits_stride,
                            int64_t width, void *stream)
{
    const Matrix x{logits, dtype, stride}, dx{dlogits, dtype, dlogits_stride};
    const sdp4::TokenGrads g{g_logp, g_entropy, g_lse};
    int rc = check_tokens(x, rows, vocab, targets);
    if (rc != SDP4_OK || rows == 0)
        return rc;
    rc = check_gradient(x, rows, vocab, targets, g, dx, width);
    if (rc != SDP4_OK)
        return rc;
    if (!lse || (g_entropy && !entropy))
        return SDP4_EINVAL;
    if (!aligned(lse, 4) || !aligned(entropy, 4))
        return SDP4_EALIGN;
    if (clash(dx.area(rows, width), {}, {flat(lse, 4 * rows), flat(entropy, 4 * rows)}))
        return SDP4_EINVAL;
    return sdp4::launch_token_logprob_grad(dtype, {logits, stride}, rows, vocab, targets, lse, entropy, g,
                                           {dlogits, dlogits_stride}, width, as_stream(stream));
}

int sdp4_token_loss(const void *logits, int dtype, int64_t stride, int64_t rows, int64_t vocab,
                    const int64_t *targets, const float *g_logp, const float *g_entropy, const float *g_lse,
                    float *logp, float *lse, float *entropy, void *dlogits, int64_t dlogits_stride, int64_t width,
                    void *workspace, int64_t workspace_bytes, void *stream)
{
    const Matrix x{logits, dtype, stride}, dx{dlogits, dtype, dlogits_stride};
    const sdp4::TokenGrads g{g_logp, g_entropy, g_lse};
    int rc = check_tokens(x, rows, vocab, targets);
    if (rc != SDP4_OK || rows == 0)
        return rc;
    rc = check_gradient(x, rows, vocab, targets, g, dx, width);
    if (rc != SDP4_OK)
        return rc;
    if (!lse || !entropy || (logp && !targets))
        return SDP4_EINVAL;
    if (!aligned(logp, 4) || !aligned(lse, 4) || !aligned(entropy, 4))
        return SDP4_EALIGN;
    const int64_t need = sdp4::token_logprob_workspace(rows, vocab, 0, false);
    rc = check_workspace(workspace, workspace_bytes, need);
    if (rc != SDP4_OK)
        return rc;
    const Area ins[6] = {x.area(rows, vocab),    flat(targets, 8 * rows),   flat(g_logp, 4 * rows),
                         flat(g_entropy, 4 * rows), flat(g_lse, 4 * rows), dx.area(rows, width)};
    const Area outs[4] = {flat(logp, 4 * rows), flat(lse, 4 * rows), flat(entropy, 4 * rows),
                          flat(need ? workspace : nullptr, need)};
    for (int i = 0; i < 4; ++i) {
        for (const Area &a : ins)
            if (overlap(outs[i], a))
                return SDP4_EINVAL;
        for (int j = 0; j < i; ++j)
            if (overlap(outs[i], outs[j]))
                return SDP4_EINVAL;
    }
    return sdp4::launch_token_loss(dtype, {logits, stride}, rows, vocab,
                                   {targets, logp, lse, entropy, 0, nullptr, nullptr}, g, {dlogits, dlogits_stride},
                                   width, workspace, as_stream(stream));
}

int sdp4_qk_norm_rope(const sdp4_heads *q, const sdp4_heads *k, const sdp4_qk_params *params, int64_t tokens,
                      const sdp4_heads *q_out, const sdp4_heads *k_out, void *stream)
{
    int rc = check_qk(params, tokens);
    if (rc != SDP4_OK)
        return rc;
    if (!q || !q_out || !k != !k_out)
        return SDP4_EINVAL;
    if (tokens == 0)
        return SDP4_OK;
    const sdp4_heads *in[2] = {q, k}, *out[2] = {q_out, k_out};
    sdp4_heads ih[2]{}, oh[2]{};
    const int dim = params->head_dim;
    const int64_t s = size_of(params->dtype);
    const int sides = k ? 2 : 1;
    for (int i = 0; i < sides; ++i) {
        if ((rc = take_heads(in[i], tokens, *params, ih[i])) || (rc = take_heads(out[i], tokens, *params, oh[i])))
            return rc;
        if (ih[i].heads != oh[i].heads)
            return SDP4_EINVAL;
    }
    for (int i = 0; i < sides; ++i) {
        const Area o = area_of(oh[i], tokens, dim, params->dtype);
        for (int j = 0; j < sides; ++j) {
            if (!(i == j && same_heads(ih[j], oh[i], tokens)) && heads_overlap(oh[i], ih[j], tokens, dim, params->dtype))
                return SDP4_EINVAL;
            if (j < i && heads_overlap(oh[i], oh[j], tokens, dim, params->dtype))
                return SDP4_EINVAL;
        }
        if (clash(o, {}, {flat(params->q_weight, s * dim), flat(params->k_weight, s * dim),
                          flat(params->rot_dim ? params->table : nullptr, 4 * params->table_rows * params->rot_dim),
                          flat(params->positions, 8 * tokens)}))
            return SDP4_EINVAL;
    }
    return sdp4::launch_qk(params->dtype, {launch_heads(ih[0]), launch_heads(ih[1])},
                           {launch_heads(oh[0]), launch_heads(oh[1])}, tokens, dim, norm_of(*params), rope_of(*params),
                           as_stream(stream));
}

int sdp4_qk_norm_rope_grad(const sdp4_heads *dq_out, const sdp4_heads *dk_out, const sdp4_heads *q,
                           const sdp4_heads *k, const sdp4_qk_params *params, int64_t tokens, const sdp4_heads *dq,
                           const sdp4_heads *dk, float *dq_weight, float *dk_weight, void *workspace,
                           int64_t workspace_bytes, void *stream)
{
    int rc = check_qk(params, tokens);
    if (rc != SDP4_OK)
        return rc;
    const bool norm = params->norm != 0;
    if (!dq_out || !dq || !dk_out != !dk || (norm && (!q || !k != !dk)))
        return SDP4_EINVAL;
    if ((dq_weight && !params->q_weight) || (dk_weight && (!params->k_weight || !dk)))
        return SDP4_EINVAL;
    if (!aligned(dq_weight, 4) || !aligned(dk_weight, 4))
        return SDP4_EALIGN;
    const int dim = params->head_dim;
    const int64_t s = size_of(params->dtype);
    if (tokens == 0) { // empty sums
        return dq_weight || dk_weight
                   ? sdp4::launch_sum_parts({{nullptr, 0, dq_weight}, {nullptr, 0, dk_weight}}, dim, dim, as_stream(stream))
                   : SDP4_OK;
    }
    const sdp4_heads *gs[2] = {dq_out, dk_out}, *xs[2] = {q, k}, *os[2] = {dq, dk};
    sdp4_heads gh[2]{}, xh[2]{}, oh[2]{};
    const int sides = dk ? 2 : 1;
    for (int i = 0; i < sides; ++i) {
        if ((rc = take_heads(gs[i], tokens, *params, gh[i])) || (rc = take_heads(os[i], tokens, *params, oh[i])) ||
            (norm && (rc = take_heads(xs[i], tokens, *params, xh[i]))))
            return rc;
        if (gh[i].heads != oh[i].heads || (norm && xh[i].heads != oh[i].heads))
            return SDP4_EINVAL;
    }
    const int64_t need = dq_weight || dk_weight ? sdp4::qk_grad_workspace(tokens, oh[0].heads, oh[1].heads, dim) : 0;
    rc = check_workspace(workspace, workspace_bytes, need);
    if (rc != SDP4_OK)
        return rc;
    const Area small[4] = {flat(params->q_weight, s * dim), flat(params->k_weight, s * dim),
                           flat(params->rot_dim ? params->table : nullptr, 4 * params->table_rows * params->rot_dim),
                           flat(params->positions, 8 * tokens)};
    const Area sums[3] = {flat(dq_weight, 4 * dim), flat(dk_weight, 4 * dim), flat(need ? workspace : nullptr, need)};
    for (int i = 0; i < 3; ++i) {
        if (clash(sums[i], {}, {small[0], small[1], small[2], small[3]}))
            return SDP4_EINVAL;
        for (int j = 0; j < i; ++j)
            if (overlap(sums[i], sums[j]))
                return SDP4_EINVAL;
    }
    for (int i = 0; i < sides; ++i) {
        const Area o = area_of(oh[i], tokens, dim, params->dtype);
        for (int j = 0; j < sides; ++j) {
            const Area g = area_of(gh[j], tokens, dim, params->dtype), x = area_of(xh[j], tokens, dim, params->dtype);
            if (!(i == j && same_heads(gh[j], oh[i], tokens)) && heads_overlap(oh[i], gh[j], tokens, dim, params->dtype))
                return SDP4_EINVAL;
            if (norm && !(i == j && same_heads(xh[j], oh[i], tokens)) && heads_overlap(oh[i], xh[j], tokens, dim, params->dtype))
                return SDP4_EINVAL;
            if (j < i && heads_overlap(oh[i], oh[j], tokens, dim, params->dtype))
                return SDP4_EINVAL;
            if (clash(g, {}, {sums[0], sums[1], sums[2]}) || (norm && clash(x, {}, {sums[0], sums[1], sums[2]})))
                return SDP4_EINVAL;
        }
        if (clash(o, {}, {small[0], small[1], small[2], small[3], sums[0], sums[1], sums[2]}))
            return SDP4_EINVAL;
    }
    return sdp4::launch_qk_grad(params->dtype, {launch_heads(gh[0]), launch_heads(gh[1])},
                                {launch_heads(xh[0]), launch_heads(xh[1])}, {launch_heads(oh[0]), launch_heads(oh[1])},
                                tokens, dim, norm_of(*params), rope_of(*params), {dq_weight, dk_weight},
                                static_cast<float *>(workspace), as_stream(stream));
}

int64_t sdp4_qk_grad_workspace(int64_t tokens, int q_heads, int k_heads, int head_dim)
{
    if (tokens < 0 || q_heads < 0 || k_heads < 0 || q_heads > (1 << 20) || k_heads > (1 << 20) || head_dim < 1 ||
        head_dim > SDP4_MAX_HEAD_DIM || !product_fits(tokens, ((int64_t)q_heads + k_heads) * head_dim))
        return -1;
    return sdp4::qk_grad_workspace(tokens, q_heads, k_heads, head_dim);
}

int sdp4_rope_table(const double *inv_freq, int half, int64_t start, int64_t rows, double scale, float *table,
                    void *stream)
{
    if (half < 1 || half > SDP4_MAX_HEAD_DIM / 2 || rows < 0 || start < 0 || start > SDP4_MAX_ELEMENTS ||
        !product_fits(rows, 2 * half) || !std::isfinite(scale))
        return SDP4_EINVAL;
    if (rows == 0)
        return SDP4_OK;
    if (!inv_freq || !table)
        return SDP4_EINVAL;
    if (!aligned(inv_freq, 8) || !aligned(table, 4))
        return SDP4_EALIGN;
    if (overlap(flat(table, 8 * rows * half), flat(inv_freq, 8 * half)))
        return SDP4_EINVAL;
    return sdp4::launch_rope_table(inv_freq, half, start, rows, scale, table, as_stream(stream));
}

} // extern "C"
