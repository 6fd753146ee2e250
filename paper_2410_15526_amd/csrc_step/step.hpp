// step.hpp -- interface between the C ABI layer (abi_step.cpp, abi_layer.cpp)
// and the launchers of the training-step operators (k_dropout.hip,
// k_logprob.hip, k_qk.hip, k_attention.hip, k_attention_grad.hip,
// k_block_norm.hip, k_embedding.hip).  Launchers assume validated arguments.
#pragma once

#include "launch.hpp"
#include "sdp4.h"

namespace sdp4 {

// launch() with a number of wavefronts known at run time: at least WAVES, at most eight.
template <int WAVES = 1, typename... Params, typename... Args>
int launch_waves(int waves, void (*kernel)(Params...), int64_t nwork_blocks, int cap, hipStream_t stream, Args... args)
{
    if constexpr (WAVES < 8)
        if (waves > WAVES)
            return launch_waves<WAVES + 1>(waves, kernel, nwork_blocks, cap, stream, args...);
    return launch<WAVES>(kernel, nwork_blocks, cap, stream, args...);
}

// A two-dimensional array with unit stride in a row.
template <class P>
struct Rows {
    P p = nullptr;
    int64_t stride = 0; // elements from one row to the next
};

struct Dropout {
    int64_t rows, cols;
    uint32_t drop; // elements whose 16-bit uniform lies below are dropped
    float scale;   // of the others
    uint64_t seed, offset;
};

// x, bias, residual -> y.  `in` and `out` are element types (SDP4_F32, SDP4_BF16).
int launch_dropout_add(const Dropout &d, int in, Rows<const void *> x, const void *bias, int out,
                       Rows<const void *> residual, Rows<void *> y, hipStream_t s);
// The same without bias and residual, and the column sums of the result in float32.
int launch_dropout_grad(const Dropout &d, int in, Rows<const void *> dy, int out, Rows<void *> dx, float *dbias,
                        float *workspace, hipStream_t s);
int64_t dropout_grad_workspace(int64_t rows, int64_t cols);

struct TokenStats {
    const int64_t *targets;
    float *logp, *lse, *entropy;
    int top_k;
    float *top_logp;
    int64_t *top_ids;
};
struct TokenGrads { // of the loss with respect to logp, entropy, lse; null where there is none
    const float *logp, *entropy, *lse;
};

int launch_token_logprob(int dtype, Rows<const void *> x, int64_t rows, int64_t vocab, const TokenStats &out,
                         void *workspace, hipStream_t s);
int launch_token_logprob_grad(int dtype, Rows<const void *> x, int64_t rows, int64_t vocab, const int64_t *targets,
                              const float *lse, const float *entropy, const TokenGrads &g, Rows<void *> dx,
                              int64_t width, hipStream_t s);
int launch_token_loss(int dtype, Rows<const void *> x, int64_t rows, int64_t vocab, const TokenStats &out,
                      const TokenGrads &g, Rows<void *> dx, int64_t width, void *workspace, hipStream_t s);
// `fewer`: the most that so many rows or fewer take.
int64_t token_logprob_workspace(int64_t rows, int64_t vocab, int top_k, bool fewer);

struct Heads {
    void *p = nullptr;
    int64_t token_stride = 0, head_stride = 0;
    int heads = 0;
};
struct Rope {
    const float *table; // [rows][rot]: rot / 2 cosines, then as many sines
    int64_t rows;
    int rot;
    bool interleaved;
    const int64_t *positions; // null: the token's index
};
struct HeadNorm {
    bool on;
    float eps;
    const void *weight[2]; // queries', keys'; null: none
};

// x[0], x[1]: queries, keys (heads = 0: none) -> y
int launch_qk(int dtype, const Heads (&x)[2], const Heads (&y)[2], int64_t tokens, int dim, const HeadNorm &norm,
              const Rope &rope, hipStream_t s);
int launch_qk_grad(int dtype, const Heads (&dy)[2], const Heads (&x)[2], const Heads (&dx)[2], int64_t tokens,
                   int dim, const HeadNorm &norm, const Rope &rope, float *const (&dw)[2], float *workspace,
                   hipStream_t s);
int64_t qk_grad_workspace(int64_t tokens, int q_heads, int k_heads, int dim);
int launch_rope_table(const double *inv_freq, int half, int64_t start, int64_t rows, double scale, float *table,
                      hipStream_t s);

// Packed sequences: sequence i has rows offsets[i] .. offsets[i + 1] - 1.
struct Sequences {
    const int64_t *offsets; // null: one sequence of all rows
    int64_t count;
    int tokens;
};
struct Attention {
    Sequences seq;
    int dim, group; // elements of a head; query heads that share a key and value head
    float scale;
};
int launch_attention(int dtype, const Attention &a, const Heads &q, const Heads &k, const Heads &v, const Heads &out,
                     float *lse, hipStream_t s);
int launch_attention_grad(int dtype, const Attention &a, const Heads &dout, const Heads &q, const Heads &k, const Heads &v,
                          const Heads &out, const float *lse, const Heads &dq, const Heads &dk, const Heads &dv,
                          float *workspace, hipStream_t s);
int64_t attention_grad_workspace(int64_t tokens, int q_heads, int k_heads, int dim);

// The joint of two blocks; arrays of the branch's element type, the residual stream's, weights of the branch's.
struct BlockNorm {
    bool post_norm;
    float post_eps, pre_eps;
    const void *post_weight, *pre_weight; // null: ones
    const float *gate;                    // of a row; null: ones
    float branch_scale, residual_scale;
};
int launch_block_norm(int x_dtype, int y_dtype, const BlockNorm &p, int64_t rows, int64_t cols, Rows<const void *> branch,
                      Rows<const void *> residual, Rows<void *> y, Rows<void *> h, hipStream_t s);
struct BlockNormArrays {
    Rows<const void *> dh, dy, branch, y;
    Rows<void *> dbranch, dresidual;
    float *dpost_weight, *dpre_weight, *dgate;
};
template <class X, class Y>
struct BlockNormGrad {
    Rows<const X *> dh;
    Rows<const Y *> dy;
    Rows<const X *> branch;
    Rows<const Y *> y;
    Rows<X *> dbranch;
    Rows<Y *> dres;
    float *dgate, *post_parts, *pre_parts;
};
int launch_block_norm_grad(int x_dtype, int y_dtype, const BlockNorm &p, int64_t rows, int64_t cols, const BlockNormArrays &a,
                           float *workspace, hipStream_t s);
int64_t block_norm_grad_workspace(int64_t rows, int64_t cols);

struct Tokens {
    const int64_t *p;
    int64_t rows, vocab;
};
int launch_embedding(const Tokens &t, int64_t cols, float scale, int in, Rows<const void *> table, int out, Rows<void *> y,
                     hipStream_t s);
int launch_embedding_grad(const Tokens &t, int64_t cols, float scale, bool accumulate, int in, Rows<const void *> dy, int out,
                          Rows<void *> dtable, void *workspace, hipStream_t s);
int64_t embedding_grad_workspace(int64_t rows, int64_t vocab, int64_t cols);

// out[c] = the sum of p[i * pitch + c] over i < count, for c < cols, in a fixed order; one or two such sums (out null: none).
struct Parts {
    const float *p = nullptr;
    int64_t count = 0;
    float *out = nullptr;
};
int launch_sum_parts(const Parts (&parts)[2], int64_t pitch, int64_t cols, hipStream_t s);

} // namespace sdp4
