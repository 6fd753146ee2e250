/*
 * sdp4.h -- C ABI of the MI355X (gfx950) compression hot path of SDP4Bit
 * (Jia et al., "SDP4Bit: Toward 4-bit Communication Quantization in Sharded
 * Data Parallelism for LLM Training", NeurIPS 2024, arXiv 2410.15526).
 *
 * Two per-GPU paths, each a few HIP kernels:
 *   - qWD (Sec. 3.1, Alg. 2): 4-bit group-wise quantization of the weight
 *     difference d = w_main - w_model before the weight all-gather, and the
 *     matching dequantize-and-accumulate into the resident model weights.
 *   - TLq-HS (Sec. 3.2, Alg. 4, Sec. 3.3): blockwise Hadamard transform and
 *     8-bit group quantization before the intra-node all-to-all; dequantize,
 *     reduce over P chunks and re-quantize to 4 bits before the inter-node
 *     all-to-all; dequantize, reduce over Q chunks and apply the inverse
 *     Hadamard transform.
 *
 * Conventions common to every entry point
 * ---------------------------------------
 *  Memory     All array arguments are device pointers (HBM), except the
 *             pointer *tables* of sdp4_dequant_reduce / sdp4_reduce_f32,
 *             which are host arrays of device pointers read during the call
 *             only.  The caller owns every buffer; the library allocates
 *             nothing, frees nothing and keeps no state between calls.
 *             The library sees addresses only: every buffer must hold
 *             the bytes its call touches (given with each entry point);
 *             a shorter one is overrun on the device.
 *  Streams    `stream` is a hipStream_t (NULL = the default stream).  Calls
 *             enqueue their kernels and return; results are visible after
 *             the usual stream synchronization.  Calls are thread-safe.
 *  Errors     Arguments are checked on the host before anything is
 *             enqueued; on any error nothing is written and nothing is
 *             launched.  Device faults surface at the caller's next sync.
 *  Sizes      n / n_chunk count elements and may be 0 (no-op), at most
 *             SDP4_MAX_ELEMENTS.  They must be multiples of
 *             lcm(group, hadamard_block), which for the allowed powers of
 *             two is max(group, hadamard_block).
 *  Alignment  Element arrays (float data, codes) must be 16-byte aligned;
 *             per-group header arrays (scales, minima) 4-byte aligned.
 *  Aliasing   Outputs must not overlap inputs, except where stated.
 *  Inputs     Must be finite; non-finite inputs give unspecified codes.
 *
 * Quantized message layout (identical on the wire and in memory)
 * ---------------------------------------------------------------
 *  8-bit codes: int8, one per element, two's complement, range [-127, 127].
 *  4-bit codes: two per byte, element 2j in the low nibble of byte j and
 *               element 2j+1 in the high nibble.  Gradient codes are signed
 *               two's-complement nibbles in [-7, 7]; weight-difference codes
 *               are unsigned in [0, 15] (signed in [-7, 7] for the
 *               symmetric qWD codec).
 *  Headers:     one float32 per group of `group` consecutive elements, in
 *               group order (scale; plus the group minimum for qWD).
 *  Chunk j of a message of n_chunk elements starts at byte
 *  j * n_chunk * bits / 8 of the codes and at float j * n_chunk / group of
 *  the headers, so a message is split for an all-to-all by pointer
 *  arithmetic alone.
 *
 * Numerics (the paper leaves these unstated; this library fixes them and
 * every kernel follows them exactly, so results are reproducible bit for bit)
 *  - symmetric quantizer (Sec. 2.2), k = 8 or 4 bits, qmax = 2^(k-1) - 1:
 *      s = max |x| over the group, scale = s / qmax, inv = qmax / s,
 *      code = clamp(rint(x * inv), -qmax, qmax), value = code * scale;
 *      a group with s = 0 (or with qmax / s overflowing) has scale 0 and
 *      all-zero codes;
 *  - asymmetric quantizer (qWD): mn, mx = min, max of the group,
 *      R = mx - mn, scale = R / 15, inv = 15 / R,
 *      code = clamp(rint((x - mn) * inv), 0, 15), value = fma(code, scale, mn);
 *      a group with R = 0 has scale 0 and all-zero codes (value = mn);
 *  - Hadamard: per block of n = hadamard_block consecutive elements,
 *      y = (H_n / sqrt(n)) x with H_n the Sylvester matrix
 *      H_n[i][j] = (-1)^popcount(i & j); computed by butterflies of width
 *      1, 2, 4, ..., n/2 followed by one multiplication by the float nearest
 *      to 1/sqrt(n).  The map is symmetric, orthogonal and its own inverse;
 *  - dequantize-reduce: r = +0, then r = fma(code_p, scale_p, r) for
 *      p = 0, 1, ..., P-1 in order;
 *  - bfloat16 model weights are widened exactly and narrowed with
 *      round-to-nearest-even.
 *  All float arithmetic is IEEE binary32 with round-to-nearest-even and no
 *  flush of denormals; division is correctly rounded.
 */
#ifndef SDP4_H
#define SDP4_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Status codes returned by every entry point. */
#define SDP4_OK 0
#define SDP4_EINVAL 1 /* null pointer, bad bit width, group, block, dtype, overlap */
#define SDP4_EALIGN 2 /* size not a multiple of lcm(group, block), or pointer misaligned */
#define SDP4_ERANGE 3 /* peer count outside [1, 16] */
#define SDP4_EHIP 4   /* a HIP launch failed; see sdp4_last_hip_error() */

/* Model-weight element types for qWD. */
#define SDP4_F32 0  /* float32 */
#define SDP4_BF16 1 /* bfloat16 stored as uint16 bit patterns */

/* Limits. */
#define SDP4_MIN_GROUP 32
#define SDP4_MAX_GROUP 4096
#define SDP4_MAX_HADAMARD 1024
#define SDP4_MAX_PEERS 16
#define SDP4_MAX_ELEMENTS ((int64_t)1 << 48) /* n above this is EINVAL (byte counts stay in range) */

/*
 * qWD encode -- Alg. 2, CompressedForwardPass, first two steps: the weight
 * difference d = w_main[p] - w_model[p] of this GPU's shard, quantized to
 * 4 bits per group (Sec. 3.1).
 *
 *   w_new   [n] float32        main (optimizer) weights of the shard
 *   w_prev  [n] prev_dtype     model weights as last communicated
 *                              (float32, or bfloat16 bits when SDP4_BF16)
 *   n                          elements; multiple of group
 *   group                      power of two in [32, 4096]
 *   codes   [n/2] uint8        out: packed unsigned 4-bit codes
 *   scale   [n/group] float32  out: (max - min) / 15 of each group
 *   minv    [n/group] float32  out: minimum of each group
 * Inputs are not modified.  Errors: EINVAL (null, bad group or dtype,
 * overlap of an output with an input), EALIGN, EHIP.
 */
int sdp4_qwd_encode(const float *w_new, const void *w_prev, int prev_dtype, int64_t n, int group,
                    uint8_t *codes, float *scale, float *minv, void *stream);

/*
 * qWD decode -- Alg. 2, CompressedForwardPass, w_model <- w_model + d after
 * the all-gather; in place on the model weights, which double as the
 * previous weights so no extra buffer is needed (Sec. 3.3, memory
 * efficiency for weight differences).
 *
 *   codes, scale, minv   a message produced by sdp4_qwd_encode (any shard)
 *   n, group             as for the encoder
 *   w_prev [n] prev_dtype  in/out: w_prev[i] <- narrow(widen(w_prev[i]) + value[i])
 * Errors: EINVAL, EALIGN, EHIP.  w_prev must not overlap the message.
 */
int sdp4_qwd_decode(const uint8_t *codes, const float *scale, const float *minv, int64_t n,
                    int group, void *w_prev, int prev_dtype, void *stream);

/*
 * Symmetric qWD encode -- the weight difference of Alg. 2 quantized with the
 * paper's own symmetric quantizer of Sec. 2.2 at 4 bits instead of the
 * asymmetric min-max codec:
 *      s = max |d| per group, scale = s / 7, inv = 7 / s,
 *      code = clamp(rint(d * inv), -7, 7), value = code * scale;
 *      a group with s = 0 has scale 0 and all-zero codes.
 *
 *   w_new, w_prev, prev_dtype, n, group   as for sdp4_qwd_encode
 *   codes   [n/2] uint8        out: packed two's-complement nibbles
 *                              (even element in the low nibble; -8 unused)
 *   scale   [n/group] float32  out: s / 7 of each group
 * The message is 4 + 32/group bits per element (no minimum).  Inputs are
 * not modified.  Errors: EINVAL, EALIGN, EHIP as for sdp4_qwd_encode.
 */
int sdp4_qwd_encode_sym(const float *w_new, const void *w_prev, int prev_dtype, int64_t n, int group,
                        uint8_t *codes, float *scale, void *stream);

/*
 * Symmetric qWD decode: w_prev[i] <- narrow(widen(w_prev[i]) + code[i] *
 * scale[i / group]) in place (the product and the sum each round once).
 *
 *   codes, scale   a message produced by sdp4_qwd_encode_sym
 *   n, group, w_prev, prev_dtype   as for sdp4_qwd_decode
 * Errors: EINVAL, EALIGN, EHIP.  w_prev must not overlap the message.
 */
int sdp4_qwd_decode_sym(const uint8_t *codes, const float *scale, int64_t n, int group, void *w_prev,
                        int prev_dtype, void *stream);

/*
 * Gradient quantization, first level -- Alg. 4, g^ <- Hadamard(grad) then
 * Quantize8Bit (bits = 8, TLq-HS); bits = 4 gives the uniform-level 4-bit
 * variant (ULq), hadamard_block = 0 the variant without smoother (TLq).
 *
 *   x      [n] float32           gradient (this GPU's full local gradient)
 *   n                            multiple of max(group, hadamard_block)
 *   bits                         8 or 4
 *   hadamard_block               0 (no transform) or a power of two in [2, 1024]
 *   group                        power of two in [32, 4096]
 *   codes  [n*bits/8] bytes      out: int8 codes, or packed signed nibbles
 *   scale  [n/group] float32     out: per-group scale
 * Errors: EINVAL, EALIGN, EHIP.
 */
int sdp4_grad_quant(const float *x, int64_t n, int bits, int hadamard_block, int group, void *codes,
                    float *scale, void *stream);

/*
 * Dequantize + Reduction over P received chunks -- Alg. 4 after each
 * all-to-all -- fused with what follows it on the path:
 *   bits_out = 4 or 8: re-quantization of the reduced values (Quantize4Bit
 *     before the inter-node all-to-all).  No Hadamard transform here: it is
 *     removed by the simplification of Sec. 3.3 (H H = I), so
 *     hadamard_block must be 0.
 *   bits_out = 0: float32 result; with hadamard_block > 0 the inverse
 *     transform (the same transform, Sec. 3.3 moves it past the reduction),
 *     then multiplication by out_scale unless out_scale == 1 (e.g. 1/(P*Q)
 *     to average instead of sum).
 *
 *   P                    number of chunks, 1..16
 *   codes  [P] (host)    device pointers to each chunk's codes (bits_in wide)
 *   scales [P] (host)    device pointers to each chunk's per-group scales
 *   n_chunk              elements per chunk; multiple of max(group, hadamard_block)
 *   bits_in              8 or 4 (signed codes)
 *   group                power of two in [32, 4096], shared by input and output
 *   bits_out             0, 4 or 8
 *   hadamard_block       0 or power of two in [2, 1024] (0 when bits_out > 0)
 *   out_scale            finite factor applied last when bits_out = 0
 *   out_codes  [n_chunk*bits_out/8]   out (bits_out > 0)
 *   out_scales [n_chunk/group] float  out (bits_out > 0)
 *   out_f32    [n_chunk] float32      out: the result when bits_out = 0;
 *                                     optional (may be NULL) when bits_out > 0,
 *                                     then it receives the reduced values
 *                                     before re-quantization
 * Errors: ERANGE (P outside 1..16), EINVAL, EALIGN, EHIP.
 */
int sdp4_dequant_reduce(int P, const void *const *codes, const float *const *scales,
                        int64_t n_chunk, int bits_in, int group, int bits_out, int hadamard_block,
                        float out_scale, void *out_codes, float *out_scales, float *out_f32,
                        void *stream);

/*
 * Stochastically rounded variants of the two gradient quantizers.  The
 * convergence analysis (Sec. 4.2: U_g in Alg. 3 is an unbiased compressor,
 * Definition of the unbiased kappa-approximate compressor) assumes unbiased
 * gradient compression; with stochastic rounding the symmetric quantizer is
 * unbiased: code = clamp(floor(fl(x * inv) + u), -qmax, qmax) with
 * u in [0, 1) drawn per element, so E[code * scale] = x (up to 2^-16 of a
 * quantization step).
 *
 * u of element e = offset + i (i the index within this call) is the 16-bit
 * uniform u = h / 65536, h = half (e % 2: 0 low, 1 high) of word (e / 2) % 4
 * of Philox4x32-10 (Salmon et al., SC'11) with counter (e / 8 as two 32-bit
 * words low first, 0, 0) and key (seed low word, seed high word).  The same
 * (seed, e) always gives the same u, so a buffer quantized in pieces with
 * matching offsets equals the one-call result.
 *
 *   seed     64-bit key of the generator (e.g. derived from the step and rank)
 *   offset   element position of x[0] in the caller's stream; multiple of 8
 * Other arguments, layouts and errors as sdp4_grad_quant / the bits_out > 0
 * mode of sdp4_dequant_reduce (bits_out must be 4 or 8; there is no
 * transform in this mode).  offset not a multiple of 8: EALIGN.
 */
int sdp4_grad_quant_sr(const float *x, int64_t n, int bits, int hadamard_block, int group, uint64_t seed,
                       uint64_t offset, void *codes, float *scale, void *stream);
int sdp4_dequant_reduce_sr(int P, const void *const *codes, const float *const *scales, int64_t n_chunk,
                           int bits_in, int group, int bits_out, uint64_t seed, uint64_t offset,
                           void *out_codes, float *out_scales, float *out_f32, void *stream);

/*
 * Standalone blockwise Hadamard transform (the unfused "HS w/o fused"
 * variant of Table 4, Sec. 5.4): y = (H_n / sqrt(n)) x per block.
 *   x, y [n] float32   y == x (in place) is allowed; partial overlap is not
 *   block              power of two in [2, 1024]; n a multiple of it
 * Errors: EINVAL, EALIGN, EHIP.
 */
int sdp4_hadamard(const float *x, float *y, int64_t n, int block, void *stream);

/*
 * Standalone float32 reduction of P chunks (the Reduction step of Alg. 4
 * for the unfused variant): y[i] = +0 + x_0[i] + ... + x_{P-1}[i], summed
 * in peer order.
 *   xs [P] (host)  device pointers; y [n] must not overlap any of them
 * Errors: ERANGE, EINVAL, EALIGN, EHIP.
 */
int sdp4_reduce_f32(int P, const float *const *xs, float *y, int64_t n, void *stream);

/*
 * Plain device copy y[i] = x[i] (no overlap), the bandwidth yardstick the
 * benchmark measures the hot path against.
 */
int sdp4_copy_f32(const float *x, float *y, int64_t n, void *stream);

/*
 * Read-only stream over x[0..n) (a bandwidth yardstick: the rate HBM gives
 * pure reads).  XOR-accumulates the bit patterns of x[i] into sink[i % 4]:
 *   x    [n] device, 16-byte aligned
 *   sink [4] device uint32, 4-byte aligned, must not overlap x; the caller
 *        clears it first (the call only XORs into it)
 * Errors: EINVAL (null pointer, n < 0 or beyond the limit, overlap), EALIGN,
 * EHIP.
 */
int sdp4_read_f32(const float *x, int64_t n, uint32_t *sink, void *stream);

/*
 * Write-only stream y[i] = value for i in [0, n) (a bandwidth yardstick: the
 * rate HBM gives pure writes).
 *   y [n] device, 16-byte aligned
 * Errors: EINVAL, EALIGN, EHIP.
 */
int sdp4_fill_f32(float *y, int64_t n, float value, void *stream);

/* ---------------------------------------------------------------------------
 * Training-step operators
 *
 * The streaming passes of a decoder's training step that stand between its
 * matrix products and make the gradients sdp4_grad_quant takes: bias +
 * dropout + residual, norm and rotation of queries and keys, the log
 * probabilities of the target tokens, attention, the norms between blocks and
 * the embedding, each with its backward pass.
 *
 * They keep the conventions above (caller-owned device memory, checked
 * arguments, one stream, no state) with these differences:
 *  Arrays     Two-dimensional arrays have unit stride in a row and any stride
 *             (in elements, >= the width) from row to row; sizes are
 *             arbitrary.  Element types are SDP4_F32 and SDP4_BF16.
 *  Alignment  Addresses need only their element's alignment; a workspace
 *             needs 16 bytes.
 *  Aliasing   An output may be the input it replaces (the same address,
 *             element type and strides), or rows of an array whose other
 *             columns are an input, and heads may lie between the heads of
 *             another set of the same strides; other overlap is EINVAL.
 *  Inputs     May be infinite or NaN, with the results stated below.
 *  Workspace  Scratch memory for one call, of at least the bytes its helper
 *             names; its contents before and after do not matter.
 *  Numerics   Arithmetic is float32, rounded once to bfloat16 at the end;
 *             sums are float32 in a fixed order (results do not depend on
 *             timing).
 * ------------------------------------------------------------------------- */

/* Limits. */
#define SDP4_MAX_TOP 32                      /* alternatives of a row */
#define SDP4_MAX_VOCAB ((int64_t)1 << 20)    /* logits of a row */
#define SDP4_MAX_HEAD_DIM 512                /* elements of a head */
#define SDP4_MIN_ATTENTION_DIM 8             /* elements of a head, for attention */
#define SDP4_MAX_ATTENTION_DIM 256
#define SDP4_MAX_TOKENS ((int64_t)1 << 30)   /* rows of a packed batch; its sequences */
#define SDP4_MAX_HIDDEN 16384                /* columns of a normed row */
#define SDP4_MAX_GRAD_TOKENS ((int64_t)1 << 21) /* rows of one embedding gradient */

/*
 * Bias, dropout and residual:
 *      y[r][c] = residual[r][c] + (keep ? (x[r][c] + bias[c]) * s : 0)
 * keep is drawn for element e = offset + r * ceil8(cols) + c, ceil8 rounding
 * up to a multiple of 8: its 16-bit uniform h (the generator of
 * sdp4_grad_quant_sr, h = 65536 u) must be at least T = rint(65536 p), and
 * s = 65536 / (65536 - T) (all is dropped for T = 65536), so E[y] = residual
 * + x + bias exactly.  The mask is not stored: the same (seed, offset) draws
 * it again.  A dropped element contributes 0 whatever it holds.
 *
 *   x         [rows][cols] x_dtype, row stride x_stride
 *   bias      [cols] x_dtype or NULL (no bias)
 *   residual  [rows][cols] y_dtype or NULL (none), row stride residual_stride
 *   p         in [0, 1]
 *   seed      64-bit key; offset: multiple of 8 (EALIGN otherwise).  Calls that
 *             must not share a mask take ranges [offset, offset + rows * ceil8(cols))
 *             that do not overlap, or other seeds.  Both are arguments by value: a
 *             call captured in a HIP graph draws the same mask in every replay, so a
 *             captured training step updates them in its node (or is captured again)
 *   y         [rows][cols] y_dtype out, row stride y_stride; may be x or residual
 */
int sdp4_dropout_add(const void *x, int x_dtype, int64_t x_stride, const void *bias, const void *residual,
                     int64_t residual_stride, int64_t rows, int64_t cols, float p, uint64_t seed, uint64_t offset,
                     void *y, int y_dtype, int64_t y_stride, void *stream);

/*
 * Its backward pass: dx[r][c] = keep ? dy[r][c] * s : 0 with the mask drawn
 * again, and dbias[c] = the float32 sum of dx[r][c] over r before rounding.
 * (The gradient of the residual is dy itself.)
 *
 *   dy     [rows][cols] y_dtype, row stride dy_stride
 *   dx     [rows][cols] x_dtype out, row stride dx_stride; may be dy
 *   dbias  [cols] float32 out, or NULL (then no workspace is needed)
 *   workspace  sdp4_dropout_grad_workspace(rows, cols) bytes
 */
int sdp4_dropout_add_grad(const void *dy, int y_dtype, int64_t dy_stride, int64_t rows, int64_t cols, float p,
                          uint64_t seed, uint64_t offset, void *dx, int x_dtype, int64_t dx_stride, float *dbias,
                          void *workspace, int64_t workspace_bytes, void *stream);
int64_t sdp4_dropout_grad_workspace(int64_t rows, int64_t cols); /* -1 for sizes out of range */

/*
 * Log probabilities of given tokens.  For each row x of `vocab` logits:
 *      lse = log sum_j exp(x_j), logp = x_target - lse,
 *      entropy = - sum_j p_j log p_j with p_j = exp(x_j - lse),
 * and its top_k largest logits (ties: the lower index first) as token ids
 * and log probabilities.  Logits of -inf have probability 0; a row of
 * nothing else has lse = logp = -inf and entropy 0; a NaN or +inf in a row
 * makes its lse, logp, entropy and top_logp NaN and its top_ids -1.  Other
 * log probabilities are never above 0 and entropies never below.  Beside the
 * rounding of the result both carry that of a float32 sum of exponentials, an
 * absolute error of a few 1e-6 at most (2.3e-6 was the largest seen), which
 * counts where -logp is as small.
 *
 *   logits   [rows][vocab] dtype, row stride `stride`; what lies between
 *            vocab and stride does not matter
 *   vocab    1 .. SDP4_MAX_VOCAB
 *   targets  [rows] or NULL; a negative target means none (logp = 0), one
 *            >= vocab is a mistake (logp = NaN)
 *   logp, lse, entropy   [rows] out, each may be NULL (logp needs targets)
 *   top_k    0 .. min(vocab, SDP4_MAX_TOP); top_logp, top_ids [rows][top_k] out
 *   workspace  sdp4_token_logprob_workspace(rows, vocab, top_k) bytes, which
 *            serve any smaller number of rows too
 */
int sdp4_token_logprob(const void *logits, int dtype, int64_t stride, int64_t rows, int64_t vocab,
                       const int64_t *targets, int top_k, float *logp, float *lse, float *entropy, float *top_logp,
                       int64_t *top_ids, void *workspace, int64_t workspace_bytes, void *stream);
int64_t sdp4_token_logprob_workspace(int64_t rows, int64_t vocab, int top_k); /* -1 for sizes out of range */

/*
 * Gradient of a loss with respect to the logits, from its gradients with
 * respect to logp, entropy and lse:
 *      dlogits_j = p_j (g_lse - g_logp - g_entropy (log p_j + entropy))
 *                  + (j = target ? g_logp : 0).
 * Columns from vocab to width (a vocabulary padded for the output product)
 * are set to 0.  A row without a finite logit gets zeros, one whose lse is
 * NaN gets NaN, and so does one whose target is >= vocab; a negative target
 * takes no g_logp.
 *
 *   logits, dtype, stride, rows, vocab, targets   as for sdp4_token_logprob
 *   lse, entropy   [rows] as it returned them (entropy only with g_entropy)
 *   g_logp, g_entropy, g_lse   [rows] or NULL for zero (g_logp needs targets)
 *   dlogits  [rows][width] dtype out, row stride dlogits_stride; may be logits
 */
int sdp4_token_logprob_grad(const void *logits, int dtype, int64_t stride, int64_t rows, int64_t vocab,
                            const int64_t *targets, const float *lse, const float *entropy, const float *g_logp,
                            const float *g_entropy, const float *g_lse, void *dlogits, int64_t dlogits_stride,
                            int64_t width, void *stream);

/*
 * Both at once for a loss whose gradients by logp, entropy and lse are known
 * before (a weighted mean of log probabilities: g_logp = -weight): the same
 * outputs as sdp4_token_logprob with top_k = 0 followed by
 * sdp4_token_logprob_grad, the logits read once where a row fits one
 * compute unit's registers (16384 chunks of 16 bytes).
 *
 *   logp  [rows] or NULL; lse, entropy [rows] out, not NULL
 *   workspace  sdp4_token_logprob_workspace(rows, vocab, 0) bytes
 */
int sdp4_token_loss(const void *logits, int dtype, int64_t stride, int64_t rows, int64_t vocab,
                    const int64_t *targets, const float *g_logp, const float *g_entropy, const float *g_lse,
                    float *logp, float *lse, float *entropy, void *dlogits, int64_t dlogits_stride, int64_t width,
                    void *workspace, int64_t workspace_bytes, void *stream);

/* Query or key heads of all tokens: element d of head h of token t lies at
 * data[t * token_stride + h * head_stride + d].  Both strides are at least
 * head_dim and heads do not overlap: token_stride >= (heads - 1) *
 * head_stride + head_dim, or the same with tokens and heads exchanged. */
typedef struct {
    void *data;
    int64_t token_stride, head_stride;
    int heads;
} sdp4_heads;

/* How heads are normed and rotated, shared by the forward and backward pass. */
typedef struct {
    int dtype;               /* of heads and weights */
    int head_dim;            /* 1 .. SDP4_MAX_HEAD_DIM */
    int norm;                /* 0: no norm (the weights are NULL) */
    float eps;               /* >= 0, finite */
    const void *q_weight;    /* [head_dim], or NULL for ones */
    const void *k_weight;
    const float *table;      /* [table_rows][rot_dim]: rot_dim / 2 cosines, then the sines; NULL with rot_dim = 0 */
    int64_t table_rows;
    int rot_dim;             /* rotated elements of a head: even, 0 .. head_dim */
    int interleaved;         /* pairs (2i, 2i+1); 0: pairs (i, i + rot_dim / 2) */
    const int64_t *positions; /* [tokens] table rows, or NULL for 0, 1, 2, ... */
} sdp4_qk_params;

/*
 * RMS norm of each head and rotation by its token's position, in one pass:
 *      u = x / sqrt(mean(x^2) + eps) * weight,
 *      pair i of the first rot_dim elements (a, b) -> (a c - b s, b c + a s)
 * with (c, s) = (table[pos][i], table[pos][rot_dim / 2 + i]); the other
 * elements are u.  A position outside the table makes the rotated elements
 * NaN (backward with a norm the head's others too).  Squares are float32:
 * mean(x^2) + eps has to be one of its normal numbers, so heads as a whole
 * stay below 1e19 and, with eps = 0, above 1e-18.
 *
 *   q, k          inputs; k may be NULL (queries only)
 *   q_out, k_out  outputs with the same numbers of heads, any strides; each
 *                 may be its input.  k_out is NULL where k is
 */
int sdp4_qk_norm_rope(const sdp4_heads *q, const sdp4_heads *k, const sdp4_qk_params *params, int64_t tokens,
                      const sdp4_heads *q_out, const sdp4_heads *k_out, void *stream);

/*
 * Its backward pass: gradients of inputs and weights from those of the
 * outputs.
 *
 *   dq_out, dk_out   gradients of q_out, k_out
 *   q, k             the inputs (not read, and may be NULL, without norm)
 *   dq, dk           out, may be dq_out, dk_out
 *   dq_weight, dk_weight   [head_dim] float32 out, sums over tokens and heads;
 *                    NULL where not wanted (each needs norm and its weight)
 *   workspace        sdp4_qk_grad_workspace() bytes, with a weight gradient
 */
int sdp4_qk_norm_rope_grad(const sdp4_heads *dq_out, const sdp4_heads *dk_out, const sdp4_heads *q,
                           const sdp4_heads *k, const sdp4_qk_params *params, int64_t tokens, const sdp4_heads *dq,
                           const sdp4_heads *dk, float *dq_weight, float *dk_weight, void *workspace,
                           int64_t workspace_bytes, void *stream);
int64_t sdp4_qk_grad_workspace(int64_t tokens, int q_heads, int k_heads, int head_dim); /* -1: out of range */

/*
 * The table of sdp4_qk_norm_rope: row r holds scale * cos and scale * sin of
 * (start + r) * inv_freq[i] for i < half, computed in float64 and rounded
 * once.  Frequencies and scale carry any rule for long contexts (stretched
 * positions, another base, a ramp between both, a factor on queries and keys).
 *   inv_freq [half] float64; table [rows][2 * half] out
 */
int sdp4_rope_table(const double *inv_freq, int half, int64_t start, int64_t rows, double scale, float *table,
                    void *stream);

/* Causal attention over packed sequences, shared by the forward and backward pass. */
typedef struct {
    int dtype;               /* of all heads */
    int head_dim;            /* SDP4_MIN_ATTENTION_DIM .. SDP4_MAX_ATTENTION_DIM */
    float scale;             /* of the scores: 2^-40 .. 2^40 */
    const int64_t *offsets;  /* [sequences + 1] on the device, never falling, 0 .. tokens; NULL: one sequence of all tokens */
    int64_t sequences;
} sdp4_attention_params;

/*
 * Attention of each row to itself and the rows before it in its sequence:
 * sequence n has rows offsets[n] .. offsets[n + 1] - 1, and for its rows j <= i
 *      s_ij = scale q_i . k_j,  lse_i = log sum_j exp(s_ij),
 *      out_i = sum_j exp(s_ij - lse_i) v_j.
 * The query heads share the key and value heads: head h uses head
 * h / (q heads / k heads), and k's heads divide q's.  Sequences may be empty.
 * Rows before the first sequence and behind the last one are not read as keys
 * (whatever they hold) and their out and lse are left as they were.  Offsets
 * that fall or leave 0 .. tokens give wrong rows, but touch nothing outside
 * the arrays.
 *
 * What a row must not see does not count, infinite or NaN or not.  An infinity
 * or NaN that a row sees (its own query included) makes elements of its result
 * infinite or NaN: those that depend on it, or the whole row.  Of a row whose
 * scores are all -inf, out is 0 and lse -inf.
 *
 * Scores, their sums and the results are float32; with bfloat16 heads the
 * probabilities are rounded to bfloat16 for their product with the values
 * (float32 heads have no rounding but float32's).
 *
 *   q, k, v   k and v have the same number of heads
 *   out       heads like q, any strides; no overlap with an input
 *   lse       [q heads][tokens] out, or NULL
 */
int sdp4_attention(const sdp4_heads *q, const sdp4_heads *k, const sdp4_heads *v, const sdp4_attention_params *params,
                   int64_t tokens, const sdp4_heads *out, float *lse, void *stream);

/*
 * Its backward pass, from the gradient of out:
 *      p_ij = exp(s_ij - lse_i),  ds_ij = p_ij (dout_i . v_j - dout_i . out_i),
 *      dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,
 *      dv_j = sum_i p_ij dout_i,
 * dk and dv summed over the query heads that share the head, too.  Rows in no
 * sequence are left as they were; what must not be seen does not count, as
 * above.  With bfloat16 heads p and ds are rounded to bfloat16 for the
 * products.
 *
 *   out, lse     as sdp4_attention left them
 *   dq, dk, dv   heads like q, k, v; no overlap with an input or each other
 *   workspace    sdp4_attention_grad_workspace() bytes, which serve any smaller
 *                number of tokens too
 */
int sdp4_attention_grad(const sdp4_heads *dout, const sdp4_heads *q, const sdp4_heads *k, const sdp4_heads *v,
                        const sdp4_heads *out, const float *lse, const sdp4_attention_params *params, int64_t tokens,
                        const sdp4_heads *dq, const sdp4_heads *dk, const sdp4_heads *dv, void *workspace,
                        int64_t workspace_bytes, void *stream);
int64_t sdp4_attention_grad_workspace(int64_t tokens, int q_heads, int k_heads, int head_dim); /* -1: out of range */

/* The joint of two blocks, shared by the forward and backward pass. */
typedef struct {
    int x_dtype;             /* of a block's output (branch), the next one's input (h) and the weights */
    int y_dtype;             /* of the residual stream */
    int post_norm;           /* 0: no norm behind the block */
    float post_eps, pre_eps; /* >= 0, finite */
    const void *post_weight; /* [cols], or NULL for ones; also without a post norm */
    const void *pre_weight;  /* [cols], or NULL for ones */
    const float *gate;       /* [rows], or NULL for ones */
    float branch_scale, residual_scale; /* finite */
} sdp4_block_params;

/*
 * The norm behind a block, its gate and scale, the residual stream, and the
 * norm in front of the next block, in one pass over the rows:
 *      u = branch / sqrt(mean(branch^2) + post_eps) * post_weight
 *          (branch * post_weight without post_norm),
 *      y = residual_scale * residual + branch_scale * gate * u,
 *      h = y / sqrt(mean(y^2) + pre_eps) * pre_weight,
 * h from y before y is rounded.  As for heads, the squares are float32.  The
 * row sums take a row as a whole: an infinity or NaN in it reaches all of it.
 *
 *   branch    [rows][cols] x_dtype, or NULL (none; then without post_norm,
 *             post_weight and gate: an RMS norm of the residual stream)
 *   residual  [rows][cols] y_dtype, or NULL (none); one of both is there
 *   y         [rows][cols] y_dtype out, or NULL (not wanted); may be an input
 *   h         [rows][cols] x_dtype out, or NULL; may be an input
 *   cols      0 .. SDP4_MAX_HIDDEN
 */
int sdp4_block_norm(const void *branch, int64_t branch_stride, const void *residual, int64_t residual_stride, int64_t rows,
                    int64_t cols, const sdp4_block_params *params, void *y, int64_t y_stride, void *h, int64_t h_stride,
                    void *stream);

/*
 * Its backward pass, from the gradients by h and by y:
 *      t = dy + the gradient of h by y, times dh,
 *      dresidual = residual_scale t,  dbranch = the gradient of u by branch, times branch_scale gate t,
 *      dpost_weight = sum over rows of branch_scale gate t branch / sqrt(...),
 *      dpre_weight = sum over rows of dh y / sqrt(...),
 *      dgate = branch_scale sum over columns of t u.
 *
 *   dh, dy     gradients of h and y; NULL: zero (one of both is there)
 *   branch     as it went in; NULL if neither dbranch through a post norm nor
 *              dpost_weight nor dgate is wanted
 *   y          as it came out (NULL without dh)
 *   dbranch, dresidual, dpost_weight [cols], dpre_weight [cols], dgate [rows]
 *              out, the last three float32; each NULL if not wanted (a weight's
 *              needs the weight, dpre_weight dh too, dgate the gate).  dbranch
 *              and dresidual may be inputs
 *   workspace  sdp4_block_norm_grad_workspace() bytes, with a weight gradient
 */
int sdp4_block_norm_grad(const void *dh, int64_t dh_stride, const void *dy, int64_t dy_stride, const void *branch,
                         int64_t branch_stride, const void *y, int64_t y_stride, int64_t rows, int64_t cols,
                         const sdp4_block_params *params, void *dbranch, int64_t dbranch_stride, void *dresidual,
                         int64_t dresidual_stride, float *dpost_weight, float *dpre_weight, float *dgate, void *workspace,
                         int64_t workspace_bytes, void *stream);
int64_t sdp4_block_norm_grad_workspace(int64_t rows, int64_t cols); /* -1 for sizes out of range */

/*
 * Rows of a table by token: out[r] = scale * table[tokens[r]].  A negative
 * token gives zeros (padding), one >= vocab is a mistake (NaN).
 *
 *   tokens  [rows]; table [vocab][cols] table_dtype; out [rows][cols] out_dtype
 *   vocab   1 .. SDP4_MAX_VOCAB; scale finite
 */
int sdp4_embedding(const int64_t *tokens, int64_t rows, const void *table, int table_dtype, int64_t table_stride, int64_t vocab,
                   int64_t cols, float scale, void *out, int out_dtype, int64_t out_stride, void *stream);

/*
 * The table's gradient: dtable[v] = scale * (the sum of dout[r] over the rows r
 * with token v), a float32 sum in an order that the tokens alone decide,
 * rounded once.  Tokens outside the table count for nothing.
 *
 *   accumulate  0: the whole of dtable is written, rows of no token with zeros;
 *               else the sums are added to what dtable holds, and rows of no
 *               token are left alone
 *   rows        0 .. SDP4_MAX_GRAD_TOKENS (more: in several calls that accumulate)
 *   dtable      [vocab][cols] dtable_dtype
 *   workspace   sdp4_embedding_grad_workspace() bytes, which serve any smaller
 *               number of rows too
 */
int sdp4_embedding_grad(const int64_t *tokens, int64_t rows, const void *dout, int dout_dtype, int64_t dout_stride, int64_t vocab,
                        int64_t cols, float scale, int accumulate, void *dtable, int dtable_dtype, int64_t dtable_stride,
                        void *workspace, int64_t workspace_bytes, void *stream);
int64_t sdp4_embedding_grad_workspace(int64_t rows, int64_t vocab, int64_t cols); /* -1 for sizes out of range */

/* Pure helpers (no device work). */
int64_t sdp4_codes_bytes(int64_t n, int bits);  /* n * bits / 8, or -1 if bits not 4 or 8 */
int64_t sdp4_num_groups(int64_t n, int group); /* n / group, or -1 if not a valid group */
const char *sdp4_status_string(int status);
const char *sdp4_version(void);
/* HIP error code of the most recent EHIP returned on the calling thread (0 if none). */
int sdp4_last_hip_error(void);

#ifdef __cplusplus
}
#endif

#endif /* SDP4_H */
