/*
 * swam_ops.h -- operators of an 8-bit, encoder-conditioned block on AMD
 * Instinct MI355X (gfx950), next to the block and step of swam.h.
 *
 * World-action backbones condition their tokens on a prompt or on an observation
 * encoder's states.  Such a block has a cross-attention sublayer beside the self
 * attention of swam_block, and a deployment in 8 bits runs its projections on
 * integer codes.  The four operators here are that sublayer,
 *   codes, s = RMSnorm(x + r)                     swam_rms_norm_i8
 *   q        = codes W_q^T (s, channel scales)    swam_gemm_i8
 *   o        = softmax(q K^T) V over the encoder  swam_cross_attention
 *   codes, s = o                                  swam_quantize_i8
 *   x        = x + gate (codes W_o^T + b)         swam_gemm_i8
 * and each is also of use alone: the quantiser makes the 8-bit weights, the
 * product serves the MLP.
 *
 * Conventions are those of swam.h: device pointers owned by the caller, every
 * call asynchronous on the context's stream, arguments validated on the host
 * before any launch, a negative swam_status and swam_last_error on failure.  No
 * call allocates, synchronises or reads anything back, so all of them can be
 * captured into a HIP graph.  Attention that is split over keys keeps its partial
 * results in the context's workspace: calls of one context (and replays of
 * graphs that captured them) must not overlap in time, as everywhere in swam.h.
 * Float tensors called "act" below have the context's dtype; strides are in
 * elements; rows of a tensor may lie further apart than they are wide (a column
 * range of a wider buffer); rows times row stride is below 2^48.  An output may not
 * overlap an input unless stated.
 * The calls run on the context's device whatever device is current.
 */
#ifndef SWAM_OPS_H
#define SWAM_OPS_H

#include "swam.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SWAM_I8_MAX_WIDTH 32768   /* elements of a row that is quantised */
#define SWAM_I8_MAX_K 131056      /* inner size of a product: 128 * 128 * K < 2^31 */

/* Residual addition and RMS norm with 8-bit output, one row per token:
 *   t = x + residual                       (t = x when residual is NULL)
 *   y = t / sqrt(mean(t^2) + eps) * gain * (1 + scale) + shift
 *   q_scale = max|y| / 127,   q = round(y / q_scale) in [-127, 127]
 * in float32 from the unrounded t; rounding is to nearest even.  Rows however small
 * keep their y, also where eps does not hide them (their squares are summed of a row
 * lifted by a power of two).  A row of zeros gets the scale 0 and zeros.  A row with a NaN or an infinity, or whose sum of
 * squares exceeds float32, gets the scale NaN and zeros, so what is made of it
 * is NaN.
 *   x        : act [rows][d], row stride x_stride >= d
 *   residual : act [rows][d] (row stride residual_stride) or NULL
 *   sum_out  : act [rows][d], receives t rounded once, or NULL.  May be x or
 *              residual itself (same pointer and stride): the residual stream is
 *              updated in place
 *   gain     : act [d] or NULL;  shift, scale : float [d], both or neither
 *   q        : int8 [rows][d], row stride q_stride;  q_scale : float [rows]
 * 1 <= d <= SWAM_I8_MAX_WIDTH, 0 <= rows < 2^31, eps >= 0 and finite.  Any alignment of
 * the element type. */
int swam_rms_norm_i8(swam_ctx* ctx, const void* x, int64_t x_stride, const void* residual,
                     int64_t residual_stride, const void* gain, const float* shift,
                     const float* scale, float eps, int64_t rows, int64_t d, void* sum_out,
                     int64_t sum_stride, int8_t* q, int64_t q_stride, float* q_scale);

/* 8-bit codes and a scale for each row: q_scale = max|x| / 127, q = round(127 x
 * / max|x|), exactly rounded (ties to even), so the codes do not depend on how
 * they are computed.  Quantises activations per token and a weight
 * [out_features][in_features] per output channel.  Zero and non-finite rows,
 * sizes and alignment as above. */
int swam_quantize_i8(swam_ctx* ctx, const void* x, int64_t x_stride, int64_t rows, int64_t d,
                     int8_t* q, int64_t q_stride, float* q_scale);

#define SWAM_GEMM_GELU 1          /* tanh-GELU of the product and bias */

/* Product of 8-bit codes with a scale for each token and output channel:
 *   z[m][n] = a_scale[m] * b_scale[n] * sum_k a[m][k] b[n][k] + bias[n]
 *   c = z;   c = GELU(z) with SWAM_GEMM_GELU;   c = residual + gate[n] * z with a
 *   residual (GELU and a residual exclude each other)
 * The sum is exact in 32-bit integers, the rest float32, rounded once.
 *   a : int8 [m][k] (row stride lda), a_scale float [m];  b : int8 [n][k] (row
 *   stride ldb), b_scale float [n];  bias : act [n] or NULL;  residual : act
 *   [m][n] (row stride ldr) or NULL, gate : float [n] or NULL (1; only with a
 *   residual);  c : act [m][n] (row stride ldc), may be residual itself (same
 *   pointer and stride)
 * k a positive multiple of 16 up to SWAM_I8_MAX_K; m, n below 2^30 and m * n below
 * 2^40 (0: nothing to do); lda, ldb below 2^22.  a, b and their row strides are
 * 16-byte aligned (SWAM_E_INVALID otherwise); the float tensors need the alignment of
 * their type only (16-byte aligned rows are moved in vectors). */
int swam_gemm_i8(swam_ctx* ctx, const int8_t* a, int64_t lda, const float* a_scale,
                 const int8_t* b, int64_t ldb, const float* b_scale, const void* bias,
                 const void* residual, int64_t ldr, const float* gate, int32_t flags, void* c,
                 int64_t ldc, int64_t m, int64_t n, int64_t k);

/* Attention of every query token to the states of an encoder:
 *   o_h(i) = sum_j p_ij v_h'(j),  p_ij = softmax_j(scale q_h(i) . k_h'(j))
 * over the visible keys j of the key sequence that i's sequence attends, with
 * h' = h / (n_heads / n_kv_heads).  lse (optional) receives the natural-log
 * normaliser of every row and head.  A row without a visible key, or whose visible
 * scores are all minus infinity, gets zeros and minus infinity.  Scores, weights and
 * sums are float32; a bf16 context rounds the weights to bf16 in front of the product
 * with v (an error of 0.0016 of the output's size beside the 0.0017 of its own rounding).
 *   q, o : act, token i, head h at q + i q_stride + h head_dim (n_q tokens)
 *   k, v : act, token j, head h' at k + j k_stride + h' head_dim (n_k tokens)
 *   key_mask : bytes [n_k], 0 hides a key (padding), or NULL.  What hidden keys
 *              and values hold does not matter, NaN and infinities included
 *   cu_q : int32 [n_seqs + 1] row offsets of the query sequences, or NULL for
 *          one sequence of n_q rows (n_seqs = 1);  cu_k : int32 [n_kv_seqs + 1]
 *          likewise.  Bounds are clamped to [0, n_q] and [0, n_k]; rows of o and
 *          lse outside every sequence are left as they are (sequences must not
 *          overlap)
 *   kv_seq : int32 [n_seqs], the key sequence that each query sequence attends
 *            (several may share one prompt; an index outside [0, n_kv_seqs) has
 *            no keys), or NULL for its own (n_kv_seqs = n_seqs)
 *   lse : float [n_q][n_heads] or NULL
 * head_dim 64 or 128; n_heads a multiple of n_kv_heads; 1..SWAM_MAX_BATCH
 * sequences; n_q * n_heads and n_k below 2^30; scale finite and > 0; row strides below
 * 2^22.  q, k, v, o and their rows are 16-byte aligned (SWAM_E_INVALID otherwise). */
int swam_cross_attention(swam_ctx* ctx, const void* q, int64_t q_stride, const void* k,
                         int64_t k_stride, const void* v, int64_t v_stride,
                         const uint8_t* key_mask, const int32_t* cu_q, const int32_t* cu_k,
                         const int32_t* kv_seq, int32_t n_seqs, int32_t n_kv_seqs, int64_t n_q,
                         int64_t n_k, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                         float scale, void* o, int64_t o_stride, float* lse);

#ifdef __cplusplus
}
#endif

#endif /* SWAM_OPS_H */
