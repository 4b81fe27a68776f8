/*
 * swam_cache.h -- operators of a streaming block on a paged cache on AMD Instinct
 * MI355X (gfx950), next to the block and step of swam.h and the operators of
 * swam_ops.h.
 *
 * A policy that acts chunk after chunk keeps the keys and values of everything it has
 * seen.  A chunk of new tokens -- one token, a frame with its action tokens, or a whole
 * context -- then passes a self-attention sublayer as
 *   q, k, v  = projection of the chunk
 *   q, cache = norm and rotation of q and k, k and v appended    swam_cache_append
 *   o        = attention of the chunk to the cache               swam_cache_attention
 * swam_qk_norm_rope is the norm and rotation alone, without a cache, and
 * swam_rope_frequencies makes the frequencies of the rotation.
 *
 * Conventions are those of swam_ops.h: device pointers owned by the caller, every
 * call asynchronous on the context's stream, arguments validated on the host before any
 * launch, a negative swam_status and swam_last_error on failure, no allocation,
 * synchronisation or read-back (so all can be captured into a HIP graph), the context's
 * device whatever device is current.  "act" tensors have the context's dtype, strides
 * are in elements, rows times row stride is below 2^48.  Attention that is split over
 * keys keeps its partial results in the context's workspace: calls of one context (and
 * replays of graphs that captured them) must not overlap in time.  An output may not
 * overlap an input unless stated.
 */
#ifndef SWAM_CACHE_H
#define SWAM_CACHE_H

#include "swam.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SWAM_CACHE_MAX_SEQS 1024  /* sequences of a call */
#define SWAM_CACHE_MAX_PAGE 4096  /* tokens of a page */
#define SWAM_QK_MAX_DIM 512       /* elements of a head that is normalised or rotated */

/* pairs of a rotation of `dims` elements: (2 i, 2 i + 1), or (i, i + dims / 2) */
enum { SWAM_ROPE_INTERLEAVED = 0, SWAM_ROPE_HALF = 1 };
/* how swam_rope_frequencies serves contexts longer than trained */
enum { SWAM_ROPE_PLAIN = 0, SWAM_ROPE_LINEAR = 1, SWAM_ROPE_NTK = 2, SWAM_ROPE_YARN = 3 };

/* Frequencies of a rotation of `dims` (even, 2..SWAM_QK_MAX_DIM) elements, a host call that needs no GPU:
 * freq[i], i < dims / 2, in radians per position, and the factor of the rotated
 * elements.  With theta_i = base^(-2 i / dims):
 *   PLAIN  : theta_i, 1
 *   LINEAR : theta_i / factor, 1 (positions interpolated)
 *   NTK    : theta_i of the base  base * factor^(dims / (dims - 2)) (dims > 2), 1
 *   YARN   : theta_i (g + (1 - g) / factor) with g = min(1, max(0, (r - 1) / 31)) of the
 *            r = trained theta_i / (2 pi) turns that the pair makes in `trained`
 *            positions, and 0.1 ln(factor) + 1 (Peng et al., 2023)
 * base > 1, factor >= 1, trained > 0 (YARN only), all finite. */
int swam_rope_frequencies(int32_t dims, double base, int32_t scaling, double factor, double trained,
                          double* freq, float* magnitude);

/* What is done to the head vectors of q and k.  With norm, a head vector x becomes
 *   y = x / sqrt(mean(x^2) + eps) * gain
 * in float32 (vectors however small or large keep their y, zeros stay zeros), and the first
 * rope_dims elements of it (or of x) are rotated in pairs (a, b) by the angle
 * t = position * freq:  a' = m (a cos t - b sin t),  b' = m (a sin t + b cos t).  The
 * angle is formed in float64, the rest in float32, rounded once.
 *   norm : 1 or 0;  eps >= 0 and finite;  q_gain, k_gain : act [head_dim] or NULL (only with
 *          norm)
 *   rope_dims : even, 0 (no rotation) to head_dim;  rope_layout : enum above
 *   rope_freq : double [rope_dims / 2] on the device;  rope_magnitude : m, finite */
typedef struct swam_qk_post {
  int32_t norm;
  float eps;
  const void* q_gain;
  const void* k_gain;
  int32_t rope_dims;
  int32_t rope_layout;
  const double* rope_freq;
  float rope_magnitude;
} swam_qk_post;

/* Norm and rotation of query and key heads.
 *   q, q_out : act, row i, head h at q + i q_stride + h head_dim (n_heads heads)
 *   k, k_out : act likewise (n_kv_heads heads); q or k may be left out (NULL, no heads).
 *              An output may be its input itself (same pointer and stride)
 *   pos      : int32 [rows], position of each row (any value), or NULL for the row's index
 * head_dim a multiple of 8 up to SWAM_QK_MAX_DIM; heads below 2^16 in all; 0 <= rows < 2^31.
 * The act tensors, their rows and the gains are 16-byte aligned (SWAM_E_INVALID
 * otherwise). */
int swam_qk_norm_rope(swam_ctx* ctx, const swam_qk_post* post, const int32_t* pos, const void* q,
                      int64_t q_stride, const void* k, int64_t k_stride, int64_t rows,
                      int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, void* q_out,
                      int64_t qo_stride, void* k_out, int64_t ko_stride);

/* A paged cache of keys and values and the chunk behind it.  Token j of sequence s
 * lies in page table[s][j / page_size] at slot j % page_size; a table entry outside
 * [0, n_pages) holds nothing, and tokens past max_pages * page_size have no place.
 *   k, v  : act, page p, slot t, head h at k + p k_page + t k_token + h k_head (any
 *           order of the three whose elements do not meet).  k and v may share a buffer -- pages,
 *           tokens or heads of both in turn -- but no element; where elements of one lie between
 *           the other's, both have the same strides there
 *   table : int32 [n_seqs][max_pages], row stride table_stride
 *   length: int32 [n_seqs], tokens of each sequence before the chunk (clamped to
 *           [0, max_pages * page_size]).  Both calls take the length before the
 *           chunk; the caller adds the chunk's once it is done with it.  A chunk that
 *           is appended again at the same length is overwritten (a chunk denoised
 *           over several steps)
 * page_size a power of two, 8..SWAM_CACHE_MAX_PAGE; max_pages * page_size below 2^30;
 * 1..SWAM_CACHE_MAX_SEQS sequences; head_dim 64 or 128; n_kv_heads below 2^16; k_token, v_token below 2^22;
 * k, v and their strides are 16-byte aligned.  Pages may be shared by sequences that only read
 * them; two tokens of one call must not be appended to one place. */
typedef struct swam_kv_cache {
  void* k;
  void* v;
  int64_t k_page, k_token, k_head;
  int64_t v_page, v_token, v_head;
  int64_t n_pages;
  int32_t page_size, n_kv_heads, head_dim;
  int32_t n_seqs, max_pages;
  int64_t table_stride;
  const int32_t* table;
  const int32_t* length;
} swam_kv_cache;

/* Appends a chunk: k, after norm and rotation, and v of token i of sequence s go to
 * position length[s] + i of it; q (optional) gets the same norm and rotation in the same
 * pass.
 *   post  : or NULL (k as it is)
 *   pos   : int32 [rows], positions of the rotation, or NULL for the token's position in
 *           its sequence
 *   cu    : int32 [n_seqs + 1], row offsets of the sequences' chunks, or NULL for one
 *           sequence of all rows.  Sequence s is the rows from cu[s] to cu[s + 1], both clamped
 *           to [0, rows], and empty where they fall (sequences must not overlap)
 *   q, q_out : act, n_heads heads (0: none, both NULL); q_out may be q itself
 *   k, v  : act, n_kv_heads heads
 * Rows outside every sequence are neither appended nor written to q_out.  Tokens without a
 * place (page or table) are not appended.  Heads below 2^16 in all, rows below 2^31; act tensors, their rows
 * and the gains 16-byte aligned. */
int swam_cache_append(swam_ctx* ctx, const swam_kv_cache* cache, const swam_qk_post* post,
                      const int32_t* pos, const int32_t* cu, const void* q, int64_t q_stride,
                      const void* k, int64_t k_stride, const void* v, int64_t v_stride, int64_t rows,
                      int32_t n_heads, void* q_out, int64_t qo_stride);

/* Attention of a chunk to everything that the cache holds, itself included (append it
 * first).  Token i of sequence s, at position p = length[s] + i, sees the keys j with
 *   j < length[s] + the chunk's tokens,   j <= p with causal,   p - j < window with a window
 * that have a place;  o_h(i) = sum_j p_ij v_h'(j), p_ij = softmax_j(scale q_h(i) . k_h'(j)),
 * h' = h / (n_heads / n_kv_heads).  A row without a visible key, or whose visible scores are
 * all minus infinity, gets zeros and the normaliser minus infinity.  Keys and values that a
 * row does not see do not matter to it, NaN and infinities included.  Scores, weights and
 * sums are float32 (weights up to 2^8 before the division: the size of v times the keys of a row
 * stays below 2^118).  In a bf16 context a sequence of up to 32 rows (tokens times n_heads / n_kv_heads) keeps
 * 16 bits of each weight in front of the product with v, whatever stands beside it in the call (outputs
 * are off by 0.0017 of their size, which is bf16's own); longer ones may round them to bf16 (0.0024).
 *   q, o : act, token i, head h at q + i q_stride + h head_dim
 *   cu   : as above; rows of o and lse outside every sequence are left as they are
 *   causal : 1 or 0 (0: a chunk whose tokens all see each other)
 *   window : keys, 0 for all
 *   lse  : float [rows][n_heads] or NULL, natural-log normalisers
 * n_heads a multiple of n_kv_heads, up to 4096; rows * n_heads below 2^30; scale finite and > 0; row strides
 * below 2^22; q, o and their rows 16-byte aligned. */
int swam_cache_attention(swam_ctx* ctx, const swam_kv_cache* cache, const int32_t* cu, const void* q,
                         int64_t q_stride, int64_t rows, int32_t n_heads, int32_t causal,
                         int32_t window, float scale, void* o, int64_t o_stride, float* lse);

#ifdef __cplusplus
}
#endif

#endif /* SWAM_CACHE_H */
