/*
 * dilated_attn_paged.h - C ABI of the head norms and of serving from a paged
 * cache: the RMS norm of query and key heads with the xPos rotation (forward
 * and backward), new keys and values into a paged cache, and dilated attention
 * of new tokens over it.  Types, limits, error codes and the operator itself
 * are those of dilated_attn.h.
 */
#ifndef DILATED_ATTN_PAGED_H
#define DILATED_ATTN_PAGED_H

#include "dilated_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * dilated_attn_qk_norm_xpos - the RMS norm of every query and key head and the
 * xPos rotation after it, in one pass (normed heads keep the attention's
 * scores in range as models grow; the rotation is that of dilated_attn_xpos):
 *   n = x * w / sqrt(mean(x^2) + eps) over the head's D elements,
 *   y = xPos(n) with sign +1 for queries and -1 for keys.
 *
 * q, k        device pointers: B * N tokens of H (q) and Hkv (k) heads of D
 *             elements of dtype, a token's heads contiguous, tokens q_stride
 *             and k_stride elements apart (H * D and Hkv * D if contiguous;
 *             larger for slices of a joint projection).  Strides times the
 *             element size are multiples of 16 bytes and below 2^32 elements.
 * qw, kw      device pointers, [D] of dtype: the norms' weights, shared by the
 *             heads.
 * qo, ko      device pointers, [B, N, H, D] and [B, N, Hkv, D] of dtype,
 *             contiguous, written; must not overlap each other or an input.
 * B, N        >= 1, B * N < 2^31.  H, Hkv in [1, 2^16), independent of each
 *             other.  D in {32, 64, 128}.  dtype DA_BF16 or DA_F32.
 * eps         finite, a normal float > 0.
 * center, base, gamma, scale_base: as for dilated_attn_xpos.
 * stream      a hipStream_t (NULL = the default stream); asynchronous.
 *
 * Arithmetic in float32, angles and scale exponents formed and reduced in
 * float64; outputs rounded to dtype once.  A head's sum of squares has to be
 * finite in float32 (elements below 1.6e18 are safe).  All device pointers
 * 16-byte aligned.  Returns DA_OK or a negative code; errors launch nothing.
 */
int dilated_attn_qk_norm_xpos(const void* q, const void* k, const void* qw, const void* kw, void* qo, void* ko,
                              int64_t B, int64_t N, int64_t H, int64_t Hkv, int64_t D, int64_t q_stride,
                              int64_t k_stride, float eps, int64_t center, float base, float gamma,
                              float scale_base, int64_t dtype, void* stream);

/*
 * dilated_attn_qk_norm_xpos_bwd - gradients of dilated_attn_qk_norm_xpos: with
 * dn the transposed xPos of the incoming gradient, rstd = 1 / sqrt(mean(x^2) +
 * eps) and xhat = x rstd (recomputed from the inputs),
 *   dx = rstd (dn w - xhat mean(dn w xhat)),   dw = sum over tokens and heads of dn xhat.
 *
 * dqo, dko    device pointers, gradients of qo and ko, contiguous.
 * q, k, qw, kw, strides, eps, center, ...: those of the forward call.
 * dq, dk      device pointers, [B, N, H, D] and [B, N, Hkv, D], contiguous,
 *             written.
 * dqw, dkw    device pointers, [D] of dtype, written.
 * workspace   device scratch of at least the bytes that
 *             dilated_attn_qk_norm_xpos_bwd_workspace reports.
 *
 * Outputs and workspace must not overlap each other or an input.  The weights'
 * gradients are summed in float32 in a fixed order (the same call gives the
 * same bits) and rounded once.  Alignment, stream and errors as above.
 */
int dilated_attn_qk_norm_xpos_bwd_workspace(int64_t B, int64_t N, int64_t D, uint64_t* bytes);
int dilated_attn_qk_norm_xpos_bwd(const void* dqo, const void* dko, const void* q, const void* k, const void* qw,
                                  const void* kw, void* dq, void* dk, void* dqw, void* dkw, int64_t B, int64_t N,
                                  int64_t H, int64_t Hkv, int64_t D, int64_t q_stride, int64_t k_stride, float eps,
                                  int64_t center, float base, float gamma, float scale_base, int64_t dtype,
                                  void* workspace, uint64_t workspace_bytes, void* stream);

/*
 * A paged cache of keys and values, and the sequences of one call.
 *
 * A call has T new tokens of B sequences (1 <= B <= 2^31 - 2^16), side by side:
 * those of sequence b are rows q_start[b] .. q_start[b + 1] - 1 of its token arrays, and they are
 * the last of the seq_lens[b] tokens that the sequence has with them.  Token p
 * (0-based) of sequence b lies in page block_table[b][p / page_size] at
 * p % page_size.  The three arrays are device memory and read by the kernels:
 * a call depends on the host's knowledge of T and B only and can be captured
 * in a graph and replayed with other lengths.
 *
 * The device arrays are not checked on the host.  Whatever they hold, nothing
 * outside the given buffers is read or written: a token of no sequence, or at
 * a position below 0 or beyond the table, is not cached and has out = 0 and
 * lse = -inf; dilated_attn_cache_append does not write to a page outside the
 * pool, and dilated_attn_paged_fwd reads the last page in its place.
 */
typedef struct {
  void* k; /* device, [num_pages, Hkv, page_size, D] of dtype, 16-byte aligned */
  void* v; /* device, the same shape                                           */
  const int32_t* block_table; /* device, [B, max_pages]                        */
  const int32_t* seq_lens;    /* device, [B]                                   */
  const int32_t* q_start;     /* device, [B + 1], ascending, from 0 to T       */
  int64_t num_pages;          /* num_pages * Hkv * page_size <= 2^32           */
  int64_t page_size;          /* a power of two, at most 2^16                  */
  int64_t max_pages;          /* entries of a table row; max_pages * page_size <= 2^31 - 2^16 */
} da_paged_cache_t;

/*
 * dilated_attn_cache_append - new keys and values into the cache, keys normed
 * and rotated on the way, and the queries of the same tokens with them:
 *   k' = xPos(norm(k), -1) and v at each token's place in the cache,
 *   qo = xPos(norm(q), +1),
 * each token at its own position (center is the same for all: fix it for the
 * life of a cache, the attention's scores do not depend on it).
 *
 * q, k, v     device pointers: T tokens of H, Hkv and Hkv heads, a token's
 *             heads contiguous, tokens q_stride, k_stride and v_stride
 *             elements apart (as above).  q may be NULL, and qo with it.
 * qw, kw      [D] norm weights, or NULL: no norm of the queries, of the keys.
 * qo          [T, H, D] contiguous, written (zeros for tokens of no sequence).
 * T           0 <= T < 2^31 (0: nothing is done).
 * eps         as above (not looked at without weights).
 * rotate      1, or 0 for no rotation (then center .. scale_base are not looked at).
 * center, base, gamma, scale_base: as for dilated_attn_xpos, with N = the
 *             positions that the table holds (max_pages * page_size).
 *
 * qo must not overlap an input, nor the cache.  Two tokens at one place of the
 * pool (a table that names a page twice) leave either's values.  v is copied
 * as it is; the rest is rounded to dtype once.
 */
int dilated_attn_cache_append(const void* q, const void* k, const void* v, const void* qw, const void* kw, void* qo,
                              const da_paged_cache_t* cache, int64_t T, int64_t B, int64_t H, int64_t Hkv, int64_t D,
                              int64_t q_stride, int64_t k_stride, int64_t v_stride, float eps, int64_t rotate,
                              int64_t center, float base, float gamma, float scale_base, int64_t dtype,
                              void* stream);

/*
 * dilated_attn_paged_fwd - causal dilated attention of the new tokens over the
 * cache, which holds them already (dilated_attn_cache_append): for the token
 * at position p of its sequence what row p of dilated_attn_fwd gives on the
 * sequence's first p + 1 rows.  Query head h reads key head h / (H / Hkv); a
 * pattern's offsets go by the query head.
 *
 * q           device pointer, T tokens of H heads, q_stride elements apart.
 * out         device pointer, [T, H, D] contiguous, written (every element).
 * lse         device pointer, [H, T] float32, written (every element).
 * H           a multiple of Hkv; H < 2^16, T * H < 2^31.
 * max_new     the most new tokens of any sequence, as far as the caller knows,
 *             or T: it only helps to choose the launches (a launch for
 *             sequences with many new tokens is left out where none has more
 *             than 4), results are right whatever it says.
 * patterns, softmax_scale: as for dilated_attn_fwd.
 * workspace   device scratch of at least the bytes that
 *             dilated_attn_paged_workspace reports for the same sizes.
 *
 * DA_BF16: scores as exact products summed in float32; probabilities rounded
 * to bf16 for the product with v, summed in float32; a sequence's tokens by
 * themselves (at most 4 new ones) mix float32 partial rows, otherwise a
 * pattern's rows are kept as in dilated_attn_fwd; out rounded once.  DA_F32
 * computes in float32 throughout.  Results are finite under the conditions of
 * dilated_attn_fwd for the sequence's own tokens; a row that sees a key whose
 * score is NaN or plus infinity is NaN in out and lse, and an element of v that is
 * not finite makes that element of the rows that see its key not finite, and of no
 * others.  What lies in the pool beyond a sequence's length is never used, whatever it
 * holds.  The same call gives the same bits every time; keys are split by the sizes of the call, so a
 * sequence alone and in a batch can differ by the rounding of its sums.
 * Outputs and workspace must not overlap each other, q or the cache.
 */
int dilated_attn_paged_workspace(int64_t T, int64_t B, int64_t H, int64_t Hkv, int64_t D, int64_t num_pages,
                                 int64_t page_size, int64_t max_pages, int64_t max_new,
                                 const da_pattern_t* patterns, int64_t num_patterns, int64_t dtype,
                                 uint64_t* bytes);
int dilated_attn_paged_fwd(const void* q, const da_paged_cache_t* cache, void* out, float* lse, int64_t T, int64_t B,
                           int64_t H, int64_t Hkv, int64_t D, int64_t q_stride, int64_t max_new,
                           const da_pattern_t* patterns, int64_t num_patterns, int64_t dtype, float softmax_scale,
                           void* workspace, uint64_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* DILATED_ATTN_PAGED_H */
