/*
 * dilated_attn_compressed.h - C ABI of serving from a compressed cache: keys and
 * values in 8 bits, and pages given up by the attention that they get.  The cache
 * is that of dilated_attn_paged.h otherwise; types, limits and error codes are
 * those of dilated_attn.h.
 */
#ifndef DILATED_ATTN_COMPRESSED_H
#define DILATED_ATTN_COMPRESSED_H

#include "dilated_attn_paged.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * A paged cache in 8 bits.  pages.k and pages.v hold e4m3 values (one sign, four
 * exponent and three mantissa bits, largest 448, no infinities), [num_pages, Hkv,
 * page_size, D] bytes, and each block of DA_CACHE_BLOCK tokens (a whole page, if
 * that is fewer) of one key head has a scale: a byte x stands for 2^(x - 127), and
 * an element is its e4m3 value times its block's scale.  The append writes
 * 1 <= x <= 253; 0 and 255 are not to be there.
 *
 * A table entry outside [0, num_pages) is a page that is not there: it holds no
 * keys.  Tokens keep their positions when pages before them go.
 */
#define DA_CACHE_BLOCK 16
typedef struct {
  da_paged_cache_t pages;
  uint8_t* k_scale; /* device, [num_pages, Hkv, page_size / block] */
  uint8_t* v_scale; /* device, the same shape                      */
} da_paged_cache_f8_t;

/*
 * dilated_attn_cache_append_f8 - dilated_attn_cache_append into an 8-bit cache:
 * keys (normed and rotated in float32) and values are rounded to e4m3, nearest even.
 * A block's scale is the least power of two, 2^-126 at least, whose 448-fold is not
 * below the block's largest finite magnitude; a block that has tokens already keeps
 * its scale or takes a larger one, its older values then multiplied by the quotient
 * (exact, but for those that fall below 2^-6 times the new scale: these are rounded
 * once more).  Scales never shrink while a block has tokens; whoever wants to take
 * an append back keeps a copy of the blocks in which its tokens follow earlier ones.
 * Infinities and NaN become NaN and do not count for the scale.  Finite magnitudes
 * have to be below 2^127.
 *
 * Arguments as for dilated_attn_cache_append, dtype the type of q, k, v, qw, kw and
 * qo; T < 2^30.  A page belongs to one sequence of the call: two sequences that name
 * one page leave either's values there, in part.
 */
int dilated_attn_cache_append_f8(const void* q, const void* k, const void* v, const void* qw, const void* kw,
                                 void* qo, const da_paged_cache_f8_t* cache, int64_t T, int64_t B, int64_t H,
                                 int64_t Hkv, int64_t D, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                                 float eps, int64_t rotate, int64_t center, float base, float gamma,
                                 float scale_base, int64_t dtype, void* stream);

/*
 * dilated_attn_paged_fwd_f8 - dilated_attn_paged_fwd over an 8-bit cache; the
 * workspace is that of dilated_attn_paged_workspace.  dtype is the type of q and
 * out.  An element of the cache of 2^-126 or more is exact in bf16 and float32 (a
 * smaller one may count as zero), so that a result is what dilated_attn_paged_fwd
 * gives (up to the rounding of its sums) on a cache that holds the same values; keys
 * of pages that are not there are left out, and a row all of whose keys are has out = 0
 * and lse = -inf.
 */
int dilated_attn_paged_fwd_f8(const void* q, const da_paged_cache_f8_t* cache, void* out, float* lse, int64_t T,
                              int64_t B, int64_t H, int64_t Hkv, int64_t D, int64_t q_stride, int64_t max_new,
                              const da_pattern_t* patterns, int64_t num_patterns, int64_t dtype,
                              float softmax_scale, void* workspace, uint64_t workspace_bytes, void* stream);

/*
 * dilated_attn_page_weights - the attention that each page gets from the new
 * tokens: weights[page] += the sum, over the page's keys, the new tokens of its
 * sequence that see them, their heads and the patterns that hold the pair, of
 * exp(softmax_scale q.k - lse).  The weights of a token's pages grow by one for
 * each head that sees a key.
 *
 * q           device pointer, T tokens of H heads, q_stride elements apart: the
 *             queries of dilated_attn_paged_fwd_f8.
 * lse         device pointer, [H, T] float32: that call's.  Rows whose lse is not
 *             finite add nothing.
 * cache       the keys (pages.v and v_scale are not looked at and may be NULL).
 * weights     device pointer, [num_pages] float32, updated.  The tables name a page
 *             once: of one that they name twice either sum may be lost.
 * max_new     the most new tokens of any sequence, 0 if the caller does not know: it
 *             chooses how the work is cut, and results differ by rounding only.
 * workspace   device scratch of at least the bytes that
 *             dilated_attn_page_weights_workspace reports for the same sizes, one
 *             call's at a time.
 *
 * Other arguments as for dilated_attn_paged_fwd_f8, with (T + 32) * H < 2^31.  Scores are sums of exact
 * products in float32 (float32 queries as three bf16 terms), sums are float32 in an
 * order that the sizes fix: the same call gives the same bits every time.
 */
int dilated_attn_page_weights_workspace(int64_t T, int64_t B, int64_t H, int64_t Hkv, int64_t D, int64_t num_pages,
                                        int64_t page_size, int64_t max_pages, int64_t max_new,
                                        const da_pattern_t* patterns, int64_t num_patterns, int64_t dtype,
                                        uint64_t* bytes);
int dilated_attn_page_weights(const void* q, const float* lse, const da_paged_cache_f8_t* cache, float* weights,
                              int64_t T, int64_t B, int64_t H, int64_t Hkv, int64_t D, int64_t q_stride,
                              int64_t max_new, const da_pattern_t* patterns, int64_t num_patterns, int64_t dtype,
                              float softmax_scale, void* workspace, uint64_t workspace_bytes, void* stream);

/*
 * dilated_attn_evict_pages - the pages of least weight out of each sequence's
 * table.  A sequence of seq_lens[b] tokens has the pages of the first
 * ceil(seq_lens[b] / page_size) entries of its row that are in [0, num_pages).  If
 * these are more than `keep`, the lightest go, of equal ones those that come first
 * in the row, until `keep` are left; but never the row's first `first` entries nor
 * the last `last` of the ceil(...) ones, even if that leaves more.  A NaN weighs
 * more than any number.
 *
 * weights     device pointer, [num_pages] float32, read only.
 * block_table, seq_lens: device pointers, int32 [B, max_pages] and [B].
 * table_out   device pointer, int32 [B, max_pages], written: the table with -1 for
 *             the pages that go; may equal block_table.
 * freed       device pointer, int32 [B, max_pages], written: the pages that go, in
 *             the order of the row, then -1.
 * count       device pointer, int32 [B], written: how many go.
 * page_size, max_pages: as in da_paged_cache_t.  keep, first, last: at least 0.
 */
int dilated_attn_evict_pages(const float* weights, const int32_t* block_table, const int32_t* seq_lens,
                             int32_t* table_out, int32_t* freed, int32_t* count, int64_t B, int64_t num_pages,
                             int64_t page_size, int64_t max_pages, int64_t keep, int64_t first, int64_t last,
                             void* stream);

#ifdef __cplusplus
}
#endif

#endif /* DILATED_ATTN_COMPRESSED_H */
