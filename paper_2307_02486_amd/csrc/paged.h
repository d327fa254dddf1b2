// Launchers of the head norms, of the append to a paged cache and of the attention over it.
#pragma once

#include <hip/hip_runtime.h>

#include "plan.h"

namespace da {

// The xPos rotation of the head operators (rotate false: none).
struct HeadRotation {
  bool rotate;
  int64_t center;
  float base, gamma, scale_base;
};

// Queries and keys of B * N tokens (or of T tokens in B sequences), strides in
// elements between tokens, norm weights [D] or null, outputs.
struct QkNormCall {
  const void *q, *k, *qw, *kw;
  void *qo, *ko;
  int64_t B, N, H, Hkv, D, q_stride, k_stride;
  float eps;
  HeadRotation rot;
  int dtype;
};

// RMS norm of every head and its rotation in one pass, and its gradients; the
// weights' gradients go through a float32 workspace.
hipError_t launch_qk_norm(const QkNormCall& c, hipStream_t stream);
uint64_t qk_norm_bwd_workspace(int64_t tokens, int64_t D);
hipError_t launch_qk_norm_bwd(const QkNormCall& c, const void* dqo, const void* dko, void* dq, void* dk, void* dqw,
                              void* dkw, void* workspace, hipStream_t stream);

// A paged cache: k and v [num_pages][Hkv][page][D], page = 2^page_log2 tokens;
// sequence b holds lens[b] tokens, token p in page table[b][p / page]; its new
// tokens are rows start[b] .. start[b + 1] of the call's token arrays, the last
// of its length.
struct PagedCache {
  void *k, *v;
  const int32_t *table, *lens, *start;
  int64_t num_pages, max_pages;
  int page_log2;
  // 8-bit caches (k and v hold e4m3 values; otherwise null): the scales' exponents,
  // biased by 127, [num_pages][Hkv][page / block], block = 2^min(page_log2, kCacheBlockLog2)
  // tokens.  Pages outside the pool hold no keys there.
  uint8_t *k_scale = nullptr, *v_scale = nullptr;
};
constexpr int kCacheBlockLog2 = 4;

hipError_t launch_cache_append(const QkNormCall& c, const void* v, int64_t v_stride, const PagedCache& cache,
                               int64_t T, hipStream_t stream);

// Dilated attention of new tokens over a paged cache.
hipError_t launch_paged(const PagedPlan& plan, const void* q, int64_t q_stride, const PagedCache& cache, void* out,
                        float* lse, void* workspace, hipStream_t stream);

// New keys and values into an 8-bit cache, and the queries beside them.
hipError_t launch_cache_append8(const QkNormCall& c, const void* v, int64_t v_stride, const PagedCache& cache,
                                int64_t T, hipStream_t stream);

// The attention weight that the pages of an 8-bit cache got from new tokens, added
// to weights [num_pages].
hipError_t launch_page_weights(const WeightPlan& plan, const void* q, int64_t q_stride, const float* lse,
                               const PagedCache& cache, float* weights, void* workspace, hipStream_t stream);

// The lightest pages out of each sequence's table.
struct EvictCall {
  const float* weights;
  const int32_t *table, *lens;
  int32_t *table_out, *freed, *count;
  int64_t B, num_pages, page_size, max_pages, keep, first, last;
};
hipError_t launch_evict(const EvictCall& c, hipStream_t stream);

}  // namespace da
