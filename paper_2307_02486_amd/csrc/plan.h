// Host-side plan of one dilated-attention forward call: validation, per-pattern
// geometry, work-item enumeration, workspace layout and exact work accounting.
// No HIP dependency, so it builds and runs with a plain host compiler.
#pragma once

#include <cstddef>
#include <cstdint>

#include "../../include/dilated_attn.h"

#if defined(__HIPCC__)
#define DA_HD __host__ __device__
#else
#define DA_HD
#endif

namespace da {

// Division by a divisor fixed at plan time, for numerators below 2^31:
// q = floor(n * mul / 2^shift) with shift = 31 + ceil(log2 d) and
// mul = ceil(2^shift / d) < 2^32 (Granlund and Montgomery, "Division by
// invariant integers using multiplication", 1994, Thm. 4.2 with N = 31).
struct FastDiv {
  uint32_t d;
  uint32_t mul;
  uint32_t shift;
  DA_HD uint32_t div(uint32_t n) const {
    return static_cast<uint32_t>((static_cast<uint64_t>(n) * mul) >> shift);
  }
};
FastDiv make_fastdiv(uint32_t d);

// Geometry of one pattern (w, r) after validation.  Segment g covers rows
// [g*w, min((g+1)*w, N)); head h keeps the rows at local offsets
// h mod r, h mod r + r, ... (Sec. 2.2 Eqs. 3-5, offset of Sec. 2.3).
struct PatternPlan {
  int64_t w;          // segment length, clamped to N (w > N means one segment)
  int64_t r;          // dilation rate
  int64_t nseg;       // ceil(N / w)
  int64_t lmax;       // kept rows of a full segment at offset 0: ceil(w / r)
  int64_t ntiles;     // query tiles per (b, h, segment) unit: ceil(lmax / block_m)
  int64_t units;      // B * H * nseg
  int64_t item_begin; // index of this pattern's first work item
  uint64_t o_off;     // byte offset of the per-pattern output in the workspace
                      // (fp16 rows scaled by a power of two for bf16 inputs,
                      // fp32 rows for fp32 inputs)
  uint64_t lse_off;   // byte offset of the per-row records (float lse, float
                      // scale: the row's values are the stored ones times it)
};

struct Plan {
  int64_t B, N, H, D;
  int causal;
  int dtype;
  float scale;        // softmax scale actually used
  int npat;
  int block_m;        // query rows per attention work item
  PatternPlan pat[DA_MAX_PATTERNS];
  int64_t total_items;
  int64_t launch_items;  // workgroups of the attention launch (XCD-balanced, >= total_items)
  bool offsets32;        // every key tile spans < 2^31 bytes: 32-bit buffer offsets suffice
  uint64_t workspace_bytes;
  int64_t covered_rows;
  double sparse_flops;
  double bytes_attn;
  double bytes_combine;
};

// Workspace of a backward call: per (b, h, row) -lse/scale and -delta
// (float32, [B][H][N] each), then per pattern the compact fp16 gradients
// of its kept rows, [units][lmax][D] for dq, dk and dv.
struct BwdLayout {
  uint64_t nl2_off;   // byte offset of -lse/scale
  uint64_t nd_off;    // byte offset of -delta
  // Per pattern, the compact gradients dq, dk, dv: fp16 rows [units*lmax][D],
  // each row scaled by a power of two per chunk of kGradChunk columns, and
  // the float scales [units*lmax][chunks] (see grad_chunks).
  uint64_t dq_off[DA_MAX_PATTERNS];
  uint64_t dk_off[DA_MAX_PATTERNS];
  uint64_t dv_off[DA_MAX_PATTERNS];
  uint64_t dq_rec_off[DA_MAX_PATTERNS];
  uint64_t dk_rec_off[DA_MAX_PATTERNS];
  uint64_t dv_rec_off[DA_MAX_PATTERNS];
  uint64_t workspace_bytes;
  double flops;          // 10*D per unmasked pair
  double bytes_grad;     // algorithmic HBM bytes of the dq and dk/dv kernels
  double bytes_combine;  // algorithmic HBM bytes of the delta and sum kernels
  bool delta_pass;       // no pattern keeps every row (r = 1): delta takes a pass of its own
};

// Columns of a compact gradient row that share one scale.
constexpr int64_t kGradChunk = 64;
inline int64_t grad_chunks(int64_t D) { return (D + kGradChunk - 1) / kGradChunk; }

// Backward workspace and work of a validated forward plan.  DA_EUNSUPPORTED
// unless the plan is bf16 (and for tiles whose offsets need 64 bits).
int make_bwd_layout(const Plan& p, BwdLayout* out);

// Query rows per work item of the attention kernel for a dtype.
int block_m_for(int dtype);

// Number of rows a pattern keeps in a segment of `seg_len` rows at offset s.
inline int64_t kept_rows(int64_t seg_len, int64_t s, int64_t r) {
  return seg_len > s ? (seg_len - s + r - 1) / r : 0;
}

// Validate and fill a plan.  Returns DA_OK or a negative DA_E* code.
int make_plan(int64_t B, int64_t N, int64_t H, int64_t D, const da_pattern_t* patterns,
              int64_t num_patterns, int64_t causal, int64_t dtype, float softmax_scale,
              Plan* out);

// Attention over a paged cache.  A sequence's new tokens are computed in one of
// two ways: each token by itself (all its keys' splits in parallel), or in
// tiles of kept query rows.  A sequence of at most kPagedFew new tokens takes
// the first, unless it is the call's only one.  (64 sequences of 500 to 8000
// tokens, the paper's patterns, 12 heads of 64: 4 tokens each by themselves 131
// us, 8 tokens 225, in tiles 9 tokens 175; 4 sequences at 31500: 8 tokens 46 us,
// 16 in tiles 37.)  Both write one partial row per (token, head) and slot, a
// slot being one split of one pattern's keys, and the join reads them.
constexpr int64_t kPagedFew = 4;
constexpr int64_t kPagedRows = 128;      // query rows of a tile
constexpr int64_t kPagedKeyTile = 64;    // its keys at a time
constexpr int64_t kPagedGroupRows = 16;  // query heads of one key head that a token's workgroup holds

struct PagedPattern {
  int32_t w, r;              // segment length (clamped to the table's reach), dilation
  FastDiv fw, fr;            // divisions by them
  FastDiv one_split;         // division by the splits of a single token's keys
  int32_t one_slot;          // its first slot there
  int32_t one_begin;         // its first workgroup among the single tokens'
  FastDiv one_heads;         // division by a token's workgroups for one split
  FastDiv tile_split;        // division by the splits of a tile's keys
  int32_t tile_slot;         // its first slot there
  int32_t tiles, run;        // bound on its query tiles per head; tiles of a unit (next to each other, of one head)
  int32_t tile_begin;        // its first workgroup among the tiles'
};

struct PagedPlan {
  int64_t T, B, H, Hkv, D, num_pages, page, max_pages;
  int dtype, page_log2, npat;
  float scale;
  bool all_few;              // every token by itself
  int full;                  // the pattern with r = 1 and the longest segment, or -1
  int64_t few;               // new tokens up to which a sequence's are computed by themselves
  int64_t singles;           // tokens computed by themselves, at most
  int64_t one_slots, tile_slots;
  int64_t one_items, tile_items;  // workgroups of the single tokens and of the tiles, at most
  int64_t grid;              // of the launch
  bool steps;                // its workgroups step through the items that there are
  uint64_t one_rec_off, one_row_off, tile_rec_off, tile_row_off, workspace_bytes;
  PagedPattern pat[DA_MAX_PATTERNS];
};

int make_paged_plan(int64_t T, int64_t B, int64_t H, int64_t Hkv, int64_t D, int64_t num_pages, int64_t page,
                    int64_t max_pages, int64_t max_new, const da_pattern_t* patterns, int64_t num_patterns,
                    int64_t dtype, float softmax_scale, PagedPlan* out);

}  // namespace da
