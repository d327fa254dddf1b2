// Which pages of an 8-bit cache the attention looks at, and which of them go.
//
// page_weights: for each page the sum, over the call's new tokens, their heads,
// the patterns that hold a pair and the page's keys, of the pair's share of its
// row's softmax, exp(scale q.k - lse) with the row's log-sum-exp from the attention.
// A workgroup is one unit of a pattern (a key head with the query heads that share
// a dilation offset: their keys are the same lattice g w + rho + t r) and one split
// of the pages that the keys lie in.  64 keys stay in registers as operands of
// v_mfma_f32_16x16x32_bf16 while columns of 16 (token, head) pairs pass by.  Then the
// keys of a page are added, and a second launch adds a page's partial sums: no
// atomics, the same bits every time.  float32 queries are three bf16 terms each, whose
// products with an e4m3 key are exact.  All sums are float32.
//
// Single tokens (64 at 1K to 32K cached, five patterns, 56 MB of keys): 33 us and the
// join's 7.0.  Waves that look their own rows up, with the next tile's keys under way
// and a segmented sum of a tile's pages, where a sum over the wave for each page took
// 45 us and 256 keys a round of the workgroup 67.  What is left is the chain of an
// item's start (lengths, table, queries, keys) and the tail, as in the attention.
// Chunks (512 tokens at 31500, 16 heads of 128 over four key heads, five patterns, 6.1
// GFLOP): 33 us and 6.8; with a tile of keys a workgroup in every pattern 45, and with
// every key operand read from LDS again for each 16 columns 159.  Bound by latency: an
// item's start and its few steps of 16 columns, at two to three waves a SIMD.
//
// evict_pages: a workgroup per sequence finds the weight up to which pages go by
// counting digits of eight bits, then lists them in the order of the table.  Bound by
// one CU's rate of single loads and LDS adds: 64 sequences of up to 512 pages 7 us, one
// of 16384 28 (with one copy of the digits' counts, and three barriers for each
// 1024 pages of the list, 36).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "heads_device.h"
#include "paged_device.h"

namespace da {
namespace {

struct WeightArgs {
  const void* q;
  const float* lse;
  const char* kc;
  const uint8_t* ks;
  const int32_t *table, *lens, *start;
  float* part;     // of each pattern [units][rows][pages], from the row's first page on
  float* weights;  // [num_pages]
  int64_t qs;
  int32_t T, B, H, Hkv, G, npat, num_pages, max_pages, page_log2, block_log2, rows, items;
  uint32_t reach;
  float scale_log2;
  int32_t begin[DA_MAX_PATTERNS];
  PagedPattern pat[DA_MAX_PATTERNS];
};

// The new tokens of row `row`: those of a sequence, or one token.
template <bool kLone>
__device__ inline NewTokens row_tokens(const WeightArgs& a, int row, int lane, int& b) {
  if constexpr (kLone) {
    const int tok[1] = {row};
    Sequence sq[1];
    find_sequences(a, tok, lane, sq);
    const int pos = position_of(a, sq[0], row);
    b = sq[0].b;
    return pos < 0 ? NewTokens{0, 0, 0} : NewTokens{pos, pos + 1, row - pos};
  } else {
    b = row;
    return new_tokens(a, row);
  }
}
// Unit u of pattern P for tokens from position c0 on: its key head and offset, and
// the query heads; false: the token has no such unit.
struct Unit {
  int hk, rho;
  KeptHeads heads;
};
template <bool kLone>
__device__ inline bool unit_of(const WeightArgs& a, const PagedPattern& P, int c0, int u, Unit& x) {
  if constexpr (kLone) {
    x.rho = lattice_of(P, c0).rho;
    x.hk = u;
    if (P.r >= a.G) {
      const int64_t h = x.rho + static_cast<int64_t>(u) * P.r;
      if (h >= a.H) return false;
      x.hk = static_cast<int>(h) / a.G;
    }
    x.heads = kept_heads(P, x.hk, a.G, x.rho);
    return x.heads.count > 0;
  } else {
    const int C = min(a.G, P.r);
    x.hk = u / C;
    const int c = u - x.hk * C, head = x.hk * a.G + c;
    x.rho = head_offset(P, head);
    x.heads = KeptHeads{head, static_cast<int>(P.fr.div(a.G - 1 - c)) + 1};
    return true;
  }
}

// Eight elements of a query as operands, the largest term first: their sum is the
// element (three bf16 terms hold a float32's 24 bits).
__device__ inline void split_terms(const u16* p, u32x4 (&t)[1]) { t[0] = load16(p); }
__device__ inline void split_terms(const float* p, u32x4 (&t)[3]) {
  const f32x8 x = *reinterpret_cast<const f32x8*>(p);
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    float r0 = x[e], r1 = x[e + 1];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const __bf16 b0 = (__bf16)r0, b1 = (__bf16)r1;
      t[i][e / 2] = static_cast<uint32_t>(__builtin_bit_cast(u16, b0)) |
                    (static_cast<uint32_t>(__builtin_bit_cast(u16, b1)) << 16);
      r0 -= static_cast<float>(b0);
      r1 -= static_cast<float>(b1);
    }
  }
}

constexpr int kWtKeys = 64;  // keys of a tile

// What an item has to do: its row's new tokens, its unit, its share of the unit's
// columns, its pages [p0, p1).
struct WeightItem {
  NewTokens c;
  Unit un;
  int b, row, u, share, seg0, p0, p1;
};
template <bool kLone>
__device__ inline bool weight_item(const WeightArgs& a, int idx, int pi, int lane, WeightItem& it) {
  const PagedPattern& P = a.pat[pi];
  // Unit number n runs with all its splits on XCD n mod 8.
  const int j = (idx - P.one_begin) >> 3, block8 = P.one_split.div(j);
  const int split = j - block8 * P.one_split.d, n = block8 * 8 + ((idx - P.one_begin) & 7);
  it.row = P.one_heads.div(n);
  it.u = n - it.row * P.one_heads.d;
  if (it.row >= a.rows) return false;
  it.c = row_tokens<kLone>(a, it.row, lane, it.b);
  const int u = P.tile_split.div(it.u);
  it.share = it.u - u * P.tile_split.d;
  if (it.c.c1 <= it.c.c0 || !unit_of<kLone>(a, P, it.c.c0, u, it.un)) return false;
  // this split's pages, of those from the first token's segment on
  it.seg0 = static_cast<int>(P.fw.div(it.c.c0)) * P.w;
  const int pg0 = it.seg0 >> a.page_log2, pages = ((it.c.c1 - 1) >> a.page_log2) + 1 - pg0;
  const int per = min(static_cast<int>(P.one_split.div(pages - 1)) + 1, static_cast<int>(kWeightPages));
  // (where a table has close to 2^31 pages, the splits past the row's end begin beyond that)
  const uint32_t skip = static_cast<uint32_t>(split) * per;
  if (skip >= static_cast<uint32_t>(pages)) return false;
  it.p0 = pg0 + static_cast<int>(skip);
  it.p1 = pg0 + min(static_cast<int>(skip) + per, pages);
  return true;
}
// The page that a row's sums begin with, if pg is its first.
__device__ inline int first_sum(int pg) { return pg & -static_cast<int>(kWeightAlign); }
// The item's partial sums: of page 0, were it among the row's.
__device__ inline float* sums_of(const WeightArgs& a, const PagedPattern& P, const WeightItem& it) {
  return a.part + P.one_slot * kWeightAlign + (static_cast<int64_t>(it.u) * a.rows + it.row) * P.tiles -
         first_sum(it.seg0 >> a.page_log2);
}
// The first t at or after segment-local position x, of those rho + t r.
__device__ inline int first_at(const PagedPattern& P, int rho, int x) {
  return x > rho ? static_cast<int>(P.fr.div(x - rho - 1)) + 1 : 0;
}

struct SmemWeights {
  uint32_t row[kPgWaves][kWtKeys];  // cache rows of a wave's tile
  float sums[kPgWaves][kWtKeys];    // what its keys got
  float psum[kWeightPages];         // what the item's pages got
};
// The rows of keys first .. first + 63 (positions base + t r), those past `last` as that
// one, into a wave's LDS; returns the keys whose page is there, a bit each.
__device__ inline uint64_t tile_rows(const WeightArgs& a, const int32_t* table, int hk, int base, int r, int first,
                                     int last, int lane, uint32_t (&rows)[kWtKeys]) {
  const int pos = base + min(first + lane, last) * r, entry = table_entry(a, table, pos);
  const uint32_t row = cache_row(a, entry, hk, pos);  // in the pool, whatever the entry
  const uint64_t live = __ballot(static_cast<uint32_t>(entry) < static_cast<uint32_t>(a.num_pages) && first + lane <= last);
  rows[lane] = row;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // (a wave's LDS operations complete in order)
  __builtin_amdgcn_wave_barrier();
  return live;
}
// Sum over the wave's lanes, in all of them.
__device__ inline float wave_sum(float v) {
  v = row_sum<16>(v);
  auto lane = [&](int l) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), l)); };
  return (lane(0) + lane(16)) + (lane(32) + lane(48));
}
// A key's sum over its 16 columns, for the 64 keys of a tile, into the wave's LDS.
__device__ inline void put_sums(f32x4 (&sum)[4], int m, int grp, float (&out)[kWtKeys]) {
#pragma unroll
  for (int u = 0; u < 4; ++u) {
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[u][e] = row_sum<16>(sum[u][e]);
    if (m == 0) *reinterpret_cast<f32x4*>(&out[16 * u + 4 * grp]) = sum[u];
  }
}
// A row's lse in log2 units; false where it is not finite: a row that sees nothing, or NaN.
__device__ inline bool lse_of(const WeightArgs& a, int head, int tok, float& l) {
  const float x = a.lse[static_cast<int64_t>(head) * a.T + tok];
  uint32_t bits = __builtin_bit_cast(uint32_t, x);
  asm("" : "+v"(bits));
  l = x * kLog2e;
  return (bits & 0x7fffffffu) < 0x7f800000u;
}

template <typename T, int D>
struct QueryFrag {
  static constexpr int kTerms = sizeof(T) == 2 ? 1 : 3;
  u32x4 q[D / 32][kTerms];
};
template <typename T, int D>
__device__ inline void load_queries(const WeightArgs& a, int tok, int head, int grp, bool there, QueryFrag<T, D>& f) {
#pragma unroll
  for (int c = 0; c < D / 32; ++c) {
    split_terms(static_cast<const T*>(a.q) + tok * a.qs + head * D + step_first<D>(c, grp), f.q[c]);
    if (!there)
#pragma unroll
      for (int i = 0; i < QueryFrag<T, D>::kTerms; ++i) f.q[c][i] = u32x4{0u, 0u, 0u, 0u};
  }
}
// Scores of 64 keys by 16 columns.
template <typename T, int D>
__device__ inline void scores(const u32x4 (&k)[4][D / 32], const QueryFrag<T, D>& f, f32x4 (&s)[4]) {
#pragma unroll
  for (int u = 0; u < 4; ++u) s[u] = f32x4{0, 0, 0, 0};
#pragma unroll
  for (int i = QueryFrag<T, D>::kTerms - 1; i >= 0; --i)
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
      for (int u = 0; u < 4; ++u)
        s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[u][c]),
                                                       __builtin_bit_cast(bf16x8, f.q[c][i]), s[u], 0, 0, 0);
}

// What the keys first .. first + 63 of a tile got, v (0 past `last`), a lane each, to their
// pages' sums.  Keys of a page are neighbours: a sum over each run of them, and its
// last lane adds it.
__device__ inline void add_pages(const WeightArgs& a, const PagedPattern& P, int base, int first, int last, int lane, float v,
                                 float* psum) {
  const int pg = (base + min(first + lane, last) * P.r) >> a.page_log2;
  const int before = __shfl_up(pg, 1);
  const uint64_t starts = __ballot(lane == 0 || before != pg);
  if (starts == 1) {
    v = wave_sum(v);
  } else {
    const int behind = lane - (63 - __builtin_clzll(starts & (~uint64_t{0} >> (63 - lane))));
    const int most = min(64, ((1 << a.page_log2) - 1) / P.r + 1);
    for (int step = 1; step < most; step <<= 1) {
      const float w = __shfl_up(v, step);
      v += behind >= step ? w : 0.0f;
    }
  }
  const int end = min(63, last - first);
  if (lane == end || (lane < end && (starts >> (lane + 1) & 1))) psum[pg] += v;
}

// Rows that are tokens: a wave has a share of the item's pages and meets no other.
template <typename T, int D>
__global__ __launch_bounds__(kPgThreads) void weight_tokens(WeightArgs a) {
  constexpr int KC = D / 32;
  __shared__ __attribute__((aligned(16))) SmemWeights sm;
  const int tid = thread_id(), lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int idx = launch_index();
  if (idx >= a.items) return;
  const int pi = pattern_at(a.begin, idx);
  const PagedPattern& P = a.pat[pi];
  WeightItem it;
  if (!weight_item<true>(a, idx, pi, lane, it)) return;
  const int rho = it.un.rho, nh = it.un.heads.count, pos = it.c.c0, tok = it.c.tok0 + pos;
  const int per = (it.p1 - it.p0 + kPgWaves - 1) / kPgWaves;
  const int p0 = it.p0 + wv * per, p1 = min(p0 + per, it.p1);
  if (p0 >= p1) return;
  for (int i = p0 + lane; i < p1; i += 64) sm.psum[i - it.p0] = 0.0f;

  const int m = lane & 15, grp = lane >> 4, base = it.seg0 + rho;
  const int32_t* table = a.table + static_cast<int64_t>(it.b) * a.max_pages;
  const float c2 = a.scale_log2;
  const int64_t end = static_cast<int64_t>(p1) << a.page_log2;
  const int t0 = first_at(P, rho, max((p0 << a.page_log2) - it.seg0, 0));
  const int t1 = first_at(P, rho, static_cast<int>(min(end, static_cast<int64_t>(pos) + 1)) - it.seg0);
  for (int h0 = 0; h0 < nh; h0 += 16) {
    QueryFrag<T, D> f;
    const bool there = h0 + m < nh;
    const int head = it.un.heads.first + (there ? h0 + m : 0) * P.r;
    load_queries<T, D>(a, tok, head, grp, there, f);
    float l;
    const bool counts = lse_of(a, head, tok, l) && there;
    // The next tile's keys are under way while one is computed.
    KeyFrag8<D> next[2];
    uint64_t live = 0;
    auto request = [&](int first) {
      live = tile_rows(a, table, it.un.hk, base, P.r, first, t1 - 1, lane, sm.row[wv]);
#pragma unroll
      for (int h = 0; h < 2; ++h) request_keys8<D>(a, sm.row[wv] + 32 * h, m, grp, next[h]);
    };
    if (t0 < t1) request(t0);
    for (int first = t0; first < t1; first += kWtKeys) {
      u32x4 k[4][KC];
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int s = 0; s < KC; ++s) k[u][s] = next[u >> 1].wide(u & 1, s);
      const uint64_t now = live;
      if (first + kWtKeys < t1) request(first + kWtKeys);
      if (!now) continue;
      f32x4 s[4];
      scores<T, D>(k, f, s);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const uint32_t mine = static_cast<uint32_t>(now >> (16 * u + 4 * grp));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][e], c2, -l));
          s[u][e] = counts && (mine >> e & 1) ? p : 0.0f;
        }
      }
      put_sums(s, m, grp, sm.sums[wv]);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      add_pages(a, P, base, first, min(first + kWtKeys, t1) - 1, lane, sm.sums[wv][lane], sm.psum - it.p0);
    }
  }
  float* part = sums_of(a, P, it);
  for (int i = p0 + lane; i < p1; i += 64) part[i] = sm.psum[i - it.p0];
}

// Rows that are sequences.  Of many columns (a long chunk has hundreds) the waves share a
// tile's keys and take 16 in turn; of few each wave has a tile of its own and all columns.
template <typename T, int D>
__global__ __launch_bounds__(kPgThreads) void weight_sequences(WeightArgs a) {
  constexpr int KC = D / 32;
  __shared__ __attribute__((aligned(16))) SmemWeights sm;
  const int tid = thread_id(), lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int idx = launch_index();
  if (idx >= a.items) return;
  const int pi = pattern_at(a.begin, idx);
  const PagedPattern& P = a.pat[pi];
  WeightItem it;
  if (!weight_item<false>(a, idx, pi, lane, it)) return;
  const NewTokens c = it.c;
  const int rho = it.un.rho, nh = it.un.heads.count;
  for (int i = tid; i < it.p1 - it.p0; i += kPgThreads) sm.psum[i] = 0.0f;

  const int m = lane & 15, grp = lane >> 4;
  const int32_t* table = a.table + static_cast<int64_t>(it.b) * a.max_pages;
  const float c2 = a.scale_log2;
  const int x0 = max(it.p0 << a.page_log2, it.seg0);
  const int x1 = static_cast<int>(min(static_cast<int64_t>(it.p1) << a.page_log2, static_cast<int64_t>(c.c1)));
  for (int g = P.fw.div(x0); g <= static_cast<int>(P.fw.div(x1 - 1)); ++g) {
    const int gs = g * P.w, base = gs + rho;
    const int t0 = first_at(P, rho, x0 - gs), t1 = first_at(P, rho, min(x1 - gs, P.w));  // keys
    const int q0 = max(first_at(P, rho, c.c0 - gs), t0), q1 = first_at(P, rho, min(c.c1 - gs, P.w));  // queries that see some
    if (q0 >= q1) continue;
    const bool apart = (q1 - q0) * nh <= kWeightApart;
    for (int k00 = t0; k00 < t1 && k00 < q1; k00 += apart ? kPgWaves * kWtKeys : kWtKeys) {
      const int k0 = apart ? k00 + wv * kWtKeys : k00;  // the wave's keys
      // Columns: tokens qa .. q1 - 1 of the nh heads, head by head (in blocks of 16
      // tokens if there are that many, so that a block's last key is near its first);
      // this item's share of them.
      const int qa = max(q0, k0), ntok = k0 < t1 ? max(q1 - qa, 0) : 0, per = ntok < 16 ? ntok : (ntok + 15) & ~15,
                cols = per * nh;
      const int share = (static_cast<int>(P.tile_split.div(((cols + 15) >> 4) + P.tile_split.d - 1))) << 4;
      const int cend = min(cols, (it.share + 1) * share), cbegin = it.share * share + (apart ? 0 : 16 * wv);
      f32x4 sum[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) sum[u] = f32x4{0, 0, 0, 0};
      uint64_t live = 0;
      if (cbegin < cend) live = tile_rows(a, table, it.un.hk, base, P.r, k0, t1 - 1, lane, sm.row[wv]);
      if (live) {
        KeyFrag8<D> kf[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) request_keys8<D>(a, sm.row[wv] + 32 * h, m, grp, kf[h]);
        struct Column {
          int last;  // its last key, -1: none
          float l;
        };
        auto column = [&](int col, QueryFrag<T, D>& f, Column& x) {
          const int h = col / per, t = col - h * per;
          const bool there = col < cols && t < ntok;
          const int token = there ? qa + t : qa, head = it.un.heads.first + (there ? h : 0) * P.r;
          const int tok = c.tok0 + base + token * P.r;
          load_queries<T, D>(a, tok, head, grp, there, f);
          x.last = lse_of(a, head, tok, x.l) && there ? token : -1;
        };
        const int step = apart ? 16 : 16 * kPgWaves;
        QueryFrag<T, D> f;
        Column x;
        column(cbegin + m, f, x);
        u32x4 k[4][KC];
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int s = 0; s < KC; ++s) k[u][s] = kf[u >> 1].wide(u & 1, s);
        const bool some = ~live != 0;
        for (int b0 = cbegin; b0 < cend; b0 += step) {
          const QueryFrag<T, D> now = f;
          const Column at = x;
          if (b0 + step < cend) column(b0 + step + m, f, x);  // the next one's on their way
          f32x4 s[4];
          scores<T, D>(k, now, s);
          const int left = at.last - k0 - 4 * grp;  // the last key that counts, from the lane's first
          if (some || !__all(left >= kWtKeys)) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              const uint32_t mine = static_cast<uint32_t>(live >> (16 * u + 4 * grp));
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (16 * u + e > left || !(mine >> e & 1)) s[u][e] = -INFINITY;
            }
          }
          const float l = at.last < 0 ? 0.0f : at.l;
#pragma unroll
          for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[u][e] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][e], c2, -l));
        }
      }
      put_sums(sum, m, grp, sm.sums[wv]);
      __syncthreads();
      if (wv == 0) {
        const float got[kPgWaves] = {sm.sums[0][lane], sm.sums[1][lane], sm.sums[2][lane], sm.sums[3][lane]};
        if (apart) {
#pragma unroll
          for (int w = 0; w < kPgWaves; ++w) {
            const int first = k00 + w * kWtKeys;
            if (first < min(t1, q1)) add_pages(a, P, base, first, min(first + kWtKeys, t1) - 1, lane, got[w], sm.psum - it.p0);
          }
        } else {
          add_pages(a, P, base, k00, min(k00 + kWtKeys, t1) - 1, lane, (got[0] + got[1]) + (got[2] + got[3]), sm.psum - it.p0);
        }
      }
      __syncthreads();
    }
  }
  __syncthreads();
  float* part = sums_of(a, P, it);
  for (int i = tid; i < it.p1 - it.p0; i += kPgThreads) part[it.p0 + i] = sm.psum[i];
}

// The partial sums of a page into its weight: a lane a page, the waves share the
// units (u, u + 4, ...) and meet in LDS, all in a fixed order.
template <bool kLone>
__global__ __launch_bounds__(kPgThreads) void weight_join(WeightArgs a) {
  __shared__ float sums[kPgWaves][64];
  const int per = (a.max_pages + 63) >> 6;
  const int idx = launch_index(), b = idx / per;
  const int tid = __builtin_amdgcn_workitem_id_x(), lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int pg = (idx - b * per) * 64 + lane;
  if (b >= a.B) return;
  const NewTokens c = new_tokens(a, b);
  if (c.c1 <= c.c0 || pg - lane > (c.c1 - 1) >> a.page_log2) return;
  const int at = min(pg, a.max_pages - 1), entry = a.table[static_cast<int64_t>(b) * a.max_pages + at];
  float s = 0.0f;
  const int rows = kLone ? c.c1 - c.c0 : 1;
  for (int i = 0; i < rows; ++i) {
    const int c0 = c.c0 + i, last = kLone ? c0 : c.c1 - 1;
    const int64_t row = kLone ? c.tok0 + c0 : b;
    for (int pi = 0; pi < a.npat; ++pi) {
      const PagedPattern& P = a.pat[pi];
      const int from = (static_cast<int>(P.fw.div(c0)) * P.w) >> a.page_log2, to = last >> a.page_log2;
      if (pg - lane > to || pg - lane + 63 < from) continue;
      const bool in = pg >= from && pg <= to;
      const int64_t step = static_cast<int64_t>(a.rows) * P.tiles;
      const float* part = a.part + P.one_slot * kWeightAlign + row * P.tiles + (min(max(pg, from), to) - first_sum(from));
      int units = P.one_heads.d;  // those that the row has
      if constexpr (kLone) {
        const int rho = lattice_of(P, c0).rho;
        if (P.r >= a.G) units = min(units, rho < a.H ? static_cast<int>(P.fr.div(a.H - 1 - rho)) + 1 : 0);
      }
      float v = 0.0f;
#pragma unroll 4
      for (int u = wv; u < units; u += kPgWaves) v += part[u * step];
      s += in ? v : 0.0f;
    }
  }
  sums[wv][lane] = s;
  __syncthreads();
  if (wv != 0 || pg > (c.c1 - 1) >> a.page_log2) return;
  if (static_cast<uint32_t>(entry) < static_cast<uint32_t>(a.num_pages))
    a.weights[entry] += (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
}

template <typename T, int D>
void launch_weights_d(const WeightPlan& p, const WeightArgs& a, hipStream_t stream) {
  const dim3 threads(kPgThreads), grid = grid_of(p.items);
  const dim3 join = grid_of(p.B * ((p.max_pages + 63) / 64));
  if (p.lone) {
    hipLaunchKernelGGL((weight_tokens<T, D>), grid, threads, 0, stream, a);
    hipLaunchKernelGGL(weight_join<true>, join, threads, 0, stream, a);
  } else {
    hipLaunchKernelGGL((weight_sequences<T, D>), grid, threads, 0, stream, a);
    hipLaunchKernelGGL(weight_join<false>, join, threads, 0, stream, a);
  }
}

// ---------------------------------------------------------------------------
// Pages that go
// ---------------------------------------------------------------------------
constexpr int64_t kEvSmall = 1024;  // pages that four waves list

struct EvictArgs {
  const float* weights;
  const int32_t *table, *lens;
  int32_t *table_out, *freed, *count;
  int32_t B, num_pages, max_pages, page_log2;
  int64_t keep, first, last;
};

// A weight's place in their order, 1 .. 2^32 - 1: both zeros are equal, NaN is the
// heaviest.  (0 marks a page that stays whatever it weighs.)
__device__ inline uint32_t order_of(float w) {
  uint32_t u = __builtin_bit_cast(uint32_t, w);
  asm("" : "+v"(u));
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
  if (u == 0x80000000u) u = 0;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// grid_of for workgroups of 1024 threads, of which 2^22 are 2^32 work-items.
inline dim3 grid_of_1024(int64_t workgroups) {
  if (workgroups < (int64_t{1} << 22)) return dim3(static_cast<unsigned>(workgroups));
  return dim3(static_cast<unsigned>(kGridRow), static_cast<unsigned>((workgroups + kGridRow - 1) / kGridRow));
}

// A wave has a run of the table's chunks of 64 pages, a lane a page.
template <int kWaves>
__global__ __launch_bounds__(kWaves * 64) void evict(EvictArgs a) {
  constexpr int kKept = kWaves == 4 ? kEvSmall : 16384;  // pages whose keys stay in LDS
  constexpr int kAtOnce = kWaves / 2;                    // chunks whose loads are under way together
  // Digits are counted in kWaves copies, a lane in one of them: most weights share
  // their first digits, and adds to one address come one after another.
  constexpr int kCopy = 260;  // words of a copy: 256, and the copies begin in different banks
  __shared__ __attribute__((aligned(16))) uint32_t keys[kKept];
  __shared__ __attribute__((aligned(16))) uint32_t hist[kWaves * kCopy];
  __shared__ int red[2][kWaves];
  __shared__ int found[2];
  const int tid = __builtin_amdgcn_workitem_id_x(), lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t b = launch_index();
  if (b >= a.B) return;
  const int32_t* table = a.table + b * a.max_pages;
  int32_t* out = a.table_out + b * a.max_pages;
  int32_t* freed = a.freed + b * a.max_pages;
  const int64_t len = max(a.lens[b], 0);
  const int n = static_cast<int>(min((len + (int64_t{1} << a.page_log2) - 1) >> a.page_log2, static_cast<int64_t>(a.max_pages)));
  const int chunks = (a.max_pages + 63) >> 6, per = (chunks + kWaves - 1) / kWaves;
  const int w0 = min(wv * per, chunks) * 64, w1 = min((wv + 1) * per, chunks) * 64;  // the wave's pages
  auto in_pool = [&](int pg, int entry) { return pg < n && static_cast<uint32_t>(entry) < static_cast<uint32_t>(a.num_pages); };
  auto may_go = [&](int pg) { return pg >= a.first && pg < n - a.last; };
  auto key_at = [&](int pg) {
    if (pg >= n) return 0u;
    if (pg < kKept) return keys[pg];
    const int entry = table[pg];
    return in_pool(pg, entry) && may_go(pg) ? order_of(a.weights[entry]) : 0u;
  };
  // The sums of x and y over the waves (of values that a wave's lanes share).
  auto both = [&](int& x, int& y) {
    if (lane == 0) {
      red[0][wv] = x;
      red[1][wv] = y;
    }
    __syncthreads();
    x = y = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      x += red[0][w];
      y += red[1][w];
    }
    __syncthreads();
  };

  int held = 0, may = 0;
  for (int c0 = w0; c0 < min(w1, n); c0 += 64 * kAtOnce) {
    int entry[kAtOnce];
    float w[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) entry[i] = table[min(c0 + 64 * i + lane, a.max_pages - 1)];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int e = in_pool(0, entry[i]) ? entry[i] : 0;
      w[i] = a.weights[e];
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int pg = c0 + 64 * i + lane;
      const bool there = in_pool(pg, entry[i]) && pg < w1, goes = there && may_go(pg);
      if (pg < min(kKept, w1)) keys[pg] = goes ? order_of(w[i]) : 0u;
      held += __popcll(__ballot(there));
      may += __popcll(__ballot(goes));
    }
  }
  both(held, may);
  const int go = static_cast<int>(max(int64_t{0}, min(held - a.keep, static_cast<int64_t>(may))));
  // The go-th lightest weight, digit by digit from the top.
  uint32_t least = 0;
  int rest = go;  // of those that have the digits so far
  for (int shift = 24; shift >= 0 && go > 0; shift -= 8) {
    for (int i = tid; i < kWaves * kCopy; i += kWaves * 64) hist[i] = 0;
    __syncthreads();
    for (int pg = w0 + lane; pg < min(w1, n); pg += 64) {
      const uint32_t k = key_at(pg);
      if (k != 0 && (shift == 24 || k >> (shift + 8) == least >> (shift + 8)))
        atomicAdd(&hist[(lane & (kWaves - 1)) * kCopy + (k >> shift & 255)], 1u);
    }
    __syncthreads();
    if (wv == 0) {  // four digits a lane
      u32x4 h = {0u, 0u, 0u, 0u};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) h += *reinterpret_cast<const u32x4*>(&hist[w * kCopy + 4 * lane]);
      const int s = static_cast<int>(h[0] + h[1] + h[2] + h[3]);
      int before = running_sum(s) - s;
      if (before < rest && before + s >= rest) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (before < rest && before + static_cast<int>(h[i]) >= rest) {
            found[0] = 4 * lane + i;
            found[1] = rest - before;
          }
          before += static_cast<int>(h[i]);
        }
      }
    }
    __syncthreads();
    least |= static_cast<uint32_t>(found[0]) << shift;
    rest = found[1];
  }
  // Lighter ones go, and the first `rest` of those that weigh as much.
  int lighter = 0, equal = 0;  // in the wave's pages
  if (go > 0)
    for (int c0 = w0; c0 < min(w1, n); c0 += 64) {
      const uint32_t k = key_at(c0 + lane);
      lighter += __popcll(__ballot(k != 0 && k < least));
      equal += __popcll(__ballot(k != 0 && k == least));
    }
  if (lane == 0) {
    red[0][wv] = lighter;
    red[1][wv] = equal;
  }
  __syncthreads();
  int place = 0, rank = 0;  // pages that go, and equal ones, before the wave's
  for (int w = 0; w < wv; ++w) {
    place += red[0][w] + max(min(rest - rank, red[1][w]), 0);
    rank += red[1][w];
  }
  const uint64_t below = (uint64_t{1} << lane) - 1;
  for (int c0 = w0; c0 < w1; c0 += 64) {
    const int pg = c0 + lane;
    const uint32_t k = go > 0 ? key_at(pg) : 0u;
    const bool eq = k != 0 && k == least;
    const uint64_t eqs = __ballot(eq);
    const bool goes = k != 0 && (k < least || (eq && rank + __popcll(eqs & below) < rest));
    const uint64_t goers = __ballot(goes);
    if (pg < a.max_pages) {
      const int entry = table[pg];
      out[pg] = goes ? -1 : entry;
      if (goes) freed[place + __popcll(goers & below)] = entry;
    }
    rank += __popcll(eqs);
    place += __popcll(goers);
  }
  for (int i = go + tid; i < a.max_pages; i += kWaves * 64) freed[i] = -1;
  if (tid == 0) a.count[b] = go;
}

}  // namespace

hipError_t launch_page_weights(const WeightPlan& p, const void* q, int64_t q_stride, const float* lse,
                               const PagedCache& cache, float* weights, void* workspace, hipStream_t stream) {
  WeightArgs a{};
  a.q = q;
  a.lse = lse;
  a.kc = static_cast<const char*>(cache.k);
  a.ks = cache.k_scale;
  a.table = cache.table;
  a.lens = cache.lens;
  a.start = cache.start;
  a.part = static_cast<float*>(workspace);
  a.weights = weights;
  a.qs = q_stride;
  a.T = static_cast<int32_t>(p.T);
  a.B = static_cast<int32_t>(p.B);
  a.H = static_cast<int32_t>(p.H);
  a.Hkv = static_cast<int32_t>(p.Hkv);
  a.G = static_cast<int32_t>(p.H / p.Hkv);
  a.npat = p.npat;
  a.num_pages = static_cast<int32_t>(p.num_pages);
  a.max_pages = static_cast<int32_t>(p.max_pages);
  a.page_log2 = p.page_log2;
  a.block_log2 = std::min(p.page_log2, kCacheBlockLog2);
  a.rows = static_cast<int32_t>(p.rows);
  a.items = static_cast<int32_t>(p.items);
  a.reach = static_cast<uint32_t>(p.max_pages * p.page);
  a.scale_log2 = p.scale * kLog2e;
  std::copy(p.pat, p.pat + p.npat, a.pat);
  for (int i = 0; i < DA_MAX_PATTERNS; ++i) a.begin[i] = i < p.npat ? p.pat[i].one_begin : 0x7fffffff;
  if (p.dtype == DA_BF16) {
    if (p.D == 32) launch_weights_d<u16, 32>(p, a, stream);
    else if (p.D == 64) launch_weights_d<u16, 64>(p, a, stream);
    else launch_weights_d<u16, 128>(p, a, stream);
  } else {
    if (p.D == 32) launch_weights_d<float, 32>(p, a, stream);
    else if (p.D == 64) launch_weights_d<float, 64>(p, a, stream);
    else launch_weights_d<float, 128>(p, a, stream);
  }
  return hipGetLastError();
}

hipError_t launch_evict(const EvictCall& c, hipStream_t stream) {
  EvictArgs a{c.weights, c.table, c.lens, c.table_out, c.freed, c.count, static_cast<int32_t>(c.B),
              static_cast<int32_t>(c.num_pages), static_cast<int32_t>(c.max_pages), 0, c.keep, c.first, c.last};
  while ((int64_t{1} << a.page_log2) < c.page_size) ++a.page_log2;
  // A table of 512 pages takes 6.7 us with four waves and 8.2 with sixteen, one of 1024
  // 9.0 and 10.6, one of 2048 13.5 and 12.3 (64 sequences; one takes about as long).
  if (c.max_pages <= kEvSmall)
    hipLaunchKernelGGL(evict<4>, grid_of(c.B), dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL(evict<16>, grid_of_1024(c.B), dim3(1024), 0, stream, a);
  return hipGetLastError();
}

}  // namespace da
