// Which pages of an 8-bit cache the attention looks at, and which of them go.
//
// page_weights: for each page the sum, over the call's new tokens, their heads,
// the patterns that hold a pair and the page's keys, of the pair's share of its
// row's softmax, exp(scale q.k - lse) with the row's log-sum-exp from the attention.
// A workgroup is one unit of a pattern (a key head with the query heads that share
// a dilation offset: their keys are the same lattice g w + rho + t r) and one split
// of the pages that the keys lie in.  Its waves take 32-key tiles in turn, which
// stay in registers as operands of v_mfma_f32_16x16x32_bf16 while columns of 16
// (token, head) pairs pass by in LDS; a key's sum over them stays in LDS.  Then a
// thread adds the keys of a page, in order, and a second launch adds the
// partial sums of a page in the order of the units: no atomics, the same bits
// every time.  float32 queries are three bf16 terms each, whose products with an
// e4m3 key are exact.  All sums are float32.
//
// evict_pages: a workgroup per sequence finds the weight up to which pages go by
// counting digits of eight bits, then lists them in the order of the table.
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
  float* part;     // [units][rows][max_pages]
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

constexpr int kWtTile = 32;    // keys of a wave's tile
constexpr int kWtRows = 1024;  // keys whose rows are looked up at once

template <typename T, int D, bool kLone>
__global__ __launch_bounds__(kPgThreads) void weight_parts(WeightArgs a) {
  constexpr int KC = D / 32, kTerms = sizeof(T) == 2 ? 1 : 3;
  constexpr int kGroups = kTerms == 1 ? 4 : 2, kCols = 16 * kGroups;  // columns in LDS at a time
  __shared__ u32x4 sq[kGroups][KC][kTerms][64];
  __shared__ float slse[kCols];  // a column's lse in log2 units
  __shared__ int slast[kCols];   // its last key, -1: none
  __shared__ uint32_t row[kWtRows];
  __shared__ uint64_t gone[kWtRows / 64];
  __shared__ __attribute__((aligned(16))) float sums[kWtRows];
  __shared__ float psum[kWeightPages];
  const int tid = thread_id(), lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int idx = launch_index();
  if (idx >= a.items) return;
  const int pi = pattern_at(a.begin, idx);
  const PagedPattern& P = a.pat[pi];
  // Unit number n runs with all its splits on XCD n mod 8.
  const int j = (idx - P.one_begin) >> 3, block8 = P.one_split.div(j);
  const int split = j - block8 * P.one_split.d, n = block8 * 8 + ((idx - P.one_begin) & 7);
  const int r0 = P.one_heads.div(n), u = n - r0 * P.one_heads.d;
  if (r0 >= a.rows) return;
  int b;
  const NewTokens c = row_tokens<kLone>(a, r0, lane, b);
  Unit un;
  if (c.c1 <= c.c0 || !unit_of<kLone>(a, P, c.c0, u, un)) return;
  const int rho = un.rho, nh = un.heads.count;
  // this split's pages, of those from the first token's segment on
  const int seg0 = static_cast<int>(P.fw.div(c.c0)) * P.w;
  const int pg0 = seg0 >> a.page_log2, pages = ((c.c1 - 1) >> a.page_log2) + 1 - pg0;
  const int per = P.one_split.div(pages + P.one_split.d - 1);
  const int p0 = pg0 + split * per, p1 = min(p0 + min(per, static_cast<int>(kWeightPages)), pg0 + pages);
  if (p0 >= p1) return;
  for (int i = tid; i < p1 - p0; i += kPgThreads) psum[i] = 0.0f;

  const int m = lane & 15, grp = lane >> 4;
  const int32_t* table = a.table + static_cast<int64_t>(b) * a.max_pages;
  const float c2 = a.scale_log2;
  const int x0 = max(p0 << a.page_log2, seg0);
  const int x1 = static_cast<int>(min(static_cast<int64_t>(p1) << a.page_log2, static_cast<int64_t>(c.c1)));
  for (int g = P.fw.div(x0); g <= static_cast<int>(P.fw.div(x1 - 1)); ++g) {
    const int gs = g * P.w;
    auto first_at = [&](int x) { return x > rho ? static_cast<int>(P.fr.div(x - rho - 1)) + 1 : 0; };
    const int t0 = first_at(x0 - gs), t1 = first_at(min(x1 - gs, P.w));  // keys
    const int q0 = max(first_at(c.c0 - gs), t0), q1 = first_at(min(c.c1 - gs, P.w));  // queries that see some
    if (t0 >= t1 || q0 >= q1) continue;
    for (int k0 = t0; k0 < t1; k0 += kWtRows) {
      const int ke = min(t1, k0 + kWtRows), ntile = (ke - k0 + kWtTile - 1) / kWtTile;
      const int qa = max(q0, k0), cols = (q1 - qa) * nh;  // the chunk's columns, token by token
      if (cols <= 0) break;
      __syncthreads();  // the chunk before is done with LDS
      look_up_rows<4, true>(a, table, un.hk, gs + rho, P.r, k0, ke - 1, ntile * kWtTile, tid, row, gone);
      for (int i = tid; i < ntile * kWtTile; i += kPgThreads) sums[i] = 0.0f;
      for (int col0 = 0; col0 < cols; col0 += kCols) {
        if (col0 > 0) __syncthreads();  // the columns before are done with
        for (int x = wv; x < kGroups * KC; x += kPgWaves) {
          const int gq = x / KC, step = x - gq * KC, col = col0 + 16 * gq + m;
          u32x4 t[kTerms];
#pragma unroll
          for (int i = 0; i < kTerms; ++i) t[i] = u32x4{0u, 0u, 0u, 0u};
          if (col < cols) {
            const int token = col / nh, pos = gs + rho + (qa + token) * P.r;
            const int head = un.heads.first + (col - token * nh) * P.r;
            split_terms(static_cast<const T*>(a.q) + (c.tok0 + pos) * a.qs + head * D + step_first<D>(step, grp), t);
          }
#pragma unroll
          for (int i = 0; i < kTerms; ++i) sq[gq][step][i][lane] = t[i];
        }
        if (tid < kCols) {
          const int col = col0 + tid;
          float x = 0.0f;
          int last = -1;
          if (col < cols) {
            const int token = col / nh, head = un.heads.first + (col - token * nh) * P.r;
            last = qa + token;
            x = a.lse[static_cast<int64_t>(head) * a.T + c.tok0 + gs + rho + last * P.r];
            uint32_t bits = __builtin_bit_cast(uint32_t, x);
            asm("" : "+v"(bits));
            if ((bits & 0x7fffffffu) >= 0x7f800000u) last = -1;  // a row that sees nothing, or NaN: adds nothing
          }
          slse[tid] = x * kLog2e;
          slast[tid] = last;
        }
        __syncthreads();
        const int groups = min(kGroups, (cols - col0 + 15) >> 4);
        const int tmax = qa + (min(cols, col0 + kCols) - 1) / nh;  // the last key that a column here sees
        KeyFrag8<D> next;
        if (wv < ntile) request_keys8<D>(a, row + wv * kWtTile, m, grp, next);
        for (int tile = wv; tile < ntile; tile += kPgWaves) {
          const int first = k0 + tile * kWtTile;
          if (first > tmax) break;
          u32x4 kf[2][KC];
#pragma unroll
          for (int u2 = 0; u2 < 2; ++u2)
#pragma unroll
            for (int s = 0; s < KC; ++s) kf[u2][s] = next.wide(u2, s);
          if (tile + kPgWaves < ntile) request_keys8<D>(a, row + (tile + kPgWaves) * kWtTile, m, grp, next);
          const uint32_t no_page = uniform(static_cast<uint32_t>(gone[tile >> 1] >> ((tile & 1) * 32)));
          const uint32_t live = ~no_page >> (4 * grp);
          f32x4 sum[2] = {f32x4{0, 0, 0, 0}, f32x4{0, 0, 0, 0}};
          for (int gq = 0; gq < groups; ++gq) {
            f32x4 s[2] = {f32x4{0, 0, 0, 0}, f32x4{0, 0, 0, 0}};
#pragma unroll
            for (int i = kTerms - 1; i >= 0; --i)
#pragma unroll
              for (int x = 0; x < KC; ++x)
#pragma unroll
                for (int u2 = 0; u2 < 2; ++u2)
                  s[u2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[u2][x]),
                                                                  __builtin_bit_cast(bf16x8, sq[gq][x][i][lane]), s[u2], 0, 0, 0);
            const float neg = -slse[16 * gq + m];
            const int left = min(slast[16 * gq + m], ke - 1) - first - 4 * grp;  // the last key that counts, from the lane's first
#pragma unroll
            for (int u2 = 0; u2 < 2; ++u2)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u2][e], c2, neg));
                sum[u2][e] += 16 * u2 + e <= left && (live >> (16 * u2 + e) & 1) ? p : 0.0f;
              }
          }
#pragma unroll
          for (int u2 = 0; u2 < 2; ++u2) {
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[u2][e] = row_sum<16>(sum[u2][e]);
            if (m == 0) {
              f32x4* at = reinterpret_cast<f32x4*>(&sums[tile * kWtTile + 16 * u2 + 4 * grp]);
              *at += sum[u2];
            }
          }
        }
      }
      __syncthreads();
      // the chunk's pages, a thread each
      const int pa = (gs + rho + k0 * P.r) >> a.page_log2, pe = (gs + rho + (ke - 1) * P.r) >> a.page_log2;
      for (int pg = pa + tid; pg <= pe; pg += kPgThreads) {
        const int from = max(first_at((pg << a.page_log2) - gs), k0);
        const int to = min(first_at(static_cast<int>(min((static_cast<int64_t>(pg) + 1) << a.page_log2, int64_t{0x7fffffff})) - gs), ke);
        float s = 0.0f;
        for (int t = from; t < to; ++t) s += sums[t - k0];
        psum[pg - p0] += s;
      }
    }
  }
  __syncthreads();
  float* part = a.part + (static_cast<int64_t>(P.one_slot + u) * a.rows + r0) * a.max_pages;
  for (int i = tid; i < p1 - p0; i += kPgThreads) part[p0 + i] = psum[i];
}

// The partial sums of a page into its weight, a thread a page of a sequence.
template <bool kLone>
__global__ __launch_bounds__(kPgThreads) void weight_join(WeightArgs a) {
  const int per = (a.max_pages + kPgThreads - 1) / kPgThreads;
  const int idx = launch_index(), b = idx / per;
  const int pg = (idx - b * per) * kPgThreads + static_cast<int>(__builtin_amdgcn_workitem_id_x());
  if (b >= a.B || pg >= a.max_pages) return;
  const NewTokens c = new_tokens(a, b);
  if (c.c1 <= c.c0 || pg > (c.c1 - 1) >> a.page_log2) return;
  const int entry = a.table[static_cast<int64_t>(b) * a.max_pages + pg];
  if (static_cast<uint32_t>(entry) >= static_cast<uint32_t>(a.num_pages)) return;
  float s = 0.0f;
  const int rows = kLone ? c.c1 - c.c0 : 1;
  for (int i = 0; i < rows; ++i) {
    const int c0 = c.c0 + i, last = kLone ? c0 : c.c1 - 1;
    const int64_t r0 = kLone ? c.tok0 + c0 : b;
    for (int pi = 0; pi < a.npat; ++pi) {
      const PagedPattern& P = a.pat[pi];
      if (pg < (static_cast<int>(P.fw.div(c0)) * P.w) >> a.page_log2 || pg > last >> a.page_log2) continue;
      const float* part = a.part + (static_cast<int64_t>(P.one_slot) * a.rows + r0) * a.max_pages + pg;
      const int units = P.one_heads.d;
      for (int u = 0; u < units; ++u) {
        Unit un;
        if (unit_of<kLone>(a, P, c0, u, un)) s += part[static_cast<int64_t>(u) * a.rows * a.max_pages];
      }
    }
  }
  a.weights[entry] += s;
}

template <typename T, int D>
void launch_weights_d(const WeightPlan& p, const WeightArgs& a, hipStream_t stream) {
  const dim3 threads(kPgThreads), grid = grid_of(p.items);
  const dim3 join = grid_of(p.B * ((p.max_pages + kPgThreads - 1) / kPgThreads));
  if (p.lone) {
    hipLaunchKernelGGL((weight_parts<T, D, true>), grid, threads, 0, stream, a);
    hipLaunchKernelGGL(weight_join<true>, join, threads, 0, stream, a);
  } else {
    hipLaunchKernelGGL((weight_parts<T, D, false>), grid, threads, 0, stream, a);
    hipLaunchKernelGGL(weight_join<false>, join, threads, 0, stream, a);
  }
}

// ---------------------------------------------------------------------------
// Pages that go
// ---------------------------------------------------------------------------
constexpr int kEvThreads = 1024;
constexpr int kEvWaves = kEvThreads / 64;
constexpr int kEvKept = 16384;  // pages whose keys stay in LDS

struct EvictArgs {
  const float* weights;
  const int32_t *table, *lens;
  int32_t *table_out, *freed, *count;
  int32_t num_pages, max_pages, page_log2;
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

__device__ inline int block_sum(int v, int tid, int (&red)[kEvWaves]) {
  const int s = __builtin_amdgcn_readlane(running_sum(v), 63);
  __syncthreads();
  if ((tid & 63) == 0) red[tid >> 6] = s;
  __syncthreads();
  int t = 0;
#pragma unroll
  for (int w = 0; w < kEvWaves; ++w) t += red[w];
  return t;
}

__global__ __launch_bounds__(kEvThreads) void evict(EvictArgs a) {
  __shared__ uint32_t keys[kEvKept];
  __shared__ int hist[256];
  __shared__ int red[kEvWaves], red2[kEvWaves];
  __shared__ int found[2];
  const int tid = __builtin_amdgcn_workitem_id_x(), lane = tid & 63, wv = tid >> 6;
  const int64_t b = launch_index();
  const int32_t* table = a.table + b * a.max_pages;
  int32_t* out = a.table_out + b * a.max_pages;
  int32_t* freed = a.freed + b * a.max_pages;
  const int64_t len = max(a.lens[b], 0);
  const int n = static_cast<int>(min((len + (int64_t{1} << a.page_log2) - 1) >> a.page_log2, static_cast<int64_t>(a.max_pages)));
  auto key_of = [&](int pg, int& there) {
    const int entry = table[pg];
    there = pg < n && static_cast<uint32_t>(entry) < static_cast<uint32_t>(a.num_pages);
    return there && pg >= a.first && pg < n - a.last ? order_of(a.weights[entry]) : 0u;
  };
  auto key_at = [&](int pg) {
    int there;
    return pg < kEvKept ? keys[pg] : key_of(pg, there);
  };
  int held = 0, may = 0;
  for (int pg = tid; pg < n; pg += kEvThreads) {
    int there;
    const uint32_t k = key_of(pg, there);
    if (pg < kEvKept) keys[pg] = k;
    held += there;
    may += k != 0;
  }
  held = block_sum(held, tid, red);
  may = block_sum(may, tid, red2);
  const int go = static_cast<int>(max(int64_t{0}, min(held - a.keep, static_cast<int64_t>(may))));
  // The go-th lightest weight, digit by digit from the top.
  uint32_t least = 0;
  int rest = go;  // of those that have the digits so far
  for (int shift = 24; shift >= 0 && go > 0; shift -= 8) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    for (int pg = tid; pg < n; pg += kEvThreads) {
      const uint32_t k = key_at(pg);
      if (k != 0 && (shift == 24 || k >> (shift + 8) == least >> (shift + 8))) atomicAdd(&hist[k >> shift & 255], 1);
    }
    __syncthreads();
    if (wv == 0) {  // four digits a lane
      int h[4], s = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) s += h[i] = hist[4 * lane + i];
      int before = running_sum(s) - s;
      if (before < rest && before + s >= rest) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (before < rest && before + h[i] >= rest) {
            found[0] = 4 * lane + i;
            found[1] = rest - before;
          }
          before += h[i];
        }
      }
    }
    __syncthreads();
    least |= static_cast<uint32_t>(found[0]) << shift;
    rest = found[1];
  }
  // Lighter ones go, and the first `rest` of those that weigh as much.
  int equal = 0, gone = 0;  // in the chunks before
  for (int c0 = 0; c0 < a.max_pages; c0 += kEvThreads) {
    const int pg = c0 + tid;
    const uint32_t k = go > 0 && pg < n ? key_at(pg) : 0u;
    const bool eq = k != 0 && k == least;
    const uint64_t before = (uint64_t{1} << lane) - 1, eqs = __ballot(eq);
    __syncthreads();
    if (lane == 0) red[wv] = __popcll(eqs);
    __syncthreads();
    int rank = equal + __popcll(eqs & before), all = 0;
#pragma unroll
    for (int w = 0; w < kEvWaves; ++w) {
      if (w < wv) rank += red[w];
      all += red[w];
    }
    equal += all;
    const bool goes = k != 0 && (k < least || (eq && rank < rest));
    const uint64_t goers = __ballot(goes);
    if (lane == 0) red2[wv] = __popcll(goers);
    __syncthreads();
    int place = gone + __popcll(goers & before);
    all = 0;
#pragma unroll
    for (int w = 0; w < kEvWaves; ++w) {
      if (w < wv) place += red2[w];
      all += red2[w];
    }
    gone += all;
    if (pg < a.max_pages) {
      const int entry = table[pg];
      out[pg] = goes ? -1 : entry;
      if (goes) freed[place] = entry;
    }
  }
  for (int i = gone + tid; i < a.max_pages; i += kEvThreads) freed[i] = -1;
  if (tid == 0) a.count[b] = gone;
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
  EvictArgs a{c.weights, c.table, c.lens, c.table_out, c.freed, c.count, static_cast<int32_t>(c.num_pages),
              static_cast<int32_t>(c.max_pages), 0, c.keep, c.first, c.last};
  while ((int64_t{1} << a.page_log2) < c.page_size) ++a.page_log2;
  hipLaunchKernelGGL(evict, grid_of(c.B), dim3(kEvThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace da
