// Dilated attention of each sequence's new tokens over its paged cache (the
// cache holds the new tokens already).  A query at position p of head h takes
// part in pattern (w, r) if (p mod w) mod r == h mod r and then sees the kept
// keys of its segment up to p; its output is one softmax over the keys of all
// patterns, a key counting once for each pattern that holds it (Sec. 2.2,
// Eqs. 3-10 of the paper, causal, in absolute positions).
//
// The lattice of a query is anchored at its own position: the keys of (w, r)
// are g w + rho + t r with rho = (p - g w) mod r and t = 0 .. (p - g w) / r, the
// same rows for every head of residue rho.  Everything is decoded on the
// device from the lengths, so that a launch needs no plan of the lengths on the
// host and can be captured in a graph.
//
// single_tokens: a workgroup is one (token, key head, pattern, split of its keys),
// for sequences with few new tokens.  Bound by HBM and, for few sequences, by
// latency: the keys are split over workgroups, and in one over its four waves,
// which take 32-key tiles in turn without a barrier.  K goes from the cache to
// registers in the operand layout of v_mfma_f32_16x16x32_bf16 (16 keys by up to
// 16 query heads), V to the wave's own LDS buffer, read transposed.
// query_tiles: a workgroup is 128 kept query rows of one (sequence, head,
// segment) of a pattern against 64-key tiles in LDS.  Bound by the matrix cores
// and the softmax's vector work.
// Both write normalised partial rows with their log-sum-exps; paged_join mixes
// a row's partials.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device_common.h"

namespace da {
namespace {

constexpr int kPgThreads = 256;
constexpr int kPgWaves = kPgThreads / 64;
constexpr float kLowest = -1.0e30f;  // finite "minus infinity" of a running maximum
constexpr float kSlack = 8.0f;       // a score this far above its row's reference (log2) moves it

struct PagedArgs {
  const void* q;
  const char *kc, *vc;
  const int32_t *table, *lens, *start;
  char* ws;
  void* out;
  float* lse;
  int64_t qs;  // elements between tokens of q
  int64_t one_rec, one_row, tile_rec, tile_row;  // byte offsets in the workspace
  int32_t T, B, H, Hkv, G, npat, num_pages, max_pages, page_log2;
  int32_t by_token, few, units, one_slots, tile_items;
  uint32_t reach;  // positions the table holds
  FastDiv fslots, funits;  // division by one_slots and by a token's units
  float scale_log2;
  PagedPattern pat[DA_MAX_PATTERNS];
};

// A sequence's new tokens: rows begin .. end - 1 of the call, the last of its
// length len.
struct Sequence {
  int b;  // -1: the token has none
  int begin, end, len;
};
// The sequences of kTokens tokens (the same in all lanes), by all lanes of a
// wave: start [B + 1] ascends and the last entry that is not above a token is
// its sequence's (empty ones before it share that value).  Whatever start
// holds, the result is below B.  Up to 63 sequences all entries arrive in one
// round of loads.
template <int kTokens>
__device__ inline void find_sequences(const PagedArgs& a, const int (&tok)[kTokens], int lane, Sequence (&sq)[kTokens]) {
  int n[kTokens];
#pragma unroll
  for (int i = 0; i < kTokens; ++i) n[i] = 0;
  int start = 0, len = 0;
  for (int b0 = 0; b0 <= a.B; b0 += 64) {
    const int b = b0 + lane;
    start = a.start[min(b, a.B)];
    len = a.lens[min(b, a.B - 1)];
#pragma unroll
    for (int i = 0; i < kTokens; ++i) n[i] += __popcll(__ballot(b <= a.B && start <= tok[i]));
  }
#pragma unroll
  for (int i = 0; i < kTokens; ++i) {
    const int b = n[i] > a.B ? -1 : n[i] - 1;
    sq[i] = Sequence{b, 0, 0, 0};
    if (b < 0) continue;
    if (a.B < 64) {
      sq[i].begin = __builtin_amdgcn_readlane(start, b);
      sq[i].end = __builtin_amdgcn_readlane(start, b + 1);
      sq[i].len = __builtin_amdgcn_readlane(len, b);
    } else {
      sq[i].begin = a.start[b];
      sq[i].end = a.start[b + 1];
      sq[i].len = a.lens[b];
    }
  }
}

// Position of row tok of its sequence; -1 where it has none in the table.
__device__ inline int position_of(const PagedArgs& a, const Sequence& sq, int tok) {
  const int64_t p = static_cast<int64_t>(sq.len) - sq.end + tok;
  return sq.b >= 0 && tok < sq.end && p >= 0 && p < a.reach ? static_cast<int>(p) : -1;
}

// A listed token: its row of q, its sequence and position.  False: not there,
// not in the cache, or computed in tiles.
struct Token {
  int tok, b, pos;
};
__device__ inline bool single_token(const PagedArgs& a, int e, int lane, Token& t) {
  Sequence sq[1];
  if (a.by_token) {
    const int tok[1] = {e};
    t.tok = e;
    find_sequences(a, tok, lane, sq);
  } else {
    const int b = e / a.few;
    sq[0] = Sequence{b, a.start[b], a.start[b + 1], a.lens[b]};
    t.tok = sq[0].begin + (e - b * a.few);
  }
  t.b = sq[0].b;
  t.pos = position_of(a, sq[0], t.tok);
  return t.pos >= 0 && t.tok >= 0 && t.tok < a.T && static_cast<int64_t>(sq[0].end) - sq[0].begin <= a.few;
}

// The heads of key head hk's group that pattern P keeps at segment-local
// offset rho: first, first + r, ... below (hk + 1) G; none: count = 0.
struct KeptHeads {
  int first, count;
};
__device__ inline KeptHeads kept_heads(const PagedPattern& P, int hk, int G, int rho) {
  const int h0 = hk * G;
  int x = rho - (h0 - static_cast<int>(P.fr.div(h0)) * P.r);
  if (x < 0) x += P.r;
  if (x >= G) return {0, 0};
  return {h0 + x, static_cast<int>(P.fr.div(G - 1 - x)) + 1};
}

// Row of key head hk in the cache for position pos of sequence b.  A page
// outside the pool reads the pool's last page: in bounds, whatever the table holds.
__device__ inline uint32_t cache_row(const PagedArgs& a, const int32_t* table, int hk, int pos) {
  const uint32_t page = min(static_cast<uint32_t>(table[pos >> a.page_log2]), static_cast<uint32_t>(a.num_pages - 1));
  return ((page * a.Hkv + hk) << a.page_log2) + (pos & ((1 << a.page_log2) - 1));
}

// Keys of split s of n keys: [first, end), whole 32-key tiles but the last.
__device__ inline int split_keys_of(const PagedPattern& P, int n) {
  return (static_cast<int>(P.one_split.div(n + P.one_split.d - 1)) + 31) & ~31;
}

__device__ inline float max_over_groups(float v) {  // over lanes 16 apart
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ inline float sum_over_groups(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

template <int N>
__device__ inline void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"i"(N) : "memory");
}

// A workgroup's place among the single tokens' items: unit u = (token, key
// head, block of 16 of its query heads) on XCD u mod 8 with all its slots.
struct OneItem {
  int e, slot, hk, block;
};
__device__ inline bool one_item(const PagedArgs& a, int idx, OneItem& it, int heads) {
  const int k = idx >> 3;
  const int j = a.fslots.div(k);
  const int unit = j * 8 + (idx & 7);
  if (unit >= a.units) return false;
  it.slot = k - j * a.one_slots;
  it.e = a.funits.div(unit);
  const int rest = unit - it.e * a.funits.d;
  it.block = rest / heads;
  it.hk = rest - it.block * heads;
  return true;
}

// A wave's K operand of a 32-key tile: two blocks of 16 keys.
template <int KC>
struct KeyFrag {
  u32x4 v[2][KC];
};

constexpr int kOneTile = 32;  // keys of a wave's tile
template <int D>
struct SmemOne {
  __attribute__((aligned(16))) char v[kPgWaves][2 * kOneTile * D * 2];  // each wave's two V tiles
  float ml[kPgWaves][2][16];
};

template <int D>
__device__ inline void single_tokens(const PagedArgs& a, int idx, SmemOne<D>& sm) {
  constexpr int KC = D / 32, DB = D / 16, kTile = kOneTile;
  using TL = TileLayout<D>;
  constexpr int kVLoads = kTile * TL::kSlots / 64;
  constexpr int kBuf = kTile * D * 2;  // bytes of a V tile
  constexpr int kJoin = D + 4;         // floats between joined rows
  static_assert(16 * kJoin * 4 <= 2 * kBuf, "the join fits a wave's V buffers");
  auto& sv = sm.v;
  auto& sml = sm.ml;

  const int tid = __builtin_amdgcn_workitem_id_x(), lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  OneItem it;
  if (!one_item(a, idx, it, a.Hkv)) return;
  int pi = 0;
  for (int i = 1; i < a.npat; ++i)
    if (it.slot >= a.pat[i].one_slot) pi = i;
  const PagedPattern& P = a.pat[pi];
  Token tk;
  if (!single_token(a, it.e, lane, tk)) return;
  const int g = P.fw.div(tk.pos), loc = tk.pos - g * P.w;
  const int tq = P.fr.div(loc), rho = loc - tq * P.r;
  KeptHeads kh = kept_heads(P, it.hk, a.G, rho);
  const int m0 = it.block * static_cast<int>(kPagedGroupRows);
  if (m0 >= kh.count) return;
  const int rows = min(static_cast<int>(kPagedGroupRows), kh.count - m0);
  const int n = tq + 1, per = split_keys_of(P, n), sp = it.slot - P.one_slot;
  const int k0 = sp * per;
  if (k0 >= n) return;
  const int ke = min(k0 + per, n), ntile = (ke - k0 + kTile - 1) / kTile;

  const int m = lane & 15, grp = lane >> 4;
  const int head = kh.first + (m0 + min(m, rows - 1)) * P.r;
  bf16x8 qf[KC];
#pragma unroll
  for (int c = 0; c < KC; ++c) {
    const u32x4 x = load16(static_cast<const u16*>(a.q) + tk.tok * a.qs + head * D + 32 * c + 8 * grp);
    qf[c] = __builtin_bit_cast(bf16x8, m < rows ? x : u32x4{0u, 0u, 0u, 0u});
  }

  const int32_t* table = a.table + static_cast<int64_t>(tk.b) * a.max_pages;
  const int base = g * P.w + rho;
  // Lanes l and l + 32 look up key l of a tile; keys past the split's end are its last.
  auto look_up = [&](int tile) {
    const int t = min(k0 + tile * kTile + (lane & 31), ke - 1);
    return cache_row(a, table, it.hk, base + t * P.r);
  };
  int vrow[kVLoads], vslot[kVLoads];
#pragma unroll
  for (int i = 0; i < kVLoads; ++i) {
    const int s = 64 * i + lane;
    vrow[i] = s / TL::kSlots;
    vslot[i] = (s % TL::kSlots) ^ TL::swz(vrow[i]);
  }
  char* my = sv[wv];
  auto load_v = [&](uint32_t row, int buf) {
#pragma unroll
    for (int i = 0; i < kVLoads; ++i) {
      const uint32_t rv = __shfl(row, vrow[i], 64);
      const int64_t at = static_cast<int64_t>(rv) * TL::kRowBytes + vslot[i] * 16;
      __builtin_amdgcn_global_load_lds(a.vc + at, (lds_void*)(my + buf * kBuf + 1024 * i), 16, 0, 0);
    }
  };
  auto load_k = [&](uint32_t row, KeyFrag<KC>& kf) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint32_t rk = __shfl(row, 16 * u + m, 64);
      const char* p = a.kc + (static_cast<int64_t>(rk) * TL::kRowBytes + 16 * grp);
#pragma unroll
      for (int c = 0; c < KC; ++c) kf.v[u][c] = *reinterpret_cast<const u32x4*>(p + 64 * c);
    }
  };
  // V^T operand: lane's d = 16 db + (lane & 15), keys 4 grp + 0..3 and 16 more.
  const int tr_r = (lane & 15) >> 2;
  int voff[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    const int d = 16 * db + (lane & 3) * 4;
    voff[db] = TL::offset(4 * grp + tr_r, d >> 3) + (d & 7) * 2;
  }

  f32x4 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = f32x4{0, 0, 0, 0};
  float m_run = kLowest, l_run = 0.0f;
  const float c2 = a.scale_log2;

  auto compute = [&](int tile, int buf, const KeyFrag<KC>& kf) {
    f32x4 s[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      s[u] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int c = 0; c < KC; ++c)
        s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf.v[u][c]), qf[c], s[u], 0, 0, 0);
    }
    const int left = ke - k0 - tile * kTile - 4 * grp;  // keys from this lane's first on
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (16 * u + e >= left) s[u][e] = -INFINITY;
    float mx = s[0][0];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[u][e]);
    mx *= c2;
    if (__any(mx > m_run + kSlack)) {
      const float m_new = fmaxf(m_run, max_over_groups(mx));
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db) acc[db] *= alpha;
    }
    bf16x8 pb;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][e], c2, -m_run));
        l_run += p;
        pb[4 * u + e] = (__bf16)p;
      }
    const uint32_t va = lds_addr(my) + buf * kBuf;
    u32x2 vf[DB][2];
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      vf[db][0] = lds_read_tr16<0>(va + voff[db]);
      vf[db][1] = lds_read_tr16<16 * TL::kRowBytes>(va + voff[db]);
    }
    lds_wait<0>();
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      lds_bind(vf[db][0]);
      lds_bind(vf[db][1]);
      const u32x4 v4 = {vf[db][0][0], vf[db][0][1], vf[db][1][0], vf[db][1][1]};
      acc[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v4), pb, acc[db], 0, 0, 0);
    }
  };

  if (wv < ntile) {
    uint32_t row = look_up(wv);
    KeyFrag<KC> ka, kb;
    load_v(row, 0);
    load_k(row, ka);
    row = look_up(wv + kPgWaves);  // clamped to the split's last key
    asm volatile("" ::: "memory");  // the counted waits below rely on this order
    __builtin_amdgcn_sched_barrier(0);
    // While a tile is computed the next one's loads are under way: all but
    // those have to have landed (the look-up is the youngest and is waited for
    // by its use).
    auto step = [&](int tile, int buf, const KeyFrag<KC>& cur, KeyFrag<KC>& nxt) {
      if (tile + kPgWaves < ntile) {
        load_v(row, buf ^ 1);
        load_k(row, nxt);
        row = look_up(tile + 2 * kPgWaves);
        wait_loads<kVLoads + 2 * KC + 1>();
      } else {
        wait_loads<0>();
      }
      __builtin_amdgcn_sched_barrier(0);
      compute(tile, buf, cur);
    };
    for (int tile = wv;; tile += 2 * kPgWaves) {
      step(tile, 0, ka, kb);
      if (tile + kPgWaves >= ntile) break;
      step(tile + kPgWaves, 1, kb, ka);
      if (tile + 2 * kPgWaves >= ntile) break;
    }
  }

  // The waves' partial rows meet in LDS, each in its wave's own V buffers.
  l_run = sum_over_groups(l_run);
  float* jo = reinterpret_cast<float*>(my);
#pragma unroll
  for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4*>(jo + m * kJoin + 16 * db + 4 * grp) = acc[db];
  if (grp == 0) {
    sml[wv][0][m] = m_run;
    sml[wv][1][m] = l_run;
  }
  __syncthreads();
  const int64_t row0 = static_cast<int64_t>(it.e) * a.H;
  for (int x = tid; x < rows * (D / 4); x += kPgThreads) {
    const int r = x / (D / 4), d = (x % (D / 4)) * 4;
    float mt = sml[0][0][r];
#pragma unroll
    for (int w = 1; w < kPgWaves; ++w) mt = fmaxf(mt, sml[w][0][r]);
    float l = 0.0f;
    f32x4 o = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < kPgWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(sml[w][0][r] - mt);
      l += f * sml[w][1][r];
      o += f * *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(sv[w]) + r * kJoin + d);
    }
    const int64_t at = (row0 + kh.first + (m0 + r) * P.r) * a.one_slots + it.slot;
    o *= l > 0.0f ? 1.0f / l : 0.0f;
    *reinterpret_cast<f32x4*>(a.ws + a.one_row + (at * D + d) * 4) = o;
    if (d == 0) reinterpret_cast<float*>(a.ws + a.one_rec)[at] = mt + __builtin_amdgcn_logf(l);
  }
}

// float32: a workgroup is one (token, query head, pattern, split).  D/4 lanes
// hold a row, each group of them its own keys and running softmax; the groups
// and waves meet in LDS.
template <int D>
__global__ __launch_bounds__(kPgThreads) void paged_one_f32(PagedArgs a) {
  constexpr int kLanes = D / 4, kGroups = kPgThreads / kLanes, kUnroll = 4;
  __shared__ __attribute__((aligned(16))) float so[kGroups][D];
  __shared__ float sml[2][kGroups];
  const int tid = __builtin_amdgcn_workitem_id_x(), lane = tid & 63;
  OneItem it;
  if (!one_item(a, launch_index(), it, a.H)) return;
  int pi = 0;
  for (int i = 1; i < a.npat; ++i)
    if (it.slot >= a.pat[i].one_slot) pi = i;
  const PagedPattern& P = a.pat[pi];
  Token tk;
  if (!single_token(a, it.e, lane, tk)) return;
  const int head = it.hk, hk = head / a.G;
  const int g = P.fw.div(tk.pos), loc = tk.pos - g * P.w;
  const int tq = P.fr.div(loc), rho = loc - tq * P.r;
  if (head - static_cast<int>(P.fr.div(head)) * P.r != rho) return;
  const int n = tq + 1, per = split_keys_of(P, n), k0 = (it.slot - P.one_slot) * per;
  if (k0 >= n) return;
  const int ke = min(k0 + per, n);
  const int grp = tid / kLanes, ch = tid % kLanes;
  const f32x4 q = *reinterpret_cast<const f32x4*>(static_cast<const float*>(a.q) + tk.tok * a.qs + head * D + 4 * ch);
  const int32_t* table = a.table + static_cast<int64_t>(tk.b) * a.max_pages;
  const int base = g * P.w + rho;
  float m_run = kLowest, l_run = 0.0f;
  f32x4 acc = f32x4{0, 0, 0, 0};
  for (int t0 = k0; t0 < ke; t0 += kUnroll * kGroups) {
    f32x4 k[kUnroll], v[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int t = min(t0 + u * kGroups + grp, ke - 1);
      const int64_t at = static_cast<int64_t>(cache_row(a, table, hk, base + t * P.r)) * D + 4 * ch;
      k[u] = *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(a.kc) + at);
      v[u] = *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(a.vc) + at);
    }
    float s[kUnroll], mx = m_run;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      float d = (q[0] * k[u][0] + q[1] * k[u][1]) + (q[2] * k[u][2] + q[3] * k[u][3]);
#pragma unroll
      for (int x = 1; x < kLanes; x <<= 1) d += __shfl_xor(d, x, 64);
      s[u] = t0 + u * kGroups + grp < ke ? d * a.scale_log2 : -INFINITY;
      mx = fmaxf(mx, s[u]);
    }
    const float alpha = __builtin_amdgcn_exp2f(m_run - mx);
    m_run = mx;
    l_run *= alpha;
    acc *= alpha;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const float p = __builtin_amdgcn_exp2f(s[u] - m_run);
      l_run += p;
      acc += p * v[u];
    }
  }
  *reinterpret_cast<f32x4*>(&so[grp][4 * ch]) = acc;
  if (ch == 0) {
    sml[0][grp] = m_run;
    sml[1][grp] = l_run;
  }
  __syncthreads();
  if (tid >= kLanes) return;
  float mt = kLowest;
#pragma unroll
  for (int w = 0; w < kGroups; ++w) mt = fmaxf(mt, sml[0][w]);
  float l = 0.0f;
  f32x4 o = f32x4{0, 0, 0, 0};
#pragma unroll 4
  for (int w = 0; w < kGroups; ++w) {
    const float f = __builtin_amdgcn_exp2f(sml[0][w] - mt);
    l += f * sml[1][w];
    o += f * *reinterpret_cast<const f32x4*>(&so[w][4 * ch]);
  }
  const int64_t at = (static_cast<int64_t>(it.e) * a.H + head) * a.one_slots + it.slot;
  o *= l > 0.0f ? 1.0f / l : 0.0f;
  *reinterpret_cast<f32x4*>(a.ws + a.one_row + (at * D + 4 * ch) * 4) = o;
  if (ch == 0) reinterpret_cast<float*>(a.ws + a.one_rec)[at] = mt + __builtin_amdgcn_logf(l);
}

// ---------------------------------------------------------------------------
// Tiles of query rows
// ---------------------------------------------------------------------------
// Entry i of start, held to the call's tokens: what a tile reads and writes stays in bounds.
__device__ inline int token_row(const PagedArgs& a, int i) { return max(0, min(a.start[i], a.T)); }

// The query tile `tile` of pattern P among all sequences' (for any head: a
// head's offset only moves the rows within a tile).
struct QueryTile {
  int b, g, j;  // sequence, segment, tile of the segment's new rows
  int c0, c1;   // positions of the sequence's new tokens
};
__device__ inline bool query_tile(const PagedArgs& a, const PagedPattern& P, int tile, int lane, QueryTile& qt) {
  constexpr int BM = kPagedRows;
  auto tiles_of = [&](int len) { return static_cast<int>(P.fr.div(len - 1)) / BM + 1; };  // len >= 1
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    const int b = b0 + lane;
    int cnt = 0, c0 = 0, c1 = 0;
    if (b < a.B) {
      const int64_t n = token_row(a, b + 1) - token_row(a, b);
      const int64_t len = a.lens[b];
      c1 = static_cast<int>(max(int64_t{0}, min(len, static_cast<int64_t>(a.reach))));
      c0 = static_cast<int>(max(int64_t{0}, min(len - n, static_cast<int64_t>(c1))));
      if (n > a.few && c1 > c0) {
        const int g0 = P.fw.div(c0), g1 = P.fw.div(c1 - 1);
        cnt = g0 == g1 ? tiles_of(c1 - c0)
                       : tiles_of((g0 + 1) * P.w - c0) + (g1 - g0 - 1) * tiles_of(P.w) + tiles_of(c1 - g1 * P.w);
      }
    }
    int upto = cnt;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const int o = __shfl_up(upto, s, 64);
      if (lane >= s) upto += o;
    }
    const int total = __shfl(upto, 63, 64);
    if (tile < total) {
      const int l = __builtin_ctzll(__ballot(upto > tile));
      qt.b = b0 + l;
      int j = tile - (__shfl(upto, l, 64) - __shfl(cnt, l, 64));
      qt.c0 = __shfl(c0, l, 64);
      qt.c1 = __shfl(c1, l, 64);
      qt.g = P.fw.div(qt.c0);
      const int g1 = P.fw.div(qt.c1 - 1);
      const int first = qt.g == g1 ? 0x7fffffff : tiles_of((qt.g + 1) * P.w - qt.c0);
      if (j >= first) {
        const int per = tiles_of(P.w);
        j -= first;
        const int skip = min(j / per, g1 - qt.g - 1);
        qt.g += 1 + skip;
        j -= skip * per;
      }
      qt.j = j;
      return true;
    }
    tile -= total;
  }
  return false;
}

template <int D>
struct SmemTile {
  __attribute__((aligned(16))) u16 k[2][kPagedKeyTile * D];
  __attribute__((aligned(16))) u16 v[2][kPagedKeyTile * D];
};

template <int D>
__device__ inline void query_tiles(const PagedArgs& a, int idx, SmemTile<D>& sm) {
  constexpr int BM = kPagedRows, BN = kPagedKeyTile;
  constexpr int KC = D / 16, DB = D / 32;
  using TL = TileLayout<D>;
  constexpr int kLoads = BN * TL::kSlots / 64 / kPgWaves;
  const int tid = __builtin_amdgcn_workitem_id_x(), lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  int pi = 0;
  for (int i = 1; i < a.npat; ++i)
    if (idx >= a.pat[i].item_begin) pi = i;
  const PagedPattern& P = a.pat[pi];
  // Heads next to each other, later (longer) tiles first.
  const int local = idx - P.item_begin;
  const int rest = local / a.H, head = local - rest * a.H;
  const int ti = rest / P.tile_splits, sp = rest - ti * P.tile_splits;
  if (ti >= P.tiles) return;
  QueryTile qt;
  if (!query_tile(a, P, P.tiles - 1 - ti, lane, qt)) return;
  qt.b = __builtin_amdgcn_readfirstlane(qt.b);
  qt.g = __builtin_amdgcn_readfirstlane(qt.g);
  qt.j = __builtin_amdgcn_readfirstlane(qt.j);
  const int gs = qt.g * P.w;
  const int off = head - static_cast<int>(P.fr.div(head)) * P.r;
  const int lo = max(__builtin_amdgcn_readfirstlane(qt.c0) - gs, 0);
  const int hi_pos = min(__builtin_amdgcn_readfirstlane(qt.c1) - gs, P.w);
  auto first_at = [&](int x) { return x > off ? static_cast<int>(P.fr.div(x - off - 1)) + 1 : 0; };  // first t at or after x
  const int q0 = first_at(lo) + qt.j * BM;
  const int qend = min(q0 + BM, first_at(hi_pos));
  if (q0 >= qend) return;
  const int hk = head / a.G;
  // this split's keys
  const int per = ((qend + P.tile_splits - 1) / P.tile_splits + BN - 1) / BN * BN;
  const int kb = sp * per, ke = min(kb + per, qend);
  const int slot = P.tile_slot + sp;
  const int base = gs + off;  // position of t = 0
  const int tok0 = token_row(a, qt.b + 1) - a.lens[qt.b];  // token row of position 0

  const int qr = lane & 31, hi = lane >> 5;
  const int wq_lo = q0 + wv * 32, tq = wq_lo + qr;
  const int tq_in = min(tq, qend - 1);
  const int my_tok = tok0 + base + tq_in * P.r;
  f32x2* rec = reinterpret_cast<f32x2*>(a.ws + a.tile_rec) + static_cast<int64_t>(slot) * a.T * a.H + head;
  if (kb >= qend) {  // no keys left for this split
    if (hi == 0 && tq < qend) rec[static_cast<int64_t>(my_tok) * a.H] = f32x2{-INFINITY, 1.0f};
    return;
  }

  u32x4 qraw[KC];
  {
    const u16* qp = static_cast<const u16*>(a.q) + my_tok * a.qs + head * D + 8 * hi;
#pragma unroll
    for (int c = 0; c < KC; ++c) qraw[c] = load16(qp + 16 * c);
  }
  const int32_t* table = a.table + static_cast<int64_t>(qt.b) * a.max_pages;
  int lrow[kLoads], lslot[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int s = 64 * (wv * kLoads + i) + lane;
    lrow[i] = s / TL::kSlots;
    lslot[i] = (s % TL::kSlots) ^ TL::swz(lrow[i]);
  }
  const int ntile = (ke - kb + BN - 1) / BN;
  uint32_t row[kLoads];
  auto look_up = [&](int jt) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) row[i] = cache_row(a, table, hk, base + min(kb + jt * BN + lrow[i], ke - 1) * P.r);
  };
  auto load_tile = [&](int buf) {
    char* kl = reinterpret_cast<char*>(&sm.k[buf][0]);
    char* vl = reinterpret_cast<char*>(&sm.v[buf][0]);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int64_t at = static_cast<int64_t>(row[i]) * TL::kRowBytes + lslot[i] * 16;
      const int lds_off = 1024 * (wv * kLoads + i);
      __builtin_amdgcn_global_load_lds(a.kc + at, (lds_void*)(kl + lds_off), 16, 0, 0);
      __builtin_amdgcn_global_load_lds(a.vc + at, (lds_void*)(vl + lds_off), 16, 0, 0);
    }
  };
  const int tr_r = (lane & 15) >> 2;
  const int tr_d = ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
  int vtr_off[DB][2];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int d = db * 32 + tr_d;
      vtr_off[db][t] = TL::offset(8 * t + 4 * hi + tr_r, d >> 3) + (d & 7) * 2;
    }
  look_up(0);
  load_tile(0);
  look_up(1);  // past the end: the last key again
  bf16x8 qreg[KC];
#pragma unroll
  for (int c = 0; c < KC; ++c) qreg[c] = __builtin_bit_cast(bf16x8, qraw[c]);

  f32x16 acc_o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) acc_o[db] = f32x16{};
  float m_run = kLowest, l_run = 0.0f;
  const float c2 = a.scale_log2;
  wait_loads<0>();
  __syncthreads();
  for (int jt = 0; jt < ntile; ++jt) {
    const int cur = jt & 1, k0 = kb + jt * BN;
    if (jt + 1 < ntile) {
      load_tile(cur ^ 1);
      look_up(jt + 2);
    }
    const char* kl = reinterpret_cast<const char*>(&sm.k[cur][0]);
    const char* vl = reinterpret_cast<const char*>(&sm.v[cur][0]);
    if (k0 <= wq_lo + 31 && wq_lo < qend) {  // not all keys after this wave's queries
      constexpr int QG = D <= 64 ? 2 : 1;
      f32x16 acc_s[2];
#pragma unroll
      for (int kb0 = 0; kb0 < 2; kb0 += QG) {
        u32x4 kf[QG][KC];
#pragma unroll
        for (int x = 0; x < QG; ++x)
#pragma unroll
          for (int c = 0; c < KC; ++c)
            kf[x][c] = *reinterpret_cast<const u32x4*>(kl + TL::offset((kb0 + x) * 32 + qr, 2 * c + hi));
        __builtin_amdgcn_sched_barrier(0);  // keep the reads ahead of the MFMAs
#pragma unroll
        for (int x = 0; x < QG; ++x) {
          acc_s[kb0 + x] = f32x16{};
#pragma unroll
          for (int c = 0; c < KC; ++c)
            acc_s[kb0 + x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[x][c]), qreg[c],
                                                                     acc_s[kb0 + x], 0, 0, 0);
        }
      }
      if (k0 + BN - 1 > wq_lo || k0 + BN > ke) {  // mask keys after the query and past the split
        int first = k0 + 4 * hi - min(tq_in, ke - 1);
        asm volatile("" : "+v"(first));  // compares made here, not hoisted into scalar masks
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (first + x * 32 + 8 * (j >> 2) + (j & 3) > 0) acc_s[x][j] = -INFINITY;
      }
      float mx = acc_s[0][0];
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int j = 0; j < 16; j += 2) mx = fmaxf(mx, fmaxf(acc_s[x][j], acc_s[x][j + 1]));
      mx *= c2;
      if (__any(mx > m_run + kSlack)) {
        const float m_new = fmaxf(m_run, fmaxf(mx, other_half(mx)));
        const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
        m_run = m_new;
        l_run *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int j = 0; j < 16; ++j) acc_o[db][j] *= alpha;
      }
      const float negm = -m_run;
      float lp[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      const uint32_t vaddr = lds_addr(vl);
      static_for<0, 2>([&](auto KB) {
        constexpr int kb2 = decltype(KB)::value;
        u32x2 vf[2][DB][2];
        static_for<0, 2>([&](auto KK) {
          static_for<0, DB>([&](auto DBI) {
            static_for<0, 2>([&](auto T) {
              constexpr int kk = decltype(KK)::value, db = decltype(DBI)::value, t = decltype(T)::value;
              constexpr int r0 = kb2 * 32 + 16 * kk;
              vf[kk][db][t] = lds_read_tr16<r0 * TL::kRowBytes>(vaddr + vtr_off[db][t]);
            });
          });
        });
        static_for<0, 2>([&](auto KK) {
          constexpr int kk = decltype(KK)::value;
          bf16x8 pb;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float pe = __builtin_amdgcn_exp2f(__builtin_fmaf(acc_s[kb2][8 * kk + e], c2, negm));
            lp[e & 3] += pe;
            pb[e] = (__bf16)pe;
          }
          lds_wait<(1 - kk) * 2 * DB>();
#pragma unroll
          for (int db = 0; db < DB; ++db) {
            lds_bind(vf[kk][db][0]);
            lds_bind(vf[kk][db][1]);
            const u32x4 a4 = {vf[kk][db][0][0], vf[kk][db][0][1], vf[kk][db][1][0], vf[kk][db][1][1]};
            acc_o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a4), pb, acc_o[db], 0, 0, 0);
          }
        });
      });
      l_run += (lp[0] + lp[1]) + (lp[2] + lp[3]);
    }
    wait_loads<0>();
    __syncthreads();
  }

  // The wave's 32 rows as fp16 times a power of two per row (within 2^-11 of
  // the row's largest element: beside bf16 outputs), staged so that whole rows
  // are stored.  A row without a visible key here stores zeros and minus infinity.
  if (wq_lo >= qend) return;
  const float l_tot = l_run + other_half(l_run);
  const float inv = l_tot > 0.0f ? 1.0f / l_tot : 0.0f;
  float amax = 0.0f;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int j = 0; j < 16; ++j) amax = fmaxf(amax, fabsf(acc_o[db][j]));
  amax = fmaxf(amax, other_half(amax));
  float mul, rscale;
  row_scale(amax * inv, inv, mul, rscale);
  char* stg = reinterpret_cast<char*>(&sm.k[0][0]) + wv * 32 * TL::kRowBytes;
  auto stg_off = [&](int r, int chunk) {
    return r * TL::kRowBytes + ((chunk ^ ((r >> 1) & (TL::kSlots - 1))) << 4);
  };
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int jj = 0; jj < 4; ++jj) {
      f16x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = (_Float16)(acc_o[db][4 * jj + e] * mul);
      *reinterpret_cast<f16x4*>(stg + stg_off(qr, db * 4 + jj) + 8 * hi) = o;
    }
  if (hi == 0 && tq < qend)
    rec[static_cast<int64_t>(my_tok) * a.H] = f32x2{m_run + __builtin_amdgcn_logf(l_tot), rscale};
  constexpr int kPasses = 32 * TL::kRowBytes / 1024;
  _Float16* obase = reinterpret_cast<_Float16*>(a.ws + a.tile_row) + static_cast<int64_t>(slot) * a.T * a.H * D;
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    const int r = (i * 64 + lane) / TL::kSlots, chunk = (i * 64 + lane) % TL::kSlots;
    const u32x4 x = *reinterpret_cast<const u32x4*>(stg + stg_off(r, chunk));
    const int64_t tok = tok0 + base + (wq_lo + r) * static_cast<int64_t>(P.r);
    if (wq_lo + r < qend) *reinterpret_cast<u32x4*>(obase + (tok * a.H + head) * D + chunk * 8) = x;
  }
}

// One launch for both: the tiles first, as they take longer.
template <int D, bool kTiles>
__global__ __launch_bounds__(kPgThreads) void paged_attn(PagedArgs a) {
  const int idx = launch_index();
  if constexpr (kTiles) {
    union Smem {
      SmemTile<D> tile;
      SmemOne<D> one;
    };
    __shared__ Smem sm;
    if (idx < a.tile_items) query_tiles<D>(a, idx, sm.tile);
    else single_tokens<D>(a, idx - a.tile_items, sm.one);
  } else {
    __shared__ SmemOne<D> sm;
    single_tokens<D>(a, idx, sm);
  }
}

// ---------------------------------------------------------------------------
// The join: a row's partials, of every pattern that keeps it and every split,
// mixed by their denominators.  D/8 lanes read a partial row; kSubs partials
// of a row at a time, so that their loads are under way together.
// ---------------------------------------------------------------------------
__device__ inline void put8(u16* p, const f32x8& v) {
  bf16x8 b;
#pragma unroll
  for (int e = 0; e < 8; ++e) b[e] = (__bf16)v[e];
  *reinterpret_cast<bf16x8*>(p) = b;
}
__device__ inline void put8(float* p, const f32x8& v) { *reinterpret_cast<f32x8*>(p) = v; }

template <typename T, int D, bool kTiles>
__global__ __launch_bounds__(kPgThreads) void paged_join(PagedArgs a) {
  constexpr int kLanes = D / 8;
  constexpr int kSubs = kTiles ? 4 : 64 / kLanes;
  constexpr int kRows = 64 / kLanes / kSubs;  // rows of a wave
  const int tid = __builtin_amdgcn_workitem_id_x(), lane = tid & 63;
  const int ch = lane % kLanes, sub = lane / kLanes % kSubs, mine = lane / (kLanes * kSubs);
  const int row0 = (launch_index() * kPgWaves + __builtin_amdgcn_readfirstlane(tid >> 6)) * kRows;
  const int total = a.T * a.H;
  if (row0 >= total) return;
  int toks[kRows];
  Sequence sq[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) toks[i] = min(row0 + i, total - 1) / a.H;
  find_sequences(a, toks, lane, sq);
  int tok = toks[0], pos = position_of(a, sq[0], toks[0]), begin = sq[0].begin, n = sq[0].end - begin, b = sq[0].b;
#pragma unroll
  for (int i = 1; i < kRows; ++i)
    if (mine == i) {
      tok = toks[i];
      pos = position_of(a, sq[i], tok);
      begin = sq[i].begin;
      n = sq[i].end - begin;
      b = sq[i].b;
    }
  const int row = row0 + mine;
  const int head = row - tok * a.H;
  const bool single = !kTiles || n <= a.few;
  const int64_t e = a.by_token ? tok : static_cast<int64_t>(b) * a.few + (tok - begin);
  const float* one_rec = reinterpret_cast<const float*>(a.ws + a.one_rec) + (e * a.H + head) * a.one_slots;
  const float* one_row = reinterpret_cast<const float*>(a.ws + a.one_row) + (e * a.H + head) * a.one_slots * D;

  float m = -INFINITY, l = 0.0f;
  f32x8 acc = f32x8{0, 0, 0, 0, 0, 0, 0, 0};
  if (pos >= 0 && row < total) {
    for (int want = sub;; want += kSubs) {  // the want-th partial of the row
      int slot = -1, before = 0;
      for (int i = 0; i < a.npat; ++i) {
        const PagedPattern& P = a.pat[i];
        const int g = P.fw.div(pos), loc = pos - g * P.w;
        const int t = P.fr.div(loc), rho = loc - t * P.r;
        if (head - static_cast<int>(P.fr.div(head)) * P.r != rho) continue;
        const int used = single ? t / split_keys_of(P, t + 1) + 1 : P.tile_splits;
        if (want >= before && want < before + used) slot = (single ? P.one_slot : P.tile_slot) + want - before;
        before += used;
      }
      if (slot < 0) break;
      float x, scale = 1.0f;
      f32x8 o;
      if (single) {
        x = one_rec[slot];
        o = *reinterpret_cast<const f32x8*>(one_row + static_cast<int64_t>(slot) * D + ch * 8);
      } else {
        const int64_t at = static_cast<int64_t>(slot) * total + row;
        const f32x2 r = reinterpret_cast<const f32x2*>(a.ws + a.tile_rec)[at];
        const f16x8 h = *reinterpret_cast<const f16x8*>(a.ws + a.tile_row + (at * D + ch * 8) * 2);
        x = r[0];
        scale = r[1];
#pragma unroll
        for (int c = 0; c < 8; ++c) o[c] = static_cast<float>(h[c]);
      }
      if (x == -INFINITY) continue;  // a split without a visible key: its row is not read
      const float mn = fmaxf(m, x);
      const float f0 = __builtin_amdgcn_exp2f(m - mn), f1 = __builtin_amdgcn_exp2f(x - mn);
      m = mn;
      l = l * f0 + f1;
      acc = acc * f0 + o * (f1 * scale);
    }
  }
#pragma unroll
  for (int x = kLanes; x < kLanes * kSubs; x <<= 1) {
    const float mo = __shfl_xor(m, x, 64), lo = __shfl_xor(l, x, 64);
    const float mn = fmaxf(m, mo);
    const float f0 = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - mn);
    const float f1 = mo == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mo - mn);
    m = mn;
    l = l * f0 + lo * f1;
#pragma unroll
    for (int c = 0; c < 8; ++c) acc[c] = acc[c] * f0 + __shfl_xor(acc[c], x, 64) * f1;
  }
  if (sub != 0 || row >= total) return;
  acc *= l > 0.0f ? 1.0f / l : 0.0f;
  put8(static_cast<T*>(a.out) + static_cast<int64_t>(row) * D + ch * 8, acc);
  if (ch == 0) a.lse[static_cast<int64_t>(head) * a.T + tok] = l > 0.0f ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
}

template <int D>
void launch_all(const PagedPlan& p, const PagedArgs& a, hipStream_t stream) {
  const dim3 threads(kPgThreads), grid = grid_of(p.tile_items + p.one_items);
  if (p.dtype == DA_F32) hipLaunchKernelGGL(paged_one_f32<D>, grid, threads, 0, stream, a);
  else if (p.all_few) hipLaunchKernelGGL((paged_attn<D, false>), grid, threads, 0, stream, a);
  else hipLaunchKernelGGL((paged_attn<D, true>), grid, threads, 0, stream, a);
  const int64_t rows = p.T * p.H, few = (rows + kPgWaves - 1) / kPgWaves;
  constexpr int kPerGroup = kPgWaves * (64 / (D / 8) / 4);  // rows of a workgroup beside tiles
  if (p.dtype == DA_F32) hipLaunchKernelGGL((paged_join<float, D, false>), grid_of(few), threads, 0, stream, a);
  else if (p.all_few) hipLaunchKernelGGL((paged_join<u16, D, false>), grid_of(few), threads, 0, stream, a);
  else hipLaunchKernelGGL((paged_join<u16, D, true>), grid_of((rows + kPerGroup - 1) / kPerGroup), threads, 0, stream, a);
}

}  // namespace

hipError_t launch_paged(const PagedPlan& p, const void* q, int64_t q_stride, const PagedCache& cache, void* out,
                        float* lse, void* workspace, hipStream_t stream) {
  PagedArgs a{};
  a.q = q;
  a.kc = static_cast<const char*>(cache.k);
  a.vc = static_cast<const char*>(cache.v);
  a.table = cache.table;
  a.lens = cache.lens;
  a.start = cache.start;
  a.ws = static_cast<char*>(workspace);
  a.out = out;
  a.lse = lse;
  a.qs = q_stride;
  a.one_rec = static_cast<int64_t>(p.one_rec_off);
  a.one_row = static_cast<int64_t>(p.one_row_off);
  a.tile_rec = static_cast<int64_t>(p.tile_rec_off);
  a.tile_row = static_cast<int64_t>(p.tile_row_off);
  a.T = static_cast<int32_t>(p.T);
  a.B = static_cast<int32_t>(p.B);
  a.H = static_cast<int32_t>(p.H);
  a.Hkv = static_cast<int32_t>(p.Hkv);
  a.G = static_cast<int32_t>(p.H / p.Hkv);
  a.npat = p.npat;
  a.num_pages = static_cast<int32_t>(p.num_pages);
  a.max_pages = static_cast<int32_t>(p.max_pages);
  a.page_log2 = p.page_log2;
  a.by_token = p.by_token;
  a.few = static_cast<int32_t>(p.few);
  a.tile_items = static_cast<int32_t>(p.tile_items);
  const int64_t per_token = p.dtype == DA_F32 ? p.H : p.Hkv * ((a.G + kPagedGroupRows - 1) / kPagedGroupRows);
  a.units = static_cast<int32_t>(p.singles * per_token);
  a.one_slots = static_cast<int32_t>(p.one_slots);
  a.reach = static_cast<uint32_t>(p.max_pages * p.page);
  a.fslots = make_fastdiv(static_cast<uint32_t>(p.one_slots));
  a.funits = make_fastdiv(static_cast<uint32_t>(per_token));
  a.scale_log2 = p.scale * kLog2e;
  std::copy(p.pat, p.pat + p.npat, a.pat);
  if (p.D == 32) launch_all<32>(p, a, stream);
  else if (p.D == 64) launch_all<64>(p, a, stream);
  else launch_all<128>(p, a, stream);
  return hipGetLastError();
}

}  // namespace da
