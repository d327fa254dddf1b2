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
// 16 query heads), V to the wave's own LDS buffer, read transposed.  Eight tokens
// of 16 heads of 128 over four key heads, 8K to 64K cached, dense: 472 MB in 91 us
// (5.2 TB/s); 64 of 12 heads of 64, 1K to 32K cached, five patterns: 277 MB in 61
// us (4.5 TB/s).
// query_tiles: a workgroup is 128 kept query rows of one (sequence, head,
// segment) of a pattern against 64-key tiles in LDS.  Bound by the matrix cores
// and the softmax's vector work where a launch is long (8192 tokens of 12 heads of
// 64, dense: 103 GFLOP in 150 us), by the start-up of an item (8 us) and the tail
// where it is short (4096 tokens at 28672, five patterns: 31.9 GFLOP in 59 us).
// Both write normalised partial rows with their log-sum-exps; paged_join mixes
// a row's partials.
//
// Fewer bits than float32, in bf16 calls only, each as in the forward pass:
// probabilities are rounded to bf16 for the product with V, as its matrix
// instruction takes them (their sums stay float32), and partial rows of tiles are
// kept as fp16 times a power of two per row, half the bytes that the join reads
// again (those of single tokens are float32).  An output as a whole is then within
// 0.0020 to 0.0024 of float64's, relatively, where float32 arithmetic rounded to bf16
// once is within 0.0016 to 0.0017.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device_common.h"
#include "paged.h"

namespace da {
namespace {

constexpr int kPgThreads = 256;
constexpr int kPgWaves = kPgThreads / 64;
constexpr float kLowest = -3.402823466e38f;  // a running maximum of no score: the lowest finite value
constexpr float kSumSlack = 1024.0f;  // a half row's sum above it moves its reference (tiles)
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
  int32_t few, singles, one_slots, one_items, tile_items, grid, join_groups;
  uint32_t reach;     // positions the table holds
  FastDiv fheads;     // division by H
  float scale_log2;
  // Single tokens: the pattern that holds every key of its segment (r = 1, the
  // longest such segment), or -1, and its segment length.
  int32_t full, full_w;
  FastDiv full_fw;
  // Where each pattern's workgroups begin, beyond all others' for patterns that
  // are not there: found without a loop over the records.
  int32_t one_begin[DA_MAX_PATTERNS], tile_begin[DA_MAX_PATTERNS];
  PagedPattern pat[DA_MAX_PATTERNS];
};

// One word of every 64 bytes of the arguments, requested together: what a
// kernel reads of them later is then near.  (Read where they are used, a launch
// of few workgroups waits for them a dozen times in turn.)
__device__ inline void touch(const PagedArgs& a) {
  const uint32_t* w = reinterpret_cast<const uint32_t*>(&a);
  uint32_t x = 0;
#pragma unroll
  for (size_t i = 0; i < sizeof(PagedArgs) / 4; i += 16) x |= w[i];
  asm volatile("" ::"s"(x));
}

// The last pattern that begins at or before x.
__device__ inline int pattern_at(const int32_t (&begin)[DA_MAX_PATTERNS], int x) {
  int n = 0;
#pragma unroll
  for (int i = 0; i < DA_MAX_PATTERNS; ++i) n += begin[i] <= x;
  return n - 1;
}

// The keys of pattern P that a query at position pos sees, if its head is kept:
// positions first + t r, t < n; rho is the head offset that is kept.
struct Lattice {
  int rho, first, n;
};
__device__ inline Lattice lattice_of(const PagedPattern& P, int pos) {
  const int seg = static_cast<int>(P.fw.div(pos)) * P.w, loc = pos - seg;
  const int t = P.fr.div(loc), rho = loc - t * P.r;
  return {rho, seg + rho, t + 1};
}
// How many of them a single token reads for P: where the list has a pattern
// that holds every key of its segment, the others leave the keys of that
// segment to it, which weights a key by the number of patterns that hold it.
// (A token's patterns overlap near its position: the paper's five at 1K to 32K
// tokens, 64 sequences, read 277 MB instead of 367.)
__device__ inline int own_keys(const PagedArgs& a, const PagedPattern& P, bool is_full, int pos, const Lattice& x) {
  if (a.full < 0 || is_full) return x.n;
  const int begin = static_cast<int>(a.full_fw.div(pos)) * a.full_w;
  return begin > x.first ? min(x.n, static_cast<int>(P.fr.div(begin - x.first - 1)) + 1) : 0;
}
__device__ inline int head_offset(const PagedPattern& P, int head) {
  return head - static_cast<int>(P.fr.div(head)) * P.r;
}

// The loads of these values begin before this point.  (A load whose value is used
// under a condition only would move there: another round to memory after those
// that the condition waits for.)
__device__ inline void here(int& v) { asm volatile("" : "+v"(v)); }

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
    here(len);
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

// Entry i of start, held to the call's tokens: what a tile reads and writes stays in bounds.
__device__ inline int token_row(const PagedArgs& a, int i) { return max(0, min(a.start[i], a.T)); }

// This thread's number, opaque to the compiler: in the loop over a workgroup's
// items what follows from it would otherwise be formed before the loop and held
// in registers over all of it (which then spill).
__device__ inline int thread_id() {
  int tid = __builtin_amdgcn_workitem_id_x();
  asm volatile("" : "+v"(tid));
  return tid;
}

// Running sum over the wave's lanes: within rows of 16 lanes by shifts on the
// vector ALU, then the rows' last sums into the rows after them.
template <int kCtrl, int kRows>
__device__ inline int add_shifted(int v) {
  return v + __builtin_amdgcn_update_dpp(0, v, kCtrl, kRows, 0xf, false);
}
__device__ inline int running_sum(int v) {
  v = add_shifted<0x111, 0xf>(v);  // row_shr 1, 2, 4, 8
  v = add_shifted<0x112, 0xf>(v);
  v = add_shifted<0x114, 0xf>(v);
  v = add_shifted<0x118, 0xf>(v);
  v = add_shifted<0x142, 0xa>(v);  // row_bcast 15 into rows 1 and 3
  return add_shifted<0x143, 0xc>(v);  // row_bcast 31 into rows 2 and 3
}

// A listed token: its row of q, its sequence and position.  kMixed: number e of
// those in sequences of at most a.few new tokens; otherwise row e of the call.
// False: not there, or not in the table.
struct Token {
  int tok, b, pos;
};
template <bool kMixed>
__device__ inline bool single_token(const PagedArgs& a, int e, int lane, Token& t) {
  Sequence sq[1] = {Sequence{-1, 0, 0, 0}};
  if constexpr (!kMixed) {
    const int tok[1] = {e};
    t.tok = e;
    find_sequences(a, tok, lane, sq);
  } else {
    t.tok = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
      const int b = min(b0 + lane, a.B - 1), begin = token_row(a, b), end = token_row(a, b + 1);
      int len = a.lens[b];
      here(len);
      const int n = b0 + lane < a.B && end - begin <= a.few ? max(end - begin, 0) : 0;
      const int upto = running_sum(n), total = __builtin_amdgcn_readlane(upto, 63);
      if (e < total) {
        const int l = __builtin_ctzll(__ballot(upto > e));
        sq[0] = Sequence{b0 + l, __builtin_amdgcn_readlane(begin, l), __builtin_amdgcn_readlane(end, l),
                         __builtin_amdgcn_readlane(len, l)};
        t.tok = sq[0].end - (__builtin_amdgcn_readlane(upto, l) - e);
        break;
      }
      e -= total;
    }
  }
  t.b = sq[0].b;
  t.pos = position_of(a, sq[0], t.tok);
  return t.pos >= 0;
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

// The table's entry for position pos of a sequence, and key head hk's row of the
// cache there.  A page outside the pool reads the pool's last page: in bounds,
// whatever the table holds.
__device__ inline int table_entry(const PagedArgs& a, const int32_t* table, int pos) { return table[pos >> a.page_log2]; }
__device__ inline uint32_t cache_row(const PagedArgs& a, int entry, int hk, int pos) {
  const uint32_t page = min(static_cast<uint32_t>(entry), static_cast<uint32_t>(a.num_pages - 1));
  return ((page * a.Hkv + hk) << a.page_log2) + (pos & ((1 << a.page_log2) - 1));
}
// The cache rows of keys first .. first + n - 1 (positions base + t r) into row,
// by a workgroup; keys past `last` are that one.  kAtOnce entries of a thread
// are on their way together.
template <int kAtOnce>
__device__ inline void look_up_rows(const PagedArgs& a, const int32_t* table, int hk, int base, int r, int first,
                                    int last, int n, int tid, uint32_t* row) {
  for (int i0 = tid; i0 < n; i0 += kAtOnce * kPgThreads) {
    int pos[kAtOnce], entry[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      pos[u] = base + min(first + i0 + u * kPgThreads, last) * r;
      entry[u] = table_entry(a, table, pos[u]);
    }
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) here(entry[u]);
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u)
      if (i0 + u * kPgThreads < n) row[i0 + u * kPgThreads] = cache_row(a, entry[u], hk, pos[u]);
  }
}

// Keys of a split of n keys: whole 32-key tiles, and two of them for each wave
// at least (64 tokens of 100 to 2000 cached, dense: 30.4 us without that, 28.9 with it).
constexpr int kOneLeast = 256;
__device__ inline int split_keys_of(const PagedPattern& P, int n) {
  return max(kOneLeast, (static_cast<int>(P.one_split.div(n + P.one_split.d - 1)) + 31) & ~31);
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

// A workgroup's place among a pattern's items for single tokens: unit u = (token
// e, number of its block of heads) runs with all its splits on XCD u mod 8
// (dealt out split by split over the XCDs, the 472 MB of 8 sequences with heads
// of 128 took 105 us instead of 90).  False: past the tokens' end.
struct OneItem {
  int pi, split, e, head;
};
__device__ inline bool one_item(const PagedArgs& a, int pi, int local, int tokens, OneItem& it) {
  const PagedPattern& P = a.pat[pi];
  const int j = local >> 3, block8 = P.one_split.div(j);
  const int unit = block8 * 8 + (local & 7);
  it.pi = pi;
  it.split = j - block8 * P.one_split.d;
  it.e = P.one_heads.div(unit);
  it.head = unit - it.e * P.one_heads.d;
  return it.e < tokens;
}

// A wave's 32 keys of K on their way: two blocks of 16 as operands.
template <int D>
struct KeyFrag {
  u32x4 k[2][D / 32];
};

constexpr int kOneTile = 32;    // keys of a wave's tile
constexpr int kOneRows = 1024;  // keys whose rows are looked up at once
template <int D>
struct SmemOne {
  __attribute__((aligned(16))) char v[kPgWaves][kOneTile * D * 2];  // each wave's V tile
  float ml[kPgWaves][2][16];
  u32x4 q[D / 32][64];     // Q^T operand, lane by lane
  uint32_t row[kOneRows];  // cache rows of the split's keys, a chunk at a time
};

template <int D, bool kMixed>
__device__ inline void single_tokens(const PagedArgs& a, const OneItem& it, SmemOne<D>& sm) {
  constexpr int KC = D / 32, DB = D / 16, kTile = kOneTile;
  using TL = TileLayout<D>;
  constexpr int kVLoads = kTile * TL::kSlots / 64;
  // Joined rows are D floats apart, 16-byte chunk c of row r at c ^ (r mod D/4).
  auto join_at = [](int r, int chunk) { return r * D + 4 * (chunk ^ (r & (D / 4 - 1))); };
  static_assert(16 * D * 4 <= kTile * D * 2, "the join fits a wave's V tile");
  auto& sv = sm.v;
  auto& sml = sm.ml;

  const int tid = thread_id(), lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int pi = it.pi;
  const PagedPattern& P = a.pat[pi];
  Token tk;
  if (!single_token<kMixed>(a, it.e, lane, tk)) return;
  const Lattice lat = lattice_of(P, tk.pos);
  // Dilations of a group's size and above keep one head of a group at most: the
  // head-th kept one; below, every group has some, in blocks.
  int hk = it.head, block = 0;
  if (P.r >= a.G) {
    const int64_t h = lat.rho + static_cast<int64_t>(it.head) * P.r;
    if (h >= a.H) return;
    hk = static_cast<int>(h) / a.G;
  } else if (a.G > static_cast<int>(kPagedGroupRows)) {
    block = it.head / a.Hkv;
    hk = it.head - block * a.Hkv;
  }
  const KeptHeads kh = kept_heads(P, hk, a.G, lat.rho);
  const int m0 = block * static_cast<int>(kPagedGroupRows);
  if (m0 >= kh.count) return;
  const int rows = min(static_cast<int>(kPagedGroupRows), kh.count - m0);
  const int n = own_keys(a, P, pi == a.full, tk.pos, lat), per = split_keys_of(P, n);
  const int k0 = it.split * per;
  if (k0 >= n) return;
  const int ke = min(k0 + per, n);

  const int m = lane & 15, grp = lane >> 4;
  const int head = kh.first + (m0 + min(m, rows - 1)) * P.r;
  // Q^T operand (kept in LDS: in registers it would spill at D = 128).
  for (int c = wv; c < KC; c += kPgWaves) {
    const u32x4 x = load16(static_cast<const u16*>(a.q) + tk.tok * a.qs + head * D + 32 * c + 8 * grp);
    sm.q[c][lane] = m < rows ? x : u32x4{0u, 0u, 0u, 0u};
  }

  const int32_t* table = a.table + static_cast<int64_t>(tk.b) * a.max_pages;
  const int base = lat.first;
  // Patterns whose keys this one reads too, for any head here and for the lane's.
  unsigned with = 0, mine = 0;
  if (pi == a.full && a.npat > 1) {
    const PagedPattern Q = a.pat[lane & 15];  // a pattern per lane
    const bool there = lane < a.npat && lane != pi;
    const int rho = there ? lattice_of(Q, tk.pos).rho : 0;
    for (int r = 0; r < rows; ++r) {
      const bool kept = there && head_offset(Q, kh.first + (m0 + r) * P.r) == rho;
      const unsigned mask = static_cast<unsigned>(__ballot(kept));
      with |= mask;
      if (m == r) mine = mask;
    }
  }
  constexpr int kVStep = 64 / TL::kSlots;  // V rows of a load
  const int vrow = lane / TL::kSlots;
  char* my = sv[wv];
  // Requests the 32 keys from `key` on (counted within the chunk whose rows are in LDS).
  auto request_k = [&](int key, KeyFrag<D>& kf) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const char* p = a.kc + (static_cast<int64_t>(sm.row[key + 16 * u + m]) * TL::kRowBytes + 16 * grp);
#pragma unroll
      for (int c = 0; c < KC; ++c) kf.k[u][c] = *reinterpret_cast<const u32x4*>(p + 64 * c);
    }
  };
  u32x4 vreg[kVLoads];
  auto request_v = [&](int key) {
#pragma unroll
    for (int i = 0; i < kVLoads; ++i)
      vreg[i] = *reinterpret_cast<const u32x4*>(
          a.vc + (static_cast<int64_t>(sm.row[key + kVStep * i + vrow]) * TL::kRowBytes + (lane % TL::kSlots) * 16));
  };
  // V^T operand: lane's d = 16 db + (lane & 15), keys 4 grp + 0..3 and 16 more.
  // Block db's 16-byte slots are 2 db and 2 db + 1 before the swizzle, an
  // exclusive or: its address is block 0's with bits of db flipped.
  const int tr_r = 4 * grp + ((lane & 15) >> 2), tr_d = (lane & 3) * 4;
  const uint32_t voff = TL::offset(tr_r, tr_d >> 3) + (tr_d & 7) * 2;

  f32x4 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = f32x4{0, 0, 0, 0};
  float m_run = kLowest, l_run = 0.0f;
  const float c2 = a.scale_log2;

  // first: the tile's first key (t); next: the next tile's, within the chunk, < 0: none
  auto compute = [&](int first, const KeyFrag<D>& kf, int next) {
    f32x4 s[2] = {f32x4{0, 0, 0, 0}, f32x4{0, 0, 0, 0}};
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      const bf16x8 qf = __builtin_bit_cast(bf16x8, sm.q[c][lane]);
#pragma unroll
      for (int u = 0; u < 2; ++u)
        s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf.k[u][c]), qf, s[u], 0, 0, 0);
    }
    const int left = ke - first - 4 * grp;  // keys from this lane's first on
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
    f32x4 count[2] = {f32x4{1, 1, 1, 1}, f32x4{1, 1, 1, 1}};
    for (unsigned rest = with; rest; rest &= rest - 1) {
      const int i = __builtin_ctz(rest);
      const PagedPattern& Q = a.pat[i];
      const int d = base + first + 4 * grp - lattice_of(Q, tk.pos).first;
      const float one = mine >> i & 1 ? 1.0f : 0.0f;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int x = d + 16 * u + e;
          const int q = Q.fr.div(max(x, 0));
          count[u][e] += x >= 0 && q * Q.r == x ? one : 0.0f;
        }
    }
    bf16x8 pb;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][e], c2, -m_run)) * count[u][e];
        l_run += p;
        pb[4 * u + e] = (__bf16)p;  // for the product alone
      }
    // V through the wave's own LDS tile, to be read transposed (LDS operations
    // of a wave complete in order: no wait between).
#pragma unroll
    for (int i = 0; i < kVLoads; ++i)
      *reinterpret_cast<u32x4*>(my + TL::offset(kVStep * i + vrow, lane % TL::kSlots)) = vreg[i];
    if (next >= 0) request_v(next);
    const uint32_t va = lds_addr(my);
    constexpr int kHalf = DB < 4 ? DB : 4;  // blocks whose V is read at once
#pragma unroll
    for (int d0 = 0; d0 < DB; d0 += kHalf) {
      u32x2 vf[kHalf][2];
#pragma unroll
      for (int x = 0; x < kHalf; ++x) {
        const uint32_t at = va + (voff ^ ((d0 + x) << 5));
        vf[x][0] = lds_read_tr16<0>(at);
        vf[x][1] = lds_read_tr16<16 * TL::kRowBytes>(at);
      }
      lds_wait<0>();
#pragma unroll
      for (int x = 0; x < kHalf; ++x) {
        lds_bind(vf[x][0]);
        lds_bind(vf[x][1]);
        const u32x4 v4 = {vf[x][0][0], vf[x][0][1], vf[x][1][0], vf[x][1][1]};
        acc[d0 + x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v4), pb, acc[d0 + x], 0, 0, 0);
      }
    }
  };

  for (int c0 = k0; c0 < ke; c0 += kOneRows) {
    const int keys = min(ke - c0, kOneRows), ntile = (keys + kTile - 1) / kTile;
    if (c0 > k0) __syncthreads();  // every wave is done with the rows before
    look_up_rows<4>(a, table, hk, base, P.r, c0, ke - 1, ntile * kTile, tid, sm.row);
    __syncthreads();
    if (wv >= ntile) continue;
    // While a tile is computed the next one's loads are under way, K's from its
    // start, V's from where its own V has left the registers.  A wave's last tile
    // is a branch of its own, so that at every use of K it is known which loads
    // are younger.
    KeyFrag<D> ka, kb;
    request_k(wv * kTile, ka);
    request_v(wv * kTile);
    for (int tile = wv;;) {
      const int next = (tile + kPgWaves) * kTile;
      if (tile + kPgWaves >= ntile) {
        compute(c0 + tile * kTile, ka, -1);
        break;
      }
      request_k(next, kb);
      compute(c0 + tile * kTile, ka, next);
      tile += kPgWaves;
      if (tile + kPgWaves >= ntile) {
        compute(c0 + tile * kTile, kb, -1);
        break;
      }
      request_k(next + kPgWaves * kTile, ka);
      compute(c0 + tile * kTile, kb, next + kPgWaves * kTile);
      tile += kPgWaves;
    }
  }

  // The waves' partial rows meet in LDS, each in its wave's own V tile.
  l_run = sum_over_groups(l_run);
  float* jo = reinterpret_cast<float*>(my);
#pragma unroll
  for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4*>(jo + join_at(m, 4 * db + grp)) = acc[db];
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
      o += f * *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(sv[w]) + join_at(r, d / 4));
    }
    const int64_t at = (row0 + kh.first + (m0 + r) * P.r) * a.one_slots + P.one_slot + it.split;
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
  const int idx = launch_index();
  if (idx >= a.one_items) return;
  const int pi = pattern_at(a.one_begin, idx);
  const PagedPattern& P = a.pat[pi];
  OneItem it;
  Token tk;
  if (!one_item(a, pi, idx - P.one_begin, a.singles, it) || !single_token<false>(a, it.e, lane, tk)) return;
  const Lattice lat = lattice_of(P, tk.pos);
  const int64_t kept = lat.rho + static_cast<int64_t>(it.head) * P.r;
  if (kept >= a.H) return;
  const int head = static_cast<int>(kept), hk = head / a.G;
  const int n = own_keys(a, P, pi == a.full, tk.pos, lat), per = split_keys_of(P, n), k0 = it.split * per;
  if (k0 >= n) return;
  const int ke = min(k0 + per, n);
  const int grp = tid / kLanes, ch = tid % kLanes;
  const f32x4 q = *reinterpret_cast<const f32x4*>(static_cast<const float*>(a.q) + tk.tok * a.qs + head * D + 4 * ch);
  const int32_t* table = a.table + static_cast<int64_t>(tk.b) * a.max_pages;
  const int base = lat.first;
  unsigned with = 0;  // patterns whose keys this one reads too
  if (pi == a.full && a.npat > 1) {
    const PagedPattern Q = a.pat[lane & 15];  // a pattern per lane
    with = static_cast<unsigned>(
        __ballot(lane < a.npat && lane != pi && head_offset(Q, head) == lattice_of(Q, tk.pos).rho));
  }
  float m_run = kLowest, l_run = 0.0f;
  f32x4 acc = f32x4{0, 0, 0, 0};
  for (int t0 = k0; t0 < ke; t0 += kUnroll * kGroups) {
    f32x4 k[kUnroll], v[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int t = min(t0 + u * kGroups + grp, ke - 1);
      const int pos = base + t * P.r;
      const int64_t at = static_cast<int64_t>(cache_row(a, table_entry(a, table, pos), hk, pos)) * D + 4 * ch;
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
    float count[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) count[u] = 1.0f;
    for (unsigned rest = with; rest; rest &= rest - 1) {
      const PagedPattern& Q = a.pat[__builtin_ctz(rest)];
      const int d = base + t0 + grp - lattice_of(Q, tk.pos).first;
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int x = d + u * kGroups;
        const int q = Q.fr.div(max(x, 0));
        count[u] += x >= 0 && q * Q.r == x ? 1.0f : 0.0f;
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const float p = __builtin_amdgcn_exp2f(s[u] - m_run) * count[u];
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
  const int64_t at = (static_cast<int64_t>(it.e) * a.H + head) * a.one_slots + P.one_slot + it.split;
  o *= l > 0.0f ? 1.0f / l : 0.0f;
  *reinterpret_cast<f32x4*>(a.ws + a.one_row + (at * D + 4 * ch) * 4) = o;
  if (ch == 0) reinterpret_cast<float*>(a.ws + a.one_rec)[at] = mt + __builtin_amdgcn_logf(l);
}

// ---------------------------------------------------------------------------
// Tiles of query rows
// ---------------------------------------------------------------------------
// The new tokens of sequences computed in tiles, sequence b0 + lane: positions
// [c0, c1), empty for the others; tok0: the token row of position 0.
struct Chunk {
  int c0, c1, tok0;
};
__device__ inline Chunk chunk_of(const PagedArgs& a, int b0, int lane) {
  const int b = min(b0 + lane, a.B - 1);
  const int end = token_row(a, b + 1), n = end - token_row(a, b), len = a.lens[b];
  const int c1 = max(0, static_cast<int>(min(static_cast<uint32_t>(max(len, 0)), a.reach)));
  const int c0 = max(0, static_cast<int>(min(static_cast<int64_t>(len) - n, static_cast<int64_t>(c1))));
  return b0 + lane < a.B && n > a.few ? Chunk{c0, c1, end - len} : Chunk{0, 0, 0};
}
// Query tiles of pattern P over `len` >= 1 positions of a segment, and over a
// sequence's new tokens, segment by segment (for any head: its offset only
// moves the rows within a tile).
__device__ inline int tiles_of(const PagedPattern& P, int len) {
  return static_cast<int>(P.fr.div(len - 1)) / static_cast<int>(kPagedRows) + 1;
}
__device__ inline int tiles_of(const PagedPattern& P, const Chunk& c) {
  if (c.c1 <= c.c0) return 0;
  const int g0 = P.fw.div(c.c0), g1 = P.fw.div(c.c1 - 1);
  return g0 == g1 ? tiles_of(P, c.c1 - c.c0)
                  : tiles_of(P, (g0 + 1) * P.w - c.c0) + (g1 - g0 - 1) * tiles_of(P, P.w) + tiles_of(P, c.c1 - g1 * P.w);
}
// Tile `tile` of pattern P among all sequences'.
struct QueryTile {
  int b, g, j;  // sequence, segment, tile of the segment's new rows
  Chunk c;
};
__device__ inline bool query_tile(const PagedArgs& a, const PagedPattern& P, int tile, int lane, QueryTile& qt) {
  qt.b = -1;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    const Chunk c = chunk_of(a, b0, lane);
    const int cnt = tiles_of(P, c), upto = running_sum(cnt), total = __builtin_amdgcn_readlane(upto, 63);
    if (tile < total) {
      const int l = __builtin_ctzll(__ballot(upto > tile));
      qt.b = b0 + l;
      qt.c = Chunk{__builtin_amdgcn_readlane(c.c0, l), __builtin_amdgcn_readlane(c.c1, l),
                   __builtin_amdgcn_readlane(c.tok0, l)};
      tile -= __builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(cnt, l);
      break;
    }
    tile -= total;
  }
  if (qt.b < 0) return false;
  qt.j = tile;
  qt.g = P.fw.div(qt.c.c0);
  const int g1 = P.fw.div(qt.c.c1 - 1);
  const int first = qt.g == g1 ? 0x7fffffff : tiles_of(P, (qt.g + 1) * P.w - qt.c.c0);
  if (qt.j >= first) {
    const int per = tiles_of(P, P.w);
    qt.j -= first;
    const int skip = min(qt.j / per, g1 - qt.g - 1);
    qt.g += 1 + skip;
    qt.j -= skip * per;
  }
  return true;
}

// A workgroup's place among a pattern's items for tiles.
struct TileItem {
  int pi, tile, head, split;
};

constexpr int kTileRows = 4096;  // keys whose rows are looked up at once (three workgroups of D = 64 fit a CU)

template <int D>
struct SmemTile {
  __attribute__((aligned(16))) u16 k[2][kPagedKeyTile * D];
  __attribute__((aligned(16))) u16 v[2][kPagedKeyTile * D];
  uint32_t row[kTileRows];  // cache rows of the keys, a chunk at a time
};

template <int D>
__device__ inline void query_tiles(const PagedArgs& a, const TileItem& it, SmemTile<D>& sm) {
  constexpr int BM = kPagedRows, BN = kPagedKeyTile;
  constexpr int KC = D / 16, DB = D / 32;
  using TL = TileLayout<D>;
  constexpr int kLoads = BN * TL::kSlots / 64 / kPgWaves;
  const int tid = thread_id(), lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const PagedPattern& P = a.pat[it.pi];
  const int head = it.head, sp = it.split;
  QueryTile qt;
  if (!query_tile(a, P, it.tile, lane, qt)) return;
  const int gs = qt.g * P.w;
  const int off = head - static_cast<int>(P.fr.div(head)) * P.r;
  const int lo = max(qt.c.c0 - gs, 0);
  const int hi_pos = min(qt.c.c1 - gs, P.w);
  auto first_at = [&](int x) { return x > off ? static_cast<int>(P.fr.div(x - off - 1)) + 1 : 0; };  // first t at or after x
  const int q0 = first_at(lo) + qt.j * BM;
  const int qend = min(q0 + BM, first_at(hi_pos));
  if (q0 >= qend) return;
  const int hk = head / a.G;
  // this split's keys
  const int per = (static_cast<int>(P.tile_split.div(qend + P.tile_split.d - 1)) + BN - 1) / BN * BN;
  const int kb = sp * per, ke = min(kb + per, qend);
  const int slot = P.tile_slot + sp;
  const int base = gs + off;  // position of t = 0
  const int tok0 = qt.c.tok0;

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
  // Tile jt of the chunk whose rows are in LDS.
  auto load_tile = [&](int jt, int buf) {
    char* kl = reinterpret_cast<char*>(&sm.k[buf][0]);
    char* vl = reinterpret_cast<char*>(&sm.v[buf][0]);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const uint64_t at = static_cast<uint64_t>(sm.row[jt * BN + lrow[i]]) * TL::kRowBytes + lslot[i] * 16;
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
  bf16x8 qreg[KC];
#pragma unroll
  for (int c = 0; c < KC; ++c) qreg[c] = __builtin_bit_cast(bf16x8, qraw[c]);

  f32x16 acc_o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) acc_o[db] = f32x16{};
  float m_run = kLowest, l_run = 0.0f;
  const float c2 = a.scale_log2;
  for (int c0 = kb; c0 < ke; c0 += kTileRows) {
    const int ntile = (min(ke - c0, kTileRows) + BN - 1) / BN;
    look_up_rows<8>(a, table, hk, base, P.r, c0, ke - 1, ntile * BN, tid, sm.row);
    __syncthreads();
    load_tile(0, 0);
    wait_loads<0>();
    __syncthreads();
    for (int jt = 0; jt < ntile; ++jt) {
      const int cur = jt & 1, k0 = c0 + jt * BN;
      if (jt + 1 < ntile) load_tile(jt + 1, cur ^ 1);
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
        // P = 2^(c S - m) for the reference m of the row so far, without looking
        // for the tile's maximum: a tile whose probabilities of half a row sum to
        // more than kSumSlack (or overflow: the first tile's do) has its scores
        // still in registers and forms them again with its maximum as reference.
        // Probabilities above 1 are held by bf16 (see above) and float32 as well as
        // those below.
        bf16x8 pb[2][2];
        float lt;
        auto probabilities = [&] {
          const float negm = -m_run;
          float lp[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const float pe = __builtin_amdgcn_exp2f(__builtin_fmaf(acc_s[x][j], c2, negm));
              lp[j & 3] += pe;
              pb[x][j >> 3][j & 7] = (__bf16)pe;
            }
          lt = (lp[0] + lp[1]) + (lp[2] + lp[3]);
        };
        probabilities();
        if (__any(!(lt <= kSumSlack))) {
          float mx = acc_s[0][0];
#pragma unroll
          for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int j = 0; j < 16; j += 2) mx = fmaxf(mx, fmaxf(acc_s[x][j], acc_s[x][j + 1]));
          const float m_new = fmaxf(m_run, fmaxf(mx, other_half(mx)) * c2);
          const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
          m_run = m_new;
          l_run *= alpha;
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int j = 0; j < 16; ++j) acc_o[db][j] *= alpha;
          probabilities();
        }
        l_run += lt;
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
            lds_wait<(1 - kk) * 2 * DB>();
#pragma unroll
            for (int db = 0; db < DB; ++db) {
              lds_bind(vf[kk][db][0]);
              lds_bind(vf[kk][db][1]);
              const u32x4 a4 = {vf[kk][db][0][0], vf[kk][db][0][1], vf[kk][db][1][0], vf[kk][db][1][1]};
              acc_o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a4), pb[kb2][kk],
                                                                  acc_o[db], 0, 0, 0);
            }
          });
        });
      }
      wait_loads<0>();
      __syncthreads();
    }
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

// Where item `local` of a pattern with `tiles` query tiles per head stands, in
// units of `run` tiles of one head with their splits: unit u runs on XCD u mod
// 8, whose L2 then serves the run's keys after their first fetch; later (longer)
// tiles first.  False: padding.
__device__ inline bool tile_item(const PagedArgs& a, int pi, int local, int tiles, int run, int splits, TileItem& it) {
  const int j = local >> 3, per = run * splits, unit8 = j / per, within = j - unit8 * per;
  const int u = unit8 * 8 + (local & 7), r = a.fheads.div(u), in_run = within / splits;
  it = TileItem{pi, tiles - 1 - (r * run + in_run), u - r * a.H, within - in_run * splits};
  return it.tile >= 0;
}

// Every token a single one.
template <int D>
__global__ __launch_bounds__(kPgThreads, D == 128 ? 2 : 3) void paged_singles(PagedArgs a) {
  __shared__ SmemOne<D> sm;
  touch(a);
  const int idx = launch_index();
  if (idx >= a.one_items) return;
  const int pi = pattern_at(a.one_begin, idx);
  OneItem it;
  if (one_item(a, pi, idx - a.pat[pi].one_begin, a.singles, it)) single_tokens<D, false>(a, it, sm);
}

template <int D>
union SmemMixed {
  SmemTile<D> tile;
  SmemOne<D> one;
  int count[DA_MAX_PATTERNS + 1];
};

// Tiles and single tokens in one launch, the tiles first, as they take longer:
// every item that the sizes allow.
template <int D>
__global__ __launch_bounds__(kPgThreads, D == 128 ? 2 : 3) void paged_mixed(PagedArgs a) {
  __shared__ SmemMixed<D> sm;
  touch(a);
  const int idx = launch_index();
  if (idx < a.tile_items) {
    const int pi = pattern_at(a.tile_begin, idx);
    const PagedPattern& P = a.pat[pi];
    TileItem it;
    if (tile_item(a, pi, idx - P.tile_begin, P.tiles, P.run, P.tile_split.d, it)) query_tiles<D>(a, it, sm.tile);
  } else if (idx - a.tile_items < a.one_items) {
    const int pi = pattern_at(a.one_begin, idx - a.tile_items);
    OneItem it;
    if (one_item(a, pi, idx - a.tile_items - a.pat[pi].one_begin, a.singles, it)) single_tokens<D, true>(a, it, sm.one);
  }
}

// The same in a launch as large as the sizes let expect: how many tiles and
// single tokens there are is known on the device only, so every workgroup counts
// them (a pattern per wave in turn, then per lane) and takes those items that
// are its index plus a multiple of the launch.  Against every item that the
// sizes allow: 16 sequences, one of them with 1000 new tokens, 50 -> 38 us; 40
// with one of 500, 102 -> 63; 64 with one of 2048, 104 -> 74.  Counted again for
// each item: held in registers over an item the counts would spill, and most
// workgroups have one.  (No least number of workgroups a CU: asking for 1, 2 or 3
// of them is within 1 % at heads of 32, 64 and 128.)
template <int D>
__global__ __launch_bounds__(kPgThreads) void paged_mixed_steps(PagedArgs a) {
  __shared__ SmemMixed<D> sm;
  touch(a);
  const uint32_t idx = launch_index();  // below 2^31, as the items and the launch are
  if (idx >= static_cast<uint32_t>(a.grid)) return;  // its items are another's
  for (uint32_t index = idx, items = idx + 1; index < items; index += a.grid) {
    const int item = static_cast<int>(index);
    const int tid = thread_id(), lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    for (int i = wv; i <= a.npat; i += kPgWaves) {  // the last: single tokens
      int cnt = 0;
      for (int b0 = 0; b0 < a.B; b0 += 64) {
        if (i < a.npat) {
          cnt += tiles_of(a.pat[i], chunk_of(a, b0, lane));
        } else if (b0 + lane < a.B) {
          const int n = token_row(a, b0 + lane + 1) - token_row(a, b0 + lane);
          cnt += n <= a.few ? max(n, 0) : 0;
        }
      }
      const int all = running_sum(cnt);
      if (lane == 63) sm.count[i] = all;
    }
    __syncthreads();
    // Lane i: pattern i's tiles, the tiles of a unit (see the plan), its items.
    // An array of starts that does not ascend can list a token twice: no more of
    // either than the plan has room for.
    const int pat = min(lane, a.npat - 1), tokens = min(sm.count[a.npat], a.singles);
    const PagedPattern P = a.pat[pat];
    const int tiles = max(0, min(sm.count[pat], P.tiles));
    const int splits = P.tile_split.d, run = max(1, min(16, static_cast<int>(static_cast<int64_t>(tiles) * a.H / 64)));
    const int units = ((tiles + run - 1) / run * a.H + 7) & ~7;
    const int singles = ((tokens * static_cast<int>(P.one_heads.d) + 7) & ~7) * P.one_split.d;
    const int mine = lane < a.npat ? units * run * splits : 0, ones = lane < a.npat ? singles : 0;
    const int tile_end = running_sum(mine), one_end = running_sum(ones);
    const int tile_items = __builtin_amdgcn_readlane(tile_end, 63);
    const int all_items = tile_items + __builtin_amdgcn_readlane(one_end, 63);
    items = all_items;
    __syncthreads();  // the counts are read
    if (item < tile_items) {
      const int pi = __builtin_ctzll(__ballot(tile_end > item));
      const int begin = __builtin_amdgcn_readlane(tile_end, pi) - __builtin_amdgcn_readlane(mine, pi);
      TileItem it;
      if (tile_item(a, pi, item - begin, __builtin_amdgcn_readlane(tiles, pi), __builtin_amdgcn_readlane(run, pi),
                    __builtin_amdgcn_readlane(splits, pi), it))
        query_tiles<D>(a, it, sm.tile);
    } else if (item < all_items) {
      const int pi = __builtin_ctzll(__ballot(one_end > item - tile_items));
      const int begin = tile_items + __builtin_amdgcn_readlane(one_end, pi) - __builtin_amdgcn_readlane(ones, pi);
      OneItem it;
      if (one_item(a, pi, item - begin, tokens, it)) single_tokens<D, true>(a, it, sm.one);
    }
    __syncthreads();  // the item is done with its LDS
  }
}

// ---------------------------------------------------------------------------
// The join: a row's partials, of every pattern that keeps it and every split,
// mixed by their denominators.
// ---------------------------------------------------------------------------
__device__ inline void put8(u16* p, const f32x8& v) {
  bf16x8 b;
#pragma unroll
  for (int e = 0; e < 8; ++e) b[e] = (__bf16)v[e];
  *reinterpret_cast<bf16x8*>(p) = b;
}
__device__ inline void put8(float* p, const f32x8& v) { *reinterpret_cast<f32x8*>(p) = v; }

// The bits of x, as the compiler cannot see through.  It takes floats for numbers
// (and a comparison of their bits for one of floats): a NaN, that of a row with a
// score that is NaN or plus infinity, may compare like any number.
__device__ inline uint32_t bits_of(float x) {
  uint32_t u = __builtin_bit_cast(uint32_t, x);
  asm("" : "+v"(u));
  return u;
}
// Whether a record marks a row that is not there.
__device__ inline bool no_row(float x) { return bits_of(x) == 0xff800000u; }

// A running mixture: m the largest log-sum-exp (log2 units) so far, l and acc
// the sums of the weights 2^(x - m) and of the weighted rows.
struct Mix {
  float m = -INFINITY, l = 0.0f;
  f32x8 acc = f32x8{0, 0, 0, 0, 0, 0, 0, 0};
  __device__ void add(float x, float scale, const f32x8& o) {  // row o * scale with weight 2^x
    if (no_row(x)) return;  // no visible key, or none with a finite score: the row is not there
    const float mn = fmaxf(m, x);
    const float f0 = __builtin_amdgcn_exp2f(m - mn), f1 = __builtin_amdgcn_exp2f(x - mn);
    m = mn;
    l = l * f0 + f1;
    acc = acc * f0 + o * (f1 * scale);
  }
  // Another mixture of the same row.
  template <typename Other>
  __device__ void meet(float mo, float lo, Other&& other) {
    const float mn = fmaxf(m, mo);
    const float f0 = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - mn);
    const float f1 = mo == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mo - mn);
    m = mn;
    l = l * f0 + lo * f1;
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = acc[i] * f0 + other(i) * f1;
  }
  __device__ void meet(int lanes) {  // of the lane `lanes` away (an exclusive or)
    meet(__shfl_xor(m, lanes, 64), __shfl_xor(l, lanes, 64), [&](int i) { return __shfl_xor(acc[i], lanes, 64); });
  }
};
template <typename T, int D>
__device__ inline void put_row(const PagedArgs& a, int tok, int head, int ch, const Mix& x) {
  const float inv = x.l > 0.0f ? 1.0f / x.l : 0.0f;
  put8(static_cast<T*>(a.out) + (static_cast<int64_t>(tok) * a.H + head) * D + ch * 8, x.acc * inv);
  // l is zero where no partial was added, and there only: the largest adds one.
  if (ch == 0)
    a.lse[static_cast<int64_t>(head) * a.T + tok] =
        bits_of(x.l) != 0 ? (x.m + __builtin_amdgcn_logf(x.l)) * kLn2 : -INFINITY;
}

// Single tokens: a wave per row (or a workgroup, kTogether), D/8 lanes across a
// partial and as many partials at a time as fit: a row has tens of them.
template <typename T, int D, bool kMixed, bool kTogether>
__device__ inline void join_singles(const PagedArgs& a, int group) {
  constexpr int kLanes = D / 8, kSubs = 64 / kLanes;
  const int tid = __builtin_amdgcn_workitem_id_x(), lane = tid & 63;
  const int ch = lane % kLanes, sub = lane / kLanes;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row = kTogether ? group : group * kPgWaves + wv;
  const int e = a.fheads.div(row), head = row - e * a.H;
  if (e >= a.singles) return;
  Token tk;
  const bool there = single_token<kMixed>(a, e, lane, tk);
  if (kMixed && !there) return;  // a row of join_tiles, if of any
  // How many partials each pattern has of the row, a pattern per lane, and
  // their running sum: partial c is slot first + c of the pattern with upto > c.
  static_assert(DA_MAX_PATTERNS == 16, "a pattern per lane");
  const PagedPattern P = a.pat[lane & 15];
  int upto = 0, first = 0;
  if (there && (lane & 15) < a.npat) {
    const Lattice x = lattice_of(P, tk.pos);
    if (head_offset(P, head) == x.rho) {
      const int n = own_keys(a, P, (lane & 15) == a.full, tk.pos, x);
      upto = n > 0 ? (n - 1) / split_keys_of(P, n) + 1 : 0;
    }
  }
  first = P.one_slot + upto;
#pragma unroll
  for (int x = 1; x < 16; x <<= 1) {
    const int o = __shfl_up(upto, x, 16);
    if ((lane & 15) >= x) upto += o;
  }
  first -= upto;
  const int count = __builtin_amdgcn_readlane(upto, 15);
  const int64_t at = (static_cast<int64_t>(e) * a.H + head) * a.one_slots;
  const float* rec = reinterpret_cast<const float*>(a.ws + a.one_rec) + at;
  const float* part = reinterpret_cast<const float*>(a.ws + a.one_row) + at * D + ch * 8;
  Mix x;
  constexpr int kAtOnce = kTogether ? kSubs * kPgWaves : kSubs;
  for (int c0 = kTogether ? kSubs * wv : 0; c0 < count; c0 += kAtOnce) {
    const int c = c0 + sub;
    int slot = 0;
    for (int i = a.npat - 1; i >= 0; --i)
      if (c < __builtin_amdgcn_readlane(upto, i)) slot = __builtin_amdgcn_readlane(first, i) + c;
    if (c < count) x.add(rec[slot], 1.0f, *reinterpret_cast<const f32x8*>(part + static_cast<int64_t>(slot) * D));
  }
#pragma unroll
  for (int s = kLanes; s < 64; s <<= 1) x.meet(s);
  if constexpr (kTogether) {
    __shared__ __attribute__((aligned(16))) float rows[kPgWaves][D];
    __shared__ float ml[kPgWaves][2];
    if (sub == 0) *reinterpret_cast<f32x8*>(&rows[wv][ch * 8]) = x.acc;
    if (lane == 0) {
      ml[wv][0] = x.m;
      ml[wv][1] = x.l;
    }
    __syncthreads();
    if (wv != 0) return;
#pragma unroll
    for (int w = 1; w < kPgWaves; ++w) x.meet(ml[w][0], ml[w][1], [&](int i) { return rows[w][ch * 8 + i]; });
  }
  if (sub == 0) put_row<T, D>(a, tk.tok, head, ch, x);
}

// Tokens of tiles, and those of no sequence: D/8 lanes a row, head by head and
// token by token, the loads of all patterns before their use.  kPats bounds the
// patterns at compile time: 5, the length of the paper's list, or all 16, whose
// records and rows in flight take 186 registers instead of 76 (lists of up to 5 with
// the second form: 4096 tokens at 28672 79 us instead of 65, 512 at 31500 30 instead
// of 26; of six patterns it takes 27 us of 90, of eight 26 of 71).  kSubs such groups of lanes share a row, each with
// every kSubs-th split.
template <int D, int kPats, int kSubs>
__device__ inline void join_tiles(const PagedArgs& a, int group) {
  constexpr int kLanes = D / 8, kRows = kPgThreads / (kLanes * kSubs);
  const int tid = __builtin_amdgcn_workitem_id_x(), lane = tid & 63;
  const int ch = tid % kLanes, sub = tid / kLanes % kSubs;
  const int total = a.T * a.H, row = min(group * kRows + tid / (kLanes * kSubs), total - 1);
  const int tok = a.fheads.div(row), head = row - tok * a.H;
  // The sequences of the wave's first and last token; a wave across more looks
  // for each lane's.
  const int ends[2] = {__builtin_amdgcn_readfirstlane(tok), __builtin_amdgcn_readlane(tok, 63)};
  Sequence sq[2];
  find_sequences(a, ends, lane, sq);
  Sequence s = tok == ends[1] ? sq[1] : sq[0];
  if ((sq[0].b != sq[1].b || sq[0].b < 0) && tok != ends[0] && tok != ends[1]) {
    int lo = max(sq[0].b, 0), hi = sq[1].b < 0 ? a.B - 1 : sq[1].b;
    while (lo < hi) {  // the last sequence that begins at or before tok
      const int mid = (lo + hi + 1) >> 1;
      if (a.start[mid] <= tok) lo = mid;
      else hi = mid - 1;
    }
    s = Sequence{lo, a.start[lo], a.start[lo + 1], a.lens[lo]};
  }
  const int pos = tok >= s.begin ? position_of(a, s, tok) : -1;
  if (pos >= 0 && s.end - s.begin <= a.few) return;  // computed by itself
  Mix x;
  if (pos >= 0) {
    int64_t at[kPats];
    int splits = 0;
#pragma unroll
    for (int i = 0; i < kPats; ++i) {
      at[i] = -1;
      if (i >= a.npat) continue;
      const PagedPattern& P = a.pat[i];
      if (head_offset(P, head) != lattice_of(P, pos).rho) continue;
      at[i] = static_cast<int64_t>(P.tile_slot) * total + row;
      splits = max(splits, static_cast<int>(P.tile_split.d));
    }
    for (int sp = sub; sp < splits; sp += kSubs) {
      f32x2 rec[kPats];
      f16x8 o[kPats];
#pragma unroll
      for (int i = 0; i < kPats; ++i) {
        rec[i] = f32x2{-INFINITY, 0.0f};
        if (at[i] < 0 || sp >= static_cast<int>(a.pat[i].tile_split.d)) continue;
        const int64_t r = at[i] + static_cast<int64_t>(sp) * total;
        rec[i] = reinterpret_cast<const f32x2*>(a.ws + a.tile_rec)[r];
        o[i] = *reinterpret_cast<const f16x8*>(a.ws + a.tile_row + (r * D + ch * 8) * 2);
      }
#pragma unroll
      for (int i = 0; i < kPats; ++i) {
        if (no_row(rec[i][0])) continue;
        f32x8 f;
#pragma unroll
        for (int c = 0; c < 8; ++c) f[c] = static_cast<float>(o[i][c]);
        x.add(rec[i][0], rec[i][1], f);
      }
    }
  }
#pragma unroll
  for (int m = kLanes; m < kLanes * kSubs; m <<= 1) x.meet(m);
  if (sub == 0 && group * kRows + tid / (kLanes * kSubs) < total) put_row<u16, D>(a, tok, head, ch, x);
}

// kTogether: the waves of a workgroup share a single token's row.
template <typename T, int D, bool kTogether>
__global__ __launch_bounds__(kPgThreads) void paged_join(PagedArgs a) {
  touch(a);
  join_singles<T, D, false, kTogether>(a, launch_index());
}
// The rows of tiles first, then the single tokens'.
template <int D, int kPats, int kSubs>
__global__ __launch_bounds__(kPgThreads) void paged_join_all(PagedArgs a) {
  touch(a);
  const int group = launch_index();
  if (group < a.join_groups) join_tiles<D, kPats, kSubs>(a, group);
  else join_singles<u16, D, true, false>(a, group - a.join_groups);
}

// Rows of single tokens: a workgroup each below this many (tens of partials
// that one wave reads in several rounds: 12 rows of a token at 32K tokens took
// 10.0 us a wave each, 5.6 a workgroup each), a wave each from there.
constexpr int64_t kShared = 512;
// Rows of tiles: lane groups that share one whose keys are split, up to this many
// rows (6144 rows of 4 to 6 splits 9.4 -> 6.8 us, 12180 of 4 splits 7.0 -> 9.4).
constexpr int kJoinSubs = 4;
constexpr int64_t kJoinShared = 8192;
template <typename T, int D>
void launch_join(int64_t rows, const PagedArgs& a, hipStream_t stream) {
  const dim3 threads(kPgThreads);
  if (rows < kShared) hipLaunchKernelGGL((paged_join<T, D, true>), grid_of(rows), threads, 0, stream, a);
  else hipLaunchKernelGGL((paged_join<T, D, false>), grid_of((rows + kPgWaves - 1) / kPgWaves), threads, 0, stream, a);
}

template <int D>
void launch_all(const PagedPlan& p, PagedArgs& a, hipStream_t stream) {
  const dim3 threads(kPgThreads), grid = grid_of(p.grid);
  const int64_t singles = p.singles * p.H;
  if (p.dtype == DA_F32) {
    hipLaunchKernelGGL(paged_one_f32<D>, grid, threads, 0, stream, a);
    launch_join<float, D>(singles, a, stream);
  } else if (p.all_few) {
    hipLaunchKernelGGL(paged_singles<D>, grid, threads, 0, stream, a);
    launch_join<u16, D>(singles, a, stream);
  } else {
    if (p.steps) hipLaunchKernelGGL(paged_mixed_steps<D>, grid, threads, 0, stream, a);
    else hipLaunchKernelGGL(paged_mixed<D>, grid, threads, 0, stream, a);
    const bool share = p.T * p.H <= kJoinShared && p.tile_slots > p.npat;
    const int64_t rows = kPgThreads / (D / 8) / (share ? kJoinSubs : 1);
    a.join_groups = static_cast<int32_t>((p.T * p.H + rows - 1) / rows);
    const dim3 join = grid_of(a.join_groups + (singles + kPgWaves - 1) / kPgWaves);
    constexpr int kMost = DA_MAX_PATTERNS;
    if (p.npat > 5 && share) hipLaunchKernelGGL((paged_join_all<D, kMost, kJoinSubs>), join, threads, 0, stream, a);
    else if (p.npat > 5) hipLaunchKernelGGL((paged_join_all<D, kMost, 1>), join, threads, 0, stream, a);
    else if (share) hipLaunchKernelGGL((paged_join_all<D, 5, kJoinSubs>), join, threads, 0, stream, a);
    else hipLaunchKernelGGL((paged_join_all<D, 5, 1>), join, threads, 0, stream, a);
  }
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
  a.few = static_cast<int32_t>(p.few);
  a.tile_items = static_cast<int32_t>(p.tile_items);
  a.grid = static_cast<int32_t>(p.grid);
  a.one_slots = static_cast<int32_t>(p.one_slots);
  a.reach = static_cast<uint32_t>(p.max_pages * p.page);
  a.one_items = static_cast<int32_t>(p.one_items);
  a.singles = static_cast<int32_t>(p.singles);
  a.fheads = make_fastdiv(static_cast<uint32_t>(p.H));
  a.scale_log2 = p.scale * kLog2e;
  std::copy(p.pat, p.pat + p.npat, a.pat);
  a.full = p.full;
  if (p.full >= 0) {
    a.full_w = p.pat[p.full].w;
    a.full_fw = p.pat[p.full].fw;
  }
  for (int i = 0; i < DA_MAX_PATTERNS; ++i) {
    a.one_begin[i] = i < p.npat ? p.pat[i].one_begin : 0x7fffffff;
    a.tile_begin[i] = i < p.npat ? p.pat[i].tile_begin : 0x7fffffff;
  }
  if (p.D == 32) launch_all<32>(p, a, stream);
  else if (p.D == 64) launch_all<64>(p, a, stream);
  else launch_all<128>(p, a, stream);
  return hipGetLastError();
}

}  // namespace da
