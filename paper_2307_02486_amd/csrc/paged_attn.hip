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
// where it is short (4096 tokens at 28672, five patterns: 31.9 GFLOP in 56 us, launch
// after launch; 65 to 69 in the first ones after a pause).
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

#include "heads_device.h"
#include "paged_device.h"

namespace da {
namespace {

constexpr float kLowest = -3.402823466e38f;  // a running maximum of no score: the lowest finite value
constexpr float kSumSlack = 1024.0f;  // a half row's sum above it moves its reference (tiles)
constexpr float kSlack = 8.0f;       // a score this far above its row's reference (log2) moves it

struct PagedArgs {
  const void* q;
  const char *kc, *vc;
  const uint8_t *ks, *vs;  // 8-bit caches: the blocks' scales
  const int32_t *table, *lens, *start;
  char* ws;
  void* out;
  float* lse;
  int64_t qs;  // elements between tokens of q
  int64_t one_rec, one_row, tile_rec, tile_row;  // byte offsets in the workspace
  int32_t T, B, H, Hkv, G, npat, num_pages, max_pages, page_log2, block_log2;
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
    // Up to 63 sequences are searched in one round of loads.  Of more, row e is most often
    // sequence e's only one: that much in one round, with the search's first entries
    // for where it is not.  (64 tokens of as many sequences, 1K to 32K cached: searched
    // 75.8 us, so 73.0, with an empty sequence before them 75.9; with the search's
    // entries requested after a guess that fails 76.6, and guessed of any number of
    // sequences four tokens of each of four 28.3 instead of 27.4.)
    int start = a.start[min(lane, a.B)], len = a.lens[min(lane, a.B - 1)];
    const int tok[1] = {e};
    t.tok = e;
    Sequence guess{min(e, a.B - 1), 0, 0, 0};
    if (a.B >= 64) {
      guess.begin = a.start[guess.b];
      guess.end = a.start[guess.b + 1];
      guess.len = a.lens[guess.b];
    }
    here(start);
    here(len);
    if (guess.begin == e && guess.end == e + 1) sq[0] = guess;
    else find_sequences(a, tok, lane, start, len, sq);
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

// What a single-token item has to do: a token, the query heads of a key head that
// share its keys, and the split [k0, ke) of these.
struct OneWork {
  Token tk;
  Lattice lat;
  KeptHeads kh;
  int hk, m0, rows, k0, ke;  // key head; first of its kept query heads here and how many
};
template <bool kMixed>
__device__ inline bool one_work(const PagedArgs& a, const OneItem& it, int lane, OneWork& w) {
  const PagedPattern& P = a.pat[it.pi];
  if (!single_token<kMixed>(a, it.e, lane, w.tk)) return false;
  w.lat = lattice_of(P, w.tk.pos);
  // Dilations of a group's size and above keep one head of a group at most: the
  // head-th kept one; below, every group has some, in blocks.
  int block = 0;
  w.hk = it.head;
  if (P.r >= a.G) {
    const int64_t h = w.lat.rho + static_cast<int64_t>(it.head) * P.r;
    if (h >= a.H) return false;
    w.hk = static_cast<int>(h) / a.G;
  } else if (a.G > static_cast<int>(kPagedGroupRows)) {
    block = it.head / a.Hkv;
    w.hk = it.head - block * a.Hkv;
  }
  w.kh = kept_heads(P, w.hk, a.G, w.lat.rho);
  w.m0 = block * static_cast<int>(kPagedGroupRows);
  if (w.m0 >= w.kh.count) return false;
  w.rows = min(static_cast<int>(kPagedGroupRows), w.kh.count - w.m0);
  const int n = own_keys(a, P, it.pi == a.full, w.tk.pos, w.lat), per = split_keys_of(P, n);
  w.k0 = it.split * per;
  w.ke = min(w.k0 + per, n);
  return w.k0 < n;
}
// Patterns whose keys this item reads too, for any head of it and for the lane's.
struct Shared {
  unsigned with, mine;
};
__device__ inline Shared shared_patterns(const PagedArgs& a, const OneItem& it, const OneWork& w, int lane) {
  Shared x{0, 0};
  if (it.pi != a.full || a.npat == 1) return x;
  const PagedPattern Q = a.pat[lane & 15];  // a pattern per lane
  const bool there = lane < a.npat && lane != it.pi;
  const int rho = there ? lattice_of(Q, w.tk.pos).rho : 0;
  for (int r = 0; r < w.rows; ++r) {
    const bool kept = there && head_offset(Q, w.kh.first + (w.m0 + r) * a.pat[it.pi].r) == rho;
    const unsigned mask = static_cast<unsigned>(__ballot(kept));
    x.with |= mask;
    if ((lane & 15) == r) x.mine = mask;
  }
  return x;
}

// The waves' partial rows (acc, reference m_run and sum l_run) meet in LDS, each in
// its wave's own V tile, and go to the workspace.
template <int D>
__device__ inline void store_one(const PagedArgs& a, const OneItem& it, const OneWork& work, const f32x4 (&acc)[D / 16],
                                 float m_run, float l_run, char (&sv)[kPgWaves][kOneTile * D * 2],
                                 float (&sml)[kPgWaves][2][16], int tid, int wv) {
  constexpr int DB = D / 16;
  // Joined rows are D floats apart, 16-byte chunk c of row r at c ^ (r mod D/4).
  auto join_at = [](int r, int chunk) { return r * D + 4 * (chunk ^ (r & (D / 4 - 1))); };
  static_assert(16 * D * 4 <= kOneTile * D * 2, "the join fits a wave's V tile");
  const PagedPattern& P = a.pat[it.pi];
  const int lane = tid & 63, m = lane & 15, grp = lane >> 4;
  l_run = sum_over_groups(l_run);
  float* jo = reinterpret_cast<float*>(sv[wv]);
#pragma unroll
  for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4*>(jo + join_at(m, 4 * db + grp)) = acc[db];
  if (grp == 0) {
    sml[wv][0][m] = m_run;
    sml[wv][1][m] = l_run;
  }
  __syncthreads();
  const int64_t row0 = static_cast<int64_t>(it.e) * a.H;
  for (int x = tid; x < work.rows * (D / 4); x += kPgThreads) {
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
    const int64_t at = (row0 + work.kh.first + (work.m0 + r) * P.r) * a.one_slots + P.one_slot + it.split;
    o *= l > 0.0f ? 1.0f / l : 0.0f;
    *reinterpret_cast<f32x4*>(a.ws + a.one_row + (at * D + d) * 4) = o;
    if (d == 0) reinterpret_cast<float*>(a.ws + a.one_rec)[at] = mt + __builtin_amdgcn_logf(l);
  }
}

template <int D, bool kMixed>
__device__ inline void single_tokens(const PagedArgs& a, const OneItem& it, SmemOne<D>& sm) {
  constexpr int KC = D / 32, DB = D / 16, kTile = kOneTile;
  using TL = TileLayout<D>;
  constexpr int kVLoads = kTile * TL::kSlots / 64;
  const int tid = thread_id(), lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  OneWork w;
  if (!one_work<kMixed>(a, it, lane, w)) return;
  const PagedPattern& P = a.pat[it.pi];
  const Token& tk = w.tk;
  const int hk = w.hk, rows = w.rows, k0 = w.k0, ke = w.ke;

  const int m = lane & 15, grp = lane >> 4;
  const int head = w.kh.first + (w.m0 + min(m, rows - 1)) * P.r;
  // Q^T operand (kept in LDS: in registers it would spill at D = 128).
  for (int c = wv; c < KC; c += kPgWaves) {
    const u32x4 x = load16(static_cast<const u16*>(a.q) + tk.tok * a.qs + head * D + 32 * c + 8 * grp);
    sm.q[c][lane] = m < rows ? x : u32x4{0u, 0u, 0u, 0u};
  }

  const int32_t* table = a.table + static_cast<int64_t>(tk.b) * a.max_pages;
  const int base = w.lat.first;
  const Shared shared = shared_patterns(a, it, w, lane);
  const unsigned with = shared.with, mine = shared.mine;
  char* my = sm.v[wv];
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

  constexpr int kVStep = 64 / TL::kSlots;  // V rows of a load
  const int vrow = lane / TL::kSlots;
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
    look_up_rows<4, false>(a, table, hk, base, P.r, c0, ke - 1, ntile * kTile, tid, sm.row, nullptr);
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

  store_one<D>(a, it, w, acc, m_run, l_run, sm.v, sm.ml, tid, wv);
}

// 8-bit caches.  A wave takes 64 keys at a time, as many bytes under way as with 32
// wide ones, and finds its own keys' rows, so that the waves meet at the end only.
// Tiles without a page are passed over.  64 tokens at 1K to 32K cached, five patterns,
// 139 MB: 47 us (32 keys at a time, rows by the workgroup: 61); with every key in one page,
// from the L2, 28; loads and nothing else 41.  So it is the start of an item (4 us: lengths,
// table, keys, one after the other) and the tail of the launch more than HBM.  Not
// faster: an item a wave (46 to 60 us at 256 to 1024 keys each), one query head's products
// on the vector ALU (45), the patterns' items mixed, twice or half the splits.
constexpr int kOneKeys = 64;   // keys of a wave's tile
constexpr int kOneAhead = 4;   // its tiles whose rows are looked up at once
template <int D>
struct SmemOne8 {
  __attribute__((aligned(16))) char v[kPgWaves][kOneTile * D * 2];  // each wave's V tile, 32 keys at a time
  float ml[kPgWaves][2][16];
  u32x4 q[kPgWaves][D / 32][64];                 // Q^T operand, lane by lane
  uint32_t row[kPgWaves][kOneAhead][kOneKeys];  // cache rows of the wave's keys
};

template <int D, bool kMixed>
__device__ inline void single_tokens8(const PagedArgs& a, const OneItem& it, SmemOne8<D>& sm) {
  constexpr int KC = D / 32, DB = D / 16, KU = kOneKeys / 16;
  constexpr int kPieces = D / 16;             // 16-byte pieces of a row
  constexpr int kHalfV = 32 * kPieces / 64;   // loads of 32 rows of V
  constexpr int kVStep = 64 / kPieces;        // rows of a load
  using TL = TileLayout<D>;
  const int tid = thread_id(), lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  OneWork w;
  if (!one_work<kMixed>(a, it, lane, w)) return;
  const PagedPattern& P = a.pat[it.pi];
  const int ke = w.ke, base = w.lat.first;
  const int m = lane & 15, grp = lane >> 4;
  const int32_t* table = a.table + static_cast<int64_t>(w.tk.b) * a.max_pages;
  char* my = sm.v[wv];
  u32x4(&q)[KC][64] = sm.q[wv];

  f32x4 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = f32x4{0, 0, 0, 0};
  float m_run = kLowest, l_run = 0.0f;
  const float c2 = a.scale_log2;
  Shared shared{0, 0};
  for (int c0 = w.k0; c0 < ke; c0 += kPgWaves * kOneAhead * kOneKeys) {
    // The rows of the wave's tiles, a key a lane; which keys have no page.
    int pos[kOneAhead], entry[kOneAhead];
#pragma unroll
    for (int t = 0; t < kOneAhead; ++t) {
      pos[t] = base + min(c0 + (t * kPgWaves + wv) * kOneKeys + lane, ke - 1) * P.r;
      entry[t] = table_entry(a, table, pos[t]);
    }
    if (c0 == w.k0) {  // meanwhile
      const int head = w.kh.first + (w.m0 + min(m, w.rows - 1)) * P.r;
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        const u32x4 x = load16(static_cast<const u16*>(a.q) + w.tk.tok * a.qs + head * D + step_first<D>(c, grp));
        q[c][lane] = m < w.rows ? x : u32x4{0u, 0u, 0u, 0u};
      }
      shared = shared_patterns(a, it, w, lane);
    }
    uint32_t left = 0, gone_lo = 0, gone_hi = 0;  // tiles with keys; lane t: tile t's keys without a page
#pragma unroll
    for (int t = 0; t < kOneAhead; ++t) {
      const uint32_t row = cache_row(a, entry[t], w.hk, pos[t]);
      const uint64_t word = __ballot(static_cast<uint32_t>(entry[t]) >= static_cast<uint32_t>(a.num_pages));
      if (c0 + (t * kPgWaves + wv) * kOneKeys < ke && ~word != 0) left |= 1u << t;
      // A key without a page has the row of one that is there: what it holds is the
      // sequence's own, and a weight of zero times it is zero.
      const uint32_t some = read_lane(row, ~word != 0 ? __builtin_ctzll(~word) : 0);
      sm.row[wv][t][lane] = word >> lane & 1 ? some : row;
      if (lane == t) {
        gone_lo = static_cast<uint32_t>(word);
        gone_hi = static_cast<uint32_t>(word >> 32);
      }
    }
    if (!left) continue;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the rows are in LDS (a wave's operations complete in order)
    __builtin_amdgcn_wave_barrier();
    // V^T operand: lane's d = 16 db + (lane & 15), keys 4 grp + 0..3 and 16 more.
    const int tr_r = 4 * grp + ((lane & 15) >> 2), tr_d = (lane & 3) * 4;
    const uint32_t voff = TL::offset(tr_r, tr_d >> 3) + (tr_d & 7) * 2;
    const int vrow = lane / kPieces, vpiece = lane % kPieces;
    // A tile's K leaves its registers with its scores and the next tile's K is then
    // requested into them, V when its second half is in LDS.
    KeyFrag8<D> kf[KU / 2];
    u32x4 vreg[2 * kHalfV];
    uint32_t vscale[2 * kHalfV];
    auto request_k = [&](int t) {
#pragma unroll
      for (int h = 0; h < KU / 2; ++h) request_keys8<D>(a, sm.row[wv][t] + 32 * h, m, grp, kf[h]);
    };
    auto request_v = [&](int t) {
#pragma unroll
      for (int i = 0; i < 2 * kHalfV; ++i) {
        const uint32_t row = sm.row[wv][t][kVStep * i + vrow];
        vreg[i] = *reinterpret_cast<const u32x4*>(a.vc + (static_cast<int64_t>(row) * D + vpiece * 16));
        vscale[i] = a.vs[row >> a.block_log2];
      }
    };
    // The wave's tile t, and if `more`, requests for its tile `next`.
    auto compute = [&](auto more, int t, int next) {
      constexpr bool kMore = decltype(more)::value;
      const int first = c0 + (t * kPgWaves + wv) * kOneKeys;
      f32x4 s[KU];
#pragma unroll
      for (int u = 0; u < KU; ++u) {
        const KeyFrag8<D>& k = kf[u >> 1];
        s[u] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k.wide(u & 1, c)),
                                                         __builtin_bit_cast(bf16x8, q[c][lane]), s[u], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);  // K is widened 16 keys at a time
      }
      __builtin_amdgcn_sched_barrier(0);  // K's registers are free from here on
      if constexpr (kMore) request_k(next);
      __builtin_amdgcn_sched_barrier(0);
      // Keys past the split and those of no page.
      const uint32_t gone[2] = {static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(gone_lo), t)),
                                static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(gone_hi), t))};
      if (first + kOneKeys > ke || (gone[0] | gone[1])) {
        const int left = ke - first - 4 * grp;
#pragma unroll
        for (int u = 0; u < KU; ++u) {
          const uint32_t out = gone[u >> 1] >> (16 * (u & 1) + 4 * grp);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (16 * u + e >= left || (out >> e & 1)) s[u][e] = -INFINITY;
        }
      }
      float mx = s[0][0];
#pragma unroll
      for (int u = 0; u < KU; ++u)
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
#pragma unroll
      for (int u = 0; u < KU; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[u][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][e], c2, -m_run));
      if (shared.with) {  // times the patterns that hold a key, a byte for each of four keys
        uint32_t count[KU];
#pragma unroll
        for (int u = 0; u < KU; ++u) count[u] = 0x01010101u;
        for (unsigned rest = shared.with; rest; rest &= rest - 1) {
          const int i = __builtin_ctz(rest);
          const PagedPattern& Q = a.pat[i];
          const int d0 = base + first - lattice_of(Q, w.tk.pos).first;
          const uint32_t row_keeps = shared.mine >> i & 1 ? 0x01010101u : 0u;
          // of four keys from a multiple of r on, those that are multiples
          const uint32_t comb = Q.r == 1 ? 0xf : Q.r == 2 ? 0x5 : Q.r == 3 ? 0x9 : 0x1;
#pragma unroll
          for (int u = 0; u < KU; ++u) {
            const int x = d0 + 4 * grp + 16 * u;
            const int over = max(x, 0) - static_cast<int>(Q.fr.div(max(x, 0))) * Q.r;
            int ahead = over > 0 ? Q.r - over : 0;  // to the next multiple
            if (x < 0) ahead = -x;                  // to the pattern's first key
            const uint32_t hits = ahead < 4 ? comb << ahead & 0xf : 0u;
            count[u] += hits * 0x00204081u & row_keeps;  // bit e to the lowest of byte e
          }
        }
#pragma unroll
        for (int u = 0; u < KU; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[u][e] *= static_cast<float>(count[u] >> (8 * e) & 0xff);
      }
      bf16x8 pb[2];
#pragma unroll
      for (int u = 0; u < KU; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          l_run += s[u][e];
          pb[u >> 1][4 * (u & 1) + e] = (__bf16)s[u][e];  // for the product alone
        }
      // V through the wave's own LDS tile, 32 keys at a time, to be read transposed
      // (LDS operations of a wave complete in order: no wait between).
      const uint32_t va = lds_addr(my);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        __builtin_amdgcn_sched_barrier(0);  // V is widened here, not before
#pragma unroll
        for (int i = 0; i < kHalfV; ++i) {
          const u32x4 x = vreg[h * kHalfV + i];
          const float scale = scale_of(vscale[h * kHalfV + i]);
          *reinterpret_cast<u32x4*>(my + TL::offset(kVStep * i + vrow, 2 * vpiece)) = widen8(x[0], x[1], scale);
          *reinterpret_cast<u32x4*>(my + TL::offset(kVStep * i + vrow, 2 * vpiece + 1)) = widen8(x[2], x[3], scale);
        }
        if constexpr (kMore) {
          if (h == 1) request_v(next);
        }
        constexpr int kAtOnce = DB < 4 ? DB : 4;  // blocks whose V is read at once
#pragma unroll
        for (int d0 = 0; d0 < DB; d0 += kAtOnce) {
          u32x2 vf[kAtOnce][2];
#pragma unroll
          for (int x = 0; x < kAtOnce; ++x) {
            const uint32_t at = va + (voff ^ ((d0 + x) << 5));
            vf[x][0] = lds_read_tr16<0>(at);
            vf[x][1] = lds_read_tr16<16 * TL::kRowBytes>(at);
          }
          lds_wait<0>();
#pragma unroll
          for (int x = 0; x < kAtOnce; ++x) {
            lds_bind(vf[x][0]);
            lds_bind(vf[x][1]);
            const u32x4 v4 = {vf[x][0][0], vf[x][0][1], vf[x][1][0], vf[x][1][1]};
            acc[d0 + x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v4), pb[h], acc[d0 + x], 0, 0, 0);
          }
        }
      }
    };
    int tile = __builtin_ctz(left);
    request_k(tile);
    request_v(tile);
    for (left &= left - 1; left; left &= left - 1) {
      const int next = __builtin_ctz(left);
      compute(std::true_type{}, tile, next);
      tile = next;
    }
    compute(std::false_type{}, tile, 0);  // at every wait it is known which loads are younger
  }
  store_one<D>(a, it, w, acc, m_run, l_run, sm.v, sm.ml, tid, wv);
}

// Four e4m3 values of a row times its scale, in float32.
__device__ inline f32x4 widen4(uint32_t w, float scale) {
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  return f32x4{lo[0] * scale, lo[1] * scale, hi[0] * scale, hi[1] * scale};
}

// float32: a workgroup is one (token, query head, pattern, split).  D/4 lanes
// hold a row, each group of them its own keys and running softmax; the groups
// and waves meet in LDS.
template <int D, bool kF8>
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
    bool gone[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int t = min(t0 + u * kGroups + grp, ke - 1);
      const int pos = base + t * P.r;
      if constexpr (kF8) {
        const int entry = table_entry(a, table, pos);
        gone[u] = static_cast<uint32_t>(entry) >= static_cast<uint32_t>(a.num_pages);
        const uint32_t row = cache_row(a, gone[u] ? 0 : entry, hk, pos);
        const int64_t at = static_cast<int64_t>(row) * D + 4 * ch;
        k[u] = widen4(*reinterpret_cast<const uint32_t*>(a.kc + at), scale_of(a.ks[row >> a.block_log2]));
        const uint32_t word = *reinterpret_cast<const uint32_t*>(a.vc + at), byte = a.vs[row >> a.block_log2];
        v[u] = widen4(gone[u] ? 0u : word, scale_of(gone[u] ? 127u : byte));  // (0 times what is there may be NaN)
        continue;
      }
      gone[u] = false;
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
      s[u] = t0 + u * kGroups + grp < ke && !gone[u] ? d * a.scale_log2 : -INFINITY;
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

// Keys whose rows are looked up at once (three workgroups of D = 64 fit a CU, two of D = 128).
template <bool kF8>
constexpr int kTileRows = kF8 ? 2048 : 4096;

template <int D, bool kF8>
struct SmemTile {
  __attribute__((aligned(16))) u16 k[2][kPagedKeyTile * D];
  __attribute__((aligned(16))) u16 v[2][kPagedKeyTile * D];
  uint32_t row[kTileRows<kF8>];  // cache rows of the keys, a chunk at a time
  uint64_t gone[kF8 ? kTileRows<kF8> / 64 : 0];  // their keys of no page
};

template <int D, bool kF8>
__device__ inline void query_tiles(const PagedArgs& a, const TileItem& it, SmemTile<D, kF8>& sm) {
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
  // 8-bit caches: a thread has a quarter of a row of K and of V, whose loads are
  // under way while a tile is computed; they go to LDS as bf16, once for the four
  // waves that read the tile.  (4096 tokens at 28672, five patterns: 60 us, and 56 with
  // a wide cache, whose rows go to LDS by themselves: 16 conversions and four stores a
  // thread and tile beside 32 exponentials.  Without rows and missing pages read a
  // tile ahead the call takes 77.0 us where it takes 75.5.)
  constexpr int kPieces = D > 32 ? D / 64 : 1;  // 16-byte loads (D = 32: of 8 bytes) of a thread's quarter
  const int brow = tid >> 2, bpart = tid & 3;
  uint32_t kbytes[kPieces * 4], vbytes[kPieces * 4], kscale = 0, vscale = 0;
  auto request_tile = [&](uint32_t row) {
    const char* kp = a.kc + (static_cast<int64_t>(row) * D + (D > 32 ? 16 : 8) * bpart);
    const char* vp = a.vc + (static_cast<int64_t>(row) * D + (D > 32 ? 16 : 8) * bpart);
    if constexpr (D == 32) {
      const u32x2 x = *reinterpret_cast<const u32x2*>(kp), y = *reinterpret_cast<const u32x2*>(vp);
      kbytes[0] = x[0], kbytes[1] = x[1], vbytes[0] = y[0], vbytes[1] = y[1];
    } else {
#pragma unroll
      for (int p = 0; p < kPieces; ++p) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(kp + 64 * p), y = *reinterpret_cast<const u32x4*>(vp + 64 * p);
#pragma unroll
        for (int i = 0; i < 4; ++i) kbytes[4 * p + i] = x[i], vbytes[4 * p + i] = y[i];
      }
    }
    kscale = a.ks[row >> a.block_log2];
    vscale = a.vs[row >> a.block_log2];
  };
  auto store_tile = [&](const uint32_t (&gone)[2], int buf) {
    if ((brow < 32 ? gone[0] : gone[1]) >> (brow & 31) & 1) {  // zeros, as a weight of zero times whatever the pool holds there may be NaN
#pragma unroll
      for (int i = 0; i < kPieces * 4; ++i) vbytes[i] = 0;
      vscale = 127;
    }
    char* kl = reinterpret_cast<char*>(&sm.k[buf][0]);
    char* vl = reinterpret_cast<char*>(&sm.v[buf][0]);
    const float ksc = scale_of(kscale), vsc = scale_of(vscale);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {  // eight elements each: slot bpart, or two of 4 p + bpart
      const int slot = D == 32 ? bpart : 2 * (bpart + 4 * (i >> 1)) + (i & 1);
      const int at = TL::offset(brow, slot);
      *reinterpret_cast<u32x4*>(kl + at) = widen8(kbytes[2 * i], kbytes[2 * i + 1], ksc);
      *reinterpret_cast<u32x4*>(vl + at) = widen8(vbytes[2 * i], vbytes[2 * i + 1], vsc);
    }
  };
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
  for (int c0 = kb; c0 < ke; c0 += kTileRows<kF8>) {
    const int ntile = (min(ke - c0, kTileRows<kF8>) + BN - 1) / BN;
    look_up_rows<8, kF8>(a, table, hk, base, P.r, c0, ke - 1, ntile * BN, tid, sm.row, sm.gone);
    __syncthreads();
    // 8 bits, read a tile ahead: the thread's row, and the keys without a page.
    uint32_t row_next = 0, gone[2] = {0, 0};
    uint64_t gone_next = 0;
    auto keep_gone = [&] {
      gone[0] = uniform(static_cast<uint32_t>(gone_next));
      gone[1] = uniform(static_cast<uint32_t>(gone_next >> 32));
    };
    if constexpr (kF8) {
      request_tile(sm.row[brow]);
      gone_next = sm.gone[0];
      row_next = sm.row[(ntile > 1 ? BN : 0) + brow];
      keep_gone();
      store_tile(gone, 0);
    } else {
      load_tile(0, 0);
      wait_loads<0>();
    }
    __syncthreads();
    for (int jt = 0; jt < ntile; ++jt) {
      const int cur = jt & 1, k0 = c0 + jt * BN;
      if (jt + 1 < ntile) {
        if constexpr (kF8) {
          request_tile(row_next);
          gone_next = sm.gone[jt + 1];
          row_next = sm.row[min(jt + 2, ntile - 1) * BN + brow];
        } else {
          load_tile(jt + 1, cur ^ 1);
        }
      }
      const char* kl = reinterpret_cast<const char*>(&sm.k[cur][0]);
      const char* vl = reinterpret_cast<const char*>(&sm.v[cur][0]);
      // not all keys after this wave's queries, nor without a page
      if (k0 <= wq_lo + 31 && wq_lo < qend && (gone[0] & gone[1]) != 0xffffffffu) {
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
        if constexpr (kF8) {  // keys of no page
          if (gone[0] | gone[1]) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const uint32_t mine = gone[x] >> (4 * hi);
#pragma unroll
              for (int j = 0; j < 16; ++j)
                if (mine >> (8 * (j >> 2) + (j & 3)) & 1) acc_s[x][j] = -INFINITY;
            }
          }
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
      if constexpr (kF8) {
        keep_gone();
        if (jt + 1 < ntile) store_tile(gone, cur ^ 1);
      } else {
        wait_loads<0>();
      }
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

template <int D, bool kF8>
using SmemSingle = typename std::conditional<kF8, SmemOne8<D>, SmemOne<D>>::type;
template <int D, bool kMixed, bool kF8>
__device__ inline void one_tokens(const PagedArgs& a, const OneItem& it, SmemSingle<D, kF8>& sm) {
  if constexpr (kF8) single_tokens8<D, kMixed>(a, it, sm);
  else single_tokens<D, kMixed>(a, it, sm);
}

// Every token a single one.
template <int D, bool kF8>
__global__ __launch_bounds__(kPgThreads, D == 128 ? 2 : kF8 ? 4 : 3) void paged_singles(PagedArgs a) {
  __shared__ SmemSingle<D, kF8> sm;
  touch(a);
  const int idx = launch_index();
  if (idx >= a.one_items) return;
  const int pi = pattern_at(a.one_begin, idx);
  OneItem it;
  if (one_item(a, pi, idx - a.pat[pi].one_begin, a.singles, it)) one_tokens<D, false, kF8>(a, it, sm);
}

template <int D, bool kF8>
union SmemMixed {
  SmemTile<D, kF8> tile;
  SmemSingle<D, kF8> one;
  int count[DA_MAX_PATTERNS + 1];
};

// Tiles and single tokens in one launch, the tiles first, as they take longer:
// every item that the sizes allow.
template <int D, bool kF8>
__global__ __launch_bounds__(kPgThreads, D == 128 ? 2 : 3) void paged_mixed(PagedArgs a) {
  __shared__ SmemMixed<D, kF8> sm;
  touch(a);
  const int idx = launch_index();
  if (idx < a.tile_items) {
    const int pi = pattern_at(a.tile_begin, idx);
    const PagedPattern& P = a.pat[pi];
    TileItem it;
    if (tile_item(a, pi, idx - P.tile_begin, P.tiles, P.run, P.tile_split.d, it)) query_tiles<D, kF8>(a, it, sm.tile);
  } else if (idx - a.tile_items < a.one_items) {
    const int pi = pattern_at(a.one_begin, idx - a.tile_items);
    OneItem it;
    if (one_item(a, pi, idx - a.tile_items - a.pat[pi].one_begin, a.singles, it)) one_tokens<D, true, kF8>(a, it, sm.one);
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
template <int D, bool kF8>
__global__ __launch_bounds__(kPgThreads) void paged_mixed_steps(PagedArgs a) {
  __shared__ SmemMixed<D, kF8> sm;
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
        query_tiles<D, kF8>(a, it, sm.tile);
    } else if (item < all_items) {
      const int pi = __builtin_ctzll(__ballot(one_end > item - tile_items));
      const int begin = tile_items + __builtin_amdgcn_readlane(one_end, pi) - __builtin_amdgcn_readlane(ones, pi);
      OneItem it;
      if (one_item(a, pi, item - begin, tokens, it)) one_tokens<D, true, kF8>(a, it, sm.one);
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
__device__ inline bool not_finite(float x) { return (bits_of(x) & 0x7f800000u) == 0x7f800000u; }
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

// Elements 8 ch .. of one row's out from its log-sum-exp (log2 units), key by key in
// float32, by the D/8 lanes of the row.  For rows that tiles leave with something that is
// not finite: a tile multiplies V by probabilities of zero where a row does not see a
// key, and zero times a V that is not finite is NaN.  (Rows that see the key come out with
// it once more.  4096 tokens at 28672, one of them with NaN in each head: 7 ms, where
// without it the call takes 0.078, with the look at a row's sums or without.  Two keys at
// a time: with four the join holds more registers, and that call takes 0.079.)
template <int D>
__device__ inline f32x8 row_by_keys(const PagedArgs& a, int b, int tok, int head, int ch, int pos, float lse2) {
  constexpr int kUnroll = 2;
  const int32_t* table = a.table + static_cast<int64_t>(b) * a.max_pages;
  const int hk = head / a.G;
  float q[8];
  unpack(load16(static_cast<const u16*>(a.q) + tok * a.qs + head * D + ch * 8), q);
  f32x8 acc = f32x8{0, 0, 0, 0, 0, 0, 0, 0};
  for (int i = 0; i < a.npat; ++i) {
    const PagedPattern& P = a.pat[i];
    const Lattice x = lattice_of(P, pos);
    if (head_offset(P, head) != x.rho) continue;
    for (int t0 = 0; t0 < x.n; t0 += kUnroll) {
      float k[kUnroll][8], v[kUnroll][8];
      bool there[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int at = x.first + min(t0 + u, x.n - 1) * P.r, entry = table_entry(a, table, at);
        there[u] = t0 + u < x.n && (!a.ks || static_cast<uint32_t>(entry) < static_cast<uint32_t>(a.num_pages));
        const int64_t row = cache_row(a, entry, hk, at);
        if (a.ks) {
          const float ks = scale_of(a.ks[row >> a.block_log2]), vs = scale_of(a.vs[row >> a.block_log2]);
          const u32x2 kw = *reinterpret_cast<const u32x2*>(a.kc + row * D + ch * 8);
          const u32x2 vw = *reinterpret_cast<const u32x2*>(a.vc + row * D + ch * 8);
          unpack(widen8(kw[0], kw[1], ks), k[u]);
          unpack(widen8(vw[0], vw[1], vs), v[u]);
        } else {
          unpack(*reinterpret_cast<const u32x4*>(a.kc + (row * D + ch * 8) * 2), k[u]);
          unpack(*reinterpret_cast<const u32x4*>(a.vc + (row * D + ch * 8) * 2), v[u]);
        }
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        float d = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) d += q[e] * k[u][e];
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(row_sum<D / 8>(d), a.scale_log2, -lse2));
        if (there[u])
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[e] += p * v[u][e];
      }
    }
  }
  return acc;
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
  if (sub != 0 || group * kRows + tid / (kLanes * kSubs) >= total) return;
  float sum = x.acc[0];  // not finite if one of them is not
#pragma unroll
  for (int i = 1; i < 8; ++i) sum += x.acc[i];
  if (const uint64_t bad = __ballot(not_finite(sum)); __builtin_expect(bad != 0, false)) {
    const float lse2 = x.m + __builtin_amdgcn_logf(x.l);
    if ((bad >> (lane - ch) & ((uint64_t{1} << kLanes) - 1)) && !not_finite(lse2)) {
      x.acc = row_by_keys<D>(a, s.b, tok, head, ch, pos, lse2);
      x.m = lse2;
      x.l = 1.0f;
    }
  }
  put_row<u16, D>(a, tok, head, ch, x);
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

template <int D, bool kF8>
void launch_all(const PagedPlan& p, PagedArgs& a, hipStream_t stream) {
  const dim3 threads(kPgThreads), grid = grid_of(p.grid);
  const int64_t singles = p.singles * p.H;
  if (p.dtype == DA_F32) {
    hipLaunchKernelGGL((paged_one_f32<D, kF8>), grid, threads, 0, stream, a);
    launch_join<float, D>(singles, a, stream);
  } else if (p.all_few) {
    hipLaunchKernelGGL((paged_singles<D, kF8>), grid, threads, 0, stream, a);
    launch_join<u16, D>(singles, a, stream);
  } else {
    if (p.steps) hipLaunchKernelGGL((paged_mixed_steps<D, kF8>), grid, threads, 0, stream, a);
    else hipLaunchKernelGGL((paged_mixed<D, kF8>), grid, threads, 0, stream, a);
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

template <bool kF8>
void launch_cached(const PagedPlan& p, PagedArgs& a, hipStream_t stream) {
  if (p.D == 32) launch_all<32, kF8>(p, a, stream);
  else if (p.D == 64) launch_all<64, kF8>(p, a, stream);
  else launch_all<128, kF8>(p, a, stream);
}

}  // namespace

hipError_t launch_paged(const PagedPlan& p, const void* q, int64_t q_stride, const PagedCache& cache, void* out,
                        float* lse, void* workspace, hipStream_t stream) {
  PagedArgs a{};
  a.q = q;
  a.kc = static_cast<const char*>(cache.k);
  a.vc = static_cast<const char*>(cache.v);
  a.ks = cache.k_scale;
  a.vs = cache.v_scale;
  a.block_log2 = std::min(cache.page_log2, kCacheBlockLog2);
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
  if (cache.k_scale) launch_cached<true>(p, a, stream);
  else launch_cached<false>(p, a, stream);
  return hipGetLastError();
}

}  // namespace da
