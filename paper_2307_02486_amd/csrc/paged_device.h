// Device-side pieces of the operators on a paged cache: a call's sequences and
// positions, the key lattice of a pattern, the cache's rows and 8-bit values.
// Args: a kernel's arguments with the fields that are used (T, B, start, lens,
// reach, page_log2, num_pages, Hkv).
#pragma once

#include <hip/hip_runtime.h>

#include "device_common.h"
#include "paged.h"

namespace da {
namespace {

constexpr int kPgThreads = 256;
constexpr int kPgWaves = kPgThreads / 64;

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
__device__ inline int head_offset(const PagedPattern& P, int head) {
  return head - static_cast<int>(P.fr.div(head)) * P.r;
}

// The loads of these values begin before this point.  (A load whose value is used
// under a condition only would move there: another round to memory after those
// that the condition waits for.)
__device__ inline void here(int& v) { asm volatile("" : "+v"(v)); }

// This thread's number, opaque to the compiler: in the loop over a workgroup's
// items what follows from it would otherwise be formed before the loop and held
// in registers over all of it (which then spill).
__device__ inline int thread_id() {
  int tid = __builtin_amdgcn_workitem_id_x();
  asm volatile("" : "+v"(tid));
  return tid;
}

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
// round of loads, which the caller has begun: lane l's entries of start and lens.
template <typename Args, int kTokens>
__device__ inline void find_sequences(const Args& a, const int (&tok)[kTokens], int lane, int start, int len,
                                      Sequence (&sq)[kTokens]) {
  int n[kTokens];
#pragma unroll
  for (int i = 0; i < kTokens; ++i) n[i] = __popcll(__ballot(lane <= a.B && start <= tok[i]));
  for (int b0 = 64; b0 <= a.B; b0 += 64) {
    const int next = a.start[min(b0 + lane, a.B)];
#pragma unroll
    for (int i = 0; i < kTokens; ++i) n[i] += __popcll(__ballot(b0 + lane <= a.B && next <= tok[i]));
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
template <typename Args, int kTokens>
__device__ inline void find_sequences(const Args& a, const int (&tok)[kTokens], int lane, Sequence (&sq)[kTokens]) {
  const int start = a.start[min(lane, a.B)];
  int len = a.lens[min(lane, a.B - 1)];
  here(len);
  find_sequences(a, tok, lane, start, len, sq);
}

// Position of row tok of its sequence; -1 where it has none in the table.
template <typename Args>
__device__ inline int position_of(const Args& a, const Sequence& sq, int tok) {
  const int64_t p = static_cast<int64_t>(sq.len) - sq.end + tok;
  return sq.b >= 0 && tok < sq.end && p >= 0 && p < a.reach ? static_cast<int>(p) : -1;
}

// Entry i of start, held to the call's tokens: what a tile reads and writes stays in bounds.
template <typename Args>
__device__ inline int token_row(const Args& a, int i) { return max(0, min(a.start[i], a.T)); }

// A sequence's new tokens in the table: positions [c0, c1), that of position p in
// row tok0 + p of the call; none: c0 = c1.  Whatever the arrays hold, these rows
// and positions are there.
struct NewTokens {
  int c0, c1, tok0;
};
template <typename Args>
__device__ inline NewTokens new_tokens(const Args& a, int seq) {
  const int b = min(seq, a.B - 1), begin = token_row(a, b), end = token_row(a, b + 1);
  int len = a.lens[b];
  here(len);
  const int n = end - begin;
  const int c1 = static_cast<int>(min(static_cast<uint32_t>(max(len, 0)), a.reach));
  const int c0 = static_cast<int>(max(int64_t{0}, min(static_cast<int64_t>(len) - n, static_cast<int64_t>(c1))));
  return seq < a.B && n > 0 ? NewTokens{c0, c1, end - len} : NewTokens{0, 0, 0};
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
template <typename Args>
__device__ inline int table_entry(const Args& a, const int32_t* table, int pos) {
  return table[pos >> a.page_log2];
}
template <typename Args>
__device__ inline uint32_t cache_row(const Args& a, int entry, int hk, int pos) {
  const uint32_t page = min(static_cast<uint32_t>(entry), static_cast<uint32_t>(a.num_pages - 1));
  return ((page * a.Hkv + hk) << a.page_log2) + (pos & ((1 << a.page_log2) - 1));
}
// The cache rows of keys first .. first + n - 1 (positions base + t r) into row,
// by a workgroup; keys past `last` are that one.  kAtOnce entries of a thread
// are on their way together.  gone (8-bit caches): a bit for each key whose page
// is outside the pool, 64 keys a word; such a key's row is the pool's first.
template <int kAtOnce, bool kF8, typename Args>
__device__ inline void look_up_rows(const Args& a, const int32_t* table, int hk, int base, int r, int first,
                                    int last, int n, int tid, uint32_t* row, uint64_t* gone) {
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
    for (int u = 0; u < kAtOnce; ++u) {
      const int i = i0 + u * kPgThreads;
      if (i >= n) continue;
      row[i] = cache_row(a, entry[u], hk, pos[u]);
      if constexpr (kF8) {
        const bool out = static_cast<uint32_t>(entry[u]) >= static_cast<uint32_t>(a.num_pages);
        if (out) row[i] = 0;
        const uint64_t word = __ballot(out);  // the wave's keys are 64 side by side, from a multiple of 64 on
        if ((i & 63) == 0) gone[i >> 6] = word;
      }
    }
  }
}

// Eight e4m3 values of a row (two words) times the row's scale, as bf16: exact,
// as their four significant bits fit eight and scales are powers of two.
__device__ inline u32x4 widen8(uint32_t lo, uint32_t hi, float scale) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true))};
}
// x, the same in all lanes, in a scalar register.
__device__ inline uint32_t uniform(uint32_t x) {
  return static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(x)));
}
// Lane l's x, the same in all lanes.
__device__ inline uint32_t read_lane(uint32_t x, int l) {
  return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(x), l));
}
// A scale's byte is the exponent of the power of two that it stands for.
__device__ inline float scale_of(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

// A wave's 32 keys of an 8-bit cache on their way: two blocks of 16, words of the
// rows and the rows' scale bytes.
// (Whole vectors: word by word, a loop that has the next tile's on their way would
// copy them, and wait for them to.)
template <int D>
struct KeyFrag8 {
  typedef typename std::conditional<D == 32, u32x2, u32x4>::type Piece;
  static constexpr int kPer = D == 32 ? 2 : 4;  // words of a piece
  Piece k[2][D / 16 / kPer];
  uint32_t scale[2];
  __device__ uint32_t word(int u, int i) const { return k[u][i / kPer][i % kPer]; }
  // Step c of block u as bf16.
  __device__ u32x4 wide(int u, int c) const { return widen8(word(u, 2 * c), word(u, 2 * c + 1), scale_of(scale[u])); }
};
// Requests the 32 keys whose cache rows are row[key .. key + 31]: block u's key m =
// lane mod 16 in lanes m, m + 16, ..., 16 bytes of every 64 each (D = 32: 8 of 32).
// As an operand these are elements 64 c + 16 grp + 0 .. 15, eight for each of two
// steps (step_first): any order of d will do that the other operand has too.
template <int D, typename Args>
__device__ inline void request_keys8(const Args& a, const uint32_t* rows, int m, int grp, KeyFrag8<D>& kf) {
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const uint32_t row = rows[16 * u + m];
    const char* p = a.kc + (static_cast<int64_t>(row) * D + (D > 32 ? 16 : 8) * grp);
#pragma unroll
    for (int c = 0; c < D / 16 / KeyFrag8<D>::kPer; ++c)
      kf.k[u][c] = *reinterpret_cast<const typename KeyFrag8<D>::Piece*>(p + 64 * c);
    kf.scale[u] = a.ks[row >> a.block_log2];
  }
}
template <int D>
__device__ inline int step_first(int c, int grp) {  // first element of a lane's eight in step c
  return D > 32 ? 64 * (c >> 1) + 16 * grp + 8 * (c & 1) : 32 * c + 8 * grp;
}

}  // namespace
}  // namespace da
