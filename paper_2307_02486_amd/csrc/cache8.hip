// New keys and values into a paged cache in 8 bits, keys normed and rotated on
// the way, and the queries of the same tokens (heads.hip has the formulas of
// both).  A block of the cache is 2^block_log2 tokens of one key head; its values
// are e4m3 times one power of two 2^e, the least with
//   max |x| <= 448 * 2^e   (448: the largest e4m3 value),  e >= -126,
// so that no value is cut off and a value keeps four significant bits down to
// 2^-13 of the block's largest (e4m3 is normal from 2^-6 on, the largest is above 224),
// and is off by 2^-10 2^e at most below.  A block that has tokens already keeps its e or
// takes a larger one, its older values then multiplied by a power of two: exact,
// but for those that fall below e4m3's least normal value, which are rounded again.
//
// A workgroup is the new tokens of one block (16 at most), of a share of the
// heads: D/8 lanes hold a row, eight elements each, the block's rows of several
// heads at once; a head's largest value meets in LDS (a maximum of bits: in any
// order the same).  Further workgroups have the queries, a token a wave.
// Only rounding to fewer bits: keys and values to e4m3, once from float32 and again
// where a block's scale grows past them.
//
// Bound by HBM where there are many tokens: three prompts, 15 thousand tokens of 16
// heads of 128 and four key heads, 133 MB in 30 us (4.4 TB/s; the wide cache's append
// moves 145 MB in 29).  64 tokens of 64 sequences, one a block: 4.7 us, a chain of
// starts, table, rows and scales.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "heads_device.h"
#include "paged_device.h"

namespace da {
namespace {

constexpr int kApThreads = 256;
constexpr int kApWaves = kApThreads / 64;
constexpr int kApPasses = 4;  // rows of a workgroup in flight: this many times the lanes' groups
constexpr int kBlockMost = 1 << kCacheBlockLog2;

struct Append8Args {
  const void *q, *k, *v;  // rows of T tokens, heads side by side
  const void *qw, *kw;    // norm weights [D], or null: no norm
  void* qo;
  uint8_t *kc, *vc, *ks, *vs;
  const int32_t *table, *lens, *start;
  int64_t qs, kst, vst;   // elements between tokens
  int32_t T, B, H, Hkv, num_pages, page_log2, block_log2, max_pages, center;
  uint32_t reach;
  int32_t blocks, parts;  // bound on the blocks with new tokens; workgroups of a block
  float eps;
};

// The bits of |x|, as the compiler cannot see through (it takes floats for
// numbers), zero for infinities and NaN.
__device__ inline uint32_t size_of(float x) {
  uint32_t u = __builtin_bit_cast(uint32_t, x);
  asm("" : "+v"(u));
  u &= 0x7fffffffu;
  return u < 0x7f800000u ? u : 0u;
}
// e of a block whose largest size is u: 448 is 1.75 * 2^8.
__device__ inline int block_exponent(uint32_t u) {
  const int e = static_cast<int>(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return max(e, -126);
}
__device__ inline float power_of_two(int e) {  // -126 <= e <= 127
  return __builtin_bit_cast(float, static_cast<uint32_t>(e + 127) << 23);
}
// Eight values to e4m3, rounded to nearest even; infinities and NaN become NaN.
__device__ inline u32x2 narrow8(const float* y, float mul) {
  int lo = 0, hi = 0;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0] * mul, y[1] * mul, lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2] * mul, y[3] * mul, lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4] * mul, y[5] * mul, hi, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6] * mul, y[7] * mul, hi, true);
  return u32x2{static_cast<uint32_t>(lo), static_cast<uint32_t>(hi)};
}

// The largest of the kLanes neighbouring lanes of a row, in every lane.
template <int kCtrl>
__device__ inline uint32_t max_dpp(uint32_t v) {
  const int u = static_cast<int>(v);
  return max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(u, u, kCtrl, 0xf, 0xf, true)));
}
template <int kLanes>
__device__ inline uint32_t row_max(uint32_t v) {
  v = max_dpp<0xB1>(v);                            // quad_perm [1,0,3,2]
  v = max_dpp<0x4E>(v);                            // quad_perm [2,3,0,1]
  if constexpr (kLanes >= 8) v = max_dpp<0x141>(v);   // row_half_mirror
  if constexpr (kLanes >= 16) v = max_dpp<0x140>(v);  // row_mirror
  return v;
}

// A row's eight elements normed (with weights w and the factor rstd) and rotated.
template <bool kRotate>
__device__ inline void turn_row(const float* f, const float* w, float rstd, const Rotation& rt, const float* s,
                                float* y) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float n0 = f[2 * e] * rstd * w[2 * e], n1 = f[2 * e + 1] * rstd * w[2 * e + 1];
    y[2 * e] = kRotate ? s[e] * (n0 * rt.cs[e] - n1 * rt.sn[e]) : n0;
    y[2 * e + 1] = kRotate ? s[e] * (n0 * rt.sn[e] + n1 * rt.cs[e]) : n1;
  }
}
template <int D>
__device__ inline float rstd_of(const float* f, float eps) {
  float ss = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) ss += f[e] * f[e];
  return __builtin_amdgcn_rsqf(row_sum<D / 8>(ss) * (1.0f / D) + eps);
}

// The queries of one token, by a wave.
template <typename T, int D, bool kRotate>
__device__ inline void query_rows(const Append8Args& a, const HeadTab<D / 2>& tab, int tok, int lane,
                                  f32x4 (&share)[D / 2]) {
  typedef typename Raw8<T>::type Raw;
  constexpr int kLanes = D / 8, kRows = 64 / kLanes, kUnroll = 3;
  const int sub = lane / kLanes, ch = lane % kLanes;
  const double turn = tab.turn[lane % (D / 2)], l2z = tab.l2z[lane % (D / 2)];
  const T* q = static_cast<const T*>(a.q) + tok * a.qs + ch * 8;
  Raw x[kUnroll];
  auto load = [&](int r0) {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int row = r0 + u * kRows + sub;
      x[u] = Raw{};
      if (row < a.H) x[u] = *reinterpret_cast<const Raw*>(q + row * D);
    }
  };
  load(0);
  const int toks[1] = {tok};
  Sequence sq[1];
  find_sequences(a, toks, lane, sq);
  const int pos = position_of(a, sq[0], tok);
  const bool live = pos >= 0;
  Rotation rt{};
  if constexpr (kRotate)
    rt = rotation<D / 2>(turn, l2z, live ? pos : 0, live ? pos - a.center : 0, share, lane, ch);
  float w[8] = {1, 1, 1, 1, 1, 1, 1, 1};
  if (a.qw) unpack(*reinterpret_cast<const Raw*>(static_cast<const T*>(a.qw) + ch * 8), w);
  for (int r0 = 0; r0 < a.H; r0 += kUnroll * kRows) {
    if (r0 > 0) load(r0);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int row = r0 + u * kRows + sub;
      if (r0 + u * kRows >= a.H) break;
      float f[8], y[8];
      unpack(x[u], f);
      const float rstd = rstd_of<D>(f, a.eps);
      turn_row<kRotate>(f, w, a.qw ? rstd : 1.0f, rt, rt.up, y);
      Raw o;
      pack(y, o);
      if (!live) o = Raw{};  // a token of no sequence
      if (row < a.H) *reinterpret_cast<Raw*>(static_cast<T*>(a.qo) + (static_cast<int64_t>(tok) * a.H + row) * D + ch * 8) = o;
    }
  }
}

template <typename T, int D, bool kRotate>
__global__ __launch_bounds__(kApThreads) void append8(Append8Args a, HeadTab<D / 2> tab) {
  typedef typename Raw8<T>::type Raw;
  constexpr int kLanes = D / 8, kPass = kApThreads / kLanes, kRows = kApPasses * kPass;
  __shared__ __attribute__((aligned(16))) f32x4 rot[kBlockMost][D / 2];
  __shared__ uint32_t most[kRows];
  const int tid = __builtin_amdgcn_workitem_id_x(), lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int idx = launch_index(), items = a.blocks * a.parts;
  if (idx >= items) {
    const int tok = (idx - items) * kApWaves + wv;
    if (a.q && tok < a.T) query_rows<T, D, kRotate>(a, tab, tok, lane, rot[wv]);
    return;
  }
  // The block: number `want` of those that the sequences' new tokens lie in.
  int want = idx / a.parts;
  const int part = idx - want * a.parts, bl = a.block_log2;
  int b = -1;
  NewTokens c{0, 0, 0};
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    const NewTokens x = new_tokens(a, b0 + lane);
    const int n = x.c1 > x.c0 ? ((x.c1 - 1) >> bl) - (x.c0 >> bl) + 1 : 0;
    const int upto = running_sum(n), total = __builtin_amdgcn_readlane(upto, 63);
    if (want < total) {
      const int l = __builtin_ctzll(__ballot(upto > want));
      b = b0 + l;
      c = NewTokens{__builtin_amdgcn_readlane(x.c0, l), __builtin_amdgcn_readlane(x.c1, l),
                    __builtin_amdgcn_readlane(x.tok0, l)};
      want -= __builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(n, l);
      break;
    }
    want -= total;
  }
  if (b < 0) return;
  const int lo = ((c.c0 >> bl) + want) << bl;  // the block's first position
  const int t0 = max(lo, c.c0), ntok = min(lo + (1 << bl), c.c1) - t0;
  const int old = max(c.c0 - lo, 0);  // tokens that it has already
  const int entry = a.table[static_cast<int64_t>(b) * a.max_pages + (lo >> a.page_log2)];
  const int units = 2 * a.Hkv, per = (units + a.parts - 1) / a.parts;  // K and V of the key heads
  const int u1 = min(units, (part + 1) * per);
  const int group = tid / kLanes, ch = tid % kLanes;
  const uint32_t split = 65536u / ntok + 1;  // i / ntok = i split >> 16 for i below 256
  const int64_t tok = static_cast<int64_t>(c.tok0) + t0;
  if (kRotate && part * per < a.Hkv) {
    for (int i = tid; i < ntok * (D / 2); i += kApThreads) {
      const int t = i / (D / 2), pair = i % (D / 2);
      rot[t][(pair & 3) * (D / 8) + (pair >> 2)] =
          pair_rotation(tab.turn[pair], tab.l2z[pair], t0 + t, t0 + t - a.center);
    }
  }
  float w[8] = {1, 1, 1, 1, 1, 1, 1, 1};
  if (a.kw) unpack(*reinterpret_cast<const Raw*>(static_cast<const T*>(a.kw) + ch * 8), w);
  if (static_cast<uint32_t>(entry) >= static_cast<uint32_t>(a.num_pages)) return;  // a page that is not there
  const uint32_t row0 = ((static_cast<uint32_t>(entry) * a.Hkv) << a.page_log2) + (lo & ((1 << a.page_log2) - 1));

  const int most_units = kRows / ntok;
  for (int u0 = part * per; u0 < u1; u0 += most_units) {
    const int rows = min(u1 - u0, most_units) * ntok;
    Raw x[kApPasses];
    int unit[kApPasses], t[kApPasses];
    uint32_t before[kApPasses];
#pragma unroll
    for (int p = 0; p < kApPasses; ++p) {
      const int i = p * kPass + group;
      const int ul = i * split >> 16;
      unit[p] = i < rows ? u0 + ul : -1;
      t[p] = i - ul * ntok;
      x[p] = Raw{};
      before[p] = 0;
      if (unit[p] < 0) continue;
      const bool is_k = unit[p] < a.Hkv;
      const int hk = is_k ? unit[p] : unit[p] - a.Hkv;
      const T* src = is_k ? static_cast<const T*>(a.k) + (tok + t[p]) * a.kst : static_cast<const T*>(a.v) + (tok + t[p]) * a.vst;
      x[p] = *reinterpret_cast<const Raw*>(src + hk * D + ch * 8);
      if (old > 0) before[p] = (is_k ? a.ks : a.vs)[(row0 + (static_cast<uint32_t>(hk) << a.page_log2)) >> bl];
    }
    if (u0 > part * per) __syncthreads();  // the maxima before are read
    for (int i = tid; i < kRows; i += kApThreads) most[i] = 0;
    __syncthreads();
    float y[kApPasses][8];
#pragma unroll
    for (int p = 0; p < kApPasses; ++p) {
      if (p * kPass >= rows) break;
      float f[8];
      unpack(x[p], f);
      const bool is_k = unit[p] < a.Hkv;
      const float rstd = rstd_of<D>(f, a.eps);
      Rotation rt{};
      if constexpr (kRotate) {
        if (is_k && unit[p] >= 0) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const f32x4 r = rot[t[p]][e * (D / 8) + ch];
            rt.cs[e] = r[0];
            rt.sn[e] = r[1];
            rt.down[e] = r[3];
          }
        }
      }
      turn_row<kRotate>(f, w, a.kw ? rstd : 1.0f, rt, rt.down, y[p]);
      uint32_t size = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (!is_k) y[p][e] = f[e];
        size = max(size, size_of(y[p][e]));
      }
      size = row_max<kLanes>(size);
      if (ch == 0 && unit[p] >= 0) atomicMax(&most[unit[p] - u0], size);
    }
#pragma unroll
    for (int p = 0; p < kApPasses; ++p) asm volatile("" : "+v"(before[p]));  // here before another wave writes it
    __syncthreads();
#pragma unroll
    for (int p = 0; p < kApPasses; ++p) {
      if (unit[p] < 0) continue;
      const bool is_k = unit[p] < a.Hkv;
      const int hk = is_k ? unit[p] : unit[p] - a.Hkv;
      const uint32_t head = row0 + (static_cast<uint32_t>(hk) << a.page_log2);
      uint8_t* cache = is_k ? a.kc : a.vc;
      const int had = static_cast<int>(before[p]) - 127;
      int e = block_exponent(most[unit[p] - u0]);
      if (old > 0) e = max(e, min(had, 126));
      const int64_t at = static_cast<int64_t>(head + (t0 - lo) + t[p]) * D + ch * 8;
      *reinterpret_cast<u32x2*>(cache + at) = narrow8(y[p], power_of_two(-e));
      if (t[p] != 0) continue;
      if (ch == 0) (is_k ? a.ks : a.vs)[head >> bl] = static_cast<uint8_t>(e + 127);
      if (old > 0 && e > had) {  // the block's older rows at its new scale
        const float less = e - had > 126 ? 0.0f : power_of_two(had - e);
        for (int r = 0; r < old; ++r) {
          u32x2* row = reinterpret_cast<u32x2*>(cache + static_cast<int64_t>(head + r) * D + ch * 8);
          const u32x2 was = *row;
          float f[8];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const f32x2 x0 = __builtin_amdgcn_cvt_pk_f32_fp8(was[h], false), x1 = __builtin_amdgcn_cvt_pk_f32_fp8(was[h], true);
            f[4 * h] = x0[0], f[4 * h + 1] = x0[1], f[4 * h + 2] = x1[0], f[4 * h + 3] = x1[1];
          }
          *row = narrow8(f, less);
        }
      }
    }
  }
}

template <typename T, int D>
void launch_d(const Append8Args& a, const HeadRotation& r, hipStream_t stream) {
  const int64_t queries = a.q ? (static_cast<int64_t>(a.T) + kApWaves - 1) / kApWaves : 0;
  const dim3 grid = grid_of(static_cast<int64_t>(a.blocks) * a.parts + queries), threads(kApThreads);
  if (r.rotate) hipLaunchKernelGGL((append8<T, D, true>), grid, threads, 0, stream, a, make_tab<D / 2>(r));
  else hipLaunchKernelGGL((append8<T, D, false>), grid, threads, 0, stream, a, HeadTab<D / 2>{});
}
template <typename T>
void launch_t(const Append8Args& a, const HeadRotation& r, int D, hipStream_t stream) {
  if (D == 32) launch_d<T, 32>(a, r, stream);
  else if (D == 64) launch_d<T, 64>(a, r, stream);
  else launch_d<T, 128>(a, r, stream);
}

}  // namespace

hipError_t launch_cache_append8(const QkNormCall& c, const void* v, int64_t v_stride, const PagedCache& cache,
                                int64_t T, hipStream_t stream) {
  Append8Args a{};
  a.q = c.q; a.k = c.k; a.v = v; a.qw = c.qw; a.kw = c.kw; a.qo = c.qo;
  a.kc = static_cast<uint8_t*>(cache.k); a.vc = static_cast<uint8_t*>(cache.v);
  a.ks = cache.k_scale; a.vs = cache.v_scale;
  a.table = cache.table; a.lens = cache.lens; a.start = cache.start;
  a.qs = c.q_stride; a.kst = c.k_stride; a.vst = v_stride;
  a.T = static_cast<int32_t>(T);
  a.B = static_cast<int32_t>(c.B);
  a.H = static_cast<int32_t>(c.H);
  a.Hkv = static_cast<int32_t>(c.Hkv);
  a.num_pages = static_cast<int32_t>(cache.num_pages);
  a.page_log2 = cache.page_log2;
  a.block_log2 = std::min(cache.page_log2, kCacheBlockLog2);
  a.max_pages = static_cast<int32_t>(cache.max_pages);
  a.reach = static_cast<uint32_t>(cache.max_pages << cache.page_log2);
  a.center = static_cast<int32_t>(c.rot.center);
  a.eps = c.eps;
  // n > 0 tokens of a sequence lie in at most min(n, (n - 1) / block + 2) blocks.
  const int64_t some = std::min(c.B, T), block = int64_t{1} << a.block_log2;
  const int64_t blocks = std::min(T, (T - some) / block + 2 * some);
  a.blocks = static_cast<int32_t>(blocks);
  a.parts = static_cast<int32_t>(std::max<int64_t>(1, std::min((2 * c.Hkv + 3) / 4, 512 / std::max<int64_t>(1, blocks))));
  if (c.dtype == DA_BF16) launch_t<u16>(a, c.rot, static_cast<int>(c.D), stream);
  else launch_t<float>(a, c.rot, static_cast<int>(c.D), stream);
  return hipGetLastError();
}

}  // namespace da
