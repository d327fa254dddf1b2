// The RMS norm of each query and key head together with the xPos rotation, in
// one pass, forward and backward, and the same pass with the keys and values
// written into a paged cache.  For a head's row x (D elements) at position p:
//   n = x w / sqrt(mean(x^2) + eps),   y = s R(a) n,
// where R(a) rotates each pair (2i, 2i+1) by a_i = p base^(-2i/D) and
// s_i = zeta_i^(sign (p - center) / scale_base), sign = +1 for queries and -1
// for keys.  Backward: dn = s R(-a) dy, xhat = x / sqrt(mean(x^2) + eps),
//   dx = rstd (dn w - xhat mean(dn w xhat)),   dw = sum over rows of dn xhat.
//
// One wave per token: D/8 lanes hold one head's row, eight elements each, and
// a wave steps through the token's heads, so that a lane keeps its four pairs,
// whose angles and scales (float64 products and a reduction to a quarter turn: as
// much work as a head's row) are formed once per token instead of once per head.
// Sums over a row are DPP exchanges within 16 lanes.  Bound by memory at training
// sizes: on inputs that no cache holds, gradients of 4 x 8192 tokens of 12 + 12 heads
// of 64 move 302 MB in 55 us (5.5 TB/s; float32 604 MB in 112), three prompts of 11800
// tokens of 24 heads of 128 into a cache 145 MB in 29 us (4.9 TB/s; float32 290 MB in
// 53).  The prompts again and again on the same inputs take 25 us: part of the
// 145 MB then comes from the Infinity Cache.  Bound by the launch at decoding sizes
// (5.3 us).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "heads_device.h"

namespace da {
namespace {

constexpr int kHeadThreads = 256;
constexpr int kHeadWaves = kHeadThreads / 64;

struct HeadFwdArgs {
  const void *q, *k, *v;    // rows of T tokens, heads side by side
  const void *qw, *kw;      // norm weights [D], or null: no norm
  void *qo, *ko;            // contiguous outputs (ko: without a cache)
  char *kc, *vc;            // the cache [num_pages][Hkv][page][D]
  const int32_t *table, *lens, *start;
  int64_t qs, ks, vs;       // elements between tokens
  int64_t T;
  int32_t B, H, Hkv, num_pages, page_log2, max_pages, center;
  float eps;
  FastDiv fn;               // division by N: a token's position without a cache
};

// The sequence that token tok belongs to, by all lanes of a wave: start [B + 1]
// ascends and the last entry that is not above tok is its sequence's (empty
// ones before it share that value).  Returns -1 before the first and after the
// last sequence; whatever start holds the result is below B.
__device__ inline int sequence_of(const int32_t* start, int B, int tok, int lane) {
  int n = 0;
  for (int b0 = 0; b0 <= B; b0 += 64) {
    const int b = b0 + lane;
    const bool before = b <= B && start[min(b, B)] <= tok;
    n += __popcll(__ballot(before));
  }
  return n > B ? -1 : n - 1;
}

// kRotate false (with a cache): no rotation.  (Not one of zero angles: those would
// make NaN of an infinite element's neighbour.  Nor a choice in the loop: three
// prompts into a cache 29.2 us instead of 28.5.)
template <typename T, int D, bool kCache, bool kRotate>
__global__ __launch_bounds__(kHeadThreads) void heads_fwd(HeadFwdArgs a, HeadTab<D / 2> tab) {
  typedef typename Raw8<T>::type Raw;
  constexpr int kLanes = D / 8;        // lanes per row
  constexpr int kRows = 64 / kLanes;   // rows a wave holds at once
  constexpr int kUnroll = 3;           // row groups in flight (12 + 12 heads of 64: all of a token's)
  const int lane = __builtin_amdgcn_workitem_id_x() & 63;
  const int64_t tok = static_cast<int64_t>(launch_index()) * kHeadWaves +
                      __builtin_amdgcn_readfirstlane(__builtin_amdgcn_workitem_id_x() >> 6);
  if (tok >= a.T) return;  // whole waves; the kernel has no barrier
  const int sub = lane / kLanes, ch = lane % kLanes;
  const int nq = a.H, nk = a.H + a.Hkv, rows = kCache ? nk + a.Hkv : nk;
  const T* q = static_cast<const T*>(a.q) + tok * a.qs + ch * 8;
  const T* k = static_cast<const T*>(a.k) + tok * a.ks + ch * 8;
  const T* v = kCache ? static_cast<const T*>(a.v) + tok * a.vs + ch * 8 : nullptr;

  auto load = [&](int row) {
    const T* p = row < nq ? q + row * D : row < nk ? k + (row - nq) * D : v + (row - nk) * D;
    return *reinterpret_cast<const Raw*>(p);
  };
  __shared__ __attribute__((aligned(16))) f32x4 share[kHeadWaves][D / 2];
  const int wv = __builtin_amdgcn_readfirstlane(__builtin_amdgcn_workitem_id_x() >> 6);
  const double turn = tab.turn[lane % (D / 2)], l2z = tab.l2z[lane % (D / 2)];
  const int first = a.q ? 0 : nq;  // without queries their rows are passed over
  Raw x[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int row = first + u * kRows + sub;
    x[u] = Raw{};
    if (row < rows) x[u] = load(row);
  }

  int pos;
  int64_t slot = -1;  // the token's row of key head 0 in the cache; < 0: none
  bool live = true;
  if constexpr (kCache) {
    const int b = sequence_of(a.start, a.B, static_cast<int>(tok), lane);
    pos = -1;
    if (b >= 0) {
      // the sequence's last new token is the last of its length
      const int64_t p = static_cast<int64_t>(a.lens[b]) - a.start[b + 1] + tok;
      if (p >= 0 && p < static_cast<int64_t>(a.max_pages) << a.page_log2) {
        pos = static_cast<int>(p);
        const int page = a.table[static_cast<int64_t>(b) * a.max_pages + (pos >> a.page_log2)];
        if (page >= 0 && page < a.num_pages)
          slot = ((static_cast<int64_t>(page) * a.Hkv) << a.page_log2) + (pos & ((1 << a.page_log2) - 1));
      }
    }
    live = pos >= 0;
  } else {
    pos = static_cast<int>(tok) - static_cast<int>(a.fn.div(static_cast<uint32_t>(tok)) * a.fn.d);
  }
  Rotation rt;
  if constexpr (kRotate)
    rt = rotation<D / 2>(turn, l2z, live ? pos : 0, live ? pos - a.center : 0, share[wv], lane, ch);
  const bool norm_q = a.qw != nullptr, norm_k = a.kw != nullptr;
  float wq[8], wk[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) wq[e] = wk[e] = 1.0f;
  if (norm_q) unpack(*reinterpret_cast<const Raw*>(static_cast<const T*>(a.qw) + ch * 8), wq);
  if (norm_k) unpack(*reinterpret_cast<const Raw*>(static_cast<const T*>(a.kw) + ch * 8), wk);

  for (int r0 = first; r0 < rows; r0 += kUnroll * kRows) {
    if (r0 > first) {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int row = r0 + u * kRows + sub;
        if (row < rows) x[u] = load(row);
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int row = r0 + u * kRows + sub;
      if (r0 + u * kRows >= rows) break;
      const bool is_q = row < nq;
      float f[8], y[8];
      unpack(x[u], f);
      float ss = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) ss += f[e] * f[e];
      ss = row_sum<kLanes>(ss);
      const float rstd = (is_q ? norm_q : norm_k) ? __builtin_amdgcn_rsqf(ss * (1.0f / D) + a.eps) : 1.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float n0 = f[2 * e] * rstd * (is_q ? wq[2 * e] : wk[2 * e]);
        const float n1 = f[2 * e + 1] * rstd * (is_q ? wq[2 * e + 1] : wk[2 * e + 1]);
        if constexpr (kRotate) {
          const float s = is_q ? rt.up[e] : rt.down[e];
          y[2 * e] = s * (n0 * rt.cs[e] - n1 * rt.sn[e]);
          y[2 * e + 1] = s * (n0 * rt.sn[e] + n1 * rt.cs[e]);
        } else {
          y[2 * e] = n0;
          y[2 * e + 1] = n1;
        }
      }
      Raw o;
      pack(y, o);
      if (row >= rows) continue;
      if (is_q) {
        if (kCache && !live) o = Raw{};  // a token of no sequence
        *reinterpret_cast<Raw*>(static_cast<T*>(a.qo) + (tok * a.H + row) * D + ch * 8) = o;
      } else if constexpr (kCache) {
        if (slot < 0) continue;
        const bool is_k = row < nk;
        const int64_t at = slot + (static_cast<int64_t>(row - (is_k ? nq : nk)) << a.page_log2);
        *reinterpret_cast<Raw*>(reinterpret_cast<T*>(is_k ? a.kc : a.vc) + at * D + ch * 8) = is_k ? o : x[u];
      } else {
        *reinterpret_cast<Raw*>(static_cast<T*>(a.ko) + (tok * a.Hkv + row - nq) * D + ch * 8) = o;
      }
    }
  }
}

struct HeadBwdArgs {
  const void *dqo, *dko, *q, *k, *qw, *kw;
  void *dq, *dk;
  float* part;  // [workgroups][2][D]: partial sums of both weights' gradients
  int64_t qs, ks, T;
  int32_t H, Hkv, center;
  int32_t groups;  // workgroups: the launch packet, where the device could read it, is in host memory
  float eps;
  FastDiv fn;
};

template <typename T, int D>
__global__ __launch_bounds__(kHeadThreads, sizeof(T) == 2 ? 4 : 3) void heads_bwd(HeadBwdArgs a, HeadTab<D / 2> tab) {
  typedef typename Raw8<T>::type Raw;
  constexpr int kLanes = D / 8, kRows = 64 / kLanes;
  __shared__ float red[kHeadWaves][2 * D];
  __shared__ __attribute__((aligned(16))) f32x4 share[kHeadWaves][D / 2];
  const int tid = __builtin_amdgcn_workitem_id_x();
  const int lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int sub = lane / kLanes, ch = lane % kLanes;
  const int nq = a.H, rows = a.H + a.Hkv;
  float wq[8], wk[8], gq[8], gk[8];
  unpack(*reinterpret_cast<const Raw*>(static_cast<const T*>(a.qw) + ch * 8), wq);
  unpack(*reinterpret_cast<const Raw*>(static_cast<const T*>(a.kw) + ch * 8), wk);
#pragma unroll
  for (int e = 0; e < 8; ++e) gq[e] = gk[e] = 0.0f;

  // A step is kRows heads of a token; the next step's rows, of this token or
  // the wave's next one, are loaded while a step is computed.
  const int64_t stride = static_cast<int64_t>(a.groups) * kHeadWaves;
  int64_t tok = static_cast<int64_t>(__builtin_amdgcn_workgroup_id_x()) * kHeadWaves + wv;
  Raw nx{}, ndy{};
  auto load = [&](int64_t t, int r0) {
    const int row = r0 + sub;
    nx = ndy = Raw{};  // lanes past the last row hold zeros
    if (t < a.T && row < rows) {
      const bool is_q = row < nq;
      const T* x = is_q ? static_cast<const T*>(a.q) + (t * a.qs + row * D)
                        : static_cast<const T*>(a.k) + (t * a.ks + (row - nq) * D);
      const T* dy = is_q ? static_cast<const T*>(a.dqo) + (t * a.H + row) * D
                         : static_cast<const T*>(a.dko) + (t * a.Hkv + row - nq) * D;
      nx = *reinterpret_cast<const Raw*>(x + ch * 8);
      ndy = *reinterpret_cast<const Raw*>(dy + ch * 8);
    }
  };
  load(tok, 0);
  const double turn = tab.turn[lane % (D / 2)], l2z = tab.l2z[lane % (D / 2)];
  for (; tok < a.T; tok += stride) {
    const int pos = static_cast<int>(tok) - static_cast<int>(a.fn.div(static_cast<uint32_t>(tok)) * a.fn.d);
    const Rotation rt = rotation<D / 2>(turn, l2z, pos, pos - a.center, share[wv], lane, ch);
    for (int r0 = 0; r0 < rows; r0 += kRows) {
      const Raw x = nx, dy = ndy;
      const bool last = r0 + kRows >= rows;
      load(last ? tok + stride : tok, last ? 0 : r0 + kRows);
      const int row = r0 + sub;
      const bool is_q = row < nq;
      float f[8], g[8], h[8];  // x, dy, then dn and dn w
      unpack(x, f);
      unpack(dy, g);
      float ss = 0.0f, dot = 0.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float s = is_q ? rt.up[e] : rt.down[e];
        const float g0 = g[2 * e], g1 = g[2 * e + 1];
        g[2 * e] = s * (g0 * rt.cs[e] + g1 * rt.sn[e]);
        g[2 * e + 1] = s * (g1 * rt.cs[e] - g0 * rt.sn[e]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        h[e] = g[e] * (is_q ? wq[e] : wk[e]);
        ss += f[e] * f[e];
        dot += h[e] * f[e];
      }
      ss = row_sum<kLanes>(ss);
      dot = row_sum<kLanes>(dot);
      const float rstd = __builtin_amdgcn_rsqf(ss * (1.0f / D) + a.eps);
      const float m = dot * rstd * (1.0f / D) * rstd;  // mean(dn w xhat) rstd
      float dx[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        dx[e] = rstd * (h[e] - f[e] * m);
        const float t = g[e] * f[e] * rstd;
        gq[e] += is_q ? t : 0.0f;
        gk[e] += is_q ? 0.0f : t;
      }
      Raw o;
      pack(dx, o);
      if (row >= rows) continue;
      T* dst = is_q ? static_cast<T*>(a.dq) + (tok * a.H + row) * D
                    : static_cast<T*>(a.dk) + (tok * a.Hkv + row - nq) * D;
      *reinterpret_cast<Raw*>(dst + ch * 8) = o;
    }
  }
  // Lanes of one ch hold the same eight columns: over the wave's row groups by
  // lane exchanges, then over the waves through LDS, in a fixed order.
#pragma unroll
  for (int e = 0; e < 8; ++e)
#pragma unroll
    for (int m = kLanes; m < 64; m <<= 1) {
      gq[e] += __shfl_xor(gq[e], m, 64);
      gk[e] += __shfl_xor(gk[e], m, 64);
    }
  if (sub == 0)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      red[wv][ch * 8 + e] = gq[e];
      red[wv][D + ch * 8 + e] = gk[e];
    }
  __syncthreads();
  if (tid < 2 * D)
    a.part[static_cast<int64_t>(__builtin_amdgcn_workgroup_id_x()) * 2 * D + tid] =
        (red[0][tid] + red[1][tid]) + (red[2][tid] + red[3][tid]);
}

// part [n][2D] -> dqw [D], dkw [D]: 16 columns per workgroup, four per thread,
// the partials over 64 threads, combined in a fixed order.
template <typename T>
__global__ __launch_bounds__(kHeadThreads) void heads_sum(const float* part, T* dqw, T* dkw, int n, int D) {
  __shared__ __attribute__((aligned(16))) float red[kHeadWaves][16];
  const int tid = __builtin_amdgcn_workitem_id_x();
  const int lane = tid & 63, wv = tid >> 6;
  const int col = __builtin_amdgcn_workgroup_id_x() * 16 + (lane & 3) * 4;
  f32x4 s = f32x4{0, 0, 0, 0};
#pragma unroll 8
  for (int r = wv * 16 + (lane >> 2); r < n; r += 64)
    s += *reinterpret_cast<const f32x4*>(part + static_cast<int64_t>(r) * 2 * D + col);
#pragma unroll
  for (int m = 4; m < 64; m <<= 1)
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] += __shfl_xor(s[e], m, 64);
  if (lane < 4) *reinterpret_cast<f32x4*>(&red[wv][4 * lane]) = s;
  __syncthreads();
  if (tid >= 16) return;
  const float t = (red[0][tid] + red[1][tid]) + (red[2][tid] + red[3][tid]);
  const int c = __builtin_amdgcn_workgroup_id_x() * 16 + tid;
  T* dst = c < D ? dqw + c : dkw + (c - D);
  if constexpr (sizeof(T) == 2) *dst = __builtin_bit_cast(u16, (__bf16)t);
  else *dst = t;
}

template <typename T, int D, bool kCache>
void launch_fwd_d(const HeadFwdArgs& a, const HeadRotation& r, hipStream_t stream) {
  const dim3 grid = grid_of((a.T + kHeadWaves - 1) / kHeadWaves), threads(kHeadThreads);
  if constexpr (kCache) {
    if (!r.rotate) {
      hipLaunchKernelGGL((heads_fwd<T, D, true, false>), grid, threads, 0, stream, a, HeadTab<D / 2>{});
      return;
    }
  }
  hipLaunchKernelGGL((heads_fwd<T, D, kCache, true>), grid, threads, 0, stream, a, make_tab<D / 2>(r));
}

template <typename T, bool kCache>
void launch_fwd(const HeadFwdArgs& a, const HeadRotation& r, int D, hipStream_t stream) {
  if (D == 32) launch_fwd_d<T, 32, kCache>(a, r, stream);
  else if (D == 64) launch_fwd_d<T, 64, kCache>(a, r, stream);
  else launch_fwd_d<T, 128, kCache>(a, r, stream);
}

template <typename T>
void launch_bwd(const HeadBwdArgs& a, const HeadRotation& r, void* dqw, void* dkw, int D, int nwg, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(nwg)), threads(kHeadThreads);
  if (D == 32) hipLaunchKernelGGL((heads_bwd<T, 32>), grid, threads, 0, stream, a, make_tab<16>(r));
  else if (D == 64) hipLaunchKernelGGL((heads_bwd<T, 64>), grid, threads, 0, stream, a, make_tab<32>(r));
  else hipLaunchKernelGGL((heads_bwd<T, 128>), grid, threads, 0, stream, a, make_tab<64>(r));
  hipLaunchKernelGGL(heads_sum<T>, dim3(static_cast<unsigned>(D / 8)), threads, 0, stream,
                     static_cast<const float*>(a.part), static_cast<T*>(dqw), static_cast<T*>(dkw), nwg, D);
}

}  // namespace

hipError_t launch_qk_norm(const QkNormCall& c, hipStream_t stream) {
  HeadFwdArgs a{};
  a.q = c.q; a.k = c.k; a.qw = c.qw; a.kw = c.kw; a.qo = c.qo; a.ko = c.ko;
  a.qs = c.q_stride; a.ks = c.k_stride;
  a.T = c.B * c.N;
  a.H = static_cast<int32_t>(c.H);
  a.Hkv = static_cast<int32_t>(c.Hkv);
  a.center = static_cast<int32_t>(c.rot.center);
  a.eps = c.eps;
  a.fn = make_fastdiv(static_cast<uint32_t>(c.N));
  if (c.dtype == DA_BF16) launch_fwd<u16, false>(a, c.rot, static_cast<int>(c.D), stream);
  else launch_fwd<float, false>(a, c.rot, static_cast<int>(c.D), stream);
  return hipGetLastError();
}

// Workgroups of the backward, each with a partial sum: four per CU, each wave
// one token at least.
static int64_t qk_norm_groups(int64_t T) { return std::min<int64_t>(1024, (T + kHeadWaves - 1) / kHeadWaves); }

uint64_t qk_norm_bwd_workspace(int64_t T, int64_t D) { return static_cast<uint64_t>(qk_norm_groups(T)) * 2 * D * 4; }

hipError_t launch_qk_norm_bwd(const QkNormCall& c, const void* dqo, const void* dko, void* dq, void* dk, void* dqw,
                              void* dkw, void* workspace, hipStream_t stream) {
  HeadBwdArgs a{};
  a.dqo = dqo; a.dko = dko; a.q = c.q; a.k = c.k; a.qw = c.qw; a.kw = c.kw; a.dq = dq; a.dk = dk;
  a.part = static_cast<float*>(workspace);
  a.qs = c.q_stride; a.ks = c.k_stride;
  a.T = c.B * c.N;
  a.H = static_cast<int32_t>(c.H);
  a.Hkv = static_cast<int32_t>(c.Hkv);
  a.center = static_cast<int32_t>(c.rot.center);
  a.eps = c.eps;
  a.fn = make_fastdiv(static_cast<uint32_t>(c.N));
  const int nwg = static_cast<int>(qk_norm_groups(a.T));
  a.groups = nwg;
  if (c.dtype == DA_BF16) launch_bwd<u16>(a, c.rot, dqw, dkw, static_cast<int>(c.D), nwg, stream);
  else launch_bwd<float>(a, c.rot, dqw, dkw, static_cast<int>(c.D), nwg, stream);
  return hipGetLastError();
}

hipError_t launch_cache_append(const QkNormCall& c, const void* v, int64_t v_stride, const PagedCache& cache,
                               int64_t T, hipStream_t stream) {
  HeadFwdArgs a{};
  a.q = c.q; a.k = c.k; a.v = v; a.qw = c.qw; a.kw = c.kw; a.qo = c.qo;
  a.kc = static_cast<char*>(cache.k); a.vc = static_cast<char*>(cache.v);
  a.table = cache.table; a.lens = cache.lens; a.start = cache.start;
  a.qs = c.q_stride; a.ks = c.k_stride; a.vs = v_stride;
  a.T = T;
  a.B = static_cast<int32_t>(c.B);
  a.H = static_cast<int32_t>(c.H);
  a.Hkv = static_cast<int32_t>(c.Hkv);
  a.num_pages = static_cast<int32_t>(cache.num_pages);
  a.page_log2 = cache.page_log2;
  a.max_pages = static_cast<int32_t>(cache.max_pages);
  a.center = static_cast<int32_t>(c.rot.center);
  a.eps = c.eps;
  if (c.dtype == DA_BF16) launch_fwd<u16, true>(a, c.rot, static_cast<int>(c.D), stream);
  else launch_fwd<float, true>(a, c.rot, static_cast<int>(c.D), stream);
  return hipGetLastError();
}

}  // namespace da
