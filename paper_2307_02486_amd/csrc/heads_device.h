// Device-side pieces of the head operators: rows of eight elements a lane, sums
// over a row's lanes, the xPos rotation of a pair, and the host's constants of it.
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>

#include "device_common.h"
#include "paged.h"

namespace da {
namespace {

// Per pair i of kPairs: quarter turns per position and log2 zeta_i /
// scale_base, in float64 (they multiply positions of up to millions).
template <int kPairs>
struct HeadTab {
  double turn[kPairs];
  double l2z[kPairs];
};
template <typename T> struct Raw8;
template <> struct Raw8<u16> { typedef u32x4 type; };
template <> struct Raw8<float> { typedef f32x8 type; };

__device__ inline void unpack(const u32x4& w, float* f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __builtin_bit_cast(float, w[i] << 16);
    f[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u);
  }
}
__device__ inline void unpack(const f32x8& w, float* f) {
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = w[i];
}
__device__ inline void pack(const float* f, u32x4& w) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = static_cast<unsigned>(__builtin_bit_cast(u16, (__bf16)f[2 * i])) |
           (static_cast<unsigned>(__builtin_bit_cast(u16, (__bf16)f[2 * i + 1])) << 16);
}
__device__ inline void pack(const float* f, f32x8& w) {
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = f[i];
}

// Sum over the kLanes (4, 8 or 16) neighbouring lanes of a row, in every lane.
template <int kCtrl>
__device__ inline float add_dpp(float v) {
  const int u = __builtin_bit_cast(int, v);
  return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(u, u, kCtrl, 0xf, 0xf, true));
}
template <int kLanes>
__device__ inline float row_sum(float v) {
  v = add_dpp<0xB1>(v);                            // quad_perm [1,0,3,2]
  v = add_dpp<0x4E>(v);                            // quad_perm [2,3,0,1]
  if constexpr (kLanes >= 8) v = add_dpp<0x141>(v);   // row_half_mirror
  if constexpr (kLanes >= 16) v = add_dpp<0x140>(v);  // row_mirror
  return v;
}

// Cosine, sine and the two scales (of a query and of a key) of one lane's four pairs.
struct Rotation {
  float cs[4], sn[4], up[4], down[4];
};
// One pair's cosine, sine and two scales at position pos, rel from the centre.
__device__ inline f32x4 pair_rotation(double turn, double l2z, int pos, int rel) {
  // The angle in quarter turns, reduced in float64 to [-1/2, 1/2]: the
  // float32 series below then have arguments of at most pi/4 and are exact
  // to a rounding (first terms left out: x^11/11! < 2e-9, x^10/10! < 3e-8).
  const double a = static_cast<double>(pos) * turn;
  const double n = rint(a);
  const int quad = static_cast<int>(n);
  const float x = static_cast<float>(a - n) * 1.57079632679489662f, x2 = x * x;
  const float s = x + x * x2 * (-1.0f / 6 + x2 * (1.0f / 120 + x2 * (-1.0f / 5040 + x2 * (1.0f / 362880))));
  const float c = 1.0f + x2 * (-0.5f + x2 * (1.0f / 24 + x2 * (-1.0f / 720 + x2 * (1.0f / 40320))));
  const float sq = quad & 1 ? c : s, cq = quad & 1 ? s : c;
  const double z = static_cast<double>(rel) * l2z;
  const double k = rint(z);
  const float f = static_cast<float>(z - k);
  f32x4 v;
  v[0] = (quad + 1) & 2 ? -cq : cq;
  v[1] = quad & 2 ? -sq : sq;
  v[2] = ldexpf(__builtin_amdgcn_exp2f(f), static_cast<int>(k));
  v[3] = ldexpf(__builtin_amdgcn_exp2f(-f), -static_cast<int>(k));
  return v;
}
// Formed a pair per lane, lane mod kPairs, whose constants turn and l2z are, and
// handed through the wave's own LDS.  (Four pairs a lane, formed by every row's
// lanes again: gradients of 4 x 8192 tokens 62.6 us instead of 61.5, three prompts
// into a cache 29.0 instead of 28.4.)
template <int kPairs>
__device__ inline Rotation rotation(double turn, double l2z, int pos, int rel, f32x4 (&share)[kPairs], int lane,
                                    int ch) {
  const f32x4 v = pair_rotation(turn, l2z, pos, rel);
  // Pair 4 c + e at e (kPairs / 4) + c: a row's lanes read 16 bytes each, side by
  // side.  A wave's LDS operations complete in order; the fences are the compiler's.
  const int pair = lane % kPairs;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  if (lane < kPairs) share[(pair & 3) * (kPairs / 4) + (pair >> 2)] = v;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  Rotation r;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const f32x4 t = share[e * (kPairs / 4) + ch];
    r.cs[e] = t[0];
    r.sn[e] = t[1];
    r.up[e] = t[2];
    r.down[e] = t[3];
  }
  __builtin_amdgcn_wave_barrier();
  return r;
}

// The constants of a rotation.  They depend on the parameters alone and are
// kept for the next call with the same ones (64 logarithms and powers take as
// long as a third of a launch).
template <int kPairs>
const HeadTab<kPairs>& make_tab(const HeadRotation& r) {
  static thread_local HeadRotation known{};
  static thread_local HeadTab<kPairs> t{};
  if (r.base != known.base || r.gamma != known.gamma || r.scale_base != known.scale_base) {
    known = r;
    const double l2b = std::log2(static_cast<double>(r.base)), gamma = r.gamma;
    for (int i = 0; i < kPairs; ++i) {
      const double x = static_cast<double>(i) / kPairs;  // 2 i / D
      t.turn[i] = std::exp2(-x * l2b) * 0.63661977236758134308;  // 2 / pi
      t.l2z[i] = std::log2((x + gamma) / (1.0 + gamma)) / r.scale_base;
    }
  }
  return t;
}

}  // namespace
}  // namespace da
