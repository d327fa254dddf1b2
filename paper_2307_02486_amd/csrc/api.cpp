// C ABI of the dilated-attention forward and backward passes (declared in include/dilated_attn.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdint>
#include <vector>

#include "../../include/dilated_attn_compressed.h"
#include "kernels.h"
#include "paged.h"
#include "plan.h"

namespace {

bool overlaps(const void* a, uint64_t na, const void* b, uint64_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a);
  const uintptr_t y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Profiling window of dilated_attn_profile_begin/end: three events per call.
struct ProfileWindow {
  bool active = false;
  int64_t capacity = 0;
  int64_t used = 0;
  std::vector<hipEvent_t> ev;  // [call][0..2]
};
ProfileWindow g_prof;

void destroy_events(ProfileWindow& w) {
  for (hipEvent_t e : w.ev)
    if (e) (void)hipEventDestroy(e);
  w.ev.clear();
  w.active = false;
  w.capacity = w.used = 0;
}

// Whether the parameters of an xPos rotation of positions 0 .. last are valid
// (see dilated_attn_xpos: the scale exponents stay within 2^+-64).
bool xpos_ok(int64_t center, int64_t last, float base, float gamma, float scale_base) {
  if (center < 0 || center > last) return false;
  if (!std::isfinite(base) || !(base > 1.0f) || !std::isfinite(gamma) || !(gamma > 0.0f) ||
      !std::isfinite(scale_base) || !(scale_base > 0.0f))
    return false;
  // zeta_i ranges over [gamma / (1 + gamma), 1): the smallest gives the
  // largest |log2 zeta| (every zeta_i < 1 for gamma > 0 and i < D/2).
  const double l2z = std::fabs(std::log2(static_cast<double>(gamma) / (1.0 + gamma)));
  return static_cast<double>(std::max(center, last - center)) / scale_base * l2z <= 64.0;
}

// Bytes of n tokens of `row` elements each, `stride` elements apart.
uint64_t strided_bytes(int64_t n, int64_t row, int64_t stride, int64_t esize) {
  return n > 0 ? static_cast<uint64_t>((n - 1) * stride + row) * esize : 0;
}

// Head counts, head size, type and token strides that the head operators take.
int head_shapes(int64_t tokens, int64_t H, int64_t Hkv, int64_t D, int64_t dtype, const int64_t* strides,
                const int64_t* heads, int n) {
  if (tokens < 0 || tokens >= (int64_t{1} << 31) || H < 1 || H >= (int64_t{1} << 16) || Hkv < 1 ||
      Hkv >= (int64_t{1} << 16))
    return DA_EINVAL;
  if (dtype != DA_BF16 && dtype != DA_F32) return DA_EUNSUPPORTED;
  if (D != 32 && D != 64 && D != 128) return DA_EUNSUPPORTED;
  for (int i = 0; i < n; ++i) {
    if (strides[i] < heads[i] * D || strides[i] >= (int64_t{1} << 32)) return DA_EINVAL;
    if (strides[i] % (dtype == DA_BF16 ? 8 : 4)) return DA_EALIGN;
  }
  return DA_OK;
}

struct Span {
  const void* p;
  uint64_t bytes;
};

// Whether an output overlaps another output or an input.
bool any_overlap(const Span* outs, int no, const Span* ins, int ni) {
  for (int i = 0; i < no; ++i) {
    for (int j = i + 1; j < no; ++j)
      if (overlaps(outs[i].p, outs[i].bytes, outs[j].p, outs[j].bytes)) return true;
    for (int j = 0; j < ni; ++j)
      if (overlaps(outs[i].p, outs[i].bytes, ins[j].p, ins[j].bytes)) return true;
  }
  return false;
}

}  // namespace

extern "C" {

int dilated_attn_plan(int64_t B, int64_t N, int64_t H, int64_t D, const da_pattern_t* patterns,
                      int64_t num_patterns, int64_t causal, int64_t dtype, float softmax_scale,
                      da_plan_info_t* info) {
  if (!info) return DA_EINVAL;
  da::Plan p;
  const int rc = da::make_plan(B, N, H, D, patterns, num_patterns, causal, dtype, softmax_scale, &p);
  if (rc != DA_OK) return rc;
  info->workspace_bytes = p.workspace_bytes;
  info->num_work_items = p.total_items;
  info->covered_rows = p.covered_rows;
  info->sparse_flops = p.sparse_flops;
  info->bytes_attn = p.bytes_attn;
  info->bytes_combine = p.bytes_combine;
  return DA_OK;
}

int dilated_attn_fwd(const void* q, const void* k, const void* v, void* out, float* lse,
                     int64_t B, int64_t N, int64_t H, int64_t D, const da_pattern_t* patterns,
                     int64_t num_patterns, int64_t causal, int64_t dtype, float softmax_scale,
                     void* workspace, uint64_t workspace_bytes, void* stream) {
  da::Plan p;
  const int rc = da::make_plan(B, N, H, D, patterns, num_patterns, causal, dtype, softmax_scale, &p);
  if (rc != DA_OK) return rc;
  if (!q || !k || !v || !out || !lse || !workspace) return DA_EINVAL;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(lse) ||
      !aligned16(workspace))
    return DA_EALIGN;
  const uint64_t esize = dtype == DA_BF16 ? 2 : 4;
  const uint64_t tensor_bytes = static_cast<uint64_t>(B * N * H * D) * esize;
  const uint64_t lse_bytes = static_cast<uint64_t>(B * H * N) * 4;
  if (overlaps(out, tensor_bytes, q, tensor_bytes) || overlaps(out, tensor_bytes, k, tensor_bytes) ||
      overlaps(out, tensor_bytes, v, tensor_bytes) || overlaps(lse, lse_bytes, out, tensor_bytes) ||
      overlaps(lse, lse_bytes, q, tensor_bytes) || overlaps(lse, lse_bytes, k, tensor_bytes) ||
      overlaps(lse, lse_bytes, v, tensor_bytes))
    return DA_EINVAL;
  if (workspace_bytes < p.workspace_bytes) return DA_EWORKSPACE;
  const void* bufs[5] = {q, k, v, out, lse};
  const uint64_t sizes[5] = {tensor_bytes, tensor_bytes, tensor_bytes, tensor_bytes, lse_bytes};
  for (int i = 0; i < 5; ++i)
    if (overlaps(workspace, p.workspace_bytes, bufs[i], sizes[i])) return DA_EINVAL;

  hipStream_t s = static_cast<hipStream_t>(stream);
  hipEvent_t* ev = nullptr;
  if (g_prof.active && g_prof.used < g_prof.capacity) ev = &g_prof.ev[3 * g_prof.used++];
  if (ev && hipEventRecord(ev[0], s) != hipSuccess) return DA_EHIP;
  if (da::launch_attention(p, q, k, v, workspace, s) != hipSuccess) return DA_EHIP;
  if (ev && hipEventRecord(ev[1], s) != hipSuccess) return DA_EHIP;
  if (da::launch_combine(p, workspace, out, lse, s) != hipSuccess) return DA_EHIP;
  if (ev && hipEventRecord(ev[2], s) != hipSuccess) return DA_EHIP;
  return DA_OK;
}

int dilated_attn_bwd_plan(int64_t B, int64_t N, int64_t H, int64_t D, const da_pattern_t* patterns,
                          int64_t num_patterns, int64_t causal, int64_t dtype, float softmax_scale,
                          da_plan_info_t* info) {
  if (!info) return DA_EINVAL;
  da::Plan p;
  int rc = da::make_plan(B, N, H, D, patterns, num_patterns, causal, dtype, softmax_scale, &p);
  if (rc != DA_OK) return rc;
  da::BwdLayout l;
  rc = da::make_bwd_layout(p, &l);
  if (rc != DA_OK) return rc;
  info->workspace_bytes = l.workspace_bytes;
  info->num_work_items = 2 * p.total_items;
  info->covered_rows = p.covered_rows;
  info->sparse_flops = l.flops;
  info->bytes_attn = l.bytes_grad;
  info->bytes_combine = l.bytes_combine;
  return DA_OK;
}

int dilated_attn_bwd(const void* q, const void* k, const void* v, const void* out, const float* lse,
                     const void* dout, void* dq, void* dk, void* dv, int64_t B, int64_t N, int64_t H,
                     int64_t D, const da_pattern_t* patterns, int64_t num_patterns, int64_t causal,
                     int64_t dtype, float softmax_scale, void* workspace, uint64_t workspace_bytes,
                     void* stream) {
  da::Plan p;
  int rc = da::make_plan(B, N, H, D, patterns, num_patterns, causal, dtype, softmax_scale, &p);
  if (rc != DA_OK) return rc;
  da::BwdLayout l;
  rc = da::make_bwd_layout(p, &l);
  if (rc != DA_OK) return rc;
  const void* ins[6] = {q, k, v, out, lse, dout};
  void* outs[3] = {dq, dk, dv};
  for (const void* x : ins)
    if (!x) return DA_EINVAL;
  for (const void* x : outs)
    if (!x) return DA_EINVAL;
  if (!workspace) return DA_EINVAL;
  for (const void* x : ins)
    if (!aligned16(x)) return DA_EALIGN;
  for (const void* x : outs)
    if (!aligned16(x)) return DA_EALIGN;
  if (!aligned16(workspace)) return DA_EALIGN;
  const uint64_t tb = static_cast<uint64_t>(B * N * H * D) * 2;
  const uint64_t lb = static_cast<uint64_t>(B * H * N) * 4;
  const uint64_t in_sizes[6] = {tb, tb, tb, tb, lb, tb};
  for (int i = 0; i < 3; ++i) {
    for (int j = 0; j < 6; ++j)
      if (overlaps(outs[i], tb, ins[j], in_sizes[j])) return DA_EINVAL;
    for (int j = i + 1; j < 3; ++j)
      if (overlaps(outs[i], tb, outs[j], tb)) return DA_EINVAL;
  }
  if (workspace_bytes < l.workspace_bytes) return DA_EWORKSPACE;
  for (int j = 0; j < 6; ++j)
    if (overlaps(workspace, l.workspace_bytes, ins[j], in_sizes[j])) return DA_EINVAL;
  for (int i = 0; i < 3; ++i)
    if (overlaps(workspace, l.workspace_bytes, outs[i], tb)) return DA_EINVAL;

  hipStream_t s = static_cast<hipStream_t>(stream);
  if (da::launch_backward(p, l, q, k, v, out, lse, dout, dq, dk, dv, workspace, s) != hipSuccess)
    return DA_EHIP;
  return DA_OK;
}

int dilated_attn_xpos(const void* x, void* y, int64_t B, int64_t N, int64_t H, int64_t D,
                      int64_t sign, int64_t transpose, int64_t center, float base, float gamma,
                      float scale_base, int64_t dtype, void* stream) {
  if (!x || !y) return DA_EINVAL;
  if (B <= 0 || N <= 0 || H <= 0 || D < 8 || D > 256 || D % 8 != 0) return DA_EINVAL;
  if (dtype != DA_BF16 && dtype != DA_F32) return DA_EUNSUPPORTED;
  if ((sign != 1 && sign != -1) || (transpose != 0 && transpose != 1)) return DA_EINVAL;
  // At most 2^34 elements: one thread per 8 keeps the grid within 2^32 work-items.
  if (B > (int64_t{1} << 34) / N || B * N > (int64_t{1} << 34) / H ||
      B * N * H > (int64_t{1} << 34) / D)
    return DA_EINVAL;
  if (!xpos_ok(center, N - 1, base, gamma, scale_base)) return DA_EINVAL;
  if (!aligned16(x) || !aligned16(y)) return DA_EALIGN;
  const uint64_t bytes = static_cast<uint64_t>(B * N * H * D) * (dtype == DA_BF16 ? 2 : 4);
  if (x != y && overlaps(x, bytes, y, bytes)) return DA_EINVAL;
  if (da::launch_xpos(x, y, B, N, H, D, static_cast<int>(sign), transpose != 0, center, base, gamma,
                      scale_base, static_cast<int>(dtype), static_cast<hipStream_t>(stream)) != hipSuccess)
    return DA_EHIP;
  return DA_OK;
}

int dilated_attn_wgrad_workspace(int64_t K, int64_t M, int64_t N, uint64_t* bytes) {
  if (!bytes) return DA_EINVAL;
  if (K < 0 || K > (int64_t{1} << 30) || M <= 0 || N <= 0 || M % 128 || N % 128 || M > 16384 || N > 16384)
    return DA_EINVAL;
  *bytes = da::wgrad_workspace(K, M, N);
  return DA_OK;
}

int dilated_attn_wgrad(const void* dy, const void* x, void* dw, void* db, int64_t K, int64_t M, int64_t N,
                       int64_t dtype, void* workspace, uint64_t workspace_bytes, void* stream) {
  uint64_t need = 0;
  if (!dw || (K > 0 && (!dy || !x))) return DA_EINVAL;
  if (dilated_attn_wgrad_workspace(K, M, N, &need) != DA_OK) return DA_EINVAL;
  if (dtype != DA_BF16) return DA_EUNSUPPORTED;
  if (need > 0 && !workspace) return DA_EINVAL;
  if (!aligned16(dy) || !aligned16(x) || !aligned16(dw) || !aligned16(db) || (need > 0 && !aligned16(workspace)))
    return DA_EALIGN;
  if (workspace_bytes < need) return DA_EWORKSPACE;
  const void* ins[2] = {dy, x};
  const uint64_t isz[2] = {static_cast<uint64_t>(K * M) * 2, static_cast<uint64_t>(K * N) * 2};
  const void* outs[3] = {dw, db, workspace};
  const uint64_t osz[3] = {static_cast<uint64_t>(M * N) * 2, db ? static_cast<uint64_t>(M) * 2 : 0, need};
  for (int i = 0; i < 3; ++i) {
    for (int j = i + 1; j < 3; ++j)
      if (overlaps(outs[i], osz[i], outs[j], osz[j])) return DA_EINVAL;
    for (int j = 0; j < 2; ++j)
      if (overlaps(outs[i], osz[i], ins[j], isz[j])) return DA_EINVAL;
  }
  if (da::launch_wgrad(dy, x, dw, db, K, M, N, workspace, static_cast<hipStream_t>(stream)) != hipSuccess)
    return DA_EHIP;
  return DA_OK;
}

int dilated_attn_layernorm_fwd(const void* x, const void* g, const void* b, void* y, float* mean, float* rstd,
                               int64_t rows, int64_t E, float eps, int64_t dtype, void* stream) {
  if (!g || !b || !y || !mean || !rstd || (rows > 0 && !x)) return DA_EINVAL;
  if (rows < 0 || rows > (int64_t{1} << 26) || E < 8 || E > 2048 || E % 8 || !std::isfinite(eps) || !(eps > 0.0f))
    return DA_EINVAL;
  if (dtype != DA_BF16) return DA_EUNSUPPORTED;
  if (!aligned16(x) || !aligned16(g) || !aligned16(b) || !aligned16(y)) return DA_EALIGN;
  const uint64_t xb = static_cast<uint64_t>(rows * E) * 2, sb = static_cast<uint64_t>(rows) * 4;
  if (x != y && overlaps(x, xb, y, xb)) return DA_EINVAL;
  const void* outs[3] = {y, mean, rstd};
  const uint64_t osz[3] = {xb, sb, sb};
  for (int i = 0; i < 3; ++i) {
    for (int j = i + 1; j < 3; ++j)
      if (overlaps(outs[i], osz[i], outs[j], osz[j])) return DA_EINVAL;
    if (overlaps(outs[i], osz[i], g, static_cast<uint64_t>(E) * 2) ||
        overlaps(outs[i], osz[i], b, static_cast<uint64_t>(E) * 2))
      return DA_EINVAL;
  }
  if (overlaps(mean, sb, x, xb) || overlaps(rstd, sb, x, xb)) return DA_EINVAL;
  if (da::launch_layernorm_fwd(x, g, b, y, mean, rstd, rows, E, eps, static_cast<hipStream_t>(stream)) !=
      hipSuccess)
    return DA_EHIP;
  return DA_OK;
}

int dilated_attn_layernorm_bwd_workspace(int64_t rows, int64_t E, uint64_t* bytes) {
  if (!bytes || rows < 0 || rows > (int64_t{1} << 26) || E < 8 || E > 2048 || E % 8) return DA_EINVAL;
  *bytes = da::layernorm_bwd_workspace(rows, E);
  return DA_OK;
}

int dilated_attn_layernorm_bwd(const void* dy, const void* x, const void* g, const float* mean, const float* rstd,
                               void* dx, void* dg, void* db, int64_t rows, int64_t E, int64_t dtype,
                               void* workspace, uint64_t workspace_bytes, void* stream) {
  uint64_t need = 0;
  if (dilated_attn_layernorm_bwd_workspace(rows, E, &need) != DA_OK) return DA_EINVAL;
  if (!g || !dg || !db || !workspace || (rows > 0 && (!dy || !x || !mean || !rstd || !dx))) return DA_EINVAL;
  if (dtype != DA_BF16) return DA_EUNSUPPORTED;
  if (!aligned16(dy) || !aligned16(x) || !aligned16(g) || !aligned16(dx) || !aligned16(workspace)) return DA_EALIGN;
  if (workspace_bytes < need) return DA_EWORKSPACE;
  const uint64_t xb = static_cast<uint64_t>(rows * E) * 2, sb = static_cast<uint64_t>(rows) * 4,
                 eb = static_cast<uint64_t>(E) * 2;
  const void* ins[5] = {dy, x, g, mean, rstd};
  const uint64_t isz[5] = {xb, xb, eb, sb, sb};
  const void* outs[4] = {dx, dg, db, workspace};
  const uint64_t osz[4] = {xb, eb, eb, need};
  for (int i = 0; i < 4; ++i) {
    for (int j = i + 1; j < 4; ++j)
      if (overlaps(outs[i], osz[i], outs[j], osz[j])) return DA_EINVAL;
    for (int j = 0; j < 5; ++j)
      if (overlaps(outs[i], osz[i], ins[j], isz[j])) return DA_EINVAL;
  }
  if (da::launch_layernorm_bwd(dy, x, g, mean, rstd, dx, dg, db, rows, E, workspace,
                               static_cast<hipStream_t>(stream)) != hipSuccess)
    return DA_EHIP;
  return DA_OK;
}

int dilated_attn_qk_norm_xpos(const void* q, const void* k, const void* qw, const void* kw, void* qo, void* ko,
                              int64_t B, int64_t N, int64_t H, int64_t Hkv, int64_t D, int64_t q_stride,
                              int64_t k_stride, float eps, int64_t center, float base, float gamma,
                              float scale_base, int64_t dtype, void* stream) {
  if (!q || !k || !qw || !kw || !qo || !ko) return DA_EINVAL;
  if (B < 1 || N < 1 || B >= (int64_t{1} << 31) / N || !std::isfinite(eps) || !(eps >= FLT_MIN)) return DA_EINVAL;
  const int64_t strides[2] = {q_stride, k_stride}, heads[2] = {H, Hkv};
  if (const int rc = head_shapes(B * N, H, Hkv, D, dtype, strides, heads, 2); rc != DA_OK) return rc;
  if (!xpos_ok(center, N - 1, base, gamma, scale_base)) return DA_EINVAL;
  for (const void* p : {q, k, qw, kw, static_cast<const void*>(qo), static_cast<const void*>(ko)})
    if (!aligned16(p)) return DA_EALIGN;
  const int64_t T = B * N, es = dtype == DA_BF16 ? 2 : 4;
  const uint64_t wb = static_cast<uint64_t>(D * es);
  const Span ins[4] = {{q, strided_bytes(T, H * D, q_stride, es)}, {k, strided_bytes(T, Hkv * D, k_stride, es)},
                       {qw, wb}, {kw, wb}};
  const Span outs[2] = {{qo, static_cast<uint64_t>(T * H * D * es)}, {ko, static_cast<uint64_t>(T * Hkv * D * es)}};
  if (any_overlap(outs, 2, ins, 4)) return DA_EINVAL;
  const da::QkNormCall c{q, k, qw, kw, qo, ko, B, N, H, Hkv, D, q_stride, k_stride, eps,
                         {true, center, base, gamma, scale_base}, static_cast<int>(dtype)};
  return da::launch_qk_norm(c, static_cast<hipStream_t>(stream)) == hipSuccess ? DA_OK : DA_EHIP;
}

int dilated_attn_qk_norm_xpos_bwd_workspace(int64_t B, int64_t N, int64_t D, uint64_t* bytes) {
  if (!bytes || B < 1 || N < 1 || B >= (int64_t{1} << 31) / N) return DA_EINVAL;
  if (D != 32 && D != 64 && D != 128) return DA_EUNSUPPORTED;
  *bytes = da::qk_norm_bwd_workspace(B * N, D);
  return DA_OK;
}

int dilated_attn_qk_norm_xpos_bwd(const void* dqo, const void* dko, const void* q, const void* k, const void* qw,
                                  const void* kw, void* dq, void* dk, void* dqw, void* dkw, int64_t B, int64_t N,
                                  int64_t H, int64_t Hkv, int64_t D, int64_t q_stride, int64_t k_stride, float eps,
                                  int64_t center, float base, float gamma, float scale_base, int64_t dtype,
                                  void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!dqo || !dko || !q || !k || !qw || !kw || !dq || !dk || !dqw || !dkw || !workspace) return DA_EINVAL;
  if (!std::isfinite(eps) || !(eps >= FLT_MIN)) return DA_EINVAL;
  uint64_t need = 0;
  if (const int rc = dilated_attn_qk_norm_xpos_bwd_workspace(B, N, D, &need); rc != DA_OK) return rc;
  const int64_t strides[2] = {q_stride, k_stride}, heads[2] = {H, Hkv};
  if (const int rc = head_shapes(B * N, H, Hkv, D, dtype, strides, heads, 2); rc != DA_OK) return rc;
  if (!xpos_ok(center, N - 1, base, gamma, scale_base)) return DA_EINVAL;
  for (const void* p : {dqo, dko, q, k, qw, kw, static_cast<const void*>(dq), static_cast<const void*>(dk),
                        static_cast<const void*>(dqw), static_cast<const void*>(dkw),
                        static_cast<const void*>(workspace)})
    if (!aligned16(p)) return DA_EALIGN;
  if (workspace_bytes < need) return DA_EWORKSPACE;
  const int64_t T = B * N, es = dtype == DA_BF16 ? 2 : 4;
  const uint64_t wb = static_cast<uint64_t>(D * es), qb = static_cast<uint64_t>(T * H * D * es),
                 kb = static_cast<uint64_t>(T * Hkv * D * es);
  const Span ins[6] = {{dqo, qb}, {dko, kb}, {q, strided_bytes(T, H * D, q_stride, es)},
                       {k, strided_bytes(T, Hkv * D, k_stride, es)}, {qw, wb}, {kw, wb}};
  const Span outs[5] = {{dq, qb}, {dk, kb}, {dqw, wb}, {dkw, wb}, {workspace, need}};
  if (any_overlap(outs, 5, ins, 6)) return DA_EINVAL;
  const da::QkNormCall c{q, k, qw, kw, nullptr, nullptr, B, N, H, Hkv, D, q_stride, k_stride, eps,
                         {true, center, base, gamma, scale_base}, static_cast<int>(dtype)};
  return da::launch_qk_norm_bwd(c, dqo, dko, dq, dk, dqw, dkw, workspace, static_cast<hipStream_t>(stream)) ==
                 hipSuccess
             ? DA_OK
             : DA_EHIP;
}

namespace {

// Cache sizes that the paged calls take; the rows fit 32-bit indices.
bool cache_ok(int64_t B, int64_t Hkv, const da_paged_cache_t* c, bool values = true) {
  if (!c || !c->k || (values && !c->v) || !c->block_table || !c->seq_lens || !c->q_start) return false;
  constexpr int64_t kMost = int64_t{1} << 31;
  return B >= 1 && B <= da::kPagedMost && c->page_size >= 1 && c->page_size <= (int64_t{1} << 16) &&
         (c->page_size & (c->page_size - 1)) == 0 && c->max_pages >= 1 &&
         c->max_pages <= da::kPagedMost / c->page_size &&
         c->num_pages >= 1 && c->num_pages < kMost && c->num_pages <= (int64_t{1} << 32) / c->page_size / Hkv;
}

da::PagedCache paged_cache(const da_paged_cache_t* c) {
  int page_log2 = 0;
  while ((int64_t{1} << page_log2) < c->page_size) ++page_log2;
  return da::PagedCache{c->k, c->v, c->block_table, c->seq_lens, c->q_start, c->num_pages, c->max_pages, page_log2};
}

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// The bytes of a cache's keys (or values), and of an 8-bit cache's scales of them.
uint64_t pool_bytes(const da_paged_cache_t* c, int64_t Hkv, int64_t row_bytes) {
  return static_cast<uint64_t>(c->num_pages * c->page_size * Hkv) * static_cast<uint64_t>(row_bytes);
}
uint64_t scale_bytes(const da_paged_cache_t* c, int64_t Hkv) {
  return static_cast<uint64_t>(c->num_pages * Hkv) *
         static_cast<uint64_t>(c->page_size / std::min<int64_t>(c->page_size, DA_CACHE_BLOCK));
}

// The append to a cache of the call's type, or (with scales) in 8 bits.
int cache_append(const void* q, const void* k, const void* v, const void* qw, const void* kw, void* qo,
                 const da_paged_cache_t* cache, const da_paged_cache_f8_t* f8, int64_t T, int64_t B, int64_t H,
                 int64_t Hkv, int64_t D, int64_t q_stride, int64_t k_stride, int64_t v_stride, float eps,
                 int64_t rotate, int64_t center, float base, float gamma, float scale_base, int64_t dtype,
                 void* stream) {
  const int64_t strides[3] = {k_stride, v_stride, q_stride}, heads[3] = {Hkv, Hkv, H};
  if (const int rc = head_shapes(T, H, Hkv, D, dtype, strides, heads, q ? 3 : 2); rc != DA_OK) return rc;
  if (!cache_ok(B, Hkv, cache) || (T > 0 && (!k || !v)) || (q != nullptr) != (qo != nullptr)) return DA_EINVAL;
  if (((qw || kw) && (!std::isfinite(eps) || !(eps >= FLT_MIN))) || (rotate != 0 && rotate != 1)) return DA_EINVAL;
  if (rotate && !xpos_ok(center, cache->max_pages * cache->page_size - 1, base, gamma, scale_base)) return DA_EINVAL;
  for (const void* p : {q, k, v, qw, kw, static_cast<const void*>(qo), static_cast<const void*>(cache->k),
                        static_cast<const void*>(cache->v)})
    if (!aligned16(p)) return DA_EALIGN;
  if (!aligned4(cache->block_table) || !aligned4(cache->seq_lens) || !aligned4(cache->q_start)) return DA_EALIGN;
  if (f8 && (!f8->k_scale || !f8->v_scale || T >= (int64_t{1} << 30))) return DA_EINVAL;
  const int64_t es = dtype == DA_BF16 ? 2 : 4;
  const uint64_t wb = static_cast<uint64_t>(D * es), cb = pool_bytes(cache, Hkv, f8 ? D : D * es),
                 sb = f8 ? scale_bytes(cache, Hkv) : 0;
  const Span ins[8] = {{q, q ? strided_bytes(T, H * D, q_stride, es) : 0}, {k, strided_bytes(T, Hkv * D, k_stride, es)},
                       {v, strided_bytes(T, Hkv * D, v_stride, es)}, {qw, qw ? wb : 0}, {kw, kw ? wb : 0},
                       {cache->block_table, static_cast<uint64_t>(B) * cache->max_pages * 4},
                       {cache->seq_lens, static_cast<uint64_t>(B) * 4}, {cache->q_start, static_cast<uint64_t>(B + 1) * 4}};
  const Span outs[5] = {{qo, qo ? static_cast<uint64_t>(T * H * D * es) : 0}, {cache->k, cb}, {cache->v, cb},
                        {f8 ? f8->k_scale : nullptr, sb}, {f8 ? f8->v_scale : nullptr, sb}};
  if (any_overlap(outs, f8 ? 5 : 3, ins, 8)) return DA_EINVAL;
  if (T == 0) return DA_OK;
  const da::QkNormCall c{q, k, qw, kw, qo, nullptr, B, 0, H, Hkv, D, q_stride, k_stride, eps,
                         {rotate != 0, rotate ? center : 0, base, gamma, scale_base}, static_cast<int>(dtype)};
  da::PagedCache pc = paged_cache(cache);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (f8) {
    pc.k_scale = f8->k_scale;
    pc.v_scale = f8->v_scale;
    return da::launch_cache_append8(c, v, v_stride, pc, T, st) == hipSuccess ? DA_OK : DA_EHIP;
  }
  return da::launch_cache_append(c, v, v_stride, pc, T, st) == hipSuccess ? DA_OK : DA_EHIP;
}

// The attention over a cache of the call's type, or (with scales) in 8 bits.
int paged_fwd(const void* q, const da_paged_cache_t* cache, const da_paged_cache_f8_t* f8, void* out, float* lse,
              int64_t T, int64_t B, int64_t H, int64_t Hkv, int64_t D, int64_t q_stride, int64_t max_new,
              const da_pattern_t* patterns, int64_t num_patterns, int64_t dtype, float softmax_scale, void* workspace,
              uint64_t workspace_bytes, void* stream) {
  if (const int rc = head_shapes(T, H, Hkv, D, dtype, &q_stride, &H, 1); rc != DA_OK) return rc;
  if (!cache_ok(B, Hkv, cache) || (f8 && (!f8->k_scale || !f8->v_scale))) return DA_EINVAL;
  da::PagedPlan p;
  if (const int rc = da::make_paged_plan(T, B, H, Hkv, D, cache->num_pages, cache->page_size, cache->max_pages,
                                         max_new, patterns, num_patterns, dtype, softmax_scale, &p);
      rc != DA_OK)
    return rc;
  if (T == 0) return DA_OK;
  if (!q || !out || !lse || !workspace) return DA_EINVAL;
  for (const void* x : {q, static_cast<const void*>(out), static_cast<const void*>(workspace),
                        static_cast<const void*>(cache->k), static_cast<const void*>(cache->v)})
    if (!aligned16(x)) return DA_EALIGN;
  if (!aligned4(cache->block_table) || !aligned4(cache->seq_lens) || !aligned4(cache->q_start) || !aligned4(lse))
    return DA_EALIGN;
  if (workspace_bytes < p.workspace_bytes) return DA_EWORKSPACE;
  const int64_t es = dtype == DA_BF16 ? 2 : 4;
  const uint64_t cb = pool_bytes(cache, Hkv, f8 ? D : D * es), sb = f8 ? scale_bytes(cache, Hkv) : 0;
  const Span ins[8] = {{q, strided_bytes(T, H * D, q_stride, es)}, {cache->k, cb}, {cache->v, cb},
                       {cache->block_table, static_cast<uint64_t>(B) * cache->max_pages * 4},
                       {cache->seq_lens, static_cast<uint64_t>(B) * 4}, {cache->q_start, static_cast<uint64_t>(B + 1) * 4},
                       {f8 ? f8->k_scale : nullptr, sb}, {f8 ? f8->v_scale : nullptr, sb}};
  const Span outs[3] = {{out, static_cast<uint64_t>(T * H * D * es)}, {lse, static_cast<uint64_t>(T * H) * 4},
                        {workspace, p.workspace_bytes}};
  if (any_overlap(outs, 3, ins, f8 ? 8 : 6)) return DA_EINVAL;
  da::PagedCache pc = paged_cache(cache);
  if (f8) {
    pc.k_scale = f8->k_scale;
    pc.v_scale = f8->v_scale;
  }
  return da::launch_paged(p, q, q_stride, pc, out, lse, workspace, static_cast<hipStream_t>(stream)) == hipSuccess
             ? DA_OK
             : DA_EHIP;
}

}  // namespace

int dilated_attn_cache_append(const void* q, const void* k, const void* v, const void* qw, const void* kw, void* qo,
                              const da_paged_cache_t* cache, int64_t T, int64_t B, int64_t H, int64_t Hkv, int64_t D,
                              int64_t q_stride, int64_t k_stride, int64_t v_stride, float eps, int64_t rotate,
                              int64_t center, float base, float gamma, float scale_base, int64_t dtype,
                              void* stream) {
  return cache_append(q, k, v, qw, kw, qo, cache, nullptr, T, B, H, Hkv, D, q_stride, k_stride, v_stride, eps, rotate,
                      center, base, gamma, scale_base, dtype, stream);
}

int dilated_attn_cache_append_f8(const void* q, const void* k, const void* v, const void* qw, const void* kw,
                                 void* qo, const da_paged_cache_f8_t* cache, int64_t T, int64_t B, int64_t H,
                                 int64_t Hkv, int64_t D, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                                 float eps, int64_t rotate, int64_t center, float base, float gamma,
                                 float scale_base, int64_t dtype, void* stream) {
  if (!cache) return DA_EINVAL;
  return cache_append(q, k, v, qw, kw, qo, &cache->pages, cache, T, B, H, Hkv, D, q_stride, k_stride, v_stride, eps,
                      rotate, center, base, gamma, scale_base, dtype, stream);
}

int dilated_attn_paged_workspace(int64_t T, int64_t B, int64_t H, int64_t Hkv, int64_t D, int64_t num_pages,
                                 int64_t page_size, int64_t max_pages, int64_t max_new, const da_pattern_t* patterns,
                                 int64_t num_patterns, int64_t dtype, uint64_t* bytes) {
  if (!bytes) return DA_EINVAL;
  da::PagedPlan p;
  const int rc = da::make_paged_plan(T, B, H, Hkv, D, num_pages, page_size, max_pages, max_new, patterns,
                                     num_patterns, dtype, 0.0f, &p);
  if (rc == DA_OK) *bytes = p.workspace_bytes;
  return rc;
}

int dilated_attn_paged_fwd(const void* q, const da_paged_cache_t* cache, void* out, float* lse, int64_t T, int64_t B,
                           int64_t H, int64_t Hkv, int64_t D, int64_t q_stride, int64_t max_new,
                           const da_pattern_t* patterns, int64_t num_patterns, int64_t dtype, float softmax_scale,
                           void* workspace, uint64_t workspace_bytes, void* stream) {
  return paged_fwd(q, cache, nullptr, out, lse, T, B, H, Hkv, D, q_stride, max_new, patterns, num_patterns, dtype,
                   softmax_scale, workspace, workspace_bytes, stream);
}

int dilated_attn_paged_fwd_f8(const void* q, const da_paged_cache_f8_t* cache, void* out, float* lse, int64_t T,
                              int64_t B, int64_t H, int64_t Hkv, int64_t D, int64_t q_stride, int64_t max_new,
                              const da_pattern_t* patterns, int64_t num_patterns, int64_t dtype,
                              float softmax_scale, void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!cache) return DA_EINVAL;
  return paged_fwd(q, &cache->pages, cache, out, lse, T, B, H, Hkv, D, q_stride, max_new, patterns, num_patterns,
                   dtype, softmax_scale, workspace, workspace_bytes, stream);
}

int dilated_attn_page_weights_workspace(int64_t T, int64_t B, int64_t H, int64_t Hkv, int64_t D, int64_t num_pages,
                                        int64_t page_size, int64_t max_pages, int64_t max_new,
                                        const da_pattern_t* patterns, int64_t num_patterns, int64_t dtype,
                                        uint64_t* bytes) {
  if (!bytes) return DA_EINVAL;
  da::WeightPlan p;
  const int rc = da::make_weight_plan(T, B, H, Hkv, D, num_pages, page_size, max_pages, max_new, patterns, num_patterns,
                                      dtype, 0.0f, &p);
  if (rc == DA_OK) *bytes = p.workspace_bytes;
  return rc;
}

int dilated_attn_page_weights(const void* q, const float* lse, const da_paged_cache_f8_t* cache, float* weights,
                              int64_t T, int64_t B, int64_t H, int64_t Hkv, int64_t D, int64_t q_stride,
                              int64_t max_new, const da_pattern_t* patterns, int64_t num_patterns, int64_t dtype,
                              float softmax_scale, void* workspace, uint64_t workspace_bytes, void* stream) {
  if (const int rc = head_shapes(T, H, Hkv, D, dtype, &q_stride, &H, 1); rc != DA_OK) return rc;
  const da_paged_cache_t* c = cache ? &cache->pages : nullptr;
  if (!cache_ok(B, Hkv, c, false) || !cache->k_scale) return DA_EINVAL;
  da::WeightPlan p;
  if (const int rc = da::make_weight_plan(T, B, H, Hkv, D, c->num_pages, c->page_size, c->max_pages, max_new,
                                          patterns, num_patterns, dtype, softmax_scale, &p);
      rc != DA_OK)
    return rc;
  if (T == 0) return DA_OK;
  if (!q || !lse || !weights || !workspace) return DA_EINVAL;
  for (const void* x : {q, static_cast<const void*>(workspace), static_cast<const void*>(c->k)})
    if (!aligned16(x)) return DA_EALIGN;
  if (!aligned4(c->block_table) || !aligned4(c->seq_lens) || !aligned4(c->q_start) || !aligned4(lse) ||
      !aligned4(weights))
    return DA_EALIGN;
  if (workspace_bytes < p.workspace_bytes) return DA_EWORKSPACE;
  const int64_t es = dtype == DA_BF16 ? 2 : 4;
  const Span ins[7] = {{q, strided_bytes(T, H * D, q_stride, es)}, {lse, static_cast<uint64_t>(T * H) * 4},
                       {c->k, pool_bytes(c, Hkv, D)}, {cache->k_scale, scale_bytes(c, Hkv)},
                       {c->block_table, static_cast<uint64_t>(B) * c->max_pages * 4},
                       {c->seq_lens, static_cast<uint64_t>(B) * 4}, {c->q_start, static_cast<uint64_t>(B + 1) * 4}};
  const Span outs[2] = {{weights, static_cast<uint64_t>(c->num_pages) * 4}, {workspace, p.workspace_bytes}};
  if (any_overlap(outs, 2, ins, 7)) return DA_EINVAL;
  da::PagedCache pc = paged_cache(c);
  pc.k_scale = cache->k_scale;
  return da::launch_page_weights(p, q, q_stride, lse, pc, weights, workspace, static_cast<hipStream_t>(stream)) ==
                 hipSuccess
             ? DA_OK
             : DA_EHIP;
}

int dilated_attn_evict_pages(const float* weights, const int32_t* block_table, const int32_t* seq_lens,
                             int32_t* table_out, int32_t* freed, int32_t* count, int64_t B, int64_t num_pages,
                             int64_t page_size, int64_t max_pages, int64_t keep, int64_t first, int64_t last,
                             void* stream) {
  constexpr int64_t kMost = int64_t{1} << 31;
  if (!weights || !block_table || !seq_lens || !table_out || !freed || !count) return DA_EINVAL;
  if (B < 1 || B >= kMost || num_pages < 1 || num_pages >= kMost || page_size < 1 ||
      page_size > (int64_t{1} << 16) || (page_size & (page_size - 1)) || max_pages < 1 ||
      max_pages > da::kPagedMost / page_size || keep < 0 || first < 0 || last < 0 || last >= kMost)
    return DA_EINVAL;
  for (const void* x : {static_cast<const void*>(weights), static_cast<const void*>(block_table),
                        static_cast<const void*>(seq_lens), static_cast<const void*>(table_out),
                        static_cast<const void*>(freed), static_cast<const void*>(count)})
    if (!aligned4(x)) return DA_EALIGN;
  const uint64_t tb = static_cast<uint64_t>(B) * max_pages * 4;
  const Span ins[3] = {{weights, static_cast<uint64_t>(num_pages) * 4}, {seq_lens, static_cast<uint64_t>(B) * 4},
                       {block_table, table_out == block_table ? 0 : tb}};
  const Span outs[3] = {{table_out, tb}, {freed, tb}, {count, static_cast<uint64_t>(B) * 4}};
  if (any_overlap(outs, 3, ins, 3)) return DA_EINVAL;
  const da::EvictCall c{weights, block_table, seq_lens, table_out, freed, count, B, num_pages, page_size, max_pages,
                        keep, first, last};
  return da::launch_evict(c, static_cast<hipStream_t>(stream)) == hipSuccess ? DA_OK : DA_EHIP;
}

int dilated_attn_profile_begin(int64_t capacity) {
  if (g_prof.active || capacity < 1 || capacity > (int64_t{1} << 20)) return DA_EINVAL;
  g_prof.ev.assign(static_cast<size_t>(3 * capacity), nullptr);
  for (hipEvent_t& e : g_prof.ev) {
    if (hipEventCreate(&e) != hipSuccess) {
      e = nullptr;
      destroy_events(g_prof);
      return DA_EHIP;
    }
  }
  g_prof.capacity = capacity;
  g_prof.used = 0;
  g_prof.active = true;
  return DA_OK;
}

int dilated_attn_profile_end(double* ms_attention, double* ms_combine, int64_t* calls) {
  if (!g_prof.active) return DA_EINVAL;
  double ta = 0.0, tc = 0.0;
  int rc = DA_OK;
  if (g_prof.used > 0 && hipEventSynchronize(g_prof.ev[3 * g_prof.used - 1]) != hipSuccess) rc = DA_EHIP;
  for (int64_t i = 0; i < g_prof.used && rc == DA_OK; ++i) {
    float a = 0.0f, c = 0.0f;
    if (hipEventElapsedTime(&a, g_prof.ev[3 * i], g_prof.ev[3 * i + 1]) != hipSuccess ||
        hipEventElapsedTime(&c, g_prof.ev[3 * i + 1], g_prof.ev[3 * i + 2]) != hipSuccess)
      rc = DA_EHIP;
    ta += a;
    tc += c;
  }
  const int64_t n = g_prof.used;
  destroy_events(g_prof);
  if (rc != DA_OK) return rc;
  if (ms_attention) *ms_attention = ta;
  if (ms_combine) *ms_combine = tc;
  if (calls) *calls = n;
  return DA_OK;
}

const char* dilated_attn_strerror(int code) {
  switch (code) {
    case DA_OK: return "success";
    case DA_EINVAL: return "invalid argument (null pointer, size, pattern list or overlapping buffers)";
    case DA_EUNSUPPORTED: return "unsupported head dimension or dtype";
    case DA_EWORKSPACE: return "workspace smaller than dilated_attn_plan requires";
    case DA_EALIGN: return "device pointer not 16-byte aligned";
    case DA_EHIP: return "HIP runtime error at kernel launch";
    case DA_ETOOLARGE: return "problem needs more workspace than the no-alloc entry point's fixed buffer";
    default: return "unknown error code";
  }
}

}  // extern "C"
