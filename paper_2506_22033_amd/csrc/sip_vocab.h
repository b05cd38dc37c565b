// Host side of the entry points declared in include/sip_head.h: argument checks, workspace carving, launches.
#pragma once
#include <algorithm>

#include "../../include/sip_head.h"
#include "sip_clip.h"
#include "sip_codes.h"
#include "sip_xent.h"

namespace {

inline size_t head_align(size_t x) { return (x + 255) / 256 * 256; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool workspace_ok(const void* p, size_t have, size_t need) {
  return p && (reinterpret_cast<uintptr_t>(p) & 255u) == 0 && have >= need;
}

// How a cross entropy of this shape is cut, and where its parts lie in the workspace.
struct XentPlan {
  int parts;                    // tiles' partial sums of a token
  int piece;                    // vocabulary entries whose dz is held at once
  size_t count, rows, target_z, part, dense, dz, sum, bytes;
};

XentPlan xent_plan(int32_t N, int32_t V, int32_t D, bool backward) {
  XentPlan p{};
  p.parts = (V + sip::kTileA - 1) / sip::kTileA * (sip::kTileA / 32);
  const long long most = std::max<long long>(256, ((1ll << 28) / N) / 256 * 256);   // dz: half a gigabyte at most, or 256 columns
  const long long pieces = (V + most - 1) / most;
  p.piece = (int)(((V + pieces - 1) / pieces + 255) / 256 * 256);
  size_t at = 0;
  auto take = [&](size_t n) { const size_t here = at; at += head_align(n); return here; };
  p.count = take(4);
  p.rows = take((size_t)N * 4);
  // the two directions' own parts share the room behind
  const size_t both = at;
  p.target_z = take((size_t)N * 4);
  p.part = take((size_t)N * p.parts * 8);
  p.bytes = at;
  if (backward) {
    at = both;
    p.dense = take((size_t)N * D * 2);
    p.dz = take((size_t)N * p.piece * 2);
    p.sum = take((size_t)N * D * 4);
    p.bytes = std::max(p.bytes, at);
  }
  return p;
}

bool xent_shape_ok(int32_t N, int32_t V, int32_t D) {
  return N > 0 && V > 0 && D > 0 && N <= SIP_MAX_TOKENS && V <= SIP_MAX_V && D <= SIP_MAX_D && D % 8 == 0;
}

sip_status xent_check(const void* hidden, int32_t N, int32_t D, int64_t hidden_stride, const void* weight, int32_t V,
                      int64_t weight_stride, const int32_t* targets) {
  if (!hidden || !weight || !targets || N <= 0 || V <= 0 || D <= 0 || D % 8 != 0) return SIP_ERR_INVALID_ARG;
  if (hidden_stride < D || weight_stride < D || hidden_stride % 8 != 0 || weight_stride % 8 != 0 || !aligned16(hidden) ||
      !aligned16(weight))
    return SIP_ERR_INVALID_ARG;
  if (!xent_shape_ok(N, V, D) || hidden_stride > (1ll << 30) / N || weight_stride > (1 << 20)) return SIP_ERR_UNSUPPORTED;
  return SIP_OK;
}

sip::XentArgs xent_args(const void* hidden, int32_t N, int32_t D, int64_t hidden_stride, const void* weight, int32_t V,
                        int64_t weight_stride, const int32_t* targets, float logit_scale, const XentPlan& pl,
                        void* workspace) {
  sip::XentArgs a{};
  char* ws = static_cast<char*>(workspace);
  a.hidden = static_cast<const uint16_t*>(hidden); a.hidden_stride = hidden_stride;
  a.weight = static_cast<const uint16_t*>(weight); a.weight_stride = weight_stride;
  a.targets = targets;
  a.N = N; a.V = V; a.D = D;
  a.logit_scale = logit_scale;
  a.count = reinterpret_cast<int*>(ws + pl.count);
  a.rows = reinterpret_cast<int*>(ws + pl.rows);
  a.target_z = reinterpret_cast<float*>(ws + pl.target_z);
  a.part = reinterpret_cast<float2*>(ws + pl.part);
  a.parts = pl.parts;
  a.dense = reinterpret_cast<uint16_t*>(ws + pl.dense);
  a.dz = reinterpret_cast<uint16_t*>(ws + pl.dz);
  a.piece = pl.piece;
  a.sum = reinterpret_cast<float*>(ws + pl.sum);
  return a;
}

inline sip_status launched() { return hipGetLastError() == hipSuccess ? SIP_OK : SIP_ERR_HIP; }
inline int tiles(int n, int tile) { return (n + tile - 1) / tile; }

}  // namespace

extern "C" {

size_t sip_xent_workspace_bytes(int32_t N, int32_t V, int32_t D, int32_t backward) {
  return xent_shape_ok(N, V, D) ? xent_plan(N, V, D, backward != 0).bytes : 0;
}

sip_status sip_xent_forward(const void* hidden, int32_t N, int32_t D, int64_t hidden_stride, const void* weight,
                            int32_t V, int64_t weight_stride, const int32_t* targets, float logit_scale, float* loss,
                            float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const sip_status ok = xent_check(hidden, N, D, hidden_stride, weight, V, weight_stride, targets);
  if (ok != SIP_OK) return ok;
  if (!loss || !lse) return SIP_ERR_INVALID_ARG;
  const XentPlan pl = xent_plan(N, V, D, false);
  if (!workspace_ok(workspace, workspace_bytes, pl.bytes)) return SIP_ERR_WORKSPACE;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  sip::XentArgs a = xent_args(hidden, N, D, hidden_stride, weight, V, weight_stride, targets, logit_scale, pl, workspace);
  a.loss = loss; a.lse = lse;
  hipLaunchKernelGGL(sip::xent_rows_kernel, dim3(1), dim3(1024), 0, stream, a);
  hipLaunchKernelGGL(sip::xent_forward_kernel, dim3(tiles(V, sip::kTileA), tiles(N, sip::kTileB)), dim3(sip::kGemmThreads), 0,
                     stream, a);
  hipLaunchKernelGGL(sip::xent_loss_kernel, dim3(tiles(N, 4)), dim3(256), 0, stream, a);
  return launched();
}

sip_status sip_xent_backward(const void* hidden, int32_t N, int32_t D, int64_t hidden_stride, const void* weight,
                             int32_t V, int64_t weight_stride, const int32_t* targets, float logit_scale,
                             const float* loss, const float* lse, const float* grad_loss, float scale,
                             void* grad_hidden, int64_t grad_hidden_stride, void* grad_weight,
                             int64_t grad_weight_stride, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const sip_status ok = xent_check(hidden, N, D, hidden_stride, weight, V, weight_stride, targets);
  if (ok != SIP_OK) return ok;
  if (!loss || !lse) return SIP_ERR_INVALID_ARG;
  if (grad_hidden && (grad_hidden_stride < D || grad_hidden_stride % 8 != 0 || !aligned16(grad_hidden))) return SIP_ERR_INVALID_ARG;
  if (grad_weight && (grad_weight_stride < D || grad_weight_stride % 8 != 0 || !aligned16(grad_weight))) return SIP_ERR_INVALID_ARG;
  const XentPlan pl = xent_plan(N, V, D, true);
  if (!workspace_ok(workspace, workspace_bytes, pl.bytes)) return SIP_ERR_WORKSPACE;
  if (!grad_hidden && !grad_weight) return SIP_OK;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  sip::XentArgs a = xent_args(hidden, N, D, hidden_stride, weight, V, weight_stride, targets, logit_scale, pl, workspace);
  a.loss_in = loss; a.lse_in = lse; a.grad_loss = grad_loss;
  a.out_scale = scale * logit_scale;
  a.grad_hidden = static_cast<uint16_t*>(grad_hidden); a.gh_stride = grad_hidden_stride;
  a.grad_weight = static_cast<uint16_t*>(grad_weight); a.gw_stride = grad_weight_stride;
  hipLaunchKernelGGL(sip::xent_rows_kernel, dim3(1), dim3(1024), 0, stream, a);
  hipLaunchKernelGGL(sip::xent_gather_kernel, dim3(N), dim3(256), 0, stream, a);
  for (int v0 = 0; v0 < V; v0 += pl.piece) {
    a.v0 = v0;
    const int left = std::min(pl.piece, V - v0);
    hipLaunchKernelGGL(sip::xent_dz_kernel, dim3(tiles(left, sip::kTileA), tiles(N, sip::kTileB)), dim3(sip::kGemmThreads), 0,
                       stream, a);
    if (grad_hidden)
      hipLaunchKernelGGL(sip::xent_grad_hidden_kernel, dim3(tiles(D, sip::kTileA), tiles(N, sip::kTileB)),
                         dim3(sip::kGemmThreads), 0, stream, a);
    if (grad_weight)
      hipLaunchKernelGGL(sip::xent_grad_weight_kernel, dim3(tiles(D, sip::kTileA), tiles(left, sip::kTileB)),
                         dim3(sip::kGemmThreads), 0, stream, a);
  }
  return launched();
}

size_t sip_grad_clip_workspace_bytes(int32_t n_tensors) {
  if (n_tensors < 0 || n_tensors > SIP_MAX_TENSORS) return 0;
  const int launches = std::max(1, tiles(n_tensors, sip::kClipTable));
  return 256 + head_align((size_t)launches * sip::kClipGroups * sizeof(double));
}

sip_status sip_grad_clip(const sip_grad* tensors, int32_t n_tensors, float max_norm, float eps, float* norm,
                         void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (n_tensors < 0 || (n_tensors > 0 && !tensors) || !norm || !(max_norm >= 0.0f) || !(eps >= 0.0f)) return SIP_ERR_INVALID_ARG;
  if (n_tensors > SIP_MAX_TENSORS) return SIP_ERR_UNSUPPORTED;
  for (int j = 0; j < n_tensors; ++j) {
    const sip_grad& t = tensors[j];
    if (t.count < 0 || (t.dtype != SIP_F32 && t.dtype != SIP_BF16)) return SIP_ERR_INVALID_ARG;
    if (t.count > 0 && (!t.grad || !t.out)) return SIP_ERR_INVALID_ARG;
    if (t.count > (1ll << 40)) return SIP_ERR_UNSUPPORTED;
    const uintptr_t mask = t.dtype == SIP_F32 ? 3 : 1;
    if (((reinterpret_cast<uintptr_t>(t.grad) | reinterpret_cast<uintptr_t>(t.out)) & mask) != 0) return SIP_ERR_INVALID_ARG;
  }
  if (!workspace_ok(workspace, workspace_bytes, sip_grad_clip_workspace_bytes(n_tensors))) return SIP_ERR_WORKSPACE;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  float* factor = static_cast<float*>(workspace);
  double* part = reinterpret_cast<double*>(static_cast<char*>(workspace) + 256);
  const int launches = std::max(1, tiles(n_tensors, sip::kClipTable));
  auto table = [&](int l) {
    sip::ClipTable t{};
    for (int j = l * sip::kClipTable; j < std::min(n_tensors, (l + 1) * sip::kClipTable); ++j, ++t.n) {
      t.grad[t.n] = tensors[j].grad;
      t.out[t.n] = tensors[j].out;
      t.count[t.n] = tensors[j].count | (tensors[j].dtype == SIP_BF16 ? sip::kClipBf16 : 0);
    }
    return t;
  };
  for (int l = 0; l < launches; ++l)
    hipLaunchKernelGGL(sip::clip_squares_kernel, dim3(sip::kClipGroups), dim3(sip::kClipThreads), 0, stream, table(l),
                       part + (size_t)l * sip::kClipGroups);
  hipLaunchKernelGGL(sip::clip_norm_kernel, dim3(1), dim3(1024), 0, stream, part, launches * sip::kClipGroups, max_norm, eps, norm,
                     factor);
  for (int l = 0; l < launches; ++l)
    hipLaunchKernelGGL(sip::clip_scale_kernel, dim3(sip::kClipGroups), dim3(sip::kClipThreads), 0, stream, table(l), factor);
  return launched();
}

namespace {
// What the quantiser and the product check alike.
sip_status codes_check(const void* codes, int64_t codes_stride, const void* scales, sip_dtype scales_dtype, int32_t V,
                       int32_t D, int32_t group) {
  if (!codes || !scales || V <= 0 || D <= 0 || (scales_dtype != SIP_F32 && scales_dtype != SIP_BF16)) return SIP_ERR_INVALID_ARG;
  if (group != 32 && group != 64 && group != 128) return group > 0 ? SIP_ERR_UNSUPPORTED : SIP_ERR_INVALID_ARG;
  if (D % group != 0 || codes_stride < D / 2 || codes_stride % 16 != 0 || !aligned16(codes)) return SIP_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(scales) & (scales_dtype == SIP_F32 ? 3 : 1)) != 0) return SIP_ERR_INVALID_ARG;
  if (V > SIP_MAX_V || D > SIP_MAX_D || codes_stride > (1 << 20)) return SIP_ERR_UNSUPPORTED;
  return SIP_OK;
}
}  // namespace

sip_status sip_head_quantize(const void* weight, int32_t V, int32_t D, int64_t weight_stride, int32_t group,
                             uint8_t* codes, int64_t codes_stride, void* scales, sip_dtype scales_dtype,
                             uint8_t* zeros, void* hip_stream) {
  if (!weight) return SIP_ERR_INVALID_ARG;
  const sip_status ok = codes_check(codes, codes_stride, scales, scales_dtype, V, D, group);
  if (ok != SIP_OK) return ok;
  if (weight_stride < D || weight_stride % 8 != 0 || !aligned16(weight)) return SIP_ERR_INVALID_ARG;
  if (weight_stride > (1 << 20)) return SIP_ERR_UNSUPPORTED;
  sip::CodesArgs a{};
  a.weight = static_cast<const uint16_t*>(weight); a.weight_stride = weight_stride;
  a.codes = codes; a.codes_stride = codes_stride;
  a.scales = scales; a.scales_bf16 = scales_dtype == SIP_BF16;
  a.zeros = zeros;
  a.V = V; a.D = D; a.group = group;
  const long long groups = (long long)V * (D / group);
  hipLaunchKernelGGL(sip::quantize_kernel, dim3((unsigned)((groups + 255) / 256)), dim3(256), 0,
                     static_cast<hipStream_t>(hip_stream), a);
  return launched();
}

size_t sip_head_workspace_bytes(int32_t B, int32_t V, int32_t D, int32_t group) {
  if (B <= 0 || V <= 0 || D <= 0 || B > SIP_MAX_B || V > SIP_MAX_V || D > SIP_MAX_D) return 0;
  if ((group != 32 && group != 64 && group != 128) || D % group != 0) return 0;
  return 256;
}

sip_status sip_head_logits(const void* hidden, int32_t B, int32_t D, int64_t hidden_stride, sip_dtype hidden_dtype,
                           const uint8_t* codes, int64_t codes_stride, const void* scales, sip_dtype scales_dtype,
                           const uint8_t* zeros, int32_t group, int32_t V, void* logits, int64_t logits_stride,
                           sip_dtype logits_dtype, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!hidden || !logits || B <= 0 || (hidden_dtype != SIP_F32 && hidden_dtype != SIP_BF16) ||
      (logits_dtype != SIP_F32 && logits_dtype != SIP_BF16))
    return SIP_ERR_INVALID_ARG;
  const sip_status ok = codes_check(codes, codes_stride, scales, scales_dtype, V, D, group);
  if (ok != SIP_OK) return ok;
  const int x_size = hidden_dtype == SIP_F32 ? 4 : 2, z_size = logits_dtype == SIP_F32 ? 4 : 2;
  if (hidden_stride < D || hidden_stride * x_size % 16 != 0 || !aligned16(hidden) || logits_stride < V ||
      reinterpret_cast<uintptr_t>(logits) % z_size != 0)
    return SIP_ERR_INVALID_ARG;
  if (B > SIP_MAX_B || hidden_stride > (1ll << 32) || logits_stride > (1ll << 32)) return SIP_ERR_UNSUPPORTED;
  if (!workspace_ok(workspace, workspace_bytes, sip_head_workspace_bytes(B, V, D, group))) return SIP_ERR_WORKSPACE;
  sip::CodesArgs a{};
  a.codes = const_cast<uint8_t*>(codes); a.codes_stride = codes_stride;
  a.scales = const_cast<void*>(scales); a.scales_bf16 = scales_dtype == SIP_BF16;
  a.zeros = const_cast<uint8_t*>(zeros);
  a.V = V; a.D = D; a.group = group;
  a.hidden = hidden; a.hidden_stride = hidden_stride; a.hidden_bf16 = hidden_dtype == SIP_BF16;
  a.B = B;
  a.logits = logits; a.logits_stride = logits_stride; a.logits_bf16 = logits_dtype == SIP_BF16;
  hipLaunchKernelGGL(sip::head_logits_kernel, dim3(tiles(B, 16), tiles(V, 16)), dim3(64), 0,
                     static_cast<hipStream_t>(hip_stream), a);
  return launched();
}

}  // extern "C"
