// Cross entropy of given tokens under a vocabulary head, and its gradient, without the logits in memory.
// Only the rows with a target in [0, V) take part: xent_rows_kernel lists them, everything after it
// works on the list.
#pragma once
#include "sip_gemm.h"

namespace sip {

constexpr float kLog2e = 1.4426950408889634f;

__device__ inline uint32_t bf16_bits(float x) {          // round to nearest even; NaN stays NaN
  const __bf16 b = (__bf16)x;
  return __builtin_bit_cast(uint16_t, b);
}
__device__ inline uint2 bf16_pack(float a, float b, float c, float d) {
  return make_uint2(bf16_bits(a) | (bf16_bits(b) << 16), bf16_bits(c) | (bf16_bits(d) << 16));
}

struct XentArgs {
  const uint16_t* hidden; long long hidden_stride;
  const uint16_t* weight; long long weight_stride;
  const int* targets;
  int N, V, D;
  float logit_scale;
  float* loss; float* lse;                // forward: out
  const float* loss_in; const float* lse_in; const float* grad_loss;
  float out_scale;                        // scale * logit_scale
  uint16_t* grad_hidden; long long gh_stride;
  uint16_t* grad_weight; long long gw_stride;
  // workspace
  int* count;                             // rows that take part
  int* rows;                              // [N] their indices, ascending
  float* target_z;                        // [N] z of the target, by place in the list
  float2* part;                           // [N][parts] maximum and sum of a tile's logits without the target
  int parts;
  uint16_t* dense;                        // [N][D] the rows that take part, one after the other
  uint16_t* dz; int piece;                // [N][piece] gradient of a piece's logits
  float* sum;                             // [N][D] of grad_hidden over the pieces
  int v0;                                 // the piece's first vocabulary entry
};

// One workgroup lists the rows.  What is read is N integers once: latency of a launch.
__global__ __launch_bounds__(1024) void xent_rows_kernel(XentArgs p) {
  __shared__ int wave_n[16];
  __shared__ int base;
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  if (t == 0) base = 0;
  for (int i0 = 0; i0 < p.N; i0 += 1024) {
    const int i = i0 + t;
    const bool live = i < p.N && (unsigned)p.targets[i] < (unsigned)p.V;
    const unsigned long long m = __ballot(live);
    if (lane == 0) wave_n[w] = __popcll(m);
    __syncthreads();
    int before = base;
    for (int j = 0; j < w; ++j) before += wave_n[j];
    if (live) p.rows[before + __popcll(m & ((1ull << lane) - 1))] = i;
    else if (i < p.N && p.loss) p.loss[i] = p.lse[i] = 0.0f;
    __syncthreads();
    if (t == 1023) base = before + wave_n[15];
    __syncthreads();
  }
  if (t == 0) *p.count = base;
}

// Row `blockIdx.x` of the list to its place in `dense`; row `blockIdx.x` of grad_hidden to zero if it is masked.
__global__ __launch_bounds__(256) void xent_gather_kernel(XentArgs p) {
  const int i = blockIdx.x;
  if (i < *p.count) {
    const uint4* src = reinterpret_cast<const uint4*>(p.hidden + p.rows[i] * p.hidden_stride);
    uint4* dst = reinterpret_cast<uint4*>(p.dense + (long long)i * p.D);
    for (int c = threadIdx.x; c < p.D / 8; c += 256) dst[c] = src[c];
  }
  if (p.grad_hidden && (unsigned)p.targets[i] >= (unsigned)p.V) {
    uint4* dst = reinterpret_cast<uint4*>(p.grad_hidden + i * p.gh_stride);
    for (int c = threadIdx.x; c < p.D / 8; c += 256) dst[c] = make_uint4(0, 0, 0, 0);
  }
}

// A tile of logits, reduced to its maximum and sum of exponentials per token.
__global__ __launch_bounds__(kGemmThreads) void xent_forward_kernel(XentArgs p) {
  const int n = *p.count, a0 = blockIdx.x * kTileA, b0 = blockIdx.y * kTileB;
  if (b0 >= n) return;
  f32x16 acc{};
  gemm_tile<kRows, kRows>(acc, Operand{p.weight, p.weight_stride, p.V, nullptr}, Operand{p.hidden, p.hidden_stride, n, p.rows},
                          a0, b0, 0, p.D);
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int v_first = a0 + 32 * (w & 1), i = b0 + 32 * (w >> 1) + (lane & 31);
  const bool live = i < n;
  const int target = live ? p.targets[p.rows[i]] : -1;
  float m = -INFINITY, s = 0.0f;
  bool nan = false;
  for (int r = 0; r < 16; ++r) {
    const int v = v_first + acc_a(r, lane);
    acc[r] *= p.logit_scale;
    if (v == target && live) p.target_z[i] = acc[r];
    if (v >= p.V || v == target) acc[r] = -INFINITY;
    nan |= acc[r] != acc[r];
    m = fmaxf(m, acc[r]);
  }
  m = fmaxf(m, __shfl_xor(m, 32));
  const float base = m == -INFINITY ? 0.0f : m;
  for (int r = 0; r < 16; ++r) s += __builtin_amdgcn_exp2f((acc[r] - base) * kLog2e);
  if (nan) s = NAN;
  s += __shfl_xor(s, 32);
  if (live && lane < 32) p.part[(long long)i * p.parts + (v_first >> 5)] = make_float2(m, s);
}

// A wave joins a token's parts.
__global__ __launch_bounds__(256) void xent_loss_kernel(XentArgs p) {
  const int i = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (i >= *p.count) return;
  const float2* part = p.part + (long long)i * p.parts;
  float m = -INFINITY, s = 0.0f;
  for (int j = lane; j < p.parts; j += 64) {
    const float2 q = part[j];
    const float top = fmaxf(m, q.x), base = top == -INFINITY ? 0.0f : top;
    s = s * __builtin_amdgcn_exp2f((m - base) * kLog2e) + q.y * __builtin_amdgcn_exp2f((q.x - base) * kLog2e);
    m = top;
  }
  for (int d = 32; d; d >>= 1) {
    const float mo = __shfl_xor(m, d), so = __shfl_xor(s, d);
    const float top = fmaxf(m, mo), base = top == -INFINITY ? 0.0f : top;
    s = s * __builtin_amdgcn_exp2f((m - base) * kLog2e) + so * __builtin_amdgcn_exp2f((mo - base) * kLog2e);
    m = top;
  }
  if (lane == 0) {
    const float zt = p.target_z[i];
    const float gap = m + logf(s) - zt;                  // ln of the others' mass over the target's
    const float loss = fmaxf(gap, 0.0f) + log1pf(expf(-fabsf(gap)));
    const int row = p.rows[i];
    p.loss[row] = gap != gap ? gap : loss;
    p.lse[row] = zt + loss;
  }
}

// dz of a tile of the piece's logits.
__global__ __launch_bounds__(kGemmThreads) void xent_dz_kernel(XentArgs p) {
  const int n = *p.count, a0 = blockIdx.x * kTileA, b0 = blockIdx.y * kTileB;
  if (b0 >= n) return;
  f32x16 acc{};
  gemm_tile<kRows, kRows>(acc, Operand{p.weight + p.v0 * p.weight_stride, p.weight_stride, p.V - p.v0, nullptr},
                          Operand{p.dense, p.D, n, nullptr}, a0, b0, 0, p.D);
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int v_first = a0 + 32 * (w & 1), i = b0 + 32 * (w >> 1) + (lane & 31);
  if (i >= n) return;
  const int row = p.rows[i], target = p.targets[row] - p.v0;
  const float lse = p.lse_in[row], g = p.grad_loss ? p.grad_loss[row] : 1.0f;
  const float at_target = expm1f(-p.loss_in[row]);
  for (int r = 0; r < 16; r += 4) {
    float d[4];
    for (int e = 0; e < 4; ++e) {
      const int v = v_first + acc_a(r + e, lane);
      d[e] = v >= p.V - p.v0 ? 0.0f : g * (v == target ? at_target : __builtin_amdgcn_exp2f((acc[r + e] * p.logit_scale - lse) * kLog2e));
    }
    *reinterpret_cast<uint2*>(p.dz + (long long)i * p.piece + v_first + acc_a(r, lane)) = bf16_pack(d[0], d[1], d[2], d[3]);
  }
}

// grad_hidden of a piece, added to what the pieces before it gave.
__global__ __launch_bounds__(kGemmThreads) void xent_grad_hidden_kernel(XentArgs p) {
  const int n = *p.count, a0 = blockIdx.x * kTileA, b0 = blockIdx.y * kTileB;
  if (b0 >= n) return;
  const int kv = min(p.piece, p.V - p.v0);
  f32x16 acc{};
  gemm_tile<kCols, kRows>(acc, Operand{p.weight + p.v0 * p.weight_stride, p.weight_stride, p.D, nullptr},
                          Operand{p.dz, p.piece, n, nullptr}, a0, b0, 0, kv);
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int d_first = a0 + 32 * (w & 1), i = b0 + 32 * (w >> 1) + (lane & 31);
  if (i >= n) return;
  const bool last = p.v0 + p.piece >= p.V;
  for (int r = 0; r < 16; r += 4) {
    const int d = d_first + acc_a(r, lane);
    if (d >= p.D) continue;
    float4* sum = reinterpret_cast<float4*>(p.sum + (long long)i * p.D + d);
    float4 s = make_float4(acc[r], acc[r + 1], acc[r + 2], acc[r + 3]);
    if (p.v0) { const float4 o = *sum; s.x += o.x; s.y += o.y; s.z += o.z; s.w += o.w; }
    if (last) {
      const float f = p.out_scale;
      *reinterpret_cast<uint2*>(p.grad_hidden + p.rows[i] * p.gh_stride + d) = bf16_pack(s.x * f, s.y * f, s.z * f, s.w * f);
    } else {
      *sum = s;
    }
  }
}

// grad_weight of a piece's rows.
__global__ __launch_bounds__(kGemmThreads) void xent_grad_weight_kernel(XentArgs p) {
  const int n = *p.count, a0 = blockIdx.x * kTileA, b0 = blockIdx.y * kTileB;
  const int left = p.V - p.v0;
  f32x16 acc{};
  gemm_tile<kCols, kCols>(acc, Operand{p.dense, p.D, p.D, nullptr}, Operand{p.dz, p.piece, p.piece, nullptr}, a0, b0, 0, n);
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int d_first = a0 + 32 * (w & 1), v = b0 + 32 * (w >> 1) + (lane & 31);
  if (v >= left) return;
  const float f = p.out_scale;
  for (int r = 0; r < 16; r += 4) {
    const int d = d_first + acc_a(r, lane);
    if (d < p.D)
      *reinterpret_cast<uint2*>(p.grad_weight + (p.v0 + (long long)v) * p.gw_stride + d) =
          bf16_pack(acc[r] * f, acc[r + 1] * f, acc[r + 2] * f, acc[r + 3] * f);
  }
}

}  // namespace sip
