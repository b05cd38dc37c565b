// A vocabulary head of 4-bit codes with group scales: the quantiser, and the product with hidden states.
#pragma once
#include "sip_gemm.h"

namespace sip {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct CodesArgs {
  const uint16_t* weight; long long weight_stride;     // quantiser: in
  uint8_t* codes; long long codes_stride;
  void* scales; int scales_bf16;
  uint8_t* zeros;
  int V, D, group;
  // product
  const void* hidden; long long hidden_stride; int hidden_bf16;
  int B;
  void* logits; long long logits_stride; int logits_bf16;
};

__device__ inline float scale_at(const CodesArgs& p, long long i) {
  return p.scales_bf16 ? __builtin_bit_cast(float, (uint32_t)static_cast<const uint16_t*>(p.scales)[i] << 16)
                       : static_cast<const float*>(p.scales)[i];
}

// A thread quantises a group.
__global__ __launch_bounds__(256) void quantize_kernel(CodesArgs p) {
  const int groups = p.D / p.group;
  const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
  if (id >= (long long)p.V * groups) return;
  const int v = (int)(id / groups), g = (int)(id % groups);
  const uint16_t* w = p.weight + v * p.weight_stride + g * p.group;
  float lo = 0.0f, hi = 0.0f;
  for (int e = 0; e < p.group; ++e) {
    const float x = __builtin_bit_cast(float, (uint32_t)w[e] << 16);
    lo = fminf(lo, x);
    hi = fmaxf(hi, x);
  }
  float s = p.zeros ? (hi - lo) / 15.0f : fmaxf(hi, -lo) / 7.0f;
  if (p.scales_bf16) s = (float)(__bf16)s;
  if (s == 0.0f) s = 1.0f;
  const float zero = p.zeros ? fminf(fmaxf(rintf(-lo / s), 0.0f), 15.0f) : 8.0f;
  if (p.scales_bf16) static_cast<__bf16*>(p.scales)[id] = (__bf16)s;
  else static_cast<float*>(p.scales)[id] = s;
  if (p.zeros) p.zeros[id] = (uint8_t)zero;
  uint8_t* c = p.codes + v * p.codes_stride + g * (p.group / 2);
  for (int e = 0; e < p.group; e += 2) {
    int q[2];
    for (int h = 0; h < 2; ++h) {
      const float x = __builtin_bit_cast(float, (uint32_t)w[e + h] << 16);
      q[h] = (int)fminf(fmaxf(rintf(x / s) + zero, 0.0f), 15.0f);
    }
    c[e / 2] = (uint8_t)(q[0] | (q[1] << 4));
  }
}

// Eight codes of a dword as the bf16 values 16 + q (q in the mantissa's bits 3 to 6 over the exponent of 16), in the
// order 0 4 1 5 2 6 3 7: no conversion, one shift and one and-or for a pair.
__device__ inline u32x4 code_values(uint32_t c) {
  constexpr uint32_t kMask = 0x00780078u, k16 = 0x41804180u;
  u32x4 r;
  r[0] = ((c << 3) & kMask) | k16;
  r[1] = ((c >> 1) & kMask) | k16;
  r[2] = ((c >> 5) & kMask) | k16;
  r[3] = ((c >> 9) & kMask) | k16;
  return r;
}

// A wave makes the logits of 16 rows and 16 vocabulary entries.  fp32 hidden states enter as three bf16 parts.
__global__ __launch_bounds__(64) void head_logits_kernel(CodesArgs p) {
  const int lane = threadIdx.x, v = blockIdx.y * 16 + (lane & 15), b = blockIdx.x * 16 + (lane & 15), q4 = lane >> 4;
  const int groups = p.D / p.group;
  const uint8_t* codes = p.codes + min(v, p.V - 1) * p.codes_stride;
  const char* x_row = static_cast<const char*>(p.hidden) + min(b, p.B - 1) * p.hidden_stride * (p.hidden_bf16 ? 2 : 4);
  f32x4 total{};
  for (int g = 0; g < groups; ++g) {
    const long long at = (long long)min(v, p.V - 1) * groups + g;
    const float s = scale_at(p, at), zero = 16.0f + (p.zeros ? (float)p.zeros[at] : 8.0f);
    f32x4 acc{}, sum{};
    for (int k = g * p.group; k < (g + 1) * p.group; k += 32) {
      const u32x4 cv = code_values(*reinterpret_cast<const uint32_t*>(codes + k / 2 + q4 * 4));
      float x[8];
      for (int e = 0; e < 8; ++e) {
        const int at_e = k + q4 * 8 + (e >> 1) + 4 * (e & 1);
        x[e] = p.hidden_bf16 ? __builtin_bit_cast(float, (uint32_t)reinterpret_cast<const uint16_t*>(x_row)[at_e] << 16)
                             : reinterpret_cast<const float*>(x_row)[at_e];
      }
      u32x4 ones;
      for (int e = 0; e < 4; ++e) ones[e] = 0x3f803f80u;
      for (int part = 0; part < (p.hidden_bf16 ? 1 : 3); ++part) {
        u32x4 xv;
        for (int e = 0; e < 8; e += 2) {
          const uint32_t h0 = __builtin_bit_cast(uint32_t, x[e]) & 0xffff0000u, h1 = __builtin_bit_cast(uint32_t, x[e + 1]) & 0xffff0000u;
          xv[e / 2] = (h0 >> 16) | h1;
          x[e] -= __builtin_bit_cast(float, h0);
          x[e + 1] -= __builtin_bit_cast(float, h1);
        }
        const bf16x8 xb = __builtin_bit_cast(bf16x8, xv);
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xb, __builtin_bit_cast(bf16x8, cv), acc, 0, 0, 0);
        sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xb, __builtin_bit_cast(bf16x8, ones), sum, 0, 0, 0);
      }
    }
    for (int r = 0; r < 4; ++r) total[r] = __builtin_fmaf(s, __builtin_fmaf(-zero, sum[r], acc[r]), total[r]);
  }
  for (int r = 0; r < 4; ++r) {
    const int row = blockIdx.x * 16 + 4 * q4 + r;
    if (row < p.B && v < p.V) {
      if (p.logits_bf16) static_cast<__bf16*>(p.logits)[row * p.logits_stride + v] = (__bf16)total[r];
      else static_cast<float*>(p.logits)[row * p.logits_stride + v] = total[r];
    }
  }
}

}  // namespace sip
