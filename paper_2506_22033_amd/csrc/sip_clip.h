// Global norm of many tensors, and clipping by it.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sip {

constexpr int kClipThreads = 256;
constexpr int kClipGroups = 2048;          // workgroups of a launch, and partial sums of it
constexpr int kClipTable = 120;            // tensors of a launch: the kernel's arguments stay below 4 KB
constexpr int kClipChunk = 8192;           // elements a workgroup takes at once

struct ClipTable {
  const void* grad[kClipTable];
  void* out[kClipTable];
  long long count[kClipTable];             // elements; the sign bit: bf16
  int n;
};
constexpr long long kClipBf16 = (long long)1 << 62;

template <class F>
__device__ inline void clip_chunks(const ClipTable& t, F f) {
  long long at = blockIdx.x;               // my next chunk, counted from the current tensor's first one
  for (int j = 0; j < t.n; ++j) {
    const long long count = t.count[j] & ~kClipBf16, chunks = (count + kClipChunk - 1) / kClipChunk;
    for (; at < chunks; at += gridDim.x) {
      const long long first = at * kClipChunk;
      f(j, (t.count[j] & kClipBf16) != 0, first, (int)min((long long)kClipChunk, count - first));
    }
    at -= chunks;
  }
}

__device__ inline float bf16_value(uint16_t b) { return __builtin_bit_cast(float, (uint32_t)b << 16); }

__global__ __launch_bounds__(kClipThreads) void clip_squares_kernel(ClipTable t, double* part) {
  __shared__ double wave_sum[kClipThreads / 64];
  double total = 0.0;
  clip_chunks(t, [&](int j, bool bf16, long long first, int n) {
    double s = 0.0;
    if (bf16) {
      const uint16_t* g = static_cast<const uint16_t*>(t.grad[j]) + first;
      for (int i = threadIdx.x; i < n; i += kClipThreads) { const double x = bf16_value(g[i]); s = __builtin_fma(x, x, s); }
    } else {
      const float* g = static_cast<const float*>(t.grad[j]) + first;
      for (int i = threadIdx.x; i < n; i += kClipThreads) { const double x = g[i]; s = __builtin_fma(x, x, s); }
    }
    total += s;
  });
  for (int d = 32; d; d >>= 1) total += __shfl_xor(total, d);
  if ((threadIdx.x & 63) == 0) wave_sum[threadIdx.x >> 6] = total;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.x] = wave_sum[0] + wave_sum[1] + wave_sum[2] + wave_sum[3];
}

__global__ __launch_bounds__(1024) void clip_norm_kernel(const double* part, int n, float max_norm, float eps, float* norm,
                                                         float* factor) {
  __shared__ double wave_sum[16];
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += 1024) s += part[i];
  for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
  if ((threadIdx.x & 63) == 0) wave_sum[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.0;
    for (int i = 0; i < 16; ++i) s += wave_sum[i];
    const float x = (float)sqrt(s);
    *norm = x;
    const float f = max_norm / (x + eps);
    *factor = f > 1.0f || max_norm == INFINITY ? 1.0f : f;   // (a NaN stays, unless nothing bounds the norm)
  }
}

__global__ __launch_bounds__(kClipThreads) void clip_scale_kernel(ClipTable t, const float* factor) {
  const float f = *factor;
  clip_chunks(t, [&](int j, bool bf16, long long first, int n) {
    if (bf16) {
      const uint16_t* g = static_cast<const uint16_t*>(t.grad[j]) + first;
      __bf16* o = static_cast<__bf16*>(t.out[j]) + first;
      for (int i = threadIdx.x; i < n; i += kClipThreads) o[i] = (__bf16)(bf16_value(g[i]) * f);
    } else {
      const float* g = static_cast<const float*>(t.grad[j]) + first;
      float* o = static_cast<float*>(t.out[j]) + first;
      for (int i = threadIdx.x; i < n; i += kClipThreads) o[i] = g[i] * f;
    }
  });
}

}  // namespace sip
