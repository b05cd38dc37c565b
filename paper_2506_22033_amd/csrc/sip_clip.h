// Global norm of many tensors, and clipping by it.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sip {

constexpr int kClipThreads = 256;
constexpr int kClipGroups = 1024;          // most workgroups of a launch, four a compute unit, and partial sums of it
constexpr int kClipTable = 120;            // tensors of a launch: the kernel's arguments stay below 4 KB
constexpr int kClipBytes = 32768;          // of a tensor that a workgroup takes at once: eight 16-byte loads a lane

struct ClipTable {
  const char* grad[kClipTable];
  char* out[kClipTable];
  long long count[kClipTable];             // elements; kClipBf16 on top: bf16
  uint32_t end[kClipTable];                // chunks of kClipBytes up to this tensor's last
  int n;
};
constexpr long long kClipBf16 = (long long)1 << 62;
inline __host__ __device__ long long clip_bytes(long long count) { return count & kClipBf16 ? 2 * (count & ~kClipBf16) : 4 * count; }

// Sixteen bytes that are aligned to an element only.
struct __attribute__((packed, aligned(2))) ClipLine { uint32_t w[4]; };

// f(tensor, first byte, bytes) for the workgroup's chunks; `back`: the last ones first.  The tensor by bisection: a walk along
// the table took 16 us for 100 tensors.
template <class F>
__device__ inline void clip_chunks(const ClipTable& t, bool back, F f) {
  const uint32_t chunks = t.n ? t.end[t.n - 1] : 0;
  for (uint32_t at = blockIdx.x; at < chunks; at += gridDim.x) {
    const uint32_t chunk = back ? chunks - 1 - at : at;
    int j = 0;                             // the first tensor that ends behind the chunk
    for (int above = t.n - 1; j < above;) {
      const int mid = (j + above) / 2;
      if (chunk < t.end[mid]) above = mid;
      else j = mid + 1;
    }
    const long long first = (long long)(chunk - (j ? t.end[j - 1] : 0)) * kClipBytes;
    f(j, first, (int)min((long long)kClipBytes, clip_bytes(t.count[j]) - first));
  }
}

__device__ inline float bf16_low(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ inline float bf16_high(uint32_t w) { return __builtin_bit_cast(float, w & 0xffff0000u); }
__device__ inline double clip_square(double s, float x) { return __builtin_fma((double)x, (double)x, s); }

// Squares in fp64, where no gradient's overflows: twelve vector operations for eight bytes of bf16, a third of what the reads
// leave time for.
// 290 tensors, 8e8 elements, a fifth of them fp32: both kernels together 1.16 ms, 5 TB/s of what is read, read again and written.
__global__ __launch_bounds__(kClipThreads) void clip_squares_kernel(ClipTable t, double* part) {
  __shared__ double wave_sum[kClipThreads / 64];
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  clip_chunks(t, false, [&](int j, long long first, int n) {
    const bool bf16 = (t.count[j] & kClipBf16) != 0;
    const char* g = t.grad[j] + first;
    auto add = [&](const ClipLine& l) {
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        if (bf16) {
          s[w] = clip_square(s[w], bf16_low(l.w[w]));
          s[w] = clip_square(s[w], bf16_high(l.w[w]));
        } else {
          s[w] = clip_square(s[w], __builtin_bit_cast(float, l.w[w]));
        }
      }
    };
    if (n == kClipBytes) {
      ClipLine l[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) l[i] = *reinterpret_cast<const ClipLine*>(g + (i * kClipThreads + threadIdx.x) * 16);
#pragma unroll
      for (int i = 0; i < 8; ++i) add(l[i]);
    } else {
      int i = threadIdx.x * 16;
      for (; i + 16 <= n; i += kClipThreads * 16) add(*reinterpret_cast<const ClipLine*>(g + i));
      for (; i < n; i += bf16 ? 2 : 4)                     // what is left of the lane's sixteen bytes
        s[0] = clip_square(s[0], bf16 ? bf16_low(*reinterpret_cast<const uint16_t*>(g + i)) : *reinterpret_cast<const float*>(g + i));
    }
  });
  double total = (s[0] + s[1]) + (s[2] + s[3]);
  for (int d = 32; d; d >>= 1) total += __shfl_xor(total, d);
  if ((threadIdx.x & 63) == 0) wave_sum[threadIdx.x >> 6] = total;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.x] = (wave_sum[0] + wave_sum[1]) + (wave_sum[2] + wave_sum[3]);
}

// Every workgroup adds up the partial sums for itself, all in the same order; the first of the first launch stores the norm.
// Tensors go back to front: what the sums read last is still in the 256 MB cache.
__global__ __launch_bounds__(kClipThreads) void clip_scale_kernel(ClipTable t, const double* part, int parts, float max_norm, float eps,
                                                                  float* norm) {
  __shared__ double wave_sum[kClipThreads / 64];
  double s = 0.0;
  for (int i = threadIdx.x; i < parts; i += kClipThreads) s += part[i];
  for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
  if ((threadIdx.x & 63) == 0) wave_sum[threadIdx.x >> 6] = s;
  __syncthreads();
  const float x = (float)sqrt((wave_sum[0] + wave_sum[1]) + (wave_sum[2] + wave_sum[3])), bound = max_norm / (x + eps);
  // (a NaN stays, unless nothing bounds the norm or there is nothing but zeros)
  const float f = bound > 1.0f || max_norm == INFINITY || x + eps == 0.0f ? 1.0f : bound;
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = x;
  clip_chunks(t, true, [&](int j, long long first, int n) {
    const bool bf16 = (t.count[j] & kClipBf16) != 0;
    if (f == 1.0f && t.grad[j] == t.out[j]) return;        // in place, and nothing to do
    const char* g = t.grad[j] + first;
    char* o = t.out[j] + first;
    auto scaled = [&](ClipLine l) {
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        if (bf16) {
          const __bf16 a = (__bf16)(bf16_low(l.w[w]) * f), b = (__bf16)(bf16_high(l.w[w]) * f);
          l.w[w] = __builtin_bit_cast(uint16_t, a) | (uint32_t)__builtin_bit_cast(uint16_t, b) << 16;
        } else {
          l.w[w] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(float, l.w[w]) * f);
        }
      }
      return l;
    };
    if (n == kClipBytes) {
      ClipLine l[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) l[i] = *reinterpret_cast<const ClipLine*>(g + (i * kClipThreads + threadIdx.x) * 16);
#pragma unroll
      for (int i = 0; i < 8; ++i) *reinterpret_cast<ClipLine*>(o + (i * kClipThreads + threadIdx.x) * 16) = scaled(l[i]);
    } else {
      int i = threadIdx.x * 16;
      for (; i + 16 <= n; i += kClipThreads * 16) *reinterpret_cast<ClipLine*>(o + i) = scaled(*reinterpret_cast<const ClipLine*>(g + i));
      for (; i < n; i += bf16 ? 2 : 4) {
        if (bf16) *reinterpret_cast<__bf16*>(o + i) = (__bf16)(bf16_low(*reinterpret_cast<const uint16_t*>(g + i)) * f);
        else *reinterpret_cast<float*>(o + i) = *reinterpret_cast<const float*>(g + i) * f;
      }
    }
  });
}

}  // namespace sip
