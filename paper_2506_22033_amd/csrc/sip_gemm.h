// Products of bf16 matrices with fp32 sums, a tile at a time, for the kernels of sip_xent.h:
//   C[b][a] = sum_k A(a, k) * B(b, k),
// either operand with its rows along k (kRows) or with k as the row index (kCols).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sip {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

enum OperandForm { kRows, kCols };

// One operand: element (i, k) of it is base[i * stride + k] (kRows) or base[k * stride + i] (kCols).  kRows with
// `rows`: row i is row rows[i] of base.
struct Operand {
  const uint16_t* base;
  long long stride;
  int n;                              // indices i from here on are zeros
  const int* rows;
};

constexpr int kGemmThreads = 256;
constexpr int kTileA = 64, kTileB = 64, kTileK = 32;
constexpr int kGemmPitch = kTileK + 8;

// The 32 x 32 block of C that a wave holds: register r of a lane is row a0 + acc_a(r, lane), column b0 + lane % 32.
__device__ inline int acc_a(int r, int lane) { return 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3); }

template <OperandForm F>
__device__ inline void stage_tile(uint16_t* lds, const Operand& m, int i0, int k0, int k_end) {
  if (F == kRows) {
    const int i = threadIdx.x >> 2, c = (threadIdx.x & 3) * 8;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (i0 + i < m.n && k0 + c < k_end) {
      const long long row = m.rows ? m.rows[i0 + i] : i0 + i;
      v = *reinterpret_cast<const uint4*>(m.base + row * m.stride + k0 + c);
    }
    *reinterpret_cast<uint4*>(lds + i * kGemmPitch + c) = v;
  } else {
    const int k = threadIdx.x >> 3, c = (threadIdx.x & 7) * 8;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (i0 + c < m.n && k0 + k < k_end) v = *reinterpret_cast<const uint4*>(m.base + (long long)(k0 + k) * m.stride + i0 + c);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    for (int e = 0; e < 8; ++e) lds[(c + e) * kGemmPitch + k] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
  }
}

// Wave w of a workgroup's four holds the block at a0 + 32 * (w & 1), b0 + 32 * (w >> 1).
template <OperandForm FA, OperandForm FB>
__device__ inline void gemm_tile(f32x16& acc, const Operand& A, const Operand& B, int a0, int b0, int k_begin, int k_end) {
  __shared__ __attribute__((aligned(16))) uint16_t la[kTileA * kGemmPitch], lb[kTileB * kGemmPitch];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  for (int k = k_begin; k < k_end; k += kTileK) {
    __syncthreads();
    stage_tile<FA>(la, A, a0, k, k_end);
    stage_tile<FB>(lb, B, b0, k, k_end);
    __syncthreads();
    for (int s = 0; s < kTileK; s += 16) {
      const bf16x8 a = *reinterpret_cast<const bf16x8*>(la + (32 * (w & 1) + (lane & 31)) * kGemmPitch + s + 8 * (lane >> 5));
      const bf16x8 b = *reinterpret_cast<const bf16x8*>(lb + (32 * (w >> 1) + (lane & 31)) * kGemmPitch + s + 8 * (lane >> 5));
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc, 0, 0, 0);
    }
  }
}

}  // namespace sip
