// Low-rank adapters of many requests: every row's own addition to its logits.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/sip_head.h"
#include "sip_embed.h"

namespace sip {

constexpr int kAdaptRows = 16;                           // rows of one adapter that a workgroup serves at once

struct AdaptArgs {
  const void* hidden; long long hidden_stride; int hidden_bf16;
  int B, D, V, rank, adapters;
  const uint16_t* down; const uint16_t* up;
  const int* adapter_of_row; const float* scales;
  void* logits; long long logits_stride; int logits_bf16;
  // workspace
  int* count;                                            // batches
  int* rows;                                             // [B] rows that have an adapter, by adapter
  int2* batch;                                           // [B] first of a batch in `rows` and its size; the adapter is that of its rows
  float* t;                                              // [B][rank] scales[a] * down[a] hidden[b]
};

// One workgroup lists the rows by adapter, in batches of up to kAdaptRows.  (The order of an adapter's rows changes no result.)
__global__ __launch_bounds__(1024) void adapt_rows_kernel(AdaptArgs p) {
  __shared__ int first[SIP_MAX_ADAPTERS], wave_n[16], wave_m[16];
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, A = p.adapters;
  for (int i = t; i < A; i += 1024) first[i] = 0;
  __syncthreads();
  for (int b = t; b < p.B; b += 1024)
    if ((unsigned)p.adapter_of_row[b] < (unsigned)A) atomicAdd(&first[p.adapter_of_row[b]], 1);
  __syncthreads();
  int rows = 0, batches = 0;                             // of the adapters before
  for (int i0 = 0; i0 < A; i0 += 1024) {
    const int i = i0 + t, n = i < A ? first[i] : 0, m = (n + kAdaptRows - 1) / kAdaptRows;
    int sn = n, sm = m;
    for (int d = 1; d < 64; d <<= 1) {
      const int on = __shfl_up(sn, d), om = __shfl_up(sm, d);
      if (lane >= d) { sn += on; sm += om; }
    }
    if (lane == 63) { wave_n[w] = sn; wave_m[w] = sm; }
    __syncthreads();
    int bn = rows + sn - n, bm = batches + sm - m;
    for (int j = 0; j < 16; ++j) {
      if (j < w) { bn += wave_n[j]; bm += wave_m[j]; }
      rows += wave_n[j];
      batches += wave_m[j];
    }
    if (i < A) {
      first[i] = bn;
      for (int j = 0; j < m; ++j) p.batch[bm + j] = make_int2(bn + j * kAdaptRows, min(kAdaptRows, n - j * kAdaptRows));
    }
    __syncthreads();
  }
  for (int b = t; b < p.B; b += 1024)
    if ((unsigned)p.adapter_of_row[b] < (unsigned)A) p.rows[atomicAdd(&first[p.adapter_of_row[b]], 1)] = b;
  if (t == 0) *p.count = batches;
}

// t of one row, eight of its entries a workgroup: two a wave.
__global__ __launch_bounds__(256) void adapt_down_kernel(AdaptArgs p) {
  const int b = blockIdx.x, lane = threadIdx.x & 63, w = threadIdx.x >> 6, adapter = p.adapter_of_row[b];
  if ((unsigned)adapter >= (unsigned)p.adapters) return;
  const float scale = p.scales ? p.scales[adapter] : 1.0f;
  for (int j = blockIdx.y * 8 + w * 2; j < blockIdx.y * 8 + w * 2 + 2; ++j) {
    float s = 0.0f;
    for (int c = lane * 8; c < p.D; c += 512) {
      const f32x8 x = as_floats(load_eight(p.hidden, b * p.hidden_stride + c, p.hidden_bf16), p.hidden_bf16);
      const f32x8 y = as_floats(load_eight(p.down, ((long long)adapter * p.rank + j) * p.D + c, true), true);
#pragma unroll
      for (int e = 0; e < 8; ++e) s += x[e] * y[e];
    }
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    if (lane == 0) p.t[(long long)b * p.rank + j] = s * scale;
  }
}

// A lane: one vocabulary entry of one batch's rows.
__global__ __launch_bounds__(256) void adapt_up_kernel(AdaptArgs p) {
  const int v = blockIdx.x * 256 + threadIdx.x;
  for (int i = blockIdx.y; i < *p.count; i += gridDim.y) {
    const int2 batch = p.batch[i];
    const int adapter = p.adapter_of_row[p.rows[batch.x]];
    if (v >= p.V) continue;
    float sum[kAdaptRows] = {};
    for (int j = 0; j < p.rank; j += 8) {
      const f32x8 u = as_floats(load_eight(p.up, ((long long)adapter * p.V + v) * p.rank + j, true), true);
#pragma unroll
      for (int r = 0; r < kAdaptRows; ++r) {
        if (r >= batch.y) break;
        const float* t = p.t + (long long)p.rows[batch.x + r] * p.rank + j;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[r] = __builtin_fmaf(u[e], t[e], sum[r]);
      }
    }
#pragma unroll
    for (int r = 0; r < kAdaptRows; ++r) {
      if (r >= batch.y) break;
      const long long at = p.rows[batch.x + r] * p.logits_stride + v;
      if (p.logits_bf16) {
        __bf16* z = static_cast<__bf16*>(p.logits) + at;
        *z = (__bf16)((float)*z + sum[r]);
      } else {
        static_cast<float*>(p.logits)[at] += sum[r];
      }
    }
  }
}

}  // namespace sip
