// Rows of an embedding by token, and their gradient.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sip_gemm.h"

namespace sip {

typedef float f32x8 __attribute__((ext_vector_type(8)));

// Eight neighbours of a row of bf16 or fp32 as floats, and back; in memory aligned to 16 bytes.
struct Eight { u32x4 w[2]; };                             // bf16: the first alone
__device__ inline Eight load_eight(const void* base, long long at, bool bf16) {
  Eight x;
  const u32x4* p = reinterpret_cast<const u32x4*>(static_cast<const char*>(base) + at * (bf16 ? 2 : 4));
  x.w[0] = p[0];
  if (!bf16) x.w[1] = p[1];
  return x;
}
__device__ inline f32x8 as_floats(const Eight& x, bool bf16) {
  f32x8 f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t w = bf16 ? (e & 1 ? x.w[0][e / 2] & 0xffff0000u : x.w[0][e / 2] << 16) : x.w[e / 4][e % 4];
    f[e] = __builtin_bit_cast(float, w);                 // (of a vector's element itself it is one of the first)
  }
  return f;
}
__device__ inline void store_eight(void* base, long long at, bool bf16, const f32x8& f) {
  u32x4* p = reinterpret_cast<u32x4*>(static_cast<char*>(base) + at * (bf16 ? 2 : 4));
  if (bf16) {
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      w[e] = __builtin_bit_cast(uint16_t, (__bf16)f[2 * e]) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)f[2 * e + 1]) << 16;
    p[0] = w;
  } else {
    f32x4* q = reinterpret_cast<f32x4*>(p);
    q[0] = __builtin_shufflevector(f, f, 0, 1, 2, 3);
    q[1] = __builtin_shufflevector(f, f, 4, 5, 6, 7);
  }
}

// ---------------------------------------------------------------- lookup

struct EmbedArgs {
  const void* weight; long long weight_stride; int weight_bf16;
  const uint8_t* codes; long long codes_stride;          // nullptr: weight
  const void* scales; int scales_bf16;
  const uint8_t* zeros;
  int group;
  int V, D, N;
  const int* ids;
  float scale;
  void* out; long long out_stride; int out_bf16;
};

// A lane takes eight neighbours of a row.
template <bool CODES>
__global__ __launch_bounds__(256) void embed_kernel(EmbedArgs a) {
  const long long per_row = a.D / 8, total = per_row * a.N;
  for (long long u = blockIdx.x * 256ll + threadIdx.x; u < total; u += gridDim.x * 256ll) {
    const int i = (int)(u / per_row), c = (int)(u - i * per_row) * 8, v = a.ids[i];
    f32x8 f = {0, 0, 0, 0, 0, 0, 0, 0};
    if ((unsigned)v < (unsigned)a.V) {
      if constexpr (CODES) {
        const uint32_t q = *reinterpret_cast<const uint32_t*>(a.codes + v * a.codes_stride + c / 2);
        const long long at = (long long)v * (a.D / a.group) + c / a.group;
        const float s = a.scales_bf16 ? (float)static_cast<const __bf16*>(a.scales)[at] : static_cast<const float*>(a.scales)[at];
        const int zero = a.zeros ? a.zeros[at] : 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = (float)((int)(q >> 4 * e & 15) - zero) * s;
      } else {
        f = as_floats(load_eight(a.weight, v * a.weight_stride + c, a.weight_bf16), a.weight_bf16);
      }
      f *= a.scale;
    }
    store_eight(a.out, i * a.out_stride + c, a.out_bf16, f);
  }
}

// ---------------------------------------------------------------- gradient
// The tokens are sorted, equal ones in the order of their positions.  The sorted list is cut into pieces; a lane sums eight
// neighbouring columns of a piece's rows, token by token.  What a token has in one piece alone is final; what crosses the
// border of a piece goes to the workspace in fp32, and a second kernel adds it up in order.

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;

struct EmbedGradArgs {
  const void* grad; long long grad_stride; int grad_bf16;
  const int* ids;
  int N, V, D;
  float scale;
  int accumulate;
  void* out; long long out_stride; int out_bf16;
  int piece;                                             // entries of a piece
  // workspace
  int* live;                                             // entries that take part
  uint32_t* key[2]; uint32_t* pos[2];                    // [N] tokens and their positions, sorted in the first pair
  float* part;                                           // [pieces][2][D] sums of what crosses a border: on the left, on the right
};

// Workgroup 0 sorts: three passes of a stable sort by seven bits each, lowest first; a wave has a run of entries.  Masked tokens come
// last.  The others fill grad_weight with zeros, unless it is added to.
__global__ __launch_bounds__(kSortThreads) void embed_sort_kernel(EmbedGradArgs a) {
  constexpr int kBits = 7, kBins = 1 << kBits;
  __shared__ uint32_t at[kBins][kSortWaves], wave_total[kSortWaves];
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  if (blockIdx.x > 0) {
    const long long per_row = a.D / 8, total = per_row * a.V, step = (gridDim.x - 1) * (long long)kSortThreads;
    const f32x8 none = {0, 0, 0, 0, 0, 0, 0, 0};
    for (long long u = (blockIdx.x - 1) * (long long)kSortThreads + t; u < total; u += step) {
      const long long v = u / per_row;
      store_eight(a.out, v * a.out_stride + (u - v * per_row) * 8, a.out_bf16, none);
    }
    return;
  }
  const int run = (a.N + kSortThreads - 1) / kSortThreads * 64, first = w * run, last = min(a.N, first + run);
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass * kBits;
    const uint32_t* key_in = pass ? a.key[(pass - 1) & 1] : nullptr;
    const uint32_t* pos_in = pass ? a.pos[(pass - 1) & 1] : nullptr;
    uint32_t* key_out = a.key[pass & 1];
    uint32_t* pos_out = a.pos[pass & 1];
    auto key_of = [&](int i) {
      if (pass) return key_in[i];
      const uint32_t v = (uint32_t)a.ids[i];
      return v < (uint32_t)a.V ? v : (uint32_t)a.V;
    };
    for (int i = t; i < kBins * kSortWaves; i += kSortThreads) at[i / kSortWaves][i % kSortWaves] = 0;
    __syncthreads();
    for (int i = first + lane; i < last; i += 64) atomicAdd(&at[key_of(i) >> shift & (kBins - 1)][w], 1u);
    __syncthreads();
    // where a wave's entries of a digit begin: those of lower digits, then those of earlier waves (2048 numbers, two a thread)
    uint32_t* flat = &at[0][0];
    const uint32_t x0 = flat[2 * t], x1 = flat[2 * t + 1];
    uint32_t sum = x0 + x1;
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t other = __shfl_up(sum, d);
      if (lane >= d) sum += other;
    }
    if (lane == 63) wave_total[w] = sum;
    __syncthreads();
    uint32_t before = sum - x0 - x1;
    for (int j = 0; j < w; ++j) before += wave_total[j];
    flat[2 * t] = before;
    flat[2 * t + 1] = before + x0;
    __syncthreads();
    for (int i0 = first; i0 < last; i0 += 64) {
      const int i = i0 + lane;
      const bool mine = i < last;
      const uint32_t key = mine ? key_of(i) : 0, digit = key >> shift & (kBins - 1);
      unsigned long long same = __ballot(mine);
#pragma unroll
      for (int b = 0; b < kBits; ++b) {
        const unsigned long long set = __ballot(digit >> b & 1);
        same &= digit >> b & 1 ? set : ~set;
      }
      const int rank = __popcll(same & ((1ull << lane) - 1));
      uint32_t base = 0;
      if (mine) base = at[digit][w];
      if (mine && rank == 0) at[digit][w] = base + __popcll(same);
      if (mine) {
        key_out[base + rank] = key;
        pos_out[base + rank] = pass ? pos_in[i] : (uint32_t)i;
      }
    }
    __syncthreads();                                     // (and what was written is read by the workgroup itself)
  }
  const uint32_t* key = a.key[0];
  if (t == 0) *a.live = 0;
  __syncthreads();
  for (int i = t; i < a.N; i += kSortThreads)
    if (key[i] < (uint32_t)a.V && (i + 1 == a.N || key[i + 1] >= (uint32_t)a.V)) *a.live = i + 1;
}

__device__ inline void embed_store(const EmbedGradArgs& a, int v, int c, f32x8 sum) {
  sum *= a.scale;
  const long long at = v * a.out_stride + c;
  if (a.accumulate) sum += as_floats(load_eight(a.out, at, a.out_bf16), a.out_bf16);
  store_eight(a.out, at, a.out_bf16, sum);
}

// A lane: eight columns of one piece.
template <bool BF16>
__global__ __launch_bounds__(256) void embed_sum_kernel(EmbedGradArgs a) {
  const int per_row = a.D / 8, n = *a.live;
  const long long u = blockIdx.x * 256ll + threadIdx.x;
  const int piece = (int)(u / per_row), c = (int)(u - (long long)piece * per_row) * 8;
  const long long first = (long long)piece * a.piece;
  if (first >= n) return;
  const int last = (int)min((long long)n, first + a.piece);
  const uint32_t* key = a.key[0];
  const uint32_t* pos = a.pos[0];
  const f32x8 none = {0, 0, 0, 0, 0, 0, 0, 0};
  f32x8 sum = none;
  bool begun = first == 0 || key[first - 1] != key[first];             // the token's first entry is in this piece
  for (int i = (int)first; i < last; ++i) {
    sum += as_floats(load_eight(a.grad, pos[i] * a.grad_stride + c, BF16), BF16);
    const bool ends = i + 1 == n || key[i + 1] != key[i];
    if (!ends && i + 1 < last) continue;
    if (begun && ends) embed_store(a, (int)key[i], c, sum);
    else store_eight(a.part, ((long long)piece * 2 + begun) * a.D + c, false, sum);
    sum = none;
    begun = true;
  }
}

// The token that piece `blockIdx.x`'s right border cuts first, if it begins in that piece: sixteen lanes of eight columns, of which each
// has sixteen workers that take every sixteenth of the pieces.
__global__ __launch_bounds__(256) void embed_join_kernel(EmbedGradArgs a) {
  __shared__ f32x8 sums[16][16];
  const int n = *a.live, piece = blockIdx.x;
  const long long border = (long long)(piece + 1) * a.piece;
  if (border >= n) return;
  const uint32_t* key = a.key[0];
  const uint32_t v = key[border];
  if (key[border - 1] != v) return;
  const long long begin = (long long)piece * a.piece;
  if (begin > 0 && key[begin] == v && key[begin - 1] == v) return;     // it began before
  long long end = n;                                     // behind its last entry
  for (long long low = border; low < end;) {
    const long long mid = (low + end) / 2;
    if (key[mid] > v) end = mid;
    else low = mid + 1;
  }
  const int pieces = (int)((end - 1) / a.piece) - piece, worker = threadIdx.x >> 4, c = (blockIdx.y * 16 + (threadIdx.x & 15)) * 8;
  f32x8 sum = {0, 0, 0, 0, 0, 0, 0, 0};
  if (c < a.D)
    for (int j = worker; j <= pieces; j += 16)
      sum += as_floats(load_eight(a.part, ((long long)(piece + j) * 2 + (j == 0)) * a.D + c, false), false);
  sums[worker][threadIdx.x & 15] = sum;
  __syncthreads();
  if (worker > 0 || c >= a.D) return;
  for (int j = 1; j < 16; ++j) sum += sums[j][threadIdx.x & 15];
  embed_store(a, (int)v, c, sum);
}

}  // namespace sip
