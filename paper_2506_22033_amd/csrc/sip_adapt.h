// Low-rank adapters of many requests: every row's own addition to its logits.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/sip_head.h"
#include "sip_embed.h"

namespace sip {

// Rows that share an adapter are served sixteen at a time, a batch: the sixteen columns of a matrix instruction, whose rows are an
// adapter's.  Both products read their adapter from memory straight into the instruction's registers.
constexpr int kAdaptRows = 16;
// Up to so many rows a wave finds its batch by itself.  One row, rank 16, V = 128256: 4.3 + 5.5 us, instead of 2.9 + 4.2 + 5.3 with a kernel that lists
// the rows.  (Near the limit listing is shorter: 59 rows of 57 adapters of rank 8, V = 125990, 10.7 + 47.2 and 4.6 + 7.4 + 36.8.)
constexpr int kAdaptDirect = 64;

struct AdaptArgs {
  const void* hidden; long long hidden_stride;
  int B, D, V, rank, adapters;
  const uint16_t* down; const uint16_t* up;
  const int* adapter_of_row; const float* scales;
  void* logits; long long logits_stride;
  // workspace
  int* count;                                            // batches
  int* rows;                                             // [B] rows that have an adapter, by adapter
  int4* batch;                                           // [B] first of a batch in `rows`, its size, its adapter
  float* t;                                              // [parts][batches][16][rank] scales[a] * down[a] hidden[b], a part of the sum over D each
  int parts, batches;
};

// One workgroup lists the rows by adapter, in batches.  (The order of an adapter's rows changes no result.)  Latency: 256 rows 4.8 us.
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
      for (int j = 0; j < m; ++j) p.batch[bm + j] = make_int4(bn + j * kAdaptRows, min(kAdaptRows, n - j * kAdaptRows), i, 0);
    }
    __syncthreads();
  }
  for (int b = t; b < p.B; b += 1024)
    if ((unsigned)p.adapter_of_row[b] < (unsigned)A) p.rows[atomicAdd(&first[p.adapter_of_row[b]], 1)] = b;
  if (t == 0) *p.count = batches;
}

// A batch as a wave sees it: its size (0: there is none), its adapter, and the row of column lane % 16 (-1: none).
struct Batch { int n, adapter, row; };
template <bool DIRECT>
__device__ inline Batch batch_of(const AdaptArgs& p, int i) {
  const int lane = threadIdx.x & 63;
  Batch x = {0, 0, -1};
  if constexpr (DIRECT) {
    // Lane b is row b; its place among its adapter's rows.  Every sixteenth leads a batch; the i-th leader's is the one.
    int a = lane < p.B ? p.adapter_of_row[lane] : -1, place = 0;
    if ((unsigned)a >= (unsigned)p.adapters) a = -1;
    for (int j = 0; j < p.B; ++j) place += j < lane && __builtin_amdgcn_readlane(a, j) == a;
    unsigned long long leaders = __ballot(a >= 0 && place % kAdaptRows == 0);
    for (int j = 0; j < i; ++j) leaders &= leaders - 1;
    if (!leaders) return x;
    const int leader = __builtin_ctzll(leaders), from = __builtin_amdgcn_readlane(place, leader);
    x.adapter = __builtin_amdgcn_readlane(a, leader);
    unsigned long long mine = __ballot(a == x.adapter && place >= from && place < from + kAdaptRows);
    x.n = __popcll(mine);
    for (int j = 0; j < (lane & 15); ++j) mine &= mine - 1;
    if ((lane & 15) < x.n) x.row = __builtin_ctzll(mine);
  } else {
    const int4 b = p.batch[i];                           // (read whether there is one or not)
    if (i >= *p.count) return x;
    x.n = b.y;
    x.adapter = b.z;
    if ((lane & 15) < x.n) x.row = p.rows[b.x + (lane & 15)];
  }
  return x;
}

// Eight floats as the sum of three bf16 each, which hold all their bits.
struct Split { bf16x8 part[3]; };
__device__ inline Split split_of(f32x8 x) {
  Split s;
#pragma unroll
  for (int i = 0; i < 3; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const __bf16 b = (__bf16)x[e];
      s.part[i][e] = b;
      x[e] -= (float)b;
    }
  return s;
}

// t of a batch, sixteen entries a workgroup: its waves share a part of the sum over D and join what they have in order.  Bound by reading:
// 32 adapters of rank 64, D = 4096, 16.8 MB, 10.3 us; one of rank 16 4.4 us in four parts, 6.9 in one.
constexpr int kDownWaves = 16, kDownParts = 4;
template <bool BF16, bool DIRECT>
__global__ __launch_bounds__(kDownWaves * 64) void adapt_down_kernel(AdaptArgs p) {
  __shared__ __align__(16) f32x4 sums[kDownWaves][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, k = 8 * (lane >> 4);
  const Batch x = batch_of<DIRECT>(p, blockIdx.x);
  if (x.n == 0) return;
  const int j = blockIdx.y * 16 + (lane & 15);
  const uint16_t* down = p.down + ((long long)x.adapter * p.rank + j) * p.D;
  const bool live = j < p.rank;
  const float scale = p.scales ? p.scales[x.adapter] : 1.0f;
  f32x4 acc = {0, 0, 0, 0};
  const bf16x8 none = {};
  constexpr int kAhead = BF16 ? 8 : 4;                   // steps whose loads are under way at once
  const int each = (p.D + p.parts * 32 - 1) / (p.parts * 32) * 32, begin = blockIdx.z * each, end = min(p.D, begin + each);
  for (int c0 = begin + w * 32; c0 < end; c0 += kAhead * kDownWaves * 32) {
    bf16x8 a[kAhead];
    Eight h[kAhead];
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
      const int c = c0 + s * kDownWaves * 32 + k;
      a[s] = live && c < end ? *reinterpret_cast<const bf16x8*>(down + c) : none;
      h[s] = Eight{};
      if (x.row >= 0 && c < end) h[s] = load_eight(p.hidden, x.row * p.hidden_stride + c, BF16);
    }
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
      if constexpr (BF16) {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[s], __builtin_bit_cast(bf16x8, h[s].w[0]), acc, 0, 0, 0);
      } else {
        const Split b = split_of(as_floats(h[s], false));
#pragma unroll
        for (int i = 2; i >= 0; --i) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[s], b.part[i], acc, 0, 0, 0);
      }
    }
  }
  sums[w][lane] = acc;
  __syncthreads();
  if (w > 0) return;
  for (int i = 1; i < kDownWaves; ++i) acc += sums[i][lane];
  const int j0 = blockIdx.y * 16 + acc_a(lane);
  if (x.row < 0 || j0 >= p.rank) return;
  const long long at = ((long long)blockIdx.z * p.batches + blockIdx.x) * kAdaptRows + (lane & 15);
  *reinterpret_cast<f32x4*>(p.t + at * p.rank + j0) = acc * scale;
}

// The additions of one batch to `tiles` of kUpWaves * 32 logits each.  A wave's share of a tile is 32 entries of the vocabulary, of
// which a lane has eight neighbours of one row, loaded and stored wherever they lie: two matrix products, one for the first four of every
// eight, one for the others (four a lane are 32 bytes of a bf16 row at once: 219 rows, 40 adapters of rank 8, V = 214517 130 us instead of 82).  ONE: tiles = 1, and t may be in parts.
// t enters as three bf16 parts, which hold its 24 bits: the products are exact, the matrix cores hardly busy.  Bound by memory: 224 rows, 32
// adapters of rank 64, V = 128256, 760 MB, 161 us, 4.7 TB/s (555 us with a lane an entry of the vocabulary and fp32 products).
constexpr int kUpWaves = 4, kUpEntries = kUpWaves * 32;
struct __attribute__((packed, aligned(4))) FourF32 { f32x4 x; };        // four logits as they may lie: aligned to one
struct __attribute__((packed, aligned(2))) EightBf16 { u32x4 x; };
template <bool BF16>
__device__ inline f32x8 load_logits(const void* logits, long long at) {
  Eight x;
  if constexpr (BF16) {
    x.w[0] = reinterpret_cast<const EightBf16*>(static_cast<const uint16_t*>(logits) + at)->x;
  } else {
    const FourF32* p = reinterpret_cast<const FourF32*>(static_cast<const float*>(logits) + at);
    x.w[0] = __builtin_bit_cast(u32x4, p[0]);
    x.w[1] = __builtin_bit_cast(u32x4, p[1]);
  }
  return as_floats(x, BF16);
}
template <bool BF16>
__device__ inline void store_logits(void* logits, long long at, const f32x8& x) {
  if constexpr (BF16) {
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = __builtin_bit_cast(uint16_t, (__bf16)x[2 * e]) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x[2 * e + 1]) << 16;
    *reinterpret_cast<EightBf16*>(static_cast<uint16_t*>(logits) + at) = EightBf16{w};
  } else {
    FourF32* p = reinterpret_cast<FourF32*>(static_cast<float*>(logits) + at);
    p[0] = FourF32{__builtin_shufflevector(x, x, 0, 1, 2, 3)};
    p[1] = FourF32{__builtin_shufflevector(x, x, 4, 5, 6, 7)};
  }
}
template <int STEPS, bool ONE, bool DIRECT, bool BF16>
__global__ __launch_bounds__(kUpWaves * 64) void adapt_up_kernel(AdaptArgs p, int batches, int tiles) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, k = 8 * (lane >> 4);
  // batches of one adapter go through the same entries one after the other on one XCD, whose L2 then has them
  const int local = blockIdx.x >> 3, i = local % batches, v0 = ((local / batches) * 8 + (blockIdx.x & 7)) * tiles * kUpEntries;
  if (v0 >= p.V) return;
  const Batch x = batch_of<DIRECT>(p, i);
  if (x.n == 0) return;
  const uint16_t* up = p.up + (long long)x.adapter * p.V * p.rank;
  const bf16x8 none = {};
  // Tiles whose loads are under way at once, kEarly while as many others are multiplied.  More waves do better where their loads are short: rank
  // 8 as above 82 us, two tiles the same, kEarly 91, four tiles 96; rank 64 as above 161 with two, 164 with one and 163 not kEarly; 220 rows of 10
  // adapters of rank 112, V = 213705, 170, 176 not kEarly and 179 with two.
  constexpr bool kEarly = ONE || STEPS > 1;
  constexpr int kAhead = ONE || STEPS != 2 ? 1 : 2;
  constexpr int kParts = ONE ? kDownParts : 1;
  struct Loads {
    bf16x8 a[kAhead][2][STEPS];
    f32x8 z[kAhead];
  };
  auto first_of = [&](int tile) { return tile < tiles ? v0 + (tile * kUpWaves + w) * 32 : p.V; };       // (V: there is none)
  // row r of a product is entry 8 (r / 4) + r % 4, and that plus 4 of the second one: lane l then has 8 (l / 16) and what follows of row l % 16
  const int entry0 = 8 * ((lane & 15) >> 2) + (lane & 3), at0 = 8 * (lane >> 4);
  auto load = [&](Loads& l, int tile0) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int v = first_of(tile0 + j), at = v + at0;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int entry = v + entry0 + 4 * half;
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
          l.a[j][half][s] = entry < p.V && 32 * s + k < p.rank ? *reinterpret_cast<const bf16x8*>(up + (long long)entry * p.rank + 32 * s + k) : none;
      }
      l.z[j] = f32x8{0, 0, 0, 0, 0, 0, 0, 0};
      if (x.row < 0 || at >= p.V) continue;
      const long long z0 = x.row * p.logits_stride + at;
      if (at + 8 <= p.V) {
        l.z[j] = load_logits<BF16>(p.logits, z0);
      } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
          if (at + e < p.V) l.z[j][e] = BF16 ? (float)static_cast<const __bf16*>(p.logits)[z0 + e] : static_cast<const float*>(p.logits)[z0 + e];
      }
    }
  };
  Eight t_part[STEPS][kParts];
#pragma unroll
  for (int s = 0; s < STEPS; ++s)
#pragma unroll
    for (int part = 0; part < kParts; ++part) {
      t_part[s][part] = Eight{};
      const long long at = (((long long)part * batches + i) * kAdaptRows + (lane & 15)) * p.rank + 32 * s + k;
      if (part < p.parts && x.row >= 0 && 32 * s + k < p.rank) t_part[s][part] = load_eight(p.t, at, false);
    }
  Loads next;
  if (kEarly) load(next, 0);
  Split t[STEPS];
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    f32x8 sum = as_floats(t_part[s][0], false);
#pragma unroll
    for (int part = 1; part < kParts; ++part) sum += as_floats(t_part[s][part], false);
    t[s] = split_of(sum);
  }
  for (int tile0 = 0; tile0 < tiles; tile0 += kAhead) {
    if (!kEarly) load(next, tile0);
    const Loads now = next;
    if (kEarly && tile0 + kAhead < tiles) load(next, tile0 + kAhead);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int at = first_of(tile0 + j) + at0;
      f32x4 acc[2];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        acc[half] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int part = 2; part >= 0; --part)
#pragma unroll
          for (int s = 0; s < STEPS; ++s) acc[half] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(now.a[j][half][s], t[s].part[part], acc[half], 0, 0, 0);
      }
      const f32x8 sum = __builtin_shufflevector(acc[0], acc[1], 0, 1, 2, 3, 4, 5, 6, 7) + now.z[j];
      if (x.row < 0 || at >= p.V) continue;
      const long long z0 = x.row * p.logits_stride + at;
      if (at + 8 <= p.V) {
        store_logits<BF16>(p.logits, z0, sum);
      } else {
#pragma unroll
        for (int e = 0; e < 7; ++e) {
          if (at + e >= p.V) break;
          if (BF16) static_cast<__bf16*>(p.logits)[z0 + e] = (__bf16)sum[e];
          else static_cast<float*>(p.logits)[z0 + e] = sum[e];
        }
      }
    }
  }
}

}  // namespace sip
