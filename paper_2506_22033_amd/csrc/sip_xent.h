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
__device__ inline u32x2 bf16_pack(f32x4 x) {
  return u32x2{bf16_bits(x[0]) | (bf16_bits(x[1]) << 16), bf16_bits(x[2]) | (bf16_bits(x[3]) << 16)};
}

// A product whose long sum is dealt out: part i has the `split` k (dealt()) from i * split on, and its sums lie behind those of the parts
// before it, [tiles] of them, tile by tile in the order of the accumulators: a lane's four neighbours, a wave's lanes in a row.
struct Parts {
  float* sum;
  int tiles, count, split;
};

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
  float2* part;                           // [N][parts] maximum and sum of a wave's logits without the target
  int parts;
  uint16_t* dense;                        // the rows that take part, one after the other, [dz_parts()][count][D]
  uint16_t* dz; int piece;                // gradient of a piece's logits, [dz_parts()][count][piece]
  Parts hidden_parts, weight_parts;
  int v0;                                 // the piece's first vocabulary entry
};

// Up to here a token's dz is held in two bf16 parts, as two rows: what bf16 holds of it, and what that leaves.  Its rounding is an error
// of its own in every gradient, and where few tokens make one up it may all go one way.  What counts is the tokens that take
// part.  These calls are bound by reading the head and writing its gradient: V = 128256, D = 4096 take 850 us instead of 762
// for 64 tokens, 735 instead of 717 for one; 41 tokens among 2048, D = 2048, 514 instead of 470.
constexpr int kTwoPartRows = 64;
__host__ __device__ inline int dz_parts(int count) { return count <= kTwoPartRows ? 2 : 1; }

// One workgroup lists the rows, eight targets a thread a turn.  What is read is N integers once: latency.
__global__ __launch_bounds__(1024) void xent_rows_kernel(XentArgs p) {
  __shared__ int wave_n[2][16];
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  int base = 0, side = 0;
  for (int first = 0; first < p.N; first += 8192, side ^= 1) {
    const int i0 = first + t * 8;
    uint32_t live = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (i0 + e < p.N && (unsigned)p.targets[i0 + e] < (unsigned)p.V) live |= 1u << e;
    const int mine = __popc(live);
    int before = mine;                                   // of the wave's lanes up to mine
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int other = __shfl_up(before, d);
      if (lane >= d) before += other;
    }
    if (lane == 63) wave_n[side][w] = before;
    __syncthreads();
    int at = base + before - mine;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const int n = wave_n[side][j];
      if (j < w) at += n;
      base += n;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (live >> e & 1) p.rows[at++] = i0 + e;
      else if (i0 + e < p.N && p.loss) p.loss[i0 + e] = p.lse[i0 + e] = 0.0f;
    }
  }
  if (t == 0) *p.count = base;
}

// Row `blockIdx.x` of the list to its place in `dense`; row `blockIdx.x` of grad_hidden to zero if it is masked.
__global__ __launch_bounds__(256) void xent_gather_kernel(XentArgs p) {
  const int i = blockIdx.x, n = *p.count;
  if (i < n) {
    const uint4* src = reinterpret_cast<const uint4*>(p.hidden + p.rows[i] * p.hidden_stride);
    for (int part = 0; part < dz_parts(n); ++part) {
      uint4* dst = reinterpret_cast<uint4*>(p.dense + (i + (long long)part * n) * p.D);
      for (int c = threadIdx.x; c < p.D / 8; c += 256) dst[c] = src[c];
    }
  }
  if (p.grad_hidden && (unsigned)p.targets[i] >= (unsigned)p.V) {
    uint4* dst = reinterpret_cast<uint4*>(p.grad_hidden + i * p.gh_stride);
    for (int c = threadIdx.x; c < p.D / 8; c += 256) dst[c] = make_uint4(0, 0, 0, 0);
  }
}

// Which tile a workgroup takes of tiles_a x tiles_b.  The eight XCDs, to which workgroups go in turn, take a run of
// tiles each; within it eight tiles along a go with one along b before the next, so that the 32 of an XCD that are under
// way share their rows of either operand in its L2.  Of `parts` such sets, one after the other, `part` is the one.  False: none is left.
__device__ inline bool tile_of(int id, int tiles_a, int tiles_b, int parts, int& ta, int& tb, int& part) {
  constexpr int kGroup = 8;
  const int total = tiles_a * tiles_b * parts, run = (total + 7) / 8;
  const int local = id >> 3, at = (id & 7) * run + local;
  if (local >= run || at >= total) return false;
  part = at / (tiles_a * tiles_b);
  const int s = at - part * (tiles_a * tiles_b);
  const int first = s / (kGroup * tiles_b) * kGroup, width = min(kGroup, tiles_a - first), r = s - first * tiles_b;
  ta = first + r % width;
  tb = r / width;
  return true;
}
__device__ inline bool tile_of(int id, int tiles_a, int tiles_b, int& ta, int& tb) {
  int part;
  return tile_of(id, tiles_a, tiles_b, 1, ta, tb, part);
}
__host__ __device__ inline int div_up(int a, int b) { return (a + b - 1) / b; }

// Where the blocks of a wave begin in the tile.
template <class S> __device__ inline int wave_a() { return (int)(threadIdx.x >> 6) % (S::kA / S::kWaveA) * S::kWaveA; }
template <class S> __device__ inline int wave_b() { return (int)(threadIdx.x >> 6) / (S::kA / S::kWaveA) * S::kWaveB; }

// The tile's values value(i, j) -- the lane's four of block (i, j) -- as bf16, row by row through LDS, to where row(b) says
// (nullptr: nowhere), columns [a0, a_end).  A lane holds four neighbours of one row: eight bytes, whose 16-byte group goes
// to place group ^ row, so that 16 rows meet every bank once; rows leave in 16-byte groups.
// `two`: of the first kTwo rows alone, and as rows kTwo + b what bf16 leaves of row b.
template <class S> constexpr int kTwo = S::kB < kTwoPartRows ? S::kB : kTwoPartRows;
template <class S, class Value, class Row>
__device__ inline void store_tile(SIP_LDS char* lds, int a0, int a_end, Value value, Row row, bool two = false) {
  constexpr int kPitch = S::kA * 2, kGroups = S::kA / 8, kMask = kGroups < 16 ? kGroups - 1 : 15;
  static_assert(2 * kTwo<S> * kPitch <= S::kLds && S::kB * kPitch <= S::kLds, "room for the rows");
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int j = 0; j < S::kTB; ++j) {
    const int b = wave_b<S>() + 16 * j + (lane & 15);
    if (two && b >= kTwo<S>) break;
#pragma unroll
    for (int i = 0; i < S::kTA; ++i) {
      const int a = wave_a<S>() + 16 * i + acc_a(lane);
      f32x4 x = value(i, j);
      auto put = [&](int r) {
        *reinterpret_cast<SIP_LDS u32x2*>(lds + r * kPitch + (((a >> 3) ^ (r & kMask)) << 4) + ((a & 4) << 1)) = bf16_pack(x);
      };
      put(b);
      if (two) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] -= (float)(__bf16)x[e];
        put(kTwo<S> + b);
      }
    }
  }
  __syncthreads();
#pragma unroll 4
  for (int g = threadIdx.x; g < (two ? 2 * kTwo<S> : S::kB) * kGroups; g += S::kThreads) {
    const int b = g / kGroups, c = g % kGroups;
    uint16_t* to = row(b);
    if (to && a0 + c * 8 < a_end)
      *reinterpret_cast<u32x4*>(to + a0 + c * 8) = *reinterpret_cast<SIP_LDS u32x4*>(lds + b * kPitch + ((c ^ (b & kMask)) << 4));
  }
}

// A tile of logits, reduced to its maximum and sum of exponentials per token and wave.  With many tokens bound by the matrix cores,
// busy for 68 % of the cycles at the 1.7 to 1.9 of 2.4 GHz that the card keeps up under them, and by the ends of the tiles: 8192
// tokens, V = 128256, D = 4096 6.5 ms, 1.32 PFLOP/s; with few by reading the head.
template <class S>
__global__ __launch_bounds__(S::kThreads) void xent_forward_kernel(XentArgs p) {
  __shared__ __attribute__((aligned(1024))) char lds[S::kLds];
  const int n = *p.count;
  int ta, tb;
  if (!tile_of(blockIdx.x, div_up(p.V, S::kA), div_up(n, S::kB), ta, tb)) return;
  const int a0 = ta * S::kA, b0 = tb * S::kB;
  typename S::Acc acc = {};
  Gemm<S, kRows, kRows>::tile(acc, Operand{p.weight, p.weight_stride, p.V, nullptr}, Operand{p.hidden, p.hidden_stride, n, p.rows},
                             a0, b0, 0, p.D, (SIP_LDS char*)lds);
  // Maxima and sums as the logits are made: acc, times f for a base of 2.  (The target's logit is made by xent_loss_kernel.)
  const int lane = threadIdx.x & 63, v0 = a0 + wave_a<S>();
  float f = p.logit_scale * kLog2e;
  if (f == 0.0f) {                                         // logits of 0, multiplied here: 0 times what marks an entry below is NaN
#pragma unroll
    for (int t = 0; t < S::kTA; ++t)
#pragma unroll
      for (int j = 0; j < S::kTB; ++j) acc[t][j] *= f;
    f = 1.0f;
  }
#pragma unroll
  for (int j = 0; j < S::kTB; ++j) {
    const int i = b0 + wave_b<S>() + 16 * j + (lane & 15);
    const bool live = i < n;
    const int target = live ? p.targets[p.rows[i]] : -1;
    // the target's own logit is left out, and so is what lies past the vocabulary: -inf, whatever the scale's sign
    if (__any(target >= v0 && target < v0 + S::kWaveA) || v0 + S::kWaveA > p.V) {
#pragma unroll
      for (int t = 0; t < S::kTA; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int v = v0 + 16 * t + acc_a(lane) + r;
          if (v >= p.V || v == target) acc[t][j][r] = f < 0.0f ? INFINITY : -INFINITY;
        }
    }
    float m = -INFINITY, s = 0.0f;
    if (f < 0.0f) {
#pragma unroll
      for (int t = 0; t < S::kTA; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) m = fmaxf(m, -acc[t][j][r]);
      m *= -f;
    } else {
#pragma unroll
      for (int t = 0; t < S::kTA; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) m = fmaxf(m, acc[t][j][r]);
      m *= f;
    }
    m = fmaxf(m, __shfl_xor(m, 16));
    m = fmaxf(m, __shfl_xor(m, 32));
    const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int t = 0; t < S::kTA; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) s += __builtin_amdgcn_exp2f(__builtin_fmaf(acc[t][j][r], f, -base));
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    if (live && lane < 16) p.part[(long long)i * p.parts + v0 / S::kWaveA] = make_float2(m, s);
  }
}

// A workgroup joins a token's parts, and makes its target's logit: in fp64, for a nearly certain token's loss is as exact as the
// difference between that logit, the largest by far, and the others'.
__global__ __launch_bounds__(256) void xent_loss_kernel(XentArgs p) {
  __shared__ double wave_zt[4];
  __shared__ float2 wave_part[4];
  const int i = blockIdx.x, t = threadIdx.x;
  if (i >= *p.count) return;
  const int row = p.rows[i];
  const u32x4* h = reinterpret_cast<const u32x4*>(p.hidden + row * p.hidden_stride);
  const u32x4* w = reinterpret_cast<const u32x4*>(p.weight + p.targets[row] * p.weight_stride);
  double zt = 0.0;
  for (int c = t; c < p.D / 8; c += 256) {
    const u32x4 x = h[c], y = w[c];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      zt += (double)(__builtin_bit_cast(float, x[e] << 16) * __builtin_bit_cast(float, y[e] << 16));                   // (exact)
      zt += (double)(__builtin_bit_cast(float, x[e] & 0xffff0000u) * __builtin_bit_cast(float, y[e] & 0xffff0000u));
    }
  }
  const float2* part = p.part + (long long)i * p.parts;
  float m = -INFINITY, s = 0.0f;
  auto join = [&](float mo, float so) {
    const float top = fmaxf(m, mo), base = top == -INFINITY ? 0.0f : top;
    s = s * __builtin_amdgcn_exp2f(m - base) + so * __builtin_amdgcn_exp2f(mo - base);
    m = top;
  };
#pragma unroll 4
  for (int j = t; j < p.parts; j += 256) join(part[j].x, part[j].y);
  for (int d = 32; d; d >>= 1) {
    zt += __shfl_xor(zt, d);
    const float mo = __shfl_xor(m, d), so = __shfl_xor(s, d);
    join(mo, so);
  }
  if ((t & 63) == 0) {
    wave_zt[t >> 6] = zt;
    wave_part[t >> 6] = make_float2(m, s);
  }
  __syncthreads();
  if (t == 0) {
    for (int o = 1; o < 4; ++o) {
      zt += wave_zt[o];
      join(wave_part[o].x, wave_part[o].y);
    }
    zt *= p.logit_scale;
    const double others = (double)m * 0.69314718055994530942 + (double)logf(s);            // ln of the others' mass
    const float gap = (float)(others - zt), rest = log1pf(expf(-fabsf(gap)));
    p.loss[row] = gap != gap ? gap : fmaxf(gap, 0.0f) + rest;
    p.lse[row] = (float)((gap > 0.0f ? others : zt) + rest);                                // (from the larger: it does not cancel)
  }
}

// dz of a tile of the piece's logits: the product of xent_forward_kernel once more, which takes a third of the backward pass (8192
// tokens, V = 128256, D = 4096: 19.5 ms together, 1.32 PFLOP/s); logits kept from the forward pass would be 4.2 GB.  Columns past the vocabulary are zeros: what multiplies dz reads groups of eight.
template <class S>
__global__ __launch_bounds__(S::kThreads) void xent_dz_kernel(XentArgs p) {
  __shared__ __attribute__((aligned(1024))) char lds[S::kLds];
  const int n = *p.count, left = min(p.piece, p.V - p.v0);
  int ta, tb;
  if (!tile_of(blockIdx.x, div_up(left, S::kA), div_up(n, S::kB), ta, tb)) return;
  const int a0 = ta * S::kA, b0 = tb * S::kB;
  typename S::Acc acc = {};
  Gemm<S, kRows, kRows>::tile(acc, Operand{p.weight + p.v0 * p.weight_stride, p.weight_stride, left, nullptr},
                             Operand{p.dense, p.D, n, nullptr}, a0, b0, 0, p.D, (SIP_LDS char*)lds);
  const int lane = threadIdx.x & 63, v0 = a0 + wave_a<S>();
  const float f = p.logit_scale * kLog2e;
#pragma unroll
  for (int j = 0; j < S::kTB; ++j) {
    const int i = b0 + wave_b<S>() + 16 * j + (lane & 15);
    const bool live = i < n;
    const int row = live ? p.rows[i] : 0;
    const int target = live ? p.targets[row] - p.v0 : -1;
    const float lse = live ? p.lse_in[row] * kLog2e : 0.0f, g = !live ? 0.0f : p.grad_loss ? p.grad_loss[row] : 1.0f;
#pragma unroll
    for (int t = 0; t < S::kTA; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[t][j][r] = g * __builtin_amdgcn_exp2f(__builtin_fmaf(acc[t][j][r], f, -lse));
    if (__any(target >= v0 && target < v0 + S::kWaveA) || v0 + S::kWaveA > left) {
      const float at_target = live ? g * expm1f(-p.loss_in[row]) : 0.0f;
#pragma unroll
      for (int t = 0; t < S::kTA; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int v = v0 + 16 * t + acc_a(lane) + r;
          if (v >= left || v == target) acc[t][j][r] = v >= left ? 0.0f : at_target;
        }
    }
  }
  const bool two = dz_parts(n) == 2;
  store_tile<S>((SIP_LDS char*)lds, a0, p.piece, [&](int i, int j) { return acc[i][j]; }, [&](int r) {
    const int part = two && r >= kTwo<S>, i = b0 + r - part * kTwo<S>;
    return i < n ? p.dz + (long long)(part * n + i) * p.piece : nullptr;
  }, two);
}

// How a launch for up to parts.tiles tiles of parts.count parts deals out `tiles` (1 .. parts.tiles) of `k` terms each: the
// workgroups and the room of rows that are masked go to those that are not.  2048 tokens of which 922 take part, V = 128256, D =
// 2048, forward and backward: 1916 us instead of 2165.
__device__ inline Parts dealt(const Parts& parts, int tiles, int k) {
  Parts p = parts;
  if (parts.count > 1) {
    p.tiles = tiles;
    p.count = max(parts.count, min(parts.tiles * parts.count / tiles, k / 256));
  }
  p.split = div_up(div_up(k, p.count), 64) * 64;
  return p;
}
template <class S>
__device__ inline f32x4* sum_tile(const Parts& parts, int part, int tile) {
  return reinterpret_cast<f32x4*>(parts.sum) + ((long long)part * parts.tiles + tile) * (S::kA * S::kB / 4) + threadIdx.x;
}

template <class S>
__device__ inline void store_grad_hidden(const XentArgs& p, SIP_LDS char* lds, const typename S::Acc& acc, int a0, int b0, int n) {
  const float f = p.out_scale;
  store_tile<S>(lds, a0, p.D, [&](int i, int j) { return acc[i][j] * f; },
                [&](int b) { return b0 + b < n ? p.grad_hidden + p.rows[b0 + b] * p.gh_stride : nullptr; });
}

// grad_hidden of a piece, or a part of its sums over the entries, added to what the pieces before it gave.  The last
// piece's kernel stores the result itself where nothing else has a part in it.
template <class S>
__global__ __launch_bounds__(S::kThreads) void xent_grad_hidden_kernel(XentArgs p) {
  __shared__ __attribute__((aligned(1024))) char lds[S::kLds];
  const int each = dz_parts(*p.count), n = *p.count * each, tiles_a = div_up(p.D, S::kA), tiles = tiles_a * div_up(n, S::kB);
  if (tiles == 0) return;
  const Parts parts = dealt(p.hidden_parts, tiles, min(p.piece, p.V));
  int ta, tb, part;
  if (!tile_of(blockIdx.y * gridDim.x + blockIdx.x, tiles_a, div_up(n, S::kB), parts.count, ta, tb, part)) return;
  const int a0 = ta * S::kA, b0 = tb * S::kB, left = min(p.piece, p.V - p.v0);
  const int k_begin = min(left, part * parts.split), k_end = min(left, k_begin + parts.split);
  typename S::Acc acc = {};
  Gemm<S, kCols, kRows>::tile(acc, Operand{p.weight + p.v0 * p.weight_stride, p.weight_stride, p.D, nullptr},
                             Operand{p.dz, p.piece, n, nullptr}, a0, b0, k_begin, k_end, (SIP_LDS char*)lds);
  f32x4* sum = sum_tile<S>(parts, part, tb * tiles_a + ta);
  const bool last = gridDim.y == 1 && each == 1 && p.v0 + p.piece >= p.V;
#pragma unroll
  for (int i = 0; i < S::kTA; ++i)
#pragma unroll
    for (int j = 0; j < S::kTB; ++j, sum += S::kThreads) {
      if (p.v0) acc[i][j] += *sum;
      if (!last) *sum = acc[i][j];
    }
  if (last) store_grad_hidden<S>(p, (SIP_LDS char*)lds, acc, a0, b0, n);
}

// The parts of grad_hidden (or of grad_weight's rows of a piece), added up in their order: workgroup (x, y) joins block y of each
// wave's in tile x.  (grad_hidden: unless xent_grad_hidden_kernel stored the result, which only the device knows.)
template <class S, bool HIDDEN>
__global__ __launch_bounds__(S::kThreads) void xent_join_kernel(XentArgs p) {
  const int tiles_a = div_up(p.D, S::kA), ta = blockIdx.x % tiles_a, tb = blockIdx.x / tiles_a, lane = threadIdx.x & 63;
  const int i = blockIdx.y / S::kTB, j = blockIdx.y % S::kTB;
  const int a = ta * S::kA + wave_a<S>() + 16 * i + acc_a(lane), b = tb * S::kB + wave_b<S>() + 16 * j + (lane & 15);
  if (a >= p.D || b >= (HIDDEN ? *p.count : min(p.piece, p.V - p.v0))) return;
  const int each = HIDDEN ? dz_parts(*p.count) : 1;
  if (HIDDEN && each == 1 && p.hidden_parts.count == 1) return;
  const Parts parts = HIDDEN ? dealt(p.hidden_parts, tiles_a * div_up(*p.count * each, S::kB), min(p.piece, p.V)) : p.weight_parts;
  f32x4 total = {};
  for (int row = each - 1; row >= 0; --row) {
    // where row b + row * count lies: its tile, its wave and block, its lane
    const int at = HIDDEN ? b + row * *p.count : b, in = at % S::kB;
    const int wave = in / S::kWaveB * (S::kA / S::kWaveA) + wave_a<S>() / S::kWaveA, block = i * S::kTB + in % S::kWaveB / 16;
    const f32x4* sum = sum_tile<S>(parts, 0, at / S::kB * tiles_a + ta) - threadIdx.x + block * S::kThreads + wave * 64 + (lane & 48) + in % 16;
    for (int k = 0; k < parts.count; ++k, sum += (long long)parts.tiles * (S::kA * S::kB / 4)) total += *sum;
  }
  uint16_t* to = HIDDEN ? p.grad_hidden + p.rows[b] * p.gh_stride : p.grad_weight + (p.v0 + (long long)b) * p.gw_stride;
  *reinterpret_cast<u32x2*>(to + a) = bf16_pack(total * p.out_scale);
}

// grad_weight of a piece's rows, or a part of its sums over the tokens.
template <class S>
__global__ __launch_bounds__(S::kThreads) void xent_grad_weight_kernel(XentArgs p) {
  __shared__ __attribute__((aligned(1024))) char lds[S::kLds];
  const int n = *p.count * dz_parts(*p.count), left = min(p.piece, p.V - p.v0), tiles_a = div_up(p.D, S::kA);
  int ta, tb, part;
  if (!tile_of(blockIdx.y * gridDim.x + blockIdx.x, tiles_a, div_up(left, S::kB), p.weight_parts.count, ta, tb, part)) return;
  const int a0 = ta * S::kA, b0 = tb * S::kB;
  const int split = div_up(div_up(n, p.weight_parts.count), 64) * 64, k_begin = min(n, part * split), k_end = min(n, k_begin + split);
  typename S::Acc acc = {};
  Gemm<S, kCols, kCols>::tile(acc, Operand{p.dense, p.D, p.D, nullptr}, Operand{p.dz, p.piece, left, nullptr}, a0, b0, k_begin, k_end,
                              (SIP_LDS char*)lds);
  if (gridDim.y > 1) {
    f32x4* sum = sum_tile<S>(p.weight_parts, part, tb * tiles_a + ta);
#pragma unroll
    for (int i = 0; i < S::kTA; ++i)
#pragma unroll
      for (int j = 0; j < S::kTB; ++j, sum += S::kThreads) *sum = acc[i][j];
    return;
  }
  const float f = p.out_scale;
  store_tile<S>((SIP_LDS char*)lds, a0, p.D, [&](int i, int j) { return acc[i][j] * f; },
                [&](int b) { return b0 + b < left ? p.grad_weight + (p.v0 + b0 + (long long)b) * p.gw_stride : nullptr; });
}

}  // namespace sip
