// Beam search: the best continuations of groups of beams, and the reordering of a sampler state's histories.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "sip_gemm.h"
#include "sip_state.h"

namespace sip {

// ---------------------------------------------------------------- selection
// total(k, v) = score_k + (c z_kv - lse_k) grows with z within a row, so that the n best logits of every row hold a group's n best
// continuations: one pass over the logits, lse and candidates together.  beam_chunk_kernel: a workgroup reads one chunk of a row once and leaves
// its maximum, its sum of exponentials and its n best logits, in order.  The merging kernels: a workgroup joins the lists of a group's
// rows, in fp64: two continuations may lie as near to one another as fp32's rounding of a sum of exponentials lets them.

constexpr int kBeamThreads = 256, kBeamWaves = kBeamThreads / 64;
constexpr int kBeamLoads = 8;                            // 16-byte loads of a lane: 32 fp32 logits, 64 bf16
constexpr int kBeamList = 512;                           // entries that a chunk's list may have before it is ranked
inline __host__ __device__ int beam_chunk(bool bf16) { return kBeamThreads * kBeamLoads * (bf16 ? 8 : 4); }

struct BeamPart { double sum; float max, off; };         // of a chunk: sum of 2^(c (z - max) + off)

struct BeamArgs {
  const void* logits; long long row_stride;
  int width, V, n;
  int chunks, chunk;                                     // of a row; logits of one
  float c;                                               // logit_scale * log2(e)
  double scale;                                          // logit_scale
  const float* scores; const uint8_t* finished; const float* rank_scale;
  int end_token;
  uint32_t wanted, wanted_last;                          // see beam_wanted()
  int* tokens; int* parents; float* out_scores;
  BeamPart* part;                                        // [rows][chunks]
  unsigned long long* cand;                              // [rows][chunks][n] keys in descending order, 0 = none
};

// How many of a wave's lanes' maxima have to reach the bound that it gives, a byte a wave: n of all, by how many of its lanes have logits among
// the chunk's `lanes`.  (0: any bound will do.)
inline uint32_t beam_wanted(int n, int lanes) {
  uint32_t wanted = 0;
  for (int w = 0; w < kBeamWaves; ++w) {
    const int live = lanes > w * 64 ? lanes - w * 64 < 64 ? lanes - w * 64 : 64 : 0;
    wanted |= (uint32_t)((n * live + lanes - 1) / lanes) << 8 * w;
  }
  return wanted;
}
static_assert(SIP_MAX_CONTINUATIONS < 256, "a byte");

// Floats as whole numbers that order alike (one zero; -inf is 0x007fffff), and back.
__device__ inline uint32_t ordered(float z) {
  const uint32_t u = __builtin_bit_cast(uint32_t, z + 0.0f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ inline float unordered(uint32_t o) {
  return __builtin_bit_cast(float, o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
__device__ inline unsigned long long ordered64(double x) {
  const unsigned long long u = __builtin_bit_cast(unsigned long long, x + 0.0);
  return u ^ ((unsigned long long)((long long)u >> 63) | 0x8000000000000000ull);
}
// A logit and its token: the larger logit first, of equal ones the lower token.  Never 0.
__device__ inline unsigned long long beam_key(float z, int token) {
  return (unsigned long long)ordered(z) << 32 | (uint32_t)~token;
}
__device__ inline int key_token(unsigned long long key) { return (int)~(uint32_t)key; }
__device__ inline float key_logit(unsigned long long key) { return unordered((uint32_t)(key >> 32)); }

// A wave's sum, in lane 63.
__device__ inline double wave_total(double x) {
  auto step = [&](auto control, auto rows) {
    const unsigned long long u = __builtin_bit_cast(unsigned long long, x);
    const uint32_t lo = dpp_mov<decltype(control)::value, decltype(rows)::value>(0u, (uint32_t)u);
    const uint32_t hi = dpp_mov<decltype(control)::value, decltype(rows)::value>(0u, (uint32_t)(u >> 32));
    x += __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
  };
  step(std::integral_constant<int, 0x111>(), std::integral_constant<int, 0xf>());        // row_shr 1, 2, 4, 8
  step(std::integral_constant<int, 0x112>(), std::integral_constant<int, 0xf>());
  step(std::integral_constant<int, 0x114>(), std::integral_constant<int, 0xf>());
  step(std::integral_constant<int, 0x118>(), std::integral_constant<int, 0xf>());
  step(std::integral_constant<int, 0x142>(), std::integral_constant<int, 0xa>());        // row_bcast 15, 31
  step(std::integral_constant<int, 0x143>(), std::integral_constant<int, 0xc>());
  return x;
}

// In a chunk's list an entry is a whole number below 2^46, the logit's and then its place from behind, as the double 2^52 + that:
// these compare in one instruction.
constexpr int kPlaceBits = 14;
__device__ inline double list_entry(float z, int place) {
  return __builtin_bit_cast(double, 0x4330000000000000ull | (unsigned long long)ordered(z) << kPlaceBits | (uint32_t)((1 << kPlaceBits) - 1 - place));
}
__device__ inline unsigned long long entry_key(double x, int first) {
  const unsigned long long u = __builtin_bit_cast(unsigned long long, x);
  return (u >> kPlaceBits & 0xffffffffu) << 32 | (uint32_t)~(first + (1 << kPlaceBits) - 1 - (int)(u & ((1u << kPlaceBits) - 1)));
}
static_assert(kBeamThreads * kBeamLoads * 8 <= 1 << kPlaceBits, "a place in the chunk");

// What a row has: continuations from its logits, one at no cost, or none.
enum BeamRow { kBeamNone, kBeamLive, kBeamFinished };
struct BeamRowInfo { float score, scale; int what; };
__device__ inline BeamRowInfo beam_row(const BeamArgs& a, int row) {
  const float score = a.scores[row], scale = a.rank_scale ? a.rank_scale[row] : 1.0f;
  const uint8_t finished = a.finished ? a.finished[row] : 0;
  const bool ok = isfinite(score) && isfinite(scale) && scale > 0.0f;
  return {score, scale, !ok ? kBeamNone : finished ? kBeamFinished : kBeamLive};
}

// The logits of a lane's 16-byte loads: logit e of those is at place beam_place(e) behind the lane's first.
template <int GROUP> constexpr int beam_place(int e) { return e / GROUP * (kBeamThreads * GROUP) + e % GROUP; }
template <int GROUP>
__device__ __forceinline__ float beam_logit(const u32x4 (&raw)[kBeamLoads], int e) {
  const uint32_t u = raw[e / GROUP][e % GROUP * 4 / GROUP], bits = GROUP == 4 ? u : e & 1 ? u & 0xffff0000u : u << 16;
  return __builtin_bit_cast(float, bits);
}

// A chunk with more than kBeamList logits from the bound on, nearly equal ones or a mask's many equal ones: its n first entries to the list
// (any order).  m is the largest; the chunk has `left` places.  The n-th largest logit is found, and among those that equal it the lowest tokens.
template <int GROUP>
__device__ __forceinline__ int select_apart(u32x4 (&raw)[kBeamLoads], double* list, int& count, int (&wave_n)[kBeamWaves], float from, float m, int n, int left) {
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  auto sum_of = [&](int mine) {                          // over the workgroup
    for (int d = 32; d; d >>= 1) mine += __shfl_xor(mine, d);
    __syncthreads();
    if (lane == 0) wave_n[w] = mine;
    __syncthreads();
    return wave_n[0] + wave_n[1] + wave_n[2] + wave_n[3];
  };
  // f(e) of all logits, a load at a time
  auto each = [&](auto f) {
#pragma unroll
    for (int i = 0; i < kBeamLoads; ++i) asm volatile("" : "+v"(raw[i]));        // (nothing of it is kept)
#pragma unroll
    for (int i = 0; i < kBeamLoads; ++i)
      if (i * kBeamThreads * GROUP < left) {
#pragma unroll
        for (int j = 0; j < GROUP; ++j) f(i * GROUP + j);
      }
  };
  // The smallest from the bound on: a mask's value, as a rule.
  float low = INFINITY;
  each([&](int e) { low = beam_logit<GROUP>(raw, e) >= from ? fminf(low, beam_logit<GROUP>(raw, e)) : low; });
  for (int d = 32; d; d >>= 1) low = fminf(low, __shfl_xor(low, d));
  __syncthreads();
  if (lane == 0) wave_n[w] = __builtin_bit_cast(int, low);
  __syncthreads();
  for (int i = 0; i < kBeamWaves; ++i) low = fminf(low, __builtin_bit_cast(float, wave_n[i]));
  int mine = 0;
  each([&](int e) { mine += beam_logit<GROUP>(raw, e) > low; });
  int above = sum_of(mine);
  if (above >= n) {
    // the n-th largest, bit by bit from the first one on in which the smallest and the largest differ: the largest value that n logits reach
    const int first = 31 - __builtin_clz(ordered(low) ^ ordered(m));
    uint32_t at = ordered(low) & ~((2ull << first) - 1);
    for (int bit = first; bit >= (GROUP == 8 ? 16 : 0); --bit) {         // (bf16 has sixteen)
      const uint32_t up = at | 1u << bit;
      if (up > 0xff800000u) continue;                    // (beyond +inf)
      const float least = unordered(up);
      mine = 0;
      if (up >= 0x007fffffu) each([&](int e) { mine += beam_logit<GROUP>(raw, e) >= least; });
      if (up < 0x007fffffu || sum_of(mine) >= n) at = up;
    }
    if (GROUP == 8 && !(at & 0x80000000u)) at |= 0xffffu;                // (those below 0 end in ones)
    low = unordered(at);
    mine = 0;
    each([&](int e) { mine += beam_logit<GROUP>(raw, e) > low; });
    above = sum_of(mine);
  }
  __syncthreads();
  if (t == 0) count = 0;
  __syncthreads();
  each([&](int e) {
    if (beam_logit<GROUP>(raw, e) > low) list[atomicAdd(&count, 1)] = list_entry(beam_logit<GROUP>(raw, e), t * GROUP + beam_place<GROUP>(e));
  });
  // Of those that equal it the n - above lowest tokens: a load after the other, whose places go by lane.  Of a mask, the first.
  int found = above;
#pragma unroll
  for (int i = 0; i < kBeamLoads; ++i)
    if (found < n) {
      mine = 0;
#pragma unroll
      for (int j = 0; j < GROUP; ++j) mine += beam_logit<GROUP>(raw, i * GROUP + j) == low;
      const int upto = (int)dpp_scan_add_u32((uint32_t)mine);
      __syncthreads();
      if (lane == 63) wave_n[w] = upto;
      __syncthreads();
      int place = found + upto - mine;
      for (int j = 0; j < kBeamWaves; ++j) {
        place += j < w ? wave_n[j] : 0;
        found += wave_n[j];
      }
#pragma unroll
      for (int j = 0; j < GROUP; ++j)
        if (beam_logit<GROUP>(raw, i * GROUP + j) == low) {
          if (place < n) list[place] = list_entry(low, t * GROUP + beam_place<GROUP>(i * GROUP + j));
          ++place;
        }
    }
  __syncthreads();
  return min(found, n);
}

// The chunk stays in registers: its maxima give the bound from which on logits can be among the n best -- n of the 256 lanes' maxima reach it,
// and few logits more --, its sum follows, and what reaches the bound is ranked in LDS.
// fp32 is bound by reading: 256 rows of V = 152064, a tenth of them finished, n = 8 28.2 us, 5 TB/s.  bf16 by vector instructions: 224 rows of
// 151643 19 us for n = 1 (floor 13), 24 for n = 64: unpacking, an exponential's four passes, the ranks.
template <bool BF16>
__global__ __launch_bounds__(kBeamThreads) void beam_chunk_kernel(BeamArgs a) {
  constexpr int kGroup = BF16 ? 8 : 4, kEach = kBeamLoads * kGroup;      // logits of a 16-byte load, of a lane
  __shared__ __align__(16) double list[kBeamList];
  __shared__ double wave_sum[kBeamWaves];
  __shared__ float wave_max[kBeamWaves];
  __shared__ uint32_t wave_least[kBeamWaves];
  __shared__ int count, wave_n[kBeamWaves];
  const int row = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  if (beam_row(a, row).what != kBeamLive) return;
  const int first = chunk * a.chunk + t * kGroup;        // my first token
  const char* z0 = static_cast<const char*>(a.logits) + ((long long)row * a.row_stride + first) * (BF16 ? 2 : 4);
  u32x4 raw[kBeamLoads];
  const uint32_t none = BF16 ? 0xff80ff80u : 0xff800000u;               // -inf
#pragma unroll
  for (int i = 0; i < kBeamLoads; ++i) {
    raw[i] = u32x4{none, none, none, none};
    if (first + beam_place<kGroup>(i * kGroup) + kGroup <= a.V) raw[i] = *reinterpret_cast<const u32x4*>(z0 + i * kBeamThreads * 16);
  }
  if (chunk == a.chunks - 1 && a.V % kGroup != 0) {      // the row's last group, in part
#pragma unroll
    for (int i = 0; i < kBeamLoads; ++i) {
      const int left = a.V - (first + beam_place<kGroup>(i * kGroup));
      if (left > 0 && left < kGroup) {
#pragma unroll
        for (int j = 0; j < kGroup; ++j)
          if (j < left) {
            const char* at = z0 + i * kBeamThreads * 16 + j * (BF16 ? 2 : 4);
            if constexpr (BF16) raw[i][j / 2] = (raw[i][j / 2] & (j & 1 ? 0xffffu : 0xffff0000u)) | (uint32_t)*reinterpret_cast<const uint16_t*>(at) << (j & 1 ? 16 : 0);
            else raw[i][j] = *reinterpret_cast<const uint32_t*>(at);
          }
      }
    }
  }
  auto value = [&](int e) { return beam_logit<kGroup>(raw, e); };
  // (else the compiler keeps all logits unpacked from one pass to the next)
  auto hide = [&]() {
#pragma unroll
    for (int i = 0; i < kBeamLoads; ++i) asm volatile("" : "+v"(raw[i]));
  };
  // Each load's largest, and the lane's.  (fmaxf drops NaNs: they show in the sum.)
  float best[kBeamLoads], m;
#pragma unroll
  for (int i = 0; i < kBeamLoads; ++i) {
    best[i] = -INFINITY;
    if constexpr (BF16) {
      // Bits of bf16 from 0 on order like whole numbers, and any below 0 is less: two at a time.
      s16x2 top = __builtin_bit_cast(s16x2, 0x80008000u);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t two = raw[i][j];                  // (a bit_cast of raw[i][j] itself is one of raw[i][0])
        top = __builtin_elementwise_max(top, __builtin_bit_cast(s16x2, two));
      }
      const int one = max((int)top[0], (int)top[1]);
      best[i] = __builtin_bit_cast(float, (uint32_t)one << 16);
      if (one < 0 || one > 0x7f80) {                     // nothing from 0 on, or a NaN
        best[i] = -INFINITY;
#pragma unroll
        for (int j = 0; j < kGroup; ++j) best[i] = fmaxf(best[i], value(i * kGroup + j));
      }
    } else {
#pragma unroll
      for (int j = 0; j < kGroup; ++j) best[i] = fmaxf(best[i], value(i * kGroup + j));
    }
    m = i ? fmaxf(m, best[i]) : best[i];
  }
  // The wave's n/4-th largest maximum of a lane (beam_wanted() in a short chunk), by its leading bits: of four waves, the smallest is at most the n-th
  // largest logit.
  const uint32_t lane_max = ordered(m);
  uint32_t least_of_wave = 0;
  const int wanted = (chunk == a.chunks - 1 ? a.wanted_last : a.wanted) >> 8 * w & 255;
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t up = least_of_wave | 1u << bit;
    if (__popcll(__ballot(lane_max >= up)) >= wanted) least_of_wave = up;
  }
  const uint32_t largest = dpp_scan_max_u32(lane_max);
  if (lane == 63) {
    wave_max[w] = unordered(largest);
    wave_least[w] = least_of_wave;
  }
  if (t == 0) count = 0;
  __syncthreads();
  m = fmaxf(fmaxf(wave_max[0], wave_max[1]), fmaxf(wave_max[2], wave_max[3]));
  const uint32_t least = min(min(wave_least[0], wave_least[1]), min(wave_least[2], wave_least[3]));
  const float from = least < 0x00800000u ? -3.402823466e38f : unordered(least);          // (-inf is no continuation)
  // My logits from the bound on go to the list: marked and counted first, so that nothing waits for a place, and read once more then, since there
  // are few: 64 tests and places of all were a third of this kernel's instructions.
  uint32_t hits[kEach == 64 ? 2 : 1] = {};               // a load's bits from the last logit's on
#pragma unroll
  for (int i = 0; i < kBeamLoads; ++i)
    if (best[i] >= from) {
      uint32_t of_load = 0;
#pragma unroll
      for (int j = 0; j < kGroup; ++j) of_load = of_load + of_load + (value(i * kGroup + j) >= from);
      hits[i * kGroup / 32] |= of_load << i * kGroup % 32;
    }
  unsigned long long marked = hits[0];
  if constexpr (kEach == 64) marked |= (unsigned long long)hits[1] << 32;
  const int mine = __popcll(marked);
  const int upto = (int)dpp_scan_add_u32((uint32_t)mine);
  int place = 0;
  if (lane == 63) place = atomicAdd(&count, upto);
  // Meanwhile the sum.  2^(c z - c max) with c rounded to 24 bits, 2^-25 of the exponent off at most; what the product c max is rounded by is
  // kept beside it.
  const float base = m == -INFINITY ? 0.0f : m, top = base * a.c;
  const bool near = fabsf(top) < 1e6f;
  float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  hide();
  if (near) {
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      s[e & 3] += __builtin_amdgcn_exp2f(__builtin_fmaf(value(e), a.c, -top));
      if (e % 8 == 7) __builtin_amdgcn_sched_barrier(0);
    }
  } else {                                               // (a row of a mask's values, or +inf)
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      s[e & 3] += __builtin_amdgcn_exp2f((value(e) - base) * a.c);
      if (e % 8 == 7) __builtin_amdgcn_sched_barrier(0);
    }
  }
  hide();
  place = __builtin_amdgcn_readlane(place, 63) + upto - mine;
  if (__builtin_amdgcn_readlane(upto, 63) > kBeamList) marked = 0;       // (the list will not be used)
  for (; marked && place < kBeamList; marked &= marked - 1, ++place) {
    const int b = __builtin_ctzll(marked), i = b / kGroup, j = kGroup - 1 - b % kGroup;
    const char* at = z0 + i * kBeamThreads * 16 + j * (BF16 ? 2 : 4);
    const float z = BF16 ? (float)*reinterpret_cast<const __bf16*>(at) : *reinterpret_cast<const float*>(at);
    list[place] = list_entry(z, (i * kBeamThreads + t) * kGroup + j);
  }
  const double sum = wave_total(((double)s[0] + (double)s[1]) + ((double)s[2] + (double)s[3]));
  if (lane == 63) wave_sum[w] = sum;
  __syncthreads();
  if (t == 0) {
    BeamPart p;
    p.sum = (wave_sum[0] + wave_sum[1]) + (wave_sum[2] + wave_sum[3]);
    p.max = m;
    p.off = near ? __builtin_fmaf(base, a.c, -top) : 0.0f;
    a.part[blockIdx.x] = p;
  }
  int listed = count;
  if (listed > kBeamList) listed = select_apart<kGroup>(raw, list, count, wave_n, from, m, a.n, a.V - chunk * a.chunk);
  unsigned long long* out = a.cand + (long long)blockIdx.x * a.n;
  for (int i = t; i < listed; i += kBeamThreads) {
    const double mine = list[i];
    int rank = 0;
#pragma unroll 8
    for (int j = 0; j < listed; ++j) rank += list[j] > mine;
    if (rank < a.n) out[rank] = entry_key(mine, chunk * a.chunk);
  }
  for (int i = listed + t; i < a.n; i += kBeamThreads) out[i] = 0;
}

// A continuation among those of its group: the larger pair comes first.
struct __align__(16) BeamRank { unsigned long long total, rest; };
__device__ inline bool operator>(const BeamRank& x, const BeamRank& y) {
  return x.total > y.total || (x.total == y.total && x.rest > y.rest);
}
__device__ inline unsigned long long beam_rest(int k, unsigned long long key) {       // lower beam, larger logit, lower token
  return (unsigned long long)(SIP_MAX_BEAMS - 1 - k) << 52 | (key >> 32) << 20 | (0xfffffu - (uint32_t)key_token(key));
}
__device__ inline int rest_beam(unsigned long long rest) { return SIP_MAX_BEAMS - 1 - (int)(rest >> 52); }
__device__ inline int rest_token(unsigned long long rest) { return (int)(0xfffffu - (uint32_t)(rest & 0xfffffu)); }
__device__ inline float rest_logit(unsigned long long rest) { return unordered((uint32_t)(rest >> 20)); }
static_assert(SIP_MAX_V <= 0xfffff && SIP_MAX_BEAMS <= 1 << 12, "beam_rest() holds a beam, a logit and a token");

// The group's rows, in LDS.  Logits count from a row's largest on, lse with them: a mask's value may be any.
struct BeamGroup {
  double lse[SIP_MAX_BEAMS];
  float top[SIP_MAX_BEAMS], score[SIP_MAX_BEAMS], scale[SIP_MAX_BEAMS];
  int what[SIP_MAX_BEAMS];
};
template <int THREADS>
__device__ inline void load_group(const BeamArgs& a, BeamGroup& rows) {
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, K = a.width, S = a.chunks, row0 = blockIdx.x * K;
  // As many rows a wave as have room for their chunks, a lane each.
  int lanes = 1;
  while (lanes < S) lanes *= 2;
  const int at_once = 64 / lanes, mine = lane / lanes, chunk = lane % lanes;
  for (int k0 = w * at_once; k0 < K; k0 += THREADS / 64 * at_once) {
    const int k = k0 + mine;
    BeamPart p = {0.0, -INFINITY, 0.0f};
    BeamRowInfo row = {0.0f, 0.0f, kBeamNone};
    if (k < K) {
      if (chunk < S) p = a.part[(long long)(row0 + k) * S + chunk];       // (of a row that is not live: anything)
      row = beam_row(a, row0 + k);
    }
    float top = p.max;
    for (int d = 1; d < lanes; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
    double s = p.max > -INFINITY ? p.sum * exp2(((double)p.max - (double)top) * (double)a.c - (double)p.off) : p.sum;
    for (int d = 1; d < lanes; d <<= 1) s += __shfl_xor(s, d);
    if (k < K && chunk == 0) {
      rows.lse[k] = log(s);
      rows.top[k] = top;
      rows.score[k] = row.score;
      rows.scale[k] = row.scale;
      // (NaN or +inf somewhere, or nothing but -inf: no continuation)
      rows.what[k] = row.what == kBeamLive && !(s > 0.0 && isfinite(s) && isfinite(top)) ? (int)kBeamNone : row.what;
    }
  }
}
__device__ inline double total_of(const BeamArgs& a, const BeamGroup& rows, int k, float z) {
  return (double)rows.score[k] + (((double)z - (double)rows.top[k]) * a.scale - rows.lse[k]);
}
// Entry e of list l (of beam l / chunks), whose key is `key`; total 0: there is none.
__device__ inline BeamRank rank_of(const BeamArgs& a, const BeamGroup& rows, int l, int e, unsigned long long key) {
  const int k = l / a.chunks, what = rows.what[k];
  if (what == kBeamLive && key) return {ordered64(total_of(a, rows, k, key_logit(key)) * (double)rows.scale[k]), beam_rest(k, key)};
  if (what == kBeamFinished && l == k * a.chunks && e == 0)
    return {ordered64((double)rows.score[k] * (double)rows.scale[k]), beam_rest(k, beam_key(0.0f, a.end_token))};
  return {0, 0};
}

// The leading bits of the n-th largest of the workgroup's values, EACH a lane: two bits a turn from the first one on in which any two of them
// differ, of which votes.at[turn] counts the values that reach the three possibilities (zeros before; a barrier a turn).  `reach` says how many
// reach it; no more than `enough` end the search.  0 is no value, unless `zeros`: then `reach` is the number of values before.  0 if there are
// fewer than n.
constexpr int kVoteTurns = 16;
struct __align__(16) BeamVotes { int at[kVoteTurns][4]; uint32_t high, low; int some; };       // low: its complement
__device__ inline void clear(BeamVotes& votes) {
  const int t = threadIdx.x;
  if (t < kVoteTurns * 4) votes.at[t / 4][t % 4] = 0;
  if (t == 0) votes.high = votes.low = votes.some = 0;
}
template <int EACH>
__device__ inline uint32_t nth_largest(const uint32_t (&x)[EACH], int n, int enough, int& reach, BeamVotes& votes, bool zeros) {
  const int lane = threadIdx.x & 63;
  uint32_t from = 0;
  int bit = 30;
  if (!zeros) {
    uint32_t high = 0, low = 0;
    int some = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      high = max(high, x[i]);
      low = max(low, x[i] ? ~x[i] : 0);
      some += __popcll(__ballot(x[i] != 0));
    }
    high = dpp_scan_max_u32(high);
    low = dpp_scan_max_u32(low);
    if (lane == 63 && high) {
      atomicMax(&votes.high, high);
      atomicMax(&votes.low, low);
      atomicAdd(&votes.some, some);
    }
    __syncthreads();
    reach = votes.some;
    if (reach < n) return 0;
    const uint32_t least = ~votes.low, differ = votes.high ^ least;
    bit = differ ? 31 - __builtin_clz(differ) & ~1 : -2;
    from = differ ? least & ~((4u << bit) - 1) : least;
  }
  for (int turn = 0; bit >= 0 && reach > enough; ++turn, bit -= 2) {
    int mine[3] = {0, 0, 0};
#pragma unroll
    for (int i = 0; i < EACH; ++i)
#pragma unroll
      for (int j = 0; j < 3; ++j) mine[j] += __popcll(__ballot(x[i] >= (from | (uint32_t)(j + 1) << bit)));
    if (lane < 3 && mine[0]) atomicAdd(&votes.at[turn][lane], lane == 0 ? mine[0] : lane == 1 ? mine[1] : mine[2]);
    __syncthreads();
    const int4 all = *reinterpret_cast<const int4*>(votes.at[turn]);
    const int step = (all.x >= n) + (all.y >= n) + (all.z >= n);
    from |= (uint32_t)step << bit;
    if (step) reach = step == 1 ? all.x : step == 2 ? all.y : all.z;
  }
  return from;
}

// Where n of a group's entries can be told by one of each list alone: if n / d lists have d entries from a bound on, n entries reach it.  Of so many
// lists a quarter decides; where there are few, by entries further down.
__device__ inline int beam_depth(int lists, int n) { return min(n, max(1, (4 * n + lists - 1) / lists)); }

// The same bound from one entry of each list, one a thread, compared with one another (their last bits make them differ), four a read: 16
// waves' reads of LDS are what it costs.  0 if there are fewer than n.
constexpr int kHeadsMost = 256;
template <int THREADS, int MOST>
__device__ inline uint32_t nth_head(uint32_t lead, int lists, int n, uint32_t (&heads)[MOST], int (&ranks)[THREADS], uint32_t& bound) {
  static_assert(MOST <= THREADS, "a thread a head");
  constexpr uint32_t kLast = MOST - 1;
  const int t = threadIdx.x;
  if (t < MOST) heads[t] = t < lists ? (lead & ~kLast) | (kLast - t) : 0;
  ranks[t] = 0;
  if (t == 0) bound = 0;
  __syncthreads();
  int wide = 64;
  while (wide < lists) wide *= 2;
  const int parts = THREADS / wide, i = t % wide;
  if (i < lists) {
    const uint32_t mine = heads[i];
    int rank = 0;
    for (int j = t / wide * 4; j < lists; j += parts * 4) {
      const uint4 four = *reinterpret_cast<const uint4*>(&heads[j]);
      rank += (four.x > mine) + (four.y > mine) + (four.z > mine) + (four.w > mine);
    }
    if (rank) atomicAdd(&ranks[i], rank);
  }
  __syncthreads();
  if (t < lists && ranks[t] == n - 1) bound = heads[t] & ~kLast;
  __syncthreads();
  return bound;
}

// Of m entries the n largest and few more, up to `enough` in all; m > enough >= n.  By the leading word of their ranks, and where that is equal
// by the next.  What it saves: two groups of 62 beams of one chunk each, n = 124, are merged in 17.5 us, in 1.2 ms with all entries ranked among one another.
template <int THREADS, int ROOM>
__device__ inline int keep_largest(BeamRank* found, int m, int n, int enough, BeamVotes& votes, int& count) {
  constexpr int kEach = (ROOM + THREADS - 1) / THREADS;
  const int t = threadIdx.x;
  BeamRank x[kEach];
  bool open[kEach], kept[kEach];                         // equal to the bound so far; above it
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    open[i] = t + i * THREADS < m;
    kept[i] = false;
    x[i] = open[i] ? found[t + i * THREADS] : BeamRank{0, 0};
  }
  int above = 0, reach = m;
  __syncthreads();                                       // (everybody has read `count`)
  for (int w = 0; w < 4; ++w) {
    uint32_t word[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) word[i] = open[i] ? (uint32_t)((w < 2 ? x[i].total : x[i].rest) >> (w & 1 ? 0 : 32)) : 0;
    clear(votes);
    if (t == 0) count = 0;
    __syncthreads();
    const uint32_t from = nth_largest(word, n - above, enough - above, reach, votes, w > 0);
    const bool last = above + reach <= enough;           // (else `from` is the n-th largest word, all of it)
    int mine = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const bool up = open[i] && (last ? word[i] >= from : word[i] > from);
      kept[i] |= up;
      mine += up;
      open[i] &= word[i] == from;
    }
    if (last) break;
    if (mine) atomicAdd(&count, mine);
    __syncthreads();
    above += count;
    reach -= count;
    __syncthreads();
  }
  __syncthreads();
  if (t == 0) count = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kEach; ++i)
    if (kept[i]) found[atomicAdd(&count, 1)] = x[i];
  __syncthreads();
  return count;
}

// f(rank, i) for each of n entries, i's place among them.  Begins and ends with the entries visible to all.
template <int THREADS, class F>
__device__ inline void rank_all(const BeamRank* found, int n, int (&ranks)[THREADS], F f) {
  const int t = threadIdx.x;
  if (n <= THREADS / 2) {
    // several threads an entry: each compares it with a part of the others
    int wide = 32;
    while (wide < n) wide *= 2;
    const int parts = THREADS / wide, i = t % wide;
    ranks[t] = 0;
    __syncthreads();
    if (i < n) {
      const BeamRank mine = found[i];
      int rank = 0;
      for (int j = t / wide; j < n; j += parts) rank += found[j] > mine;
      if (rank) atomicAdd(&ranks[i], rank);
    }
    __syncthreads();
    if (t < n) f(ranks[t], t);
  } else {
    for (int i = t; i < n; i += THREADS) {
      const BeamRank mine = found[i];
      int rank = 0;
      for (int j = 0; j < n; ++j) rank += found[j] > mine;
      f(rank, i);
    }
  }
  __syncthreads();
}

__device__ inline void store_selected(const BeamArgs& a, const BeamGroup& rows, const BeamRank& x, int rank) {
  if (rank >= a.n) return;
  const int k = rest_beam(x.rest), at = blockIdx.x * a.n + rank;
  a.tokens[at] = rest_token(x.rest);
  a.parents[at] = k;
  a.out_scores[at] = rows.what[k] == kBeamFinished ? rows.score[k] : (float)total_of(a, rows, k, rest_logit(x.rest));
}
__device__ inline void store_missing(const BeamArgs& a, int kept) {
  for (int i = kept + threadIdx.x; i < a.n; i += blockDim.x) {
    const int at = blockIdx.x * a.n + i;
    a.tokens[at] = a.parents[at] = -1;
    a.out_scores[at] = -INFINITY;
  }
}

// A group whose lists have up to kMergeFew entries together: all of them in registers.  Latency, of the loads and a dozen barriers: 64 groups
// with 608 entries 6.8 us, one with 64 4.2 (with the kernel for any group 8.0 and 5.8).
constexpr int kMergeFew = 1024, kRankFew = 192;           // (entries that are ranked among one another at most)
static_assert(kRankFew >= SIP_MAX_CONTINUATIONS, "all that are selected");
__global__ __launch_bounds__(256) void beam_merge_few_kernel(BeamArgs a) {
  constexpr int kEach = kMergeFew / 256;
  __shared__ BeamGroup rows;
  __shared__ BeamRank found[kMergeFew];
  __shared__ int ranks[256], count;
  __shared__ uint32_t first[kHeadsMost], bound;
  __shared__ __align__(16) uint32_t heads[kHeadsMost];
  __shared__ BeamVotes votes;
  const int t = threadIdx.x, entries = a.width * a.chunks * a.n;
  const unsigned long long* cand = a.cand + (long long)blockIdx.x * entries;
  unsigned long long key[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) key[i] = t + i * 256 < entries ? cand[t + i * 256] : 0;
  if (t == 0) count = 0;
  clear(votes);
  load_group<256>(a, rows);
  __syncthreads();
  BeamRank x[kEach];
  uint32_t lead[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int at = t + i * 256;
    x[i] = {0, 0};
    if (at < entries) x[i] = rank_of(a, rows, at / a.n, at % a.n, key[i]);
    lead[i] = (uint32_t)(x[i].total >> 32);
  }
  const int lists = a.width * a.chunks;
  uint32_t from = 0;
  if (entries <= 64) from = 0;                           // (so few are compared with one another at once)
  else if (lists <= kHeadsMost) {
    // entry d - 1 of list t is entry t * n + d - 1 of all
    const int depth = beam_depth(lists, a.n);
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (t + i * 256 < entries && (t + i * 256) % a.n == depth - 1) first[(t + i * 256) / a.n] = lead[i];
    __syncthreads();
    from = nth_head<256, kHeadsMost>(t < lists ? first[t] : 0, lists, (a.n + depth - 1) / depth, heads, ranks, bound);
  } else {
    int reach;
    from = nth_largest(lead, a.n, max(a.n, 64), reach, votes, false);
  }
  from = max(from, 1u);                                  // (0: there is none)
#pragma unroll
  for (int i = 0; i < kEach; ++i)
    if (lead[i] >= from) found[atomicAdd(&count, 1)] = x[i];
  __syncthreads();
  int kept = count;
  if (kept > kRankFew) kept = keep_largest<256, kMergeFew>(found, kept, a.n, kRankFew, votes, count);
  rank_all<256>(found, kept, ranks, [&](int rank, int i) { store_selected(a, rows, found[i], rank); });
  store_missing(a, kept);
}

// Any group.  The lists are in order, so one entry of each bounds what can be selected, and a list whose head is the r-th best
// can give its n - r first entries at most.  7 groups of 32 beams, 320 lists of 64 each: 14.6 us, latency too.
constexpr int kMergeThreads = 1024, kRankMost = 256, kHeadsMany = 512;
constexpr int kMergeLists = SIP_MAX_BEAMS * 64;
constexpr int kMergeRoom = SIP_MAX_CONTINUATIONS * (SIP_MAX_CONTINUATIONS + 1) / 2;
static_assert(kMergeRoom >= kMergeLists, "room for all heads");
__global__ __launch_bounds__(kMergeThreads) void beam_merge_kernel(BeamArgs a) {
  constexpr int kHeads = kMergeLists / kMergeThreads;
  __shared__ BeamGroup rows;
  __shared__ BeamRank found[kMergeRoom];
  __shared__ int ranks[kMergeThreads], chosen[SIP_MAX_CONTINUATIONS], count;
  __shared__ uint32_t bound;
  __shared__ __align__(16) uint32_t leads[kHeadsMany];
  __shared__ BeamVotes votes;
  const int t = threadIdx.x, S = a.chunks, n = a.n, lists = a.width * S;
  const unsigned long long* cand = a.cand + (long long)blockIdx.x * lists * n;
  static_assert(kHeads == 4, "and as many entries at once");
  unsigned long long key[kHeads], deep = 0;
  const int depth = beam_depth(lists, n);
#pragma unroll
  for (int i = 0; i < kHeads; ++i) key[i] = t + i * kMergeThreads < lists ? cand[(long long)(t + i * kMergeThreads) * n] : 0;
  if (t < lists && depth > 1) deep = cand[(long long)t * n + depth - 1];
  if (t == 0) count = 0;
  clear(votes);
  load_group<kMergeThreads>(a, rows);
  __syncthreads();
  uint32_t lead[kHeads];
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    const int l = t + i * kMergeThreads;
    lead[i] = l < lists ? (uint32_t)(rank_of(a, rows, l, 0, key[i]).total >> 32) : 0;
  }
  uint32_t from;
  if (lists <= kHeadsMany) {
    const uint32_t mine = depth > 1 && t < lists ? (uint32_t)(rank_of(a, rows, t, depth - 1, deep).total >> 32) : lead[0];
    from = nth_head<kMergeThreads, kHeadsMany>(mine, lists, (n + depth - 1) / depth, leads, ranks, bound);
  } else {
    int reach;
    from = nth_largest(lead, n, n + n / 4, reach, votes, false);
  }
  from = max(from, 1u);
#pragma unroll
  for (int i = 0; i < kHeads; ++i)
    if (lead[i] >= from) found[atomicAdd(&count, 1)] = rank_of(a, rows, t + i * kMergeThreads, 0, key[i]);
  __syncthreads();
  int heads = count;
  if (heads > kRankMost) heads = keep_largest<kMergeThreads, kMergeLists>(found, heads, n, kRankMost, votes, count);
  const int selected = min(heads, n);
  rank_all<kMergeThreads>(found, heads, ranks, [&](int rank, int i) {
    const unsigned long long rest = found[i].rest;
    const int k = rest_beam(rest);
    if (rank < n) chosen[rank] = k * S + (rows.what[k] == kBeamFinished ? 0 : rest_token(rest) / a.chunk);
  });
  if (t == 0) count = 0;
  __syncthreads();
  constexpr int kAhead = kHeads;                         // entries whose loads are under way at once
  for (int i0 = t; i0 < selected * n; i0 += kAhead * kMergeThreads) {
    int list[kAhead], e[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int i = i0 + j * kMergeThreads, r = i / n;
      e[j] = i - r * n;
      list[j] = i < selected * n && r + e[j] < n ? chosen[r] : -1;
      key[j] = list[j] >= 0 ? cand[(long long)list[j] * n + e[j]] : 0;
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (list[j] < 0) continue;
      const BeamRank x = rank_of(a, rows, list[j], e[j], key[j]);
      if (x.total >> 32 >= from) found[atomicAdd(&count, 1)] = x;
    }
  }
  __syncthreads();
  int kept = count;
  if (kept > kRankMost) kept = keep_largest<kMergeThreads, kMergeRoom>(found, kept, n, kRankMost, votes, count);
  rank_all<kMergeThreads>(found, kept, ranks, [&](int rank, int i) { store_selected(a, rows, found[i], rank); });
  store_missing(a, kept);
}

// ---------------------------------------------------------------- reordering of a state

struct ReorderArgs {
  StateHeader* head;
  int* len; int* ndist; int* tokens; uint32_t* table;
  int slots, L_max, width;
  const int* slot_of_row; const int* parents; const int* new_tokens;
};

// Where the rows of a group take their histories from, lane k row k's: its parent's slot (-1: an empty history), its own, and how long that history
// is.  to < 0: nothing is appended, nor moved; a row whose parent is itself moves nothing.  For a whole wave.
struct Move { int from, to, length; };
__device__ inline int length_of(const ReorderArgs& a, int slot) {
  return slot < 0 ? 0 : min(max(a.len[slot], 0), a.L_max);
}
__device__ inline Move move_of(const ReorderArgs& a, int group, bool lengths) {
  const int k = threadIdx.x & 63, row = group * a.width + k;
  int p = -1, to = -1;
  if (k < a.width) {
    p = a.parents[row];
    to = a.slot_of_row[row];
  }
  const int from = __shfl(to, p & 63);
  unsigned long long same = __ballot((unsigned)to < (unsigned)a.slots);                    // the rows of my slot, by its bits
  for (int b = 0; (a.slots - 1) >> b; ++b) {
    const unsigned long long set = __ballot(to >> b & 1);
    same &= to >> b & 1 ? set : ~set;
  }
  const bool taken = same & ((1ull << k) - 1);           // an earlier one's
  Move m = {-1, -1, 0};
  if ((unsigned)p >= (unsigned)a.width || (unsigned)to >= (unsigned)a.slots) return m;
  m.from = (unsigned)from < (unsigned)a.slots ? from : -1;
  m.to = taken ? -1 : to;
  if (lengths) m.length = length_of(a, m.from);
  return m;
}

// Sixteen bytes that are aligned to four.
struct __attribute__((packed, aligned(4))) StateLine { uint32_t w[4]; };

// A lane takes the same 16 bytes of every slot of a group of up to kGroupWidth, of the tables or of the tokens: it reads them all before it writes any,
// and nobody else touches them, so that the slots change places without room beside them.  The moves come from the wave's lanes, as scalars, and are
// fetched where all lanes are active (fetch_moves(); fetch_lengths() where these are wanted, since they arrive later): what a lane's register
// holds that has left a loop is not defined.
constexpr int kGroupWidth = 8;
struct Moves { int from[kGroupWidth], to[kGroupWidth], length[kGroupWidth]; };       // to < 0: nothing moves
__device__ inline void fetch_moves(Moves& all, const Move& m) {
  const int to = m.to == m.from ? -1 : m.to;
#pragma unroll
  for (int k = 0; k < kGroupWidth; ++k) {
    all.from[k] = __builtin_amdgcn_readlane(m.from, k);
    all.to[k] = __builtin_amdgcn_readlane(to, k);
  }
}
__device__ inline void fetch_lengths(Moves& all, const Move& m) {
#pragma unroll
  for (int k = 0; k < kGroupWidth; ++k) all.length[k] = __builtin_amdgcn_readlane(m.length, k);
}
__device__ inline void move_table(const ReorderArgs& a, const Moves& m, int column) {
  StateLine x[kGroupWidth];
#pragma unroll
  for (int k = 0; k < kGroupWidth; ++k) {
    if (m.to[k] < 0) continue;
    const uint32_t empty = column < kTableSlots ? kTableEmpty : 0u;
    x[k] = StateLine{{empty, empty, empty, empty}};
    if (m.from[k] >= 0) x[k] = *reinterpret_cast<const StateLine*>(a.table + (long long)m.from[k] * (2 * kTableSlots) + column);
  }
#pragma unroll
  for (int k = 0; k < kGroupWidth; ++k)
    if (m.to[k] >= 0) *reinterpret_cast<StateLine*>(a.table + (long long)m.to[k] * (2 * kTableSlots) + column) = x[k];
}
__device__ inline void move_tokens(const ReorderArgs& a, const Moves& m, int column) {
  StateLine x[kGroupWidth];
#pragma unroll
  for (int k = 0; k < kGroupWidth; ++k) {
    if (m.to[k] < 0 || column >= m.length[k]) continue;
    x[k] = *reinterpret_cast<const StateLine*>(a.tokens + (long long)m.from[k] * a.L_max + column);
  }
#pragma unroll
  for (int k = 0; k < kGroupWidth; ++k) {
    if (m.to[k] < 0 || column >= m.length[k]) continue;
    int* out = a.tokens + (long long)m.to[k] * a.L_max + column;
    if (column + 4 <= m.length[k]) *reinterpret_cast<StateLine*>(out) = x[k];
    else
      for (int j = 0; j < 3; ++j)
        if (column + j < m.length[k]) out[j] = (int)x[k].w[j];
  }
}
// A row's length and number of distinct tokens (`n`, `nd` as its parent had them), and its new token, once the copies are there.
__device__ inline void append_token(const ReorderArgs& a, int to, int n, int nd, int token) {
  if (token >= 0) {
    if (n < a.L_max) {
      a.tokens[(long long)to * a.L_max + n] = token;
      ++n;
      if (nd >= 0) {
        uint32_t* key = a.table + (long long)to * (2 * kTableSlots);
        const int r = table_insert_single(key, key + kTableSlots, (uint32_t)token);
        nd = r < 0 ? -1 : nd + r;
        if (nd > kTableMaxDistinct) nd = -1;
      }
    } else {
      atomicAdd(&a.head->overflow, 1u);
    }
  }
  a.len[to] = n;
  a.ndist[to] = nd;
}
struct Appended { int nd, token; };
__device__ inline Appended appended_of(const ReorderArgs& a, int group, const Move& m) {
  Appended x = {0, -1};
  if ((int)threadIdx.x >= a.width || m.to < 0) return x;
  if (m.from >= 0) x.nd = a.ndist[m.from];
  if (a.new_tokens) x.token = a.new_tokens[group * a.width + threadIdx.x];
  return x;
}

// A workgroup a group, and all in one launch.  (sip_search.h has the figures of both ways.)
constexpr int kGroupThreads = 1024;
static_assert(kGroupThreads * 4 == kTableSlots, "four entries of a table a thread");
__global__ __launch_bounds__(kGroupThreads) void state_reorder_group_kernel(ReorderArgs a) {
  const int t = threadIdx.x;
  const Move m = move_of(a, blockIdx.x, true);
  const Appended x = appended_of(a, blockIdx.x, m);
  Moves all;
  fetch_moves(all, m);
  move_table(a, all, t * 4);
  move_table(a, all, kTableSlots + t * 4);
  fetch_lengths(all, m);
  for (int column = t * 4; column < a.L_max; column += kGroupThreads * 4) move_tokens(a, all, column);
  __syncthreads();                                       // (everybody has read, and written)
  if (t < a.width && m.to >= 0) append_token(a, m.to, m.length, x.nd, x.token);
}

// The same in many workgroups, 4 KB of a group's slots each, without the new tokens.  Latency: slots, then lengths, then the loads, then the stores.  64
// groups of 8 slots with 3000 tokens each: 9.5 us for 33 MB read and written.
constexpr int kReorderThreads = 256, kReorderTables = 2 * kTableSlots / (kReorderThreads * 4);
__global__ __launch_bounds__(kReorderThreads) void state_reorder_few_kernel(ReorderArgs a) {
  const int block = blockIdx.y - kReorderTables;         // (below 0: of the tables)
  const Move m = move_of(a, blockIdx.x, block >= 0);
  const int column = ((block < 0 ? blockIdx.y : block) * kReorderThreads + threadIdx.x) * 4;
  Moves all;
  fetch_moves(all, m);
  if (block < 0) {
    move_table(a, all, column);
  } else {
    fetch_lengths(all, m);
    move_tokens(a, all, column);
  }
}

// Wider groups: a workgroup takes 1 KB of a group's slots, a wave that of kReorderEach of them, and all are read before any is written.  2 groups
// of 64 slots, L_max = 2097, 6.7 us; 24 with all slots in every lane's registers: the instructions of so many are what costs.  64 groups of 8 10.8 us.
constexpr int kReorderEach = 4, kReorderWords = 64 * 4;
constexpr int kReorderTableBlocks = 2 * kTableSlots / kReorderWords;
__global__ __launch_bounds__(SIP_MAX_BEAMS / kReorderEach * 64) void state_reorder_kernel(ReorderArgs a) {
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, block = blockIdx.y - kReorderTableBlocks;       // (below 0: of the tables)
  const bool table = block < 0;
  const Move m = move_of(a, blockIdx.x, !table);
  const int column = (table ? blockIdx.y : block) * kReorderWords + lane * 4;
  uint32_t* rows = table ? a.table : reinterpret_cast<uint32_t*>(a.tokens);
  const long long pitch = table ? 2 * kTableSlots : a.L_max;
  const uint32_t empty = column < kTableSlots ? kTableEmpty : 0u;
  StateLine x[kReorderEach];
  int from[kReorderEach], to[kReorderEach], left[kReorderEach];          // words from mine on that move
#pragma unroll
  for (int j = 0; j < kReorderEach; ++j) {               // (with all lanes active, before any load of some)
    const int k = w * kReorderEach + j, length = __builtin_amdgcn_readlane(m.length, k);
    from[j] = __builtin_amdgcn_readlane(m.from, k);
    to[j] = __builtin_amdgcn_readlane(m.to, k);
    left[j] = to[j] < 0 || to[j] == from[j] ? 0 : table ? 4 : length - column;
  }
#pragma unroll
  for (int j = 0; j < kReorderEach; ++j) {
    x[j] = StateLine{{empty, empty, empty, empty}};
    if (left[j] > 0 && from[j] >= 0) x[j] = *reinterpret_cast<const StateLine*>(rows + from[j] * pitch + column);
  }
#pragma unroll
  for (int j = 0; j < kReorderEach; ++j) asm volatile("" : "+v"(x[j].w[0]), "+v"(x[j].w[1]), "+v"(x[j].w[2]), "+v"(x[j].w[3]) :: "memory");      // (they are here)
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kReorderEach; ++j) {
    uint32_t* out = rows + to[j] * pitch + column;
    if (left[j] >= 4) *reinterpret_cast<StateLine*>(out) = x[j];
    else
      for (int i = 0; i < 3; ++i)
        if (i < left[j]) out[i] = x[j].w[i];
  }
}
// And behind either one wave a group for the rest: lengths and numbers of distinct tokens, all read before any is written, and
// the new tokens.
__global__ __launch_bounds__(64) void state_reorder_append_kernel(ReorderArgs a) {
  const Move m = move_of(a, blockIdx.x, true);
  const Appended x = appended_of(a, blockIdx.x, m);
  __syncthreads();
  if (m.to >= 0) append_token(a, m.to, m.length, x.nd, x.token);
}

}  // namespace sip
