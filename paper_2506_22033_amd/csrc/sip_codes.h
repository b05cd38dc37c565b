// A vocabulary head of 4-bit codes with group scales: the quantiser, and the product with hidden states.
#pragma once
#include <type_traits>

#include "sip_gemm.h"

namespace sip {


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
  char* states;                                        // workspace: see ManyLayout
};

// The largest of each half of `x` over the GROUP / 8 lanes of a group, by exchange of neighbours, pairs, quads and eights.
template <int GROUP>
__device__ inline s16x2 group_max(s16x2 x) {
  auto with = [&](auto pattern) {
    x = __builtin_elementwise_max(x, __builtin_bit_cast(s16x2, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), decltype(pattern)::value, 0xf, 0xf, true)));
  };
  with(std::integral_constant<int, 0xb1>());                            // quad_perm 1 0 3 2
  with(std::integral_constant<int, 0x4e>());                            // quad_perm 2 3 0 1
  if constexpr (GROUP >= 64) with(std::integral_constant<int, 0x141>());  // row_half_mirror
  if constexpr (GROUP >= 128) with(std::integral_constant<int, 0x140>()); // row_mirror
  return x;
}

// Eight weights a lane, a group in group / 8 neighbouring lanes.  Reads 16 bytes a lane and writes 4.
// Bounds: a bf16 that is not negative is the larger the larger its bits as an int16; a negative one the smaller, and with its
// sign flipped its bits order likewise.
// Quotients: with r = fl(1 / s), t the product w r corrected once by its remainder, fl(t + r (w - t s)) is w / s correctly rounded
// (Markstein, 1990), six operations instead of an IEEE division's dozen; for s in the middle of fp32's range, where
// nothing that matters underflows.
// Bound by vector instructions, 180 for a lane's eight weights, close to memory's rate: V = 256000, D = 4096, groups of 128 594 to
// 644 us, 4.1 to 4.4 TB/s read and written (a plain copy moves 4.9).  With IEEE divisions, and bounds in fp32 by shuffles, it
// was 220 instructions and 751 us.
template <int GROUP>
__global__ __launch_bounds__(256) void quantize_kernel(CodesArgs p) {
  const uint32_t per_row = (uint32_t)p.D / 8, total = (uint32_t)p.V * per_row;              // (below 2^31)
  const uint32_t lanes = (total + 63) & ~63u, step = gridDim.x * 256u;
  for (uint32_t id = blockIdx.x * 256 + threadIdx.x; id < lanes; id += step) {
    const bool live = id < total;
    const uint32_t v = live ? id / per_row : 0, c = live ? id - v * per_row : 0;
    const u32x4 w = *reinterpret_cast<const u32x4*>(p.weight + v * p.weight_stride + c * 8);
    s16x2 above = {0, 0}, below = {0, 0};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t two = w[e];                           // (a bit_cast of w[e] itself is one of w[0])
      above = __builtin_elementwise_max(above, __builtin_bit_cast(s16x2, two));
      below = __builtin_elementwise_max(below, __builtin_bit_cast(s16x2, two ^ 0x80008000u));
    }
    const s16x2 bounds = group_max<GROUP>(__builtin_elementwise_max(s16x2{above[0], below[0]}, s16x2{above[1], below[1]}));
    const uint32_t bits = __builtin_bit_cast(uint32_t, bounds);
    const float hi = __builtin_bit_cast(float, bits << 16), minus_lo = __builtin_bit_cast(float, bits & 0xffff0000u);
    float s = p.zeros ? (hi + minus_lo) / 15.0f : fmaxf(hi, minus_lo) / 7.0f;
    if (p.scales_bf16) s = (float)(__bf16)s;
    if (s == 0.0f) s = 1.0f;
    const float zero = p.zeros ? fminf(fmaxf(rintf(minus_lo / s), 0.0f), 15.0f) : 8.0f;
    float ratio[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) ratio[e] = __builtin_bit_cast(float, e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
    if (s > 0x1p-60f && s < 0x1p60f) {
      const float r = 1.0f / s;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float t = ratio[e] * r;
#pragma unroll
        for (int i = 0; i < 2; ++i) t = __builtin_fmaf(__builtin_fmaf(-t, s, ratio[e]), r, t);
        ratio[e] = t;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) ratio[e] /= s;
    }
    // four codes at a time as a number below 2^16, which fp32 holds
    uint32_t half[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float sum = 0.0f;
#pragma unroll
      for (int e = 3; e >= 0; --e) sum = __builtin_fmaf(sum, 16.0f, fminf(fmaxf(rintf(ratio[4 * h + e]) + zero, 0.0f), 15.0f));
      half[h] = (uint32_t)sum;
    }
    const uint32_t q = half[0] | half[1] << 16;
    if (live) {
      *reinterpret_cast<uint32_t*>(p.codes + v * p.codes_stride + c * 4) = q;
      if (c % (GROUP / 8) == 0) {
        const long long at = (long long)v * (per_row / (GROUP / 8)) + c / (GROUP / 8);
        if (p.scales_bf16) static_cast<__bf16*>(p.scales)[at] = (__bf16)s;
        else static_cast<float*>(p.scales)[at] = s;
        if (p.zeros) p.zeros[at] = (uint8_t)zero;
      }
    }
  }
}

// Eight codes of a dword as the bf16 values 16 + q (q in the mantissa's bits 3 to 6 over the exponent of 16), in the
// order 0 4 1 5 2 6 3 7: no conversion, one shift and one and-or for a pair.
// (The constants from registers that the compiler cannot see through: it then has an instruction for the and-or.)
struct CodeValues {
  uint32_t mask, k16;
  __device__ CodeValues() {
    asm("s_mov_b32 %0, 0x00780078" : "=s"(mask));
    asm("v_mov_b32 %0, 0x41804180" : "=v"(k16));
  }
  __device__ u32x4 operator()(uint32_t c) const {
    u32x4 r;
    r[0] = ((c << 3) & mask) | k16;
    r[1] = ((c >> 1) & mask) | k16;
    r[2] = ((c >> 5) & mask) | k16;
    r[3] = ((c >> 9) & mask) | k16;
    return r;
  }
};

// ---- few rows: the head is read once, and nothing else takes as long

constexpr int kFewWaves = 8;
#define SIP_GLOBAL __attribute__((address_space(1)))
template <class T, int N> struct __attribute__((packed)) Packed { T w[N]; };

// WORDS * 4 bytes from any address on, as the aligned words they lie in: a load of several words from an odd place takes twice the
// time.  `odd`: whether there are such places (uniform); where not, the one more word that they need is not read.  (That word
// holds a byte that is wanted, or it is the last one once more: nothing behind the array is touched.)
template <int WORDS>
struct Unaligned {
  uint32_t w[WORDS], more, shift;

  __device__ void load(const SIP_GLOBAL uint8_t* from, bool odd) {
    const uint64_t at = (uint64_t)from;
    shift = (uint32_t)(at & 3) * 8;
    const auto* words = (const SIP_GLOBAL Packed<uint32_t, WORDS>*)(at & ~3ull);
#pragma unroll
    for (int i = 0; i < WORDS; ++i) w[i] = words->w[i];
    more = 0;
    if (odd) more = *((const SIP_GLOBAL uint32_t*)words + (shift ? WORDS : WORDS - 1));
  }
  __device__ void get(uint32_t (&out)[WORDS]) const {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) out[i] = __builtin_amdgcn_alignbit(i + 1 < WORDS ? w[i + 1] : more, w[i], shift);
  }
};

// Scales and zero points of N neighbouring groups, aligned to their element; whole words of them if there are any.
__device__ const uint32_t kEights[8] = {0x08080808u, 0x08080808u, 0x08080808u, 0x08080808u,
                                        0x08080808u, 0x08080808u, 0x08080808u, 0x08080808u};   // a head without zero points
template <int N, int BYTES>
struct Elements {                        // N of BYTES each
  static constexpr bool kWhole = N * BYTES % 4 == 0;
  static constexpr int kWords = kWhole ? N * BYTES / 4 : 1;
  typedef std::conditional_t<BYTES == 1, uint8_t, uint16_t> Single;
  // (singles as wide as they were read: widened before its time, a load under way would be waited for)
  Unaligned<kWords> read;
  Single single[N];
  uint32_t words[kWords];

  __device__ void load(const SIP_GLOBAL uint8_t* from, bool odd) {
    if constexpr (kWhole) read.load(from, odd);
    else
#pragma unroll
      for (int i = 0; i < N; ++i) single[i] = ((const SIP_GLOBAL Single*)from)[i];
  }
  __device__ uint32_t get(int i) const {         // after settle()
    if constexpr (!kWhole) return single[i];
    const uint32_t word = words[i * BYTES / 4];
    return BYTES == 4 ? word : (word >> (i * BYTES % 4 * 8)) & (BYTES == 1 ? 0xffu : 0xffffu);
  }
  __device__ void settle() {
    if constexpr (kWhole) read.get(words);
  }
};
template <int N, bool SCALES_BF16>
struct GroupScales {
  Elements<N, SCALES_BF16 ? 2 : 4> s;
  Elements<N, 1> z;

  __device__ void settle() { s.settle(); z.settle(); }
  __device__ float scale(int g) const {
    if constexpr (SCALES_BF16) return __builtin_bit_cast(float, s.get(g) << 16);
    else return __builtin_bit_cast(float, s.get(g));
  }
  __device__ float zero(int g) const { return (float)z.get(g); }
};

// How a wave of UNITS * 128 entries reads its codes.  Units in pairs: of a row's 128 bytes a lane takes 16 at 32 * quad and the 16
// behind, so that a load touches whole lines (half lines are as many requests for half as much); a last unit without a
// partner: 16 at 16 * quad.  Dwords are then exchanged between the quarters of the wave until the four of a product hold
// entries of one group: between its halves (group 128), or as a 4 x 4 transposition; a unit alone needs less.
template <int GROUP, int UNITS>
struct UnitOrder {
  static __device__ constexpr bool paired(int u) { return (u | 1) < UNITS; }
  // byte of load u, from the row's first one in the wave's window on
  static __device__ int byte_of(int u, int quad) { return paired(u) ? (u >> 1) * 128 + quad * 32 + (u & 1) * 16 : u * 64 + quad * 16; }
  // entry at which the eight of dword j of load u begin, after order()
  static __device__ int entry_of(int u, int j, int quad) {
    if (paired(u))
      return (u >> 1) * 256 + (u & 1) * 32 +
             (GROUP == 128 ? (2 * (j >> 1) + (quad & 1)) * 64 + ((j & 1) + 2 * (quad >> 1)) * 8 : j * 64 + quad * 8);
    return u * 128 + (GROUP == 128 ? 32 * quad + 8 * j
                      : GROUP == 64 ? 64 * (j >> 1) + 32 * (quad & 1) + 8 * ((j & 1) + 2 * (quad >> 1)) : 32 * j + 8 * quad);
  }
  static __device__ u32x4 order(int u, u32x4 c) {
    if (GROUP == 128 && !paired(u)) return c;
    const u32x2 a = __builtin_amdgcn_permlane32_swap(c[0], c[2], false, false), b = __builtin_amdgcn_permlane32_swap(c[1], c[3], false, false);
    if (GROUP == (paired(u) ? 128 : 64)) return u32x4{a[0], b[0], a[1], b[1]};
    const u32x2 l = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false), h = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    return u32x4{l[0], l[1], h[0], h[1]};
  }
  // group of dword j of load u, counted in the window
  static __device__ constexpr int group_of(int u, int j) {
    return paired(u) ? ((u >> 1) * 256 + (u & 1) * 32 + j * 64) / GROUP : (u * 128 + j * 32) / GROUP;
  }
};

// Row r of the hidden states as the products take them, eight entries from k on in the order of CodeValues; zeros if not
// `wanted`.  A bf16 state is a row; an fp32 one is three, of 8 bits each: all 24.
__device__ inline bf16x8 hidden_row(const CodesArgs& p, int r, int k, bool wanted) {
  u32x4 out;
  if (p.hidden_bf16) {
    u32x4 w = {0, 0, 0, 0};
    if (wanted) w = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p.hidden) + r * p.hidden_stride + k);
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = e & 1 ? (w[e >> 1] >> 16) | (w[(e >> 1) + 2] & 0xffff0000u) : (w[e >> 1] & 0xffffu) | (w[(e >> 1) + 2] << 16);
  } else {
    const int b = r / 3, part = r - 3 * b;
    const float* from = static_cast<const float*>(p.hidden) + b * p.hidden_stride + k;
    uint32_t bits[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float x = wanted ? from[e] : 0.0f;
      for (int i = 0; i < 2; ++i)
        if (i < part) x -= __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, x) & 0xffff0000u);
      bits[e] = __builtin_bit_cast(uint32_t, x) >> 16;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = bits[e] | (bits[e + 4] << 16);
  }
  return __builtin_bit_cast(bf16x8, out);
}
__host__ __device__ inline int rows_of_state(bool hidden_bf16) { return hidden_bf16 ? 1 : 3; }

// Tiles a turn: as many as leave room in the registers beside the states (16 registers a unit and row of tiles).
constexpr int few_tiles(int group, bool scales_bf16, int units, int mt) {
  const int bytes = units * 128 / group * (scales_bf16 ? 3 : 5), states = 16 * units * mt;
  for (int nt = 4; nt > 1; nt /= 2)
    if (states + nt * (4 * units + 2 * ((bytes + 3) / 4) + 8 * mt) <= 200) return nt;
  return 1;
}

// Up to 16 * MT rows (hidden_row()), D from 128 on.  A workgroup a compute unit, which takes NT tiles of 16 vocabulary entries a turn; a
// wave keeps its eighth of the hidden states -- up to UNITS units of 128 entries -- in registers for all turns, reads its
// eighth of the tiles' codes, loading the next turn's into the registers it has just used, and the eight waves' sums meet
// in LDS.  Codes are the only thing read in quantity, 8 * NT * UNITS KB ahead of their use on each compute unit.
// A wave's window has UNITS units whatever its share; where that is more, it begins earlier if it would end behind the row,
// and what is another wave's share meets zeros.  (All waves have the same loads, and a wait for one can be told by
// how many came after it.)
// Products: 16 + q against the states, from - (16 + zero) times the group's sum of the states on; the scale on the fp32
// sum of a group.
// Bound by reading the head: one row, V = 128256, D = 4096, groups of 128 51 us, 5.3 TB/s.  With groups of 32, fp32 scales and
// 7 fp32 states (two rows of tiles), V = 151643, D = 2080, 106 us, 2.0 TB/s: a tile a turn is all that registers hold then,
// scales, sums by group and the codes' conversion take the vector units longer than the reads take, and of the 17 units the last
// wave has three where the others have two, which wait for it every turn.
template <int GROUP, bool SCALES_BF16, int UNITS, int MT>
__global__ __launch_bounds__(kFewWaves * 64) void head_few_kernel(CodesArgs p) {
  constexpr int NT = few_tiles(GROUP, SCALES_BF16, UNITS, MT);
  constexpr int kGroups = UNITS * 128 / GROUP;                          // of the window
  typedef UnitOrder<GROUP, UNITS> Order;
  __shared__ f32x4 sums[kFewWaves][kGroups][MT][4];                     // of the hidden states by group, as the accumulators lie
  __shared__ f32x4 part[2][kFewWaves][NT * MT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quad = lane >> 4;
  const int units = (p.D + 127) / 128, groups = p.D / GROUP;
  const int mine = wave * units / kFewWaves * 128, others = (wave + 1) * units / kFewWaves * 128;   // my share: [mine, others)
  const int first = min(mine, p.D - UNITS * 128);                       // of the window
  const bool last = others - mine == UNITS * 128;                        // whether the last unit is mine
  const int turns = (p.V + 16 * NT - 1) / (16 * NT);

  u32x4 codes[NT][UNITS];
  GroupScales<kGroups, SCALES_BF16> scales[NT], next[NT];
  const SIP_GLOBAL uint8_t* my_codes = (const SIP_GLOBAL uint8_t*)p.codes + first / 2;
  const SIP_GLOBAL uint8_t* zeros = (const SIP_GLOBAL uint8_t*)(p.zeros ? p.zeros : reinterpret_cast<const uint8_t*>(kEights));
  const uint32_t stride = (uint32_t)p.codes_stride, zeros_mask = p.zeros ? ~0u : 0u;
  constexpr int kScaleBytes = SCALES_BF16 ? 2 : 4;
  const SIP_GLOBAL uint8_t* scale_bytes = (const SIP_GLOBAL uint8_t*)p.scales;
  const bool odd_scales = (((uint64_t)scale_bytes | (uint64_t)(groups * kScaleBytes) | (uint64_t)(first / GROUP * kScaleBytes)) & 3) != 0;
  const bool odd_zeros = p.zeros && (((uint64_t)p.zeros | (uint64_t)groups | (uint64_t)(first / GROUP)) & 3) != 0;
  int step = gridDim.x;
  asm("" : "+s"(step));                                    // (read once: a load per use is what the compiler prefers)
  auto row_of = [&](int t, int turn) { return (uint32_t)min((turn * NT + t) * 16 + (lane & 15), p.V - 1); };
  auto load = [&](int t, int u, int turn) {
    codes[t][u] = *(const SIP_GLOBAL u32x4*)(my_codes + (uint64_t)row_of(t, turn) * stride + Order::byte_of(u, quad));
  };
  auto load_scales = [&](int t, int turn) {
    const uint32_t at = row_of(t, turn) * groups + first / GROUP;       // (below 2^28)
    next[t].s.load(scale_bytes + at * (uint32_t)kScaleBytes, odd_scales);
    next[t].z.load(zeros + (at & zeros_mask), odd_zeros);
  };
#pragma unroll
  for (int t = 0; t < NT; ++t) load_scales(t, blockIdx.x);
#pragma unroll
  for (int u = 0; u < UNITS; ++u)
#pragma unroll
    for (int t = 0; t < NT; ++t) load(t, u, blockIdx.x);

  const int each = rows_of_state(p.hidden_bf16), rows = p.B * each;
  bf16x8 x[UNITS][4][MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
#pragma unroll
    for (int u = 0; u < UNITS; ++u)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int k = first + Order::entry_of(u, j, quad);
        x[u][j][m] = hidden_row(p, min(m * 16 + (lane & 15), rows - 1), k, k >= mine && k < others && k < p.D);
      }
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const u32x4 ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
      f32x4 sum = {};
#pragma unroll
      for (int u = 0; u < UNITS; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (Order::group_of(u, j) == g)
            sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[u][j][m], __builtin_bit_cast(bf16x8, ones), sum, 0, 0, 0);
      if ((lane & 15) == 0) sums[wave][g][m][quad] = sum;
    }
  }
  // (a wave reads what it wrote itself)
  const CodeValues code_values;
  int side = 0;
  // `more`: whether there is a next turn to load for.
  auto take = [&](int turn, auto more) {
    f32x4 total[NT][MT] = {};
    // the next turn's scales ahead of its codes: loads arrive in the order of their issue, and the scales are wanted first
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      scales[t] = next[t];
      scales[t].settle();
      if constexpr (decltype(more)::value) load_scales(t, turn + step);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < UNITS; u += Order::paired(u) ? 2 : 1) {
      const int width = Order::paired(u) ? 2 : 1;
      if (width == 1 && UNITS > 1 && !last) break;         // (a unit alone, another wave's)
      // two tiles at once: a chain of products waits for its own sums
#pragma unroll
      for (int t0 = 0; t0 < NT; t0 += 2) {
        constexpr int kPair = NT > 1 ? 2 : 1;
        u32x4 c[kPair][2];
#pragma unroll
        for (int t = 0; t < kPair; ++t)
#pragma unroll
          for (int e = 0; e < width; ++e) c[t][e] = Order::order(u + e, codes[t0 + t][u + e]);
        // a group's sums are scaled when the next group's products are under way; the sums of the states are read as far ahead
        const int first_group = Order::group_of(u, 0), last_group = Order::group_of(u + width - 1, 3);
        f32x4 acc[2][kPair][MT], sum[2][MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) sum[0][m] = sums[wave][first_group][m][quad];
#pragma unroll
        for (int g = first_group; g <= last_group + 1; ++g) {
          const int now = (g - first_group) & 1;
          if (g < last_group) {
#pragma unroll
            for (int m = 0; m < MT; ++m) sum[now ^ 1][m] = sums[wave][g + 1][m][quad];
          }
          if (g <= last_group) {
#pragma unroll
            for (int t = 0; t < kPair; ++t) {
              const float zero = -16.0f - scales[t0 + t].zero(g);
#pragma unroll
              for (int m = 0; m < MT; ++m) acc[now][t][m] = sum[now][m] * zero;
#pragma unroll
              for (int e = 0; e < width; ++e)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  if (Order::group_of(u + e, j) != g) continue;
                  const bf16x8 w = __builtin_bit_cast(bf16x8, code_values(c[t][e][j]));
#pragma unroll
                  for (int m = 0; m < MT; ++m)
                    acc[now][t][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[u + e][j][m], w, acc[now][t][m], 0, 0, 0);
                }
            }
          }
          __builtin_amdgcn_sched_barrier(0);
          if (g > first_group) {
#pragma unroll
            for (int t = 0; t < kPair; ++t) {
              const float s = scales[t0 + t].scale(g - 1);
#pragma unroll
              for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int r = 0; r < 4; ++r) total[t0 + t][m][r] = __builtin_fmaf(s, acc[now ^ 1][t][m][r], total[t0 + t][m][r]);
            }
          }
        }
        // Here and nowhere else: earlier they would need registers of their own, later they would be waited for.
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (decltype(more)::value)
#pragma unroll
          for (int t = t0; t < t0 + 2 && t < NT; ++t) {
#pragma unroll
            for (int e = 0; e < width; ++e) load(t, u + e, turn + step);
          }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int m = 0; m < MT; ++m) part[side][wave][t * MT + m][lane] = total[t][m];
    __builtin_amdgcn_s_waitcnt(0xC07F);                    // (LDS alone: what was loaded for the next turn stays under way)
    __builtin_amdgcn_s_barrier();                          // (the other side's sums were read before this turn's)
    // row r of entry v: quarter (r % 16) / 4, register r % 4
    for (int o = threadIdx.x; o < NT * 16 * p.B; o += kFewWaves * 64) {
      const int b = o / (NT * 16), e = o % (NT * 16);
      float z = 0.0f;
      for (int r = (b + 1) * each - 1; r >= b * each; --r)
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) z += part[side][w][(e >> 4) * MT + (r >> 4)][((r & 15) >> 2) * 16 + (e & 15)][r & 3];
      const int v = turn * NT * 16 + e;
      if (v < p.V) {
        if (p.logits_bf16) static_cast<__bf16*>(p.logits)[b * p.logits_stride + v] = (__bf16)z;
        else static_cast<float*>(p.logits)[b * p.logits_stride + v] = z;
      }
    }
    side ^= 1;
  };
  // (else the compiler, which takes the loads up to here for still under way, waits for all of them in every turn)
  __builtin_amdgcn_s_waitcnt(0x0F70);                      // vmcnt(0)
  int turn = blockIdx.x;
  for (; turn + step < turns; turn += step) take(turn, std::true_type());
  take(turn, std::false_type());
}

// ---- more rows: tiles of the product, the hidden states through LDS

// Rows of a block of MT * 16: as many whole states as fit it.
__host__ __device__ inline int block_states(int mt, bool hidden_bf16) { return mt * 16 / rows_of_state(hidden_bf16); }
__host__ __device__ inline int many_units(int D) { return (D + 255) / 256 * 2; }             // of 128 entries
__host__ __device__ inline int many_groups(int D, int group) { return many_units(D) * 128 / group; }   // zeros behind the last ones

// The states in the order of the products, by block: [pair of units][product][tile of rows][lane], 16 bytes a lane: eight products of
// the states, and behind them zero_products() of the states' sums by group, as SumParts says.
__host__ __device__ constexpr int zero_products(int group) { return group == 32 ? 2 : 1; }
struct ManyLayout {
  size_t pair, block;                                     // bytes
  __host__ __device__ ManyLayout(int D, int group, int mt) {
    pair = (size_t)(8 + zero_products(group)) * mt * 1024;
    block = many_units(D) / 2 * pair;
  }
};

// Products x y of fp32 values, four groups a matrix product, from bf16 parts that are a value's next 8 bits each.  Of a group
// quarter j of the wave has a pair of terms, dword i that of group i: x0 y0; x0 y1 and x1 y0; x0 y2 and x2 y0; x1 y1 and x1 y2.
// (The instruction aligns the eight terms of a quarter with their largest and cuts off what is below 24 bits, but rounds the
// quarters' sums: terms of all sizes in one quarter lost 2^-23 of the product, always to the same side.)
struct SumParts {
  uint32_t part[3];                                        // bf16 in the upper half
  __device__ explicit SumParts(float x) {
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      part[i] = __builtin_bit_cast(uint32_t, x) & 0xffff0000u;
      x -= __builtin_bit_cast(float, part[i]);
    }
  }
  __device__ uint32_t two(int low, int high) const { return (part[low] >> 16) | part[high]; }
  __device__ u32x4 x() const { return u32x4{part[0] >> 16, two(0, 1), two(0, 2), two(1, 1)}; }     // by quarter
  __device__ u32x4 y() const { return u32x4{part[0] >> 16, two(1, 0), two(2, 0), two(1, 2)}; }
};

// A wave takes a tile of 16 rows and a group.
template <int GROUP>
__global__ __launch_bounds__(256) void head_rows_kernel(CodesArgs p, int mt) {
  const int lane = threadIdx.x & 63, quad = lane >> 4, g = blockIdx.y * 4 + (threadIdx.x >> 6);
  if (g >= many_groups(p.D, GROUP)) return;
  const int block = blockIdx.x / mt, tile = blockIdx.x % mt, each = rows_of_state(p.hidden_bf16), states = block_states(mt, p.hidden_bf16);
  const int r = tile * 16 + (lane & 15), state = block * states + r / each;
  const bool live = r < states * each && state < p.B;
  const ManyLayout layout(p.D, GROUP, mt);
  constexpr int kGroups = 256 / GROUP;                     // of a pair
  char* out = p.states + block * layout.block + g / kGroups * layout.pair + tile * 1024;
  float sum = 0.0f;
  for (int c = g * (GROUP / 32); c < (g + 1) * (GROUP / 32); ++c) {
    const int k = c * 32 + quad * 8;
    const bf16x8 x = hidden_row(p, live ? state * each + r % each : 0, k, live && k < p.D);
    *reinterpret_cast<bf16x8*>(out + c % 8 * mt * 1024 + lane * 16) = x;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += (float)x[e];
  }
  sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
  // (of 128 there are two groups, and two of zeros)
  uint32_t* to = reinterpret_cast<uint32_t*>(out + (8 + g % kGroups / 4) * mt * 1024 + lane * 16) + g % kGroups % 4;
  const u32x4 terms = SumParts(sum).x();
  to[0] = quad == 0 ? terms[0] : quad == 1 ? terms[1] : quad == 2 ? terms[2] : terms[3];
  if (GROUP == 128) to[2] = 0;
}

// WAVES * NT * 16 vocabulary entries by MT * 16 rows: 256 entries, or 64 where tiles of 256 would leave compute units without
// one (31 fp32 states, V = 5164, D = 5568: 60 us instead of 116).  A wave has NT * 16 of the entries and all rows, so that a
// code becomes a bf16 value once.  It goes through a pair of units -- 256 entries of a state, a line of each row's codes -- at a
// time: states through LDS, codes and scales straight into registers, all of the next pair's loaded while this one's products
// are made.
//   sum_g s (sum_d (16 + q) x - (16 + zero) sum_d x)
// The second part of a pair is a product over its groups, in bf16 parts (SumParts), ahead of the first: with 8 row tiles it saves 32
// multiplications a group and tile of entries.  What cancels between the two, the more the further the states' mean is from
// zero, cancels within 256 entries.  States of mean 1, D = 4096, groups of 128 and 32: off by 4.3e-7 and 1.0e-6 of the result; with a
// row's second part added as a whole 2.2e-6 and 9.8e-6, for 3 to 10 % less time.
// 256 rows, V = 152064, D = 4096, fp32 logits, groups of 128, 64, 32: 393, 450, 647 us, 811, 709, 493 TFLOP/s.  In groups of 64
// matrix cores are busy for 33 % of it and vector units for 43 (half of that the scales' multiplications), which two waves of a
// SIMD do not hide behind each other altogether; reads further ahead or four waves of half the entries changed nothing.
template <int GROUP, bool SCALES_BF16, int MT, int WAVES, int NT>
__global__ __launch_bounds__(WAVES * 64) void head_many_kernel(CodesArgs p) {
  constexpr int kEntries = WAVES * NT * 16, kGroups = 256 / GROUP, kZero = zero_products(GROUP);
  constexpr int kPieces = (8 + kZero) * MT, kPairBytes = kPieces * 1024, kLoads = (kPieces + WAVES - 1) / WAVES;
  constexpr int kPitch = kEntries + 4;
  constexpr int kRing = 2 * kPairBytes, kOut = MT * 16 * kPitch * 4;
  __shared__ __attribute__((aligned(1024))) char lds_bytes[kRing > kOut ? kRing : kOut];
  SIP_LDS char* lds = (SIP_LDS char*)lds_bytes;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quad = lane >> 4;
  const int each = rows_of_state(p.hidden_bf16), states = block_states(MT, p.hidden_bf16), blocks = (p.B + states - 1) / states;
  // the blocks of one tile of entries on one XCD, one after the other
  const int tile = (int)(blockIdx.x >> 3) / blocks * 8 + (blockIdx.x & 7), block = (int)(blockIdx.x >> 3) % blocks;
  if (tile * kEntries >= p.V) return;
  const ManyLayout layout(p.D, GROUP, MT);
  const char* from = p.states + block * layout.block;
  const int pairs = many_units(p.D) / 2, groups = p.D / GROUP;
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
  auto load_states = [&](int pair) {
    const uint64_t at = reinterpret_cast<uint64_t>(from + (size_t)pair * kPairBytes);
    const u32x4 buffer = {(uint32_t)at, (uint32_t)(at >> 32) & 0xffff, kPairBytes, 0x00020000};
#pragma unroll
    for (int l = 0; l < kLoads; ++l) {
      if (kPieces % WAVES != 0 && l * WAVES + wave >= kPieces) break;
      const uint32_t piece = (l * WAVES + wave) * 1024;
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                   :: "s"(lds0 + (uint32_t)(pair & 1) * kPairBytes + piece), "v"(piece + lane * 16), "s"(buffer) : "memory");
    }
  };
  uint32_t row[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) row[t] = min(tile * kEntries + (wave * NT + t) * 16 + (lane & 15), p.V - 1);
  const SIP_GLOBAL uint8_t* zeros = (const SIP_GLOBAL uint8_t*)(p.zeros ? p.zeros : reinterpret_cast<const uint8_t*>(kEights));
  const uint32_t stride = (uint32_t)p.codes_stride;
  u32x4 next_codes[NT][2];
  auto load_codes = [&](int pair) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 2; ++e)
        next_codes[t][e] = *(const SIP_GLOBAL u32x4*)((const SIP_GLOBAL uint8_t*)p.codes + (uint64_t)row[t] * stride +
                                                      min(pair * 128 + quad * 32 + e * 16, p.D / 2 - 16));
  };
  float scales[NT][kGroups];
  uint32_t next_scales[NT][kGroups];                       // as they are loaded: to shift them there would wait for them
  auto load_scales = [&](int pair) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        const uint32_t at = row[t] * groups + min(pair * kGroups + g, groups - 1);
        if constexpr (SCALES_BF16) next_scales[t][g] = ((const SIP_GLOBAL uint16_t*)p.scales)[at];
        else next_scales[t][g] = ((const SIP_GLOBAL uint32_t*)p.scales)[at];
      }
  };
  uint32_t next_zeros[NT][kZero];                          // of group 4 c + my quarter
  const uint32_t zeros_mask = p.zeros ? ~0u : 0u;
  auto load_zeros = [&](int pair) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int c = 0; c < kZero; ++c)
        next_zeros[t][c] = zeros[(row[t] * groups + min(pair * kGroups + c * 4 + quad % kGroups, groups - 1)) & zeros_mask];
  };
  load_states(0);
  load_scales(0);
  load_zeros(0);
  load_codes(0);

  f32x4 total[NT][MT] = {};
  // A step: the products of a tile of rows and a group -- with the tile's first group the zero points' --, and with them the
  // multiplications of the step before and the reads of the one behind.
  constexpr int kEach = GROUP / 32, kSteps = MT * kGroups;
  const CodeValues code_values;
  for (int pair = 0; pair < pairs; ++pair) {
    bf16x8 w[NT][8], w_zero[NT][kZero];                    // product c of the pair: dword c / 2 of load c % 2
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const u32x4 codes = UnitOrder<32, 2>::order(e, next_codes[t][e]);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[t][2 * j + e] = __builtin_bit_cast(bf16x8, code_values(codes[j]));
      }
#pragma unroll
      for (int g = 0; g < kGroups; ++g) scales[t][g] = __builtin_bit_cast(float, SCALES_BF16 ? next_scales[t][g] << 16 : next_scales[t][g]);
#pragma unroll
      for (int c = 0; c < kZero; ++c) {
        float s = scales[t][c * 4];
#pragma unroll
        for (int q = 1; q < 4 && q < kGroups; ++q) s = quad == q ? scales[t][c * 4 + q] : s;
        if (quad >= kGroups) s = 0.0f;
        w_zero[t][c] = __builtin_bit_cast(bf16x8, UnitOrder<32, 1>::order(0, SumParts(s * (-16.0f - (float)next_zeros[t][c])).y()));
      }
    }
    // this pair's states have arrived, and everybody has read the last one's
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    const uint32_t states_at = lds0 + (uint32_t)(pair & 1) * kPairBytes + lane * 16;
    bf16x8 x[2][kEach], sums[2][kZero];
    f32x4 acc[2][NT];
    auto read = [&](int step) {
#pragma unroll
      for (int j = 0; j < kEach; ++j)
        x[step & 1][j] = *(const SIP_LDS bf16x8*)(uintptr_t)(states_at + ((step % kGroups * kEach + j) * MT + step / kGroups) * 1024);
      if (step % kGroups == 0)
#pragma unroll
        for (int c = 0; c < kZero; ++c)
          sums[step / kGroups & 1][c] = *(const SIP_LDS bf16x8*)(uintptr_t)(states_at + ((8 + c) * MT + step / kGroups) * 1024);
    };
    auto scale = [&](int step) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          total[t][step / kGroups][r] = __builtin_fmaf(scales[t][step % kGroups], acc[step & 1][t][r], total[t][step / kGroups][r]);
    };
    read(0);
    if (pair + 1 < pairs) {
      load_states(pair + 1);
      load_scales(pair + 1);
      load_zeros(pair + 1);
      load_codes(pair + 1);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int step = 0; step < kSteps; ++step) {
      const bool first = step % kGroups == 0, reads_sums = step + 1 < kSteps && (step + 1) % kGroups == 0;
      if (step + 1 < kSteps) read(step + 1);
      if (first)
#pragma unroll
        for (int c = 0; c < kZero; ++c)
#pragma unroll
          for (int t = 0; t < NT; ++t)
            total[t][step / kGroups] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(sums[step / kGroups & 1][c], w_zero[t][c], total[t][step / kGroups], 0, 0, 0);
#pragma unroll
      for (int j = 0; j < kEach; ++j)
#pragma unroll
        for (int t = 0; t < NT; ++t)
          acc[step & 1][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[step & 1][j], w[t][step % kGroups * kEach + j], j == 0 ? f32x4{} : acc[step & 1][t], 0, 0, 0);
      if (step > 0) scale(step - 1);
      __builtin_amdgcn_sched_group_barrier(0x100, kEach, 0);
      if (reads_sums) __builtin_amdgcn_sched_group_barrier(0x100, kZero, 0);
      if (first) __builtin_amdgcn_sched_group_barrier(0x008, kZero * NT, 0);
#pragma unroll
      for (int n = 0; n < kEach * NT; ++n) {               // in turn: a product, and multiplications while it runs
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 4 / kEach, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    scale(kSteps - 1);
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
  SIP_LDS float* out = (SIP_LDS float*)lds;
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int r = 0; r < 4; ++r) out[(m * 16 + quad * 4 + r) * kPitch + (wave * NT + t) * 16 + (lane & 15)] = total[t][m][r];
  __syncthreads();
  const int v = tile * kEntries + (threadIdx.x & (kEntries - 1));
  for (int b = threadIdx.x / kEntries; b < states && block * states + b < p.B; b += WAVES * 64 / kEntries) {
    float z = 0.0f;
    for (int r = (b + 1) * each - 1; r >= b * each; --r) z += out[r * kPitch + (threadIdx.x & (kEntries - 1))];
    if (v < p.V) {
      const long long at = (block * states + b) * p.logits_stride + v;
      if (p.logits_bf16) static_cast<__bf16*>(p.logits)[at] = (__bf16)z;
      else static_cast<float*>(p.logits)[at] = z;
    }
  }
}

}  // namespace sip
