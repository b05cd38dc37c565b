// Products of bf16 matrices with fp32 sums, a tile at a time, for the kernels of sip_xent.h:
//   C[b][a] = sum_k A(a, k) * B(b, k),
// either operand with its rows along k (kRows) or with k as the row index (kCols).
//
// Tiles of both operands go from memory to LDS without passing registers, a unit of 64 k at a time -- whole 128-byte lines
// of either form --, one unit of B and two of A ahead of their use in the widest tile: a unit's products take 2048 cycles of the
// matrix cores, a load that misses the L2 some 2500.  There eight waves hold 128 x 64 each (128 accumulators a lane), two a SIMD,
// for which LDS serves 96 bytes a cycle of the 128 it has.  What an element is read as 16-byte groups
// for, eight of its neighbours along k, a kCols tile delivers by transposing reads.  Groups lie in LDS permuted (swizzled) so
// that the lanes of a read meet every bank once.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sip {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int16_t s16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

#define SIP_LDS __attribute__((address_space(3)))

enum OperandForm { kRows, kCols };

// One operand: element (i, k) of it is base[i * stride + k] (kRows) or base[k * stride + i] (kCols).  Indices from n on
// are zeros.  kRows with `rows`: row i is row rows[i] of base (ascending).
struct Operand {
  const uint16_t* base;
  long long stride;
  int n;
  const int* rows;
};


constexpr int kUnit = 64;                                // k of a unit

// A tile of kA x kB, in waves of kWaveA x kWaveB, with room for SLOTS_A and SLOTS_B units.
template <int A, int B, int WA, int WB, int SLOTS_A, int SLOTS_B>
struct GemmShape {
  static constexpr int kA = A, kB = B, kWaveA = WA, kWaveB = WB, kSlotsA = SLOTS_A, kSlotsB = SLOTS_B;
  static constexpr int kTA = WA / 16, kTB = WB / 16;                  // 16 x 16 blocks of a wave
  static constexpr int kWaves = (A / WA) * (B / WB), kThreads = kWaves * 64;
  typedef f32x4 Acc[kTA][kTB];
  static constexpr int kBytesA = A * kUnit * 2, kBytesB = B * kUnit * 2;
  static constexpr int kLds = SLOTS_A * kBytesA + SLOTS_B * kBytesB;
  static constexpr int kLoadsA = kBytesA / (kWaves * 1024), kLoadsB = kBytesB / (kWaves * 1024);
  static constexpr int kLoads = kLoadsA + kLoadsB;                    // of a wave, 1 KB each
  static_assert(kBytesA % (kWaves * 1024) == 0 && kBytesB % (kWaves * 1024) == 0, "the waves share a tile's loads evenly");
  static_assert(SLOTS_B >= 2 && (SLOTS_A == SLOTS_B || SLOTS_A == SLOTS_B + 1) && kLds <= 160 * 1024, "see Gemm::tile()");
};

// The 16 x 16 block of C that a wave holds: register r of a lane is row a + acc_a(lane) + r, column b + lane % 16.
__device__ inline int acc_a(int lane) { return 4 * (lane >> 4); }

constexpr uint32_t kOutside = 0x80000000u;               // an offset that the buffer's bounds check turns into zeros

// Where 16-byte group c of the eight of LDS row i (kRows) lies: at c ^ its swizzle.  LDS serves sixteen lanes of a read at a
// time, of which eight read one group and eight its neighbour (c ^ 1), of the other eight rows: 256 bytes, every bank once.
__device__ inline int swizzle_rows(int i) { return i & 6; }
// The same for row k of a kCols tile of 128 entries a row or more: a transposing read takes 32 bytes of each of four rows k,
// and of four more for every eight.
__device__ inline int swizzle_cols(int k) { return ((k & 3) << 1) ^ (((k >> 3) & 1) << 3); }

// The loads of a wave for one operand's I indices.
template <OperandForm F, int I, int WAVES>
struct TileLoader {
  static constexpr int K = kUnit, THREADS = WAVES * 64, LOADS = I * K * 2 / (WAVES * 1024);
  const char* base;                    // of the tile at its first k
  long long step;                      // bytes from a unit to the next
  uint32_t offset[LOADS];              // of my 16 bytes, kOutside where the index is
  int k;                               // their k within the unit: load j's is k + j * kStep
  static constexpr int kStep = F == kRows ? 0 : THREADS / (I / 8);

  __device__ void init(const Operand& m, int i0, int k0, int wave, int lane) {
    const int first = m.rows ? m.rows[min(i0, m.n - 1)] : i0;
    base = reinterpret_cast<const char*>(m.base + (F == kRows ? first * m.stride + k0 : k0 * m.stride + i0));
    step = F == kRows ? (long long)K * 2 : (long long)K * m.stride * 2;
    const int at0 = wave * 64 + lane;
    k = F == kRows ? ((at0 % (K / 8)) ^ swizzle_rows(at0 / (K / 8))) * 8 : at0 / (I / 8);
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int at = j * THREADS + at0;                        // 16-byte group of the tile's LDS image
      if constexpr (F == kRows) {
        static_assert(THREADS / (K / 8) % 16 == 0, "a load's rows repeat the swizzle");
        const int i = at / (K / 8);
        const long long row = m.rows ? m.rows[min(i0 + i, m.n - 1)] - first : i;
        offset[j] = i0 + i < m.n ? (uint32_t)(row * m.stride * 2 + k * 2) : kOutside;
      } else {
        static_assert(I >= 128, "room for the swizzle");
        const int c = (at % (I / 8)) ^ swizzle_cols(k + j * kStep);
        offset[j] = i0 + c * 8 < m.n ? (uint32_t)((k + j * kStep) * m.stride * 2 + c * 16) : kOutside;
      }
    }
  }
  // Load j of unit t into the LDS image at `lds` (uniform); `left`: how many k there are from the unit's first one on.
  // Assembly: the compiler would have every transposing read wait for all of them.  unit_barrier() waits.  (m0 is nobody's:
  // the compiler sets it where it needs it.)
  __device__ void load(int j, int t, int left, uint32_t lds, int wave) const {
    const uint64_t at = reinterpret_cast<uint64_t>(base + t * step);
    const u32x4 buffer = {(uint32_t)at, (uint32_t)(at >> 32) & 0xffff, kOutside, 0x00020000};
    const uint32_t from = k < left - j * kStep ? offset[j] : kOutside;
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :: "s"(lds + (j * WAVES + wave) * 1024), "v"(from), "s"(buffer) : "memory");
  }
};

// The reads of a lane for 16 * T entries from i0 on, 32 k at a time: entry lane % 16 of a block, k 8 * (lane / 16) to + 7.
template <OperandForm F, int I, int T>
struct FragmentReader {
  static constexpr int K = kUnit;
  int at[F == kRows ? K / 32 : 1];     // byte offsets in the operand's LDS image

  __device__ void init(int i0, int lane) {
    if constexpr (F == kRows) {
      const int i = i0 + (lane & 15);
#pragma unroll
      for (int s = 0; s < K / 32; ++s) at[s] = i * K * 2 + (((4 * s + (lane >> 4)) ^ swizzle_rows(i)) << 4);
    } else {
      // (i0 a multiple of 16 T, T a power of two: block t's 16-byte groups are those of block 0 with 2 t in bits that are clear there)
      const int k = 8 * (lane >> 4) + ((lane & 15) >> 2), i = i0 + ((lane & 3) << 2);
      at[0] = k * I * 2 + (((i >> 3) ^ swizzle_cols(k)) << 4) + ((i & 4) << 1);
    }
  }
  __device__ bf16x8 read(uint32_t lds, int s, int t) const {
    if constexpr (F == kRows) {
      return *(const SIP_LDS bf16x8*)(uintptr_t)(lds + at[s] + t * 16 * K * 2);
    } else {
      const uint32_t p = ((lds + at[0]) ^ (t << 5)) + s * 32 * I * 2;
      s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SIP_LDS s16x4*)(uintptr_t)p);
      s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SIP_LDS s16x4*)(uintptr_t)(p + 4 * I * 2));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
};

// vmcnt(n), lgkmcnt(0) and the barrier: my loads but the last n have arrived, my LDS reads are done, and so are the others'.
template <int N>
__device__ inline void unit_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// acc[i][j] of wave w: the block at a0 + (w % (kA / kWaveA)) * kWaveA + 16 i, b0 + (w / (kA / kWaveA)) * kWaveB + 16 j.
// All of the workgroup's waves leave together, with nothing under way to LDS.
template <class S, OperandForm FA, OperandForm FB>
struct Gemm {
  __device__ static void tile(typename S::Acc& acc, const Operand& A, const Operand& B, int a0, int b0, int k_begin,
                              int k_end, SIP_LDS char* lds) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wa = wave % (S::kA / S::kWaveA), wb = wave / (S::kA / S::kWaveA);
    TileLoader<FA, S::kA, S::kWaves> la;
    TileLoader<FB, S::kB, S::kWaves> lb;
    la.init(A, a0, k_begin, wave, lane);
    lb.init(B, b0, k_begin, wave, lane);
    FragmentReader<FA, S::kA, S::kTA> ra;
    FragmentReader<FB, S::kB, S::kTB> rb;
    ra.init(wa * S::kWaveA, lane);
    rb.init(wb * S::kWaveB, lane);
    const int n = k_end - k_begin, units = (n + kUnit - 1) / kUnit;
    const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
    constexpr int kLdsB = S::kSlotsA * S::kBytesA;         // where B's slots begin
    auto load_a = [&](int j, int u) { la.load(j, u, n - u * kUnit, lds0 + (uint32_t)u % S::kSlotsA * S::kBytesA, wave); };
    auto load_b = [&](int j, int u) { lb.load(j, u, n - u * kUnit, lds0 + kLdsB + (uint32_t)u % S::kSlotsB * S::kBytesB, wave); };
    // Load j of the kLoads that a wave issues between the barrier of unit u - 1 and that of unit u: B's first, which is needed
    // first.  (Past the end: zeros into slots that nobody reads.)
    auto load = [&](int j, int u) { j < S::kLoadsB ? load_b(j, u + S::kSlotsB - 1) : load_a(j - S::kLoadsB, u + S::kSlotsA - 1); };
    // A step is 32 k: a row of blocks after the other, its fragment of A read anew for the next step when its products are
    // done; B's fragments, which every row needs, in two sets.
    bf16x8 fa[S::kTA], fb[2][S::kTB];
    auto read_a = [&](int i, int u, int s) { fa[i] = ra.read(lds0 + (uint32_t)u % S::kSlotsA * S::kBytesA, s, i); };
    auto read_b = [&](int j, int u, int s) { fb[s & 1][j] = rb.read(lds0 + kLdsB + (uint32_t)u % S::kSlotsB * S::kBytesB, s, j); };
    constexpr int kRow = S::kTB, kProducts = S::kTA * kRow;
    constexpr int kBefore = S::kTA > 2 ? 2 : 1;            // rows of a unit's second step that come before its barrier
    // Of the loads between two barriers, those that are issued before product q behind the first: evenly spread.  (All in a row
    // they wait for the address unit, 16 cycles a load, and the products behind them too.)
    auto issued = [](int q) constexpr { return q * S::kLoads / (2 * kProducts); };
#pragma unroll
    for (int u = 0; u < S::kSlotsA - 1; ++u) {
#pragma unroll
      for (int j = 0; j < S::kLoadsA; ++j) load_a(j, u);
      if (u < S::kSlotsB - 1)
#pragma unroll
        for (int j = 0; j < S::kLoadsB; ++j) load_b(j, u);
    }
    constexpr int kFirst = issued(kProducts - kBefore * kRow);   // of the first window, those that belong to the unit before
#pragma unroll
    for (int j = 0; j < kFirst; ++j) load(j, 0);
    unit_barrier<S::kLoadsA * (S::kSlotsA - 2) + S::kLoadsB * (S::kSlotsB - 2) + kFirst>();
#pragma unroll
    for (int j = 0; j < S::kTB; ++j) read_b(j, 0, 0);
#pragma unroll
    for (int i = 0; i < S::kTA; ++i) read_a(i, 0, 0);
    // (else the compiler takes what it loaded up to here for still under way inside the loop, and waits for everything)
    __builtin_amdgcn_s_waitcnt(0xC07F);                    // lgkmcnt(0)
    for (int u = 0; u < units; ++u) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
#pragma unroll
        for (int i = 0; i < S::kTA; ++i) {
#pragma unroll
          for (int j = 0; j < kRow; ++j) {
            // The order is that of the source.
            const int m = i * kRow + j, after = m - kBefore * kRow;
            const int q = s == 0 ? 2 * kProducts - kProducts - kBefore * kRow + m : after < 0 ? 2 * kProducts + after : after;
#pragma unroll
            for (int l = issued(q); l < issued(q + 1); ++l) load(l, s == 1 && after >= 0 ? u + 1 : u);
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[i], fb[s][j], acc[i][j], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
          }
          if (s == 0) {
            if (i * 2 < S::kTB) {
              read_b(i * 2, u, 1);
              if (i * 2 + 1 < S::kTB) read_b(i * 2 + 1, u, 1);
            }
            read_a(i, u, 1);
          } else if (i + 1 == kBefore) {
            // The next unit's reads begin: it has arrived -- what was issued after it may be under way --, and everybody has
            // read the last of this one, whose slots are free from here on.
            unit_barrier<S::kLoads * (S::kSlotsB - 2) + (S::kSlotsA > S::kSlotsB ? S::kLoadsA : 0)>();
#pragma unroll
            for (int j = 0; j < S::kTB; ++j) read_b(j, u + 1, 0);
#pragma unroll
            for (int k = 0; k <= i; ++k) read_a(k, u + 1, 0);
          } else if (i + 1 > kBefore) {
            read_a(i, u + 1, 0);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    unit_barrier<0>();
  }
};

}  // namespace sip
