// Rows of an embedding by token, and their gradient.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/sip_head.h"
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
  int group_shift;                                       // log2 of a group's entries
  int V, D, N;
  const int* ids;
  float scale;
  void* out; long long out_stride; int out_bf16;
};

// A lane takes eight neighbours of a row, or of kEmbedAhead rows, all under way at once.  Bound by memory: 16000 tokens of 4096 bf16 40 us, 4.5 TB/s
// of the distinct rows and what is written; a few tokens by a launch and two reads, 2.8 us.
template <bool CODES, int kEmbedAhead>
__global__ __launch_bounds__(256) void embed_kernel(EmbedArgs a) {
  const uint32_t per_row = a.D / 8, total = per_row * (uint32_t)a.N;                        // (up to 2^31)
  const uint32_t u0 = blockIdx.x * (kEmbedAhead * 256) + threadIdx.x;
  int v[kEmbedAhead], c[kEmbedAhead];
  long long to[kEmbedAhead];
#pragma unroll
  for (int j = 0; j < kEmbedAhead; ++j) {
    const uint32_t u = u0 + j * 256, i = u / per_row;
    c[j] = (int)(u - i * per_row) * 8;
    to[j] = u < total ? i * a.out_stride + c[j] : -1;
    v[j] = u < total ? a.ids[i] : -1;
  }
  if constexpr (CODES) {
    uint32_t q[kEmbedAhead];
    float s[kEmbedAhead];
    int zero[kEmbedAhead];
#pragma unroll
    for (int j = 0; j < kEmbedAhead; ++j) {
      q[j] = 0; s[j] = 0.0f; zero[j] = 8;
      if ((unsigned)v[j] >= (unsigned)a.V) continue;
      const long long at = (long long)v[j] * (a.D >> a.group_shift) + (c[j] >> a.group_shift);
      q[j] = *reinterpret_cast<const uint32_t*>(a.codes + v[j] * a.codes_stride + c[j] / 2);
      s[j] = a.scales_bf16 ? (float)static_cast<const __bf16*>(a.scales)[at] : static_cast<const float*>(a.scales)[at];
      if (a.zeros) zero[j] = a.zeros[at];
    }
#pragma unroll
    for (int j = 0; j < kEmbedAhead; ++j) {
      f32x8 f;
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = (float)((int)(q[j] >> 4 * e & 15) - zero[j]) * s[j] * a.scale;
      if ((unsigned)v[j] >= (unsigned)a.V) f = f32x8{0, 0, 0, 0, 0, 0, 0, 0};
      if (to[j] >= 0) store_eight(a.out, to[j], a.out_bf16, f);
    }
  } else {
    Eight x[kEmbedAhead];
#pragma unroll
    for (int j = 0; j < kEmbedAhead; ++j) {
      x[j] = Eight{};
      if ((unsigned)v[j] < (unsigned)a.V) x[j] = load_eight(a.weight, v[j] * a.weight_stride + c[j], a.weight_bf16);
    }
#pragma unroll
    for (int j = 0; j < kEmbedAhead; ++j) {
      f32x8 f = as_floats(x[j], a.weight_bf16) * a.scale;
      if ((unsigned)v[j] >= (unsigned)a.V) f = f32x8{0, 0, 0, 0, 0, 0, 0, 0};            // (whatever the scale)
      if (to[j] >= 0) store_eight(a.out, to[j], a.out_bf16, f);
    }
  }
}

// ---------------------------------------------------------------- gradient
// The tokens are sorted, equal ones in the order of their positions.  The sorted list is cut into pieces; a lane sums eight
// neighbouring columns of a piece's rows, token by token.  A cut that would fall into a token of few entries (`whole`) moves to its
// end, so that a token is in one piece, and its sum final; sums of a longer one's parts go to the workspace in fp32, and a third kernel
// adds them up in order.

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kSortPairs = 256;                          // entries of a bucket that are compared with one another
constexpr int kSortBits = 6, kSortBins = 1 << kSortBits; // most of a digit
constexpr int kBucketMost = 4096;                        // tokens of a bucket
constexpr int kPosBits = 16;                             // an entry: the token within its bucket, and the position below

struct EmbedGradArgs {
  const void* grad; long long grad_stride;
  const int* ids;
  int N, V, D;
  float scale;
  void* out; long long out_stride; int out_bf16;
  int shift, buckets;                                    // bucket of a token: its bits from `shift` on
  int pieces, piece, whole;                              // entries of a piece, and of a token that is not cut: powers of two
  // workspace
  int* live;                                             // entries that take part
  uint32_t* key; uint32_t* pos;                          // [N + 2 kSumAhead] tokens and their positions, sorted; the last are looked at, and may be anything
  int* cut;                                              // [pieces + 1] where a piece begins
  uint32_t* spare[2];                                    // [N] for buckets that LDS does not hold
  float* part;                                           // [pieces][2][D] sums of what crosses a border: on the left, on the right
};

// What the wave's lanes did to its own part of LDS comes before what they do next.  (LDS takes a wave's accesses in order: no instruction, only
// the compiler's order.)
__device__ inline void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Stable sort of n entries by `bits` of the token, a digit after the other; from and to are LDS or global memory.  Returns where the
// result is.  A wave has a run of entries, and counters of its own (their rows in LDS a bank apart).
typedef uint32_t SortCounters[kSortWaves][kSortBins + 1];
template <class P>
__device__ inline P sort_entries(P from, P to, int n, int bits, SortCounters& at, uint32_t* wave_total) {
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  const int run = (n + kSortThreads - 1) / kSortThreads * 64, first = min(n, w * run), last = min(n, first + run);
  const int digits = (bits + kSortBits - 1) / kSortBits;
  const unsigned long long below = (1ull << lane) - 1;
  static_assert(kSortBins == 64 && kSortBins * kSortWaves == kSortThreads, "a number a thread");
  for (int d = 0, low = 0; d < digits; ++d) {
    const int wide = (bits - low + digits - d - 1) / (digits - d), shift = kPosBits + low;
    const uint32_t mask = (1u << wide) - 1;
    low += wide;
    // the lanes with my digit
    auto match = [&](uint32_t digit, bool mine) {
      unsigned long long same = __ballot(mine);
      for (int b = 0; b < wide; ++b) {
        const unsigned long long set = __ballot(digit >> b & 1);
        same &= digit >> b & 1 ? set : ~set;
      }
      return same;
    };
    at[w][lane] = 0;
    for (int i0 = first; i0 < last; i0 += 64) {
      const bool mine = i0 + lane < last;
      const uint32_t digit = (mine ? from[i0 + lane] : 0) >> shift & mask;
      const unsigned long long same = match(digit, mine);
      wave_order();                                      // (another lane's zero, or its count of the turn before)
      if (mine && !(same & below)) at[w][digit] += __popcll(same);
    }
    __syncthreads();
    // where a wave's entries of a digit begin: those of lower digits, then those of earlier waves
    uint32_t& mine_at = at[t % kSortWaves][t / kSortWaves];
    const uint32_t x = mine_at;
    uint32_t sum = x;
    for (int s = 1; s < 64; s <<= 1) {
      const uint32_t other = __shfl_up(sum, s);
      if (lane >= s) sum += other;
    }
    if (lane == 63) wave_total[w] = sum;
    __syncthreads();
    uint32_t before = lane < w ? wave_total[lane] : 0;
    for (int s = 1; s < kSortWaves; s <<= 1) before += __shfl_xor(before, s);
    mine_at = __shfl(before, 0) + sum - x;
    __syncthreads();
    for (int i0 = first; i0 < last; i0 += 64) {
      const bool mine = i0 + lane < last;
      const uint32_t entry = mine ? from[i0 + lane] : 0, digit = entry >> shift & mask;
      const unsigned long long same = match(digit, mine);
      uint32_t base = 0;
      wave_order();                                      // (the first lane's place of the turn before)
      if (mine) base = at[w][digit];
      wave_order();                                      // (all have read it)
      if (mine && !(same & below)) at[w][digit] = base + __popcll(same);
      if (mine) to[base + __popcll(same & below)] = entry;
    }
    __syncthreads();                                     // (and what was written is read by the workgroup itself)
    const P other = from;
    from = to;
    to = other;
  }
  return from;
}

// Zeros in all rows of grad_weight: 16 bytes a lane (up to 2^31 in all), of `lanes` lanes mine.
__device__ inline void clear_rows(const EmbedGradArgs& a, uint32_t mine, uint32_t lanes) {
  const uint32_t size = a.out_bf16 ? 2 : 4, per_row = a.D * size / 16, end = per_row * (uint32_t)a.V;
  u32x4* out = static_cast<u32x4*>(a.out);
  if (a.out_stride == a.D) {
#pragma unroll 4
    for (uint32_t u = mine; u < end; u += lanes) out[u] = u32x4{0, 0, 0, 0};
  } else {
    const long long pitch = a.out_stride * size / 16;
    for (uint32_t u = mine; u < end; u += lanes) {
      const uint32_t v = u / per_row;
      out[v * pitch + (u - v * per_row)] = u32x4{0, 0, 0, 0};
    }
  }
}

struct __attribute__((packed, aligned(4))) FourIds { uint32_t x[4]; };
struct BucketShared {
  SortCounters at;
  uint32_t wave_total[kSortWaves], wave_before[kSortWaves];
};
// What a workgroup finds of its bucket of the vocabulary: how many entries, how many are in the buckets before.
struct Bucket { uint32_t low, size, n, start; };
// It reads all tokens, lists those of its bucket in order -- put(place, bucket, entry) -- and counts those of the buckets before.
template <class F>
__device__ inline Bucket list_bucket(const EmbedGradArgs& a, int bucket, BucketShared& s, F put) {
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  // A wave's run of ids, four neighbours a lane, kQuads loads under way at once.
  constexpr int kQuads = 4;
  const int run = (a.N + kSortThreads * 4 - 1) / (kSortThreads * 4) * 256, first = __builtin_amdgcn_readfirstlane(w) * run, last = min(a.N, first + run);
  Bucket b;
  b.low = (uint32_t)bucket << a.shift;
  b.size = min((uint32_t)a.V - b.low, 1u << a.shift);
  FourIds id[kQuads];
  auto load = [&](int i0) {
#pragma unroll
    for (int j = 0; j < kQuads; ++j) {
      const int i = i0 + j * 256 + lane * 4;
      id[j] = FourIds{{0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu}};
      if (i + 4 <= last) id[j] = *reinterpret_cast<const FourIds*>(a.ids + i);
      else
        for (int e = 0; e < 3; ++e)
          if (i + e < last) id[j].x[e] = (uint32_t)a.ids[i + e];
    }
  };
  uint32_t n = 0, before = 0;                            // of the wave's ids
  for (int i0 = first; i0 < last; i0 += kQuads * 256) {
    load(i0);
#pragma unroll
    for (int j = 0; j < kQuads; ++j)
      if (i0 + j * 256 < last) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          n += __popcll(__ballot(id[j].x[e] - b.low < b.size));
          before += __popcll(__ballot(id[j].x[e] < b.low));
        }
      }
  }
  if (lane == 0) { s.wave_total[w] = n; s.wave_before[w] = before; }
  __syncthreads();
  uint32_t all = lane < kSortWaves ? s.wave_total[lane] : 0, base = lane < w ? all : 0, start = lane < kSortWaves ? s.wave_before[lane] : 0;
  for (int d = 1; d < kSortWaves; d <<= 1) {
    all += __shfl_xor(all, d);
    base += __shfl_xor(base, d);
    start += __shfl_xor(start, d);
  }
  b.n = __shfl(all, 0);
  b.start = __shfl(start, 0);
  base = __shfl(base, 0);
  const unsigned long long below = (1ull << lane) - 1;
  for (int i0 = first; i0 < last; i0 += kQuads * 256) {
    if (run > kQuads * 256) load(i0);
#pragma unroll
    for (int j = 0; j < kQuads; ++j) {
      if (i0 + j * 256 >= last) continue;
      unsigned long long mine[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) mine[e] = __ballot(id[j].x[e] - b.low < b.size);
      if (mine[0] | mine[1] | mine[2] | mine[3]) {
        uint32_t to = base;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          to += __popcll(mine[e] & below);
          base += __popcll(mine[e]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (mine[e] >> lane & 1) put(to++, b, (id[j].x[e] - b.low) << kPosBits | (uint32_t)(i0 + j * 256 + lane * 4 + e));
      }
    }
  }
  __syncthreads();
  return b;
}
// The n entries in `from`, sorted: there or in `to` (LDS).
typedef SIP_LDS uint32_t* LdsEntries;
__device__ inline LdsEntries sort_bucket(const EmbedGradArgs& a, LdsEntries from, LdsEntries to, int n, BucketShared& s) {
  if (n > kSortPairs) return sort_entries<LdsEntries>(from, to, n, a.shift, s.at, s.wave_total);
  if ((int)threadIdx.x < n) {
    const uint32_t mine = from[threadIdx.x];
    uint32_t rank = 0;
    for (int j = 0; j < n; ++j) rank += from[j] < mine;
    to[rank] = mine;
  }
  __syncthreads();
  return to;
}

// A workgroup a bucket, up to 128 of them, each of which reads all tokens: no counts are exchanged, and none waits for another.  The
// workgroups behind fill grad_weight with zeros meanwhile, unless it is added to.  ROOM: entries of a bucket that LDS holds, twice; larger buckets
// are sorted in the workspace.
// 8192 tokens 7 to 9 us, 65536 22, and 39 where one token is an eighth of them: reading, and the largest bucket.  Beside 1.24 GB of zeros
// that is hidden: 215 us, 5.8 TB/s.
template <int ROOM>
__global__ __launch_bounds__(kSortThreads) void embed_sort_kernel(EmbedGradArgs a) {
  __shared__ uint32_t room[2][ROOM];
  __shared__ BucketShared shared;
  const int t = threadIdx.x;
  if ((int)blockIdx.x >= a.buckets) {
    clear_rows(a, (blockIdx.x - a.buckets) * kSortThreads + t, (gridDim.x - a.buckets) * kSortThreads);
    return;
  }
  const int bucket = blockIdx.x;
  const Bucket b = list_bucket(a, bucket, shared, [&](uint32_t to, const Bucket& b, uint32_t entry) {
    if (b.n <= ROOM) room[0][to] = entry;
    else a.spare[0][b.start + to] = entry;
  });
  const uint32_t n = b.n, start = b.start;
  if (bucket == a.buckets - 1 && t == 0) *a.live = (int)(start + n);
  // what is sorted goes out, and where the pieces' borders among it lie
  auto finish = [&](auto sorted) {
    for (uint32_t i = t; i < n; i += kSortThreads) {
      const uint32_t entry = sorted[i];
      a.key[start + i] = (uint32_t)bucket << a.shift | entry >> kPosBits;
      a.pos[start + i] = entry & ((1u << kPosBits) - 1);
    }
    for (uint32_t border = (start + a.piece - 1) / a.piece * a.piece + t * a.piece; border < start + n; border += kSortThreads * a.piece) {
      const int i = (int)(border - start), token = sorted[i] >> kPosBits;
      auto is = [&](int j) { return j >= 0 && j < (int)n && (int)(sorted[j] >> kPosBits) == token; };
      int cut = i;
      if (is(i - 1) && !is(i - a.whole) && !is(i + a.whole)) {           // (else it has more than that many entries, or begins here)
        int before = 1, behind = 0;                      // as many of its entries are ahead of the border for certain, and behind
        for (int step = a.whole / 2; step; step /= 2) {
          if (is(i - before - step)) before += step;
          if (is(i + behind + step)) behind += step;
        }
        if (before + behind + 1 <= a.whole) cut = i + behind + 1;
      }
      a.cut[border / a.piece] = (int)start + cut;
    }
  };
  if (n <= ROOM) finish(sort_bucket(a, (LdsEntries)&room[0][0], (LdsEntries)&room[1][0], (int)n, shared));
  else finish(sort_entries<uint32_t*>(a.spare[0] + start, a.spare[1] + start, (int)n, a.shift, shared.at, shared.wave_total));
}

__device__ inline void embed_store(const EmbedGradArgs& a, long long at, f32x8 sum, const Eight* old) {
  sum *= a.scale;
  if (old) sum += as_floats(*old, a.out_bf16);
  store_eight(a.out, at, a.out_bf16, sum);
}

// A lane: eight columns of one piece, eight rows under way at once, and where they are added to the rows of grad_weight that end there.
// Bound by memory: 8192 rows of 4096 bf16, a tenth masked, added to 3500 rows of bf16 26 us, 4.5 TB/s; 65536 of 2048 to 53000 rows of fp32 240 us,
// 4.7 TB/s.
constexpr int kSumAhead = 8;
template <bool BF16, bool ADD>
__global__ __launch_bounds__(256) void embed_sum_kernel(EmbedGradArgs a) {
  const uint32_t per_row = a.D / 8, u = blockIdx.x * 256 + threadIdx.x;                     // (up to 2^21)
  const int n = *a.live, piece = (int)(u / per_row), c = (int)(u - piece * per_row) * 8;
  if (piece >= a.pieces) return;
  const int first = a.cut[piece], end = a.cut[piece + 1];               // (from the last entry on: anything)
  if ((long long)piece * a.piece >= n) return;
  const int last = (piece + 1ll) * a.piece < n ? end : n;
  if (first >= last) return;
  f32x8 sum = {0, 0, 0, 0, 0, 0, 0, 0};
  bool begun = first == 0 || a.key[first - 1] != a.key[first];         // the token's first entry is in this piece
  struct __attribute__((packed, aligned(4))) Ahead { uint32_t x[kSumAhead]; };
  Ahead next_key, next_pos;
  uint32_t next_last;
  auto look = [&](int i0) {                              // (what lies behind the last entry may be anything)
    next_key = *reinterpret_cast<const Ahead*>(a.key + i0);
    next_pos = *reinterpret_cast<const Ahead*>(a.pos + i0);
    next_last = a.key[i0 + kSumAhead];
  };
  look(first);
  for (int i0 = first; i0 < last; i0 += kSumAhead) {
    uint32_t key[kSumAhead + 1], pos[kSumAhead];
#pragma unroll
    for (int j = 0; j < kSumAhead; ++j) {
      key[j] = next_key.x[j];
      pos[j] = next_pos.x[j];
    }
    key[kSumAhead] = next_last;
    if (i0 + kSumAhead < last) look(i0 + kSumAhead);
#pragma unroll
    for (int j = 0; j <= kSumAhead; ++j)
      if (i0 + j >= n) key[j] = 0xffffffffu;
    Eight x[kSumAhead], old[kSumAhead];
    bool fresh = begun;
#pragma unroll
    for (int j = 0; j < kSumAhead; ++j) {
      x[j] = Eight{};
      if (i0 + j < last) x[j] = load_eight(a.grad, pos[j] * a.grad_stride + c, BF16);
      if constexpr (ADD) {
        old[j] = Eight{};
        if (i0 + j < last && key[j + 1] != key[j]) {
          if (fresh) old[j] = load_eight(a.out, key[j] * a.out_stride + c, a.out_bf16);
          fresh = true;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < kSumAhead; ++j) {
      if (i0 + j < last) {
        sum += as_floats(x[j], BF16);
        const bool ends = key[j + 1] != key[j];
        if (ends || i0 + j + 1 == last) {
          if (begun && ends) embed_store(a, key[j] * a.out_stride + c, sum, ADD ? &old[j] : nullptr);
          else store_eight(a.part, ((long long)piece * 2 + begun) * a.D + c, false, sum);
          sum = f32x8{0, 0, 0, 0, 0, 0, 0, 0};
          begun = true;
        }
      }
    }
  }
}

// A small gradient in one launch: a workgroup a bucket, which sums its tokens' rows itself and clears the bucket's others.  The sorted
// entries go to groups of waves that cover a row each, a run of entries a group; what crosses the end of a run goes through LDS.
// 384 tokens, 4096 x 512 fp32: 8.5 us instead of the three kernels' 16.
constexpr int kSmallTokens = 1024, kSmallWidth = kSortWaves * 512;
template <bool BF16, bool ADD>
__global__ __launch_bounds__(kSortThreads) void embed_small_kernel(EmbedGradArgs a) {
  __shared__ uint32_t room[2][kSmallTokens];
  __shared__ BucketShared shared;
  __shared__ __align__(16) uint8_t hit[kBucketMost];
  __shared__ f32x8 part[2][kSortThreads];                // of a group's run: what begins before it, what goes on behind it
  const int t = threadIdx.x;
  reinterpret_cast<uint32_t*>(hit)[t] = 0;
  static_assert(kBucketMost == 4 * kSortThreads, "four a thread");
  const Bucket b = list_bucket(a, blockIdx.x, shared, [&](uint32_t to, const Bucket&, uint32_t entry) {
    room[0][to] = entry;
    hit[entry >> kPosBits] = 1;
  });
  if constexpr (!ADD) {
    const uint32_t per_row = a.D * (a.out_bf16 ? 2 : 4) / 16;
    const long long pitch = a.out_stride * (a.out_bf16 ? 2 : 4) / 16;
    u32x4* out = static_cast<u32x4*>(a.out) + b.low * pitch;
    for (uint32_t u = t; u < b.size * per_row; u += kSortThreads) {
      const uint32_t v = u / per_row;
      if (!hit[v]) out[v * pitch + (u - v * per_row)] = u32x4{0, 0, 0, 0};
    }
  }
  const int n = (int)b.n;
  if (n == 0) return;
  const LdsEntries sorted = sort_bucket(a, (LdsEntries)&room[0][0], (LdsEntries)&room[1][0], n, shared);
  const int waves = (a.D + 511) / 512, groups = kSortWaves / waves, group = (t >> 6) / waves, c = (t - group * waves * 64) * 8;
  const int run = (n + groups - 1) / groups, first = group * run, last = min(n, first + run);
  auto token = [&](int i) { return sorted[i] >> kPosBits; };
  const f32x8 none = {0, 0, 0, 0, 0, 0, 0, 0};
  f32x8 sum = none;
  constexpr int kAhead = ADD ? 4 : kSumAhead;            // (128 registers a lane)
  if (c < a.D && first < last) {
    bool begun = first == 0 || token(first - 1) != token(first);
    for (int i0 = first; i0 < last; i0 += kAhead) {
      Eight x[kAhead], old[kAhead];
      bool fresh = begun;
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        x[j] = old[j] = Eight{};
        if (i0 + j >= last) continue;
        x[j] = load_eight(a.grad, (sorted[i0 + j] & ((1u << kPosBits) - 1)) * a.grad_stride + c, BF16);
        if (ADD && (i0 + j + 1 == n || token(i0 + j + 1) != token(i0 + j))) {
          if (fresh) old[j] = load_eight(a.out, (b.low + token(i0 + j)) * a.out_stride + c, a.out_bf16);
          fresh = true;
        }
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        if (i0 + j >= last) continue;
        sum += as_floats(x[j], BF16);
        const bool ends = i0 + j + 1 == n || token(i0 + j + 1) != token(i0 + j);
        if (!ends && i0 + j + 1 < last) continue;
        if (begun && ends) embed_store(a, (b.low + token(i0 + j)) * a.out_stride + c, sum, ADD ? &old[j] : nullptr);
        else part[begun][t] = sum;
        sum = none;
        begun = true;
      }
    }
  }
  __syncthreads();
  // the token that goes on behind the run, if it begins in it
  if (c >= a.D || first >= last || last == n) return;
  const uint32_t v = token(last);
  if (token(last - 1) != v || (first > 0 && token(first - 1) == v)) return;
  sum = part[1][t];
  for (int at = last, there = t + waves * 64; at < n && token(at) == v; at += run, there += waves * 64) sum += part[0][there];
  Eight old = {};
  const long long to = (b.low + v) * a.out_stride + c;
  if (ADD) old = load_eight(a.out, to, a.out_bf16);
  embed_store(a, to, sum, ADD ? &old : nullptr);
}

// The tokens that begin in a piece and go on behind its right border.  A workgroup looks at kJoinPieces of them, kJoinLanes lanes of eight
// columns, of which each has kJoinWorkers workers that take every sixteenth of the token's pieces: one that is a fifth of all tokens has a thousand.
// Latency, 2 to 5 us where there is nothing to join, 8 for the 18 most frequent tokens of 8192, and 23 where 50000 tokens of 568 columns are drawn with
// 1 / rank^1.2 (64 lanes, 1024 threads: 8.5 and 54; 8 lanes: 13 and 26).
constexpr int kJoinPieces = 4, kJoinThreads = 256, kJoinLanes = 16, kJoinWorkers = kJoinThreads / kJoinLanes;
template <bool ADD>
__global__ __launch_bounds__(kJoinThreads) void embed_join_kernel(EmbedGradArgs a) {
  __shared__ f32x8 sums[kJoinThreads / 64][kJoinLanes];
  const int t = threadIdx.x, lane = t & 63, n = *a.live, worker = t / kJoinLanes, c = (blockIdx.y * kJoinLanes + t % kJoinLanes) * 8, piece0 = blockIdx.x * kJoinPieces;
  uint32_t token = 0;                                    // lane j: that of piece0 + j
  bool cut = false;
  if (lane < kJoinPieces && piece0 + lane + 1 < a.pieces) {
    const int border = (piece0 + lane + 1) * a.piece;                    // (within the list: what lies behind the last entry may be anything)
    const int begin = a.cut[piece0 + lane], moved = a.cut[piece0 + lane + 1];
    token = a.key[border];
    const uint32_t behind = a.key[border - 1];
    if (border < n && moved == border && begin < border && behind == token) cut = begin == 0 || a.key[begin - 1] != token;
  }
  for (unsigned long long left = __ballot(cut); left; left &= left - 1) {
    const int j0 = __builtin_ctzll(left), piece = piece0 + j0;
    const uint32_t v = __builtin_amdgcn_readlane(token, j0);
    // Pieces behind this one that begin with the token: 64 at a time by every one, 4096 by every 64th.
    int pieces = 1;
    auto same = [&](int step) {
      const long long at = (long long)(piece + pieces + (lane + 1) * step) * a.piece;
      return __ballot(at < n && a.key[min(at, (long long)n - 1)] == v);
    };
    auto count = [](unsigned long long same) { return ~same ? __builtin_ctzll(~same) : 64; };
    unsigned long long next = same(1), far = same(64);
    if (!~next) {
      while (far) {
        const int more = count(far);
        pieces += more * 64;
        if (more < 64) break;
        far = same(64);
      }
      next = same(1);
    }
    pieces += count(next);
    f32x8 sum = {0, 0, 0, 0, 0, 0, 0, 0};
    Eight old = {};
    if (c < a.D) {
      if (ADD && worker == 0) old = load_eight(a.out, v * a.out_stride + c, a.out_bf16);
#pragma unroll 8
      for (int j = worker; j <= pieces; j += kJoinWorkers)
        sum += as_floats(load_eight(a.part, ((long long)(piece + j) * 2 + (j == 0)) * a.D + c, false), false);
    }
    for (int d = kJoinLanes; d < 64; d <<= 1) {
      f32x8 other;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = sum[e];
        other[e] = __shfl_xor(x, d);
      }
      sum += other;
    }
    __syncthreads();
    if (lane < kJoinLanes) sums[t >> 6][lane] = sum;
    __syncthreads();
    if (t >= kJoinLanes || c >= a.D) continue;
    for (int j = 1; j < kJoinThreads / 64; ++j) sum += sums[j][lane];
    embed_store(a, v * a.out_stride + c, sum, ADD ? &old : nullptr);
  }
}

}  // namespace sip
