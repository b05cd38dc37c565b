// Beam search: the best continuations of groups of beams, and the reordering of a sampler state's histories.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sip_state.h"

namespace sip {

// ---------------------------------------------------------------- selection
// beam_chunk_kernel: a workgroup reads one chunk of a row once and leaves its maximum, its sum of exponentials and its n best
// logits, in order.  beam_merge_kernel: a workgroup joins the lists of a group's rows.

constexpr int kBeamThreads = 256;
constexpr int kBeamEach = 32;                            // logits of a lane, in registers
constexpr int kBeamChunk = kBeamThreads * kBeamEach;
constexpr int kBeamList = 512;                           // entries that a chunk's list may have before it is ranked
constexpr int kMergeThreads = 1024;

struct BeamPart { double sum; float max; float pad; };   // of a chunk: sum of 2^(c (z - max))

struct BeamArgs {
  const void* logits; long long row_stride;
  int groups, width, V, n;
  int chunks;                                            // of a row
  float c_hi, c_lo;                                      // logit_scale * log2(e) = c_hi + c_lo, c_lo > 0
  double scale;                                          // logit_scale
  const float* scores; const uint8_t* finished; const float* rank_scale;
  int end_token;
  int* tokens; int* parents; float* out_scores;
  BeamPart* part;                                        // [rows][chunks]
  unsigned long long* cand;                              // [rows][chunks][n] keys in descending order, 0 = none
};

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

// What a row has: continuations from its logits, one at no cost, or none.
enum BeamRow { kBeamNone, kBeamLive, kBeamFinished };
__device__ inline BeamRow beam_row(const BeamArgs& a, int row) {
  if (!isfinite(a.scores[row])) return kBeamNone;
  if (a.rank_scale && !(a.rank_scale[row] > 0.0f && isfinite(a.rank_scale[row]))) return kBeamNone;
  return a.finished && a.finished[row] ? kBeamFinished : kBeamLive;
}

template <bool BF16>
__global__ __launch_bounds__(kBeamThreads) void beam_chunk_kernel(BeamArgs a) {
  constexpr int kGroup = BF16 ? 8 : 4, kLoads = kBeamEach / kGroup;      // logits of a 16-byte load; loads of a lane
  __shared__ __align__(16) uint32_t lane_max[kBeamThreads];
  __shared__ __align__(16) unsigned long long list[kBeamList];
  __shared__ double wave_sum[kBeamThreads / 64];
  __shared__ float wave_max[kBeamThreads / 64], least;
  __shared__ int count;
  const int row = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  if (beam_row(a, row) != kBeamLive) return;
  // logit j of load i is token first + i * 256 * kGroup + j
  const int first = chunk * kBeamChunk + t * kGroup;
  auto token = [&](int e) { return first + e / kGroup * (kBeamThreads * kGroup) + e % kGroup; };
  const char* z0 = static_cast<const char*>(a.logits) + ((long long)row * a.row_stride + first) * (BF16 ? 2 : 4);
  float z[kBeamEach];
  uint4 raw[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i)
    if (token(i * kGroup + kGroup - 1) < a.V) raw[i] = *reinterpret_cast<const uint4*>(z0 + i * kBeamThreads * 16);
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const uint32_t u[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
    for (int j = 0; j < kGroup; ++j) {
      const int e = i * kGroup + j;
      const uint32_t bits = BF16 ? (j & 1 ? u[j / 2] & 0xffff0000u : u[j / 2] << 16) : u[j];
      z[e] = token(i * kGroup + kGroup - 1) < a.V ? __builtin_bit_cast(float, bits) : -INFINITY;
    }
    if (token(i * kGroup) < a.V && token(i * kGroup + kGroup - 1) >= a.V) {              // the row's last group, in part
#pragma unroll
      for (int j = 0; j < kGroup; ++j) {
        const char* at = z0 + i * kBeamThreads * 16 + j * (BF16 ? 2 : 4);
        if (token(i * kGroup + j) < a.V)
          z[i * kGroup + j] = BF16 ? __builtin_bit_cast(float, (uint32_t)*reinterpret_cast<const uint16_t*>(at) << 16)
                                   : *reinterpret_cast<const float*>(at);
      }
    }
  }
  float m = z[0];
#pragma unroll
  for (int e = 1; e < kBeamEach; ++e) m = fmaxf(m, z[e]);
  lane_max[t] = ordered(fmaxf(m, -INFINITY));            // (a lane of NaNs alone)
  for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
  if (lane == 0) wave_max[w] = fmaxf(m, -INFINITY);
  if (t == 0) count = 0;
  __syncthreads();
  // The n-th largest of the lanes' maxima is at most the n-th largest logit: by its leading bits, from wave 0 alone.
  if (w == 0) {
    const uint4 k = reinterpret_cast<const uint4*>(lane_max)[lane];
    uint32_t at = 0;
    for (int bit = 31; bit >= 12; --bit) {
      const uint32_t up = at | 1u << bit;
      const int n = __popcll(__ballot(k.x >= up)) + __popcll(__ballot(k.y >= up)) + __popcll(__ballot(k.z >= up)) +
                    __popcll(__ballot(k.w >= up));
      if (n >= a.n) at = up;
    }
    if (lane == 0) least = at < 0x00800000u ? -3.402823466e38f : unordered(at);          // (-inf is no continuation)
  }
  m = fmaxf(fmaxf(wave_max[0], wave_max[1]), fmaxf(wave_max[2], wave_max[3]));
  const float base = m == -INFINITY ? 0.0f : m;
  float s[2] = {0.0f, 0.0f};
#pragma unroll
  for (int e = 0; e < kBeamEach; ++e) {
    const float d = z[e] - base;
    s[e & 1] += __builtin_amdgcn_exp2f(__builtin_fmaf(d, a.c_lo, d * a.c_hi));
  }
  double sum = (double)s[0] + (double)s[1];
  for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
  if (lane == 0) wave_sum[w] = sum;
  __syncthreads();
  if (t == 0) {
    BeamPart p;
    p.sum = (wave_sum[0] + wave_sum[1]) + (wave_sum[2] + wave_sum[3]);
    p.max = m;
    p.pad = 0.0f;
    a.part[blockIdx.x] = p;
  }
  const float from = least;
#pragma unroll
  for (int e = 0; e < kBeamEach; ++e) {
    if (z[e] >= from) {
      const int at = atomicAdd(&count, 1);
      if (at < kBeamList) list[at] = beam_key(z[e], token(e));
    }
  }
  __syncthreads();
  int listed = count;
  if (listed > kBeamList) {
    // Thousands of nearly equal logits: the n-th largest key, bit by bit, over all of them.
    unsigned long long at = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const unsigned long long up = at | 1ull << bit;
      int n = 0;
#pragma unroll
      for (int e = 0; e < kBeamEach; ++e) n += z[e] >= from && beam_key(z[e], token(e)) >= up;
      for (int d = 32; d; d >>= 1) n += __shfl_xor(n, d);
      __syncthreads();
      if (lane == 0) lane_max[w] = n;
      __syncthreads();
      if ((int)(lane_max[0] + lane_max[1] + lane_max[2] + lane_max[3]) >= a.n) at = up;
    }
    __syncthreads();
    if (t == 0) count = 0;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kBeamEach; ++e)
      if (z[e] >= from && beam_key(z[e], token(e)) >= at) list[atomicAdd(&count, 1)] = beam_key(z[e], token(e));
    __syncthreads();
    listed = count;
  }
  unsigned long long* out = a.cand + (long long)blockIdx.x * a.n;
  for (int i = t; i < listed; i += kBeamThreads) {
    const unsigned long long mine = list[i];
    int rank = 0;
    for (int j = 0; j < listed; ++j) rank += list[j] > mine;
    if (rank < a.n) out[rank] = mine;
  }
  for (int i = listed + t; i < a.n; i += kBeamThreads) out[i] = 0;
}

// A continuation among those of its group: the larger pair comes first.
struct BeamRank { unsigned long long total, rest; };
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

// Room for LISTS heads, and for what the selected lists hold at most: of the list with the r-th best head entries r + e < n.
constexpr int merge_room(int lists, int n) { return lists > n * (n + 1) / 2 ? lists : n * (n + 1) / 2; }

// One workgroup a group.  The lists are in order, so the n-th best of their heads bounds what can be selected, and a list whose
// head is the r-th best can give its n - r first entries at most.
template <int ROOM>
__global__ __launch_bounds__(kMergeThreads) void beam_merge_kernel(BeamArgs a) {
  __shared__ BeamRank found[ROOM];
  __shared__ double lse[SIP_MAX_BEAMS];
  __shared__ float score[SIP_MAX_BEAMS], scale[SIP_MAX_BEAMS];
  __shared__ int what[SIP_MAX_BEAMS], chosen[SIP_MAX_CONTINUATIONS], wave_n[2][kMergeThreads / 64], count, lists_chosen;
  const int g = blockIdx.x, t = threadIdx.x, lane = t & 63, w = t >> 6, K = a.width, S = a.chunks, n = a.n;
  const int lists = K * S, row0 = g * K;
  if (t < K) {
    what[t] = beam_row(a, row0 + t);
    score[t] = a.scores[row0 + t];
    scale[t] = a.rank_scale ? a.rank_scale[row0 + t] : 1.0f;
  }
  if (t == 0) count = lists_chosen = 0;
  __syncthreads();
  for (int k = w; k < K; k += kMergeThreads / 64) {
    if (what[k] != kBeamLive) continue;
    const BeamPart* part = a.part + (long long)(row0 + k) * S;
    float m = -INFINITY;
    double s = 0.0;
    if (lane < S) { m = part[lane].max; s = part[lane].sum; }
    float top = m;
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    if (m > -INFINITY) s *= exp2(((double)m - (double)top) * ((double)a.c_hi + (double)a.c_lo));
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    if (lane == 0) {
      lse[k] = (double)top * a.scale + log(s);
      if (!isfinite(s) || !(s > 0.0) || !isfinite(top)) what[k] = kBeamNone;     // NaN or +inf somewhere, or nothing but -inf
    }
  }
  __syncthreads();
  // Entry e of list l (of beam l / S); total = 0: there is none.
  auto total_of = [&](int k, float z) { return (double)score[k] + ((double)z * a.scale - lse[k]); };
  auto entry = [&](int l, int e) {
    const int k = l / S;
    BeamRank r = {0, 0};
    if (what[k] == kBeamLive) {
      const unsigned long long key = a.cand[((long long)row0 * S + l) * n + e];
      if (key) r = {ordered64(total_of(k, key_logit(key)) * (double)scale[k]), beam_rest(k, key)};
    } else if (what[k] == kBeamFinished && l == k * S && e == 0) {
      r = {ordered64((double)score[k] * (double)scale[k]), beam_rest(k, beam_key(0.0f, a.end_token))};
    }
    return r;
  };
  constexpr int kHeads = SIP_MAX_BEAMS * 64 / kMergeThreads;
  uint32_t head[kHeads];
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    const int l = t + i * kMergeThreads;
    head[i] = l < lists ? (uint32_t)(entry(l, 0).total >> 32) : 0;
  }
  uint32_t from = 0;                                     // the leading bits of the n-th best head
  for (int bit = 31, side = 0; bit >= 8; --bit, side ^= 1) {
    const uint32_t up = from | 1u << bit;
    int mine = 0;
#pragma unroll
    for (int i = 0; i < kHeads; ++i) mine += __popcll(__ballot(head[i] >= up));
    if (lane == 0) wave_n[side][w] = mine;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int j = 0; j < kMergeThreads / 64; ++j) all += wave_n[side][j];
    if (all >= n) from = up;
    if (all == n) break;
  }
  if (from == 0) from = 1;                               // (fewer than n lists: every one that has an entry)
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    const int l = t + i * kMergeThreads;
    if (head[i] >= from) found[atomicAdd(&count, 1)] = {entry(l, 0).total, entry(l, 0).rest};
  }
  __syncthreads();
  const int heads = count;
  // their order, and their lists' numbers by it
  for (int i = t; i < heads; i += kMergeThreads) {
    const BeamRank mine = found[i];
    int rank = 0;
    for (int j = 0; j < heads; ++j) rank += found[j] > mine;
    if (rank < n) {
      const int k = rest_beam(mine.rest);
      chosen[rank] = k * S + (what[k] == kBeamFinished ? 0 : rest_token(mine.rest) / kBeamChunk);
      atomicAdd(&lists_chosen, 1);
    }
  }
  __syncthreads();
  if (t == 0) count = 0;
  __syncthreads();
  const int pairs = lists_chosen * n;
  for (int i = t; i < pairs; i += kMergeThreads) {
    const int r = i / n, e = i % n;
    if (r + e >= n) continue;
    const BeamRank x = entry(chosen[r], e);
    if (x.total >> 32 >= from) found[atomicAdd(&count, 1)] = x;
  }
  __syncthreads();
  const int kept = count;
  for (int i = t; i < kept; i += kMergeThreads) {
    const BeamRank mine = found[i];
    int rank = 0;
    for (int j = 0; j < kept; ++j) rank += found[j] > mine;
    if (rank >= n) continue;
    const int k = rest_beam(mine.rest), at = g * n + rank;
    a.tokens[at] = rest_token(mine.rest);
    a.parents[at] = k;
    a.out_scores[at] = what[k] == kBeamFinished ? score[k] : (float)total_of(k, rest_logit(mine.rest));
  }
  for (int i = kept + t; i < n; i += kMergeThreads) {
    a.tokens[g * n + i] = a.parents[g * n + i] = -1;
    a.out_scores[g * n + i] = -INFINITY;
  }
}

// ---------------------------------------------------------------- reordering of a state

struct ReorderArgs {
  StateHeader* head;
  int* len; int* ndist; int* tokens; uint32_t* table;
  int slots, L_max, groups, width;
  const int* slot_of_row; const int* parents; const int* new_tokens;
  int token_blocks;                                      // of 4 KB of a slot's token row; the table has eight more
};

// Where row k of a group takes its history from: its own slot and its parent's (-1: an empty history).  to < 0: nothing moves.
struct Move { int from, to; };
__device__ inline Move move_of(const ReorderArgs& a, int row0, int k) {
  const int p = a.parents[row0 + k], to = a.slot_of_row[row0 + k];
  if ((unsigned)p >= (unsigned)a.width || (unsigned)to >= (unsigned)a.slots) return {-1, -1};
  for (int j = 0; j < k; ++j)
    if (a.slot_of_row[row0 + j] == to) return {-1, -1};  // an earlier row's
  const int from = a.slot_of_row[row0 + p];
  return {(unsigned)from < (unsigned)a.slots ? from : -1, to};
}
__device__ inline int length_of(const ReorderArgs& a, int slot) {
  return slot < 0 ? 0 : min(max(a.len[slot], 0), a.L_max);
}

// Sixteen bytes that are aligned to four.
struct __attribute__((packed, aligned(4))) StateLine { uint32_t w[4]; };

constexpr int kReorderThreads = 256;

// A lane takes the same 16 bytes of every slot of a group: it reads them all before it writes any, and nobody else touches
// them, so that the slots change places without room beside them.
template <int WIDTH>
__global__ __launch_bounds__(kReorderThreads) void state_reorder_kernel(ReorderArgs a) {
  __shared__ Move move[WIDTH];
  __shared__ int keep[WIDTH];                            // tokens that move; a valid table
  const int blocks = a.token_blocks + 8, g = blockIdx.x / blocks, block = blockIdx.x % blocks, t = threadIdx.x;
  const bool table = block >= a.token_blocks;
  if (t < a.width) {
    Move m = move_of(a, g * a.width, t);
    if (m.from == m.to) m.to = -1;
    move[t] = m;
    keep[t] = table ? (m.from < 0 || a.ndist[m.from] >= 0) : length_of(a, m.from);
  }
  __syncthreads();
  StateLine x[WIDTH];
  const int column = ((table ? block - a.token_blocks : block) * kReorderThreads + t) * 4;
#pragma unroll
  for (int k = 0; k < WIDTH; ++k) {
    if (k >= a.width || move[k].to < 0) continue;
    const long long from = move[k].from;
    if (!table) {
      if (column < keep[k]) x[k] = *reinterpret_cast<const StateLine*>(a.tokens + from * a.L_max + column);
    } else if (keep[k]) {
      if (from >= 0) x[k] = *reinterpret_cast<const StateLine*>(a.table + from * (2 * kTableSlots) + column);
      else
        for (int j = 0; j < 4; ++j) x[k].w[j] = column < kTableSlots ? kTableEmpty : 0u;
    }
  }
#pragma unroll
  for (int k = 0; k < WIDTH; ++k) {
    if (k >= a.width || move[k].to < 0) continue;
    const long long to = move[k].to;
    if (!table) {
      int* out = a.tokens + to * a.L_max + column;
      if (column + 4 <= keep[k]) *reinterpret_cast<StateLine*>(out) = x[k];
      else
        for (int j = 0; j < 4; ++j)
          if (column + j < keep[k]) out[j] = (int)x[k].w[j];
    } else if (keep[k]) {
      *reinterpret_cast<StateLine*>(a.table + to * (2 * kTableSlots) + column) = x[k];
    }
  }
}

// One wave a group, behind the copies: lengths and numbers of distinct tokens, all read before any is written, and the new tokens.
__global__ __launch_bounds__(64) void state_reorder_append_kernel(ReorderArgs a) {
  const int row0 = blockIdx.x * a.width, k = threadIdx.x;
  Move m = {-1, -1};
  int n = 0, nd = 0, token = -1;
  if (k < a.width) {
    m = move_of(a, row0, k);
    n = length_of(a, m.from);
    if (m.from >= 0) nd = a.ndist[m.from];
    if (a.new_tokens) token = a.new_tokens[row0 + k];
  }
  __syncthreads();
  if (m.to < 0) return;
  if (token >= 0) {
    if (n < a.L_max) {
      a.tokens[(long long)m.to * a.L_max + n] = token;
      ++n;
      if (nd >= 0) {
        uint32_t* key = a.table + (long long)m.to * (2 * kTableSlots);
        const int r = table_insert_single(key, key + kTableSlots, (uint32_t)token);
        nd = r < 0 ? -1 : nd + r;
        if (nd > kTableMaxDistinct) nd = -1;
      }
    } else {
      atomicAdd(&a.head->overflow, 1u);
    }
  }
  a.len[m.to] = n;
  a.ndist[m.to] = nd;
}

}  // namespace sip
