// Host side of the entry points of include/sip_head.h on the way from tokens to vectors, and of the adapters: argument checks,
// workspace carving, launches.
#pragma once
#include <algorithm>
#include <type_traits>

#include "../../include/sip_head.h"
#include "sip_adapt.h"
#include "sip_embed.h"
#include "sip_host.h"

namespace {

bool matrix_shape_ok(int32_t V, int32_t D) { return V > 0 && D > 0 && D % 8 == 0 && V <= SIP_MAX_V && D <= SIP_MAX_D; }

sip_status embed_check(int32_t V, int32_t D, const int32_t* ids, int32_t N, const void* out, int64_t out_stride, sip_dtype out_dtype) {
  if (V <= 0 || D <= 0 || D % 8 != 0 || N < 0 || !dtype_ok(out_dtype)) return SIP_ERR_INVALID_ARG;
  if (N > 0 && (!ids || !rows_ok(out, D, out_stride, out_dtype))) return SIP_ERR_INVALID_ARG;
  if (V > SIP_MAX_V || D > SIP_MAX_D || N > SIP_MAX_B || out_stride > (1ll << 32)) return SIP_ERR_UNSUPPORTED;
  return SIP_OK;
}
sip::EmbedArgs embed_args(int32_t V, int32_t D, const int32_t* ids, int32_t N, float scale, void* out, int64_t out_stride,
                          sip_dtype out_dtype) {
  sip::EmbedArgs a{};
  a.V = V; a.D = D; a.N = N; a.ids = ids; a.scale = scale;
  a.out = out; a.out_stride = out_stride; a.out_bf16 = out_dtype == SIP_BF16;
  return a;
}
// Four rows' pieces a lane where that leaves every compute unit eight workgroups: 16000 rows of 4096 bf16 take 40 us so, 49 with one a lane;
// 32 rows from codes 4.4 and 2.8.
template <bool CODES>
void launch_embed(const sip::EmbedArgs& a, hipStream_t stream) {
  const long long units = (long long)a.N * (a.D / 8);
  if (units >= 8 * kChip * 4 * 256) hipLaunchKernelGGL((sip::embed_kernel<CODES, 4>), dim3(tiles(units, 4 * 256)), dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((sip::embed_kernel<CODES, 1>), dim3(tiles(units, 256)), dim3(256), 0, stream, a);
}

// Entries of a piece of the sorted tokens: 8 to 64, as many as leave every SIMD four waves.  65536 tokens drawn with 1 / rank^1.1, 2048 columns, 140 us of
// sums and 9 of joining with pieces of 64, 130 and 48 with 8; evenly drawn ones, added to fp32, 240 + 5 and 232 + 12.
constexpr int kPieceLeast = sip::kSumAhead, kPieceMost = 64;
constexpr long long kEmbedLanes = kChip * 4 * 64 * 4;
int embed_piece(int32_t N, int32_t D) {
  int piece = kPieceLeast;
  while (piece < kPieceMost && (long long)N * (D / 8) >= 2 * piece * kEmbedLanes) piece *= 2;
  return piece;
}
// The most pieces of N tokens or fewer.
int embed_pieces_most(int32_t N, int32_t D) {
  int most = tiles(N, embed_piece(N, D));
  for (int piece = kPieceLeast; piece < embed_piece(N, D); piece *= 2)
    most = std::max(most, tiles((2 * piece * kEmbedLanes - 1) / (D / 8), piece));
  return most;
}
// Buckets of the vocabulary: up to 128, each a power of two wide.
int embed_shift(int32_t V) {
  int shift = 0;
  while (tiles(V, 1 << shift) > 128) ++shift;
  return shift;
}
static_assert(SIP_MAX_TOKENS <= 1 << sip::kPosBits && SIP_MAX_V <= 128 * sip::kBucketMost && sip::kBucketMost <= 1 << (32 - sip::kPosBits),
              "an entry is 32 bits");
// One launch instead of three where that is shorter, and the buckets' workgroups clear the matrix in it too.  Kernels in us, one launch and three:
// 1024 random tokens of 512 7.3 and 13.3, all of them the same -- which one compute unit reads -- 33 and 15 (8192 of 64: 159 and 30).
bool embed_is_small(int32_t N, int32_t V, int32_t D, sip_dtype dtype, bool accumulate) {
  return N <= sip::kSmallTokens && D <= sip::kSmallWidth && (long long)N * D <= 512 << 10 &&
         (accumulate || (long long)V * D * dtype_bytes(dtype) <= 32ll << 20);
}
struct EmbedPlan { int piece, pieces; size_t live, key, pos, cut, spare[2], part, bytes; };
EmbedPlan embed_plan(int32_t N, int32_t D) {             // (room for N tokens or fewer)
  EmbedPlan p{};
  size_t at = 0;
  auto take = [&](size_t n) { const size_t here = at; at += head_align(n); return here; };
  p.live = take(4);
  p.key = take(((size_t)N + 2 * sip::kSumAhead) * 4);
  p.pos = take(((size_t)N + 2 * sip::kSumAhead) * 4);
  p.cut = take((size_t)N / kPieceLeast * 4 + 8);
  for (size_t& s : p.spare) s = take((size_t)N * 4);
  p.piece = embed_piece(N, D);
  p.pieces = tiles(N, p.piece);
  p.part = take((size_t)embed_pieces_most(N, D) * 2 * D * 4);
  p.bytes = at;
  return p;
}

// Batches of B rows at most: one for every adapter that a row has, and one more for every sixteen rows.
int adapt_batches(int32_t B, int32_t adapters) { return std::min(B, adapters + B / sip::kAdaptRows); }
// Into how many parts the sum over D is dealt out: as many as compute units are free, of 512 entries or more.  (An adapter of rank 16, D = 4096,
// 4.4 us in four parts, 6.9 in one.)
int adapt_parts(int batches, int32_t rank, int32_t D) {
  return std::max(1, std::min({sip::kDownParts, D / 512, kChip / (batches * tiles(rank, 16))}));
}
struct AdaptPlan { size_t count, rows, batch, t, bytes; };
AdaptPlan adapt_plan(int32_t B, int32_t adapters, int32_t rank) {
  AdaptPlan p{};
  size_t at = 0;
  auto take = [&](size_t n) { const size_t here = at; at += head_align(n); return here; };
  p.count = take(4);
  p.rows = take((size_t)B * 4);
  p.batch = take((size_t)B * 16);
  p.t = take((size_t)std::max(adapt_batches(B, adapters), kChip) * sip::kAdaptRows * rank * 4);           // (batches of all parts)
  p.bytes = at;
  return p;
}
bool adapt_shape_ok(int32_t B, int32_t adapters, int32_t rank, int32_t D) {
  return B > 0 && adapters > 0 && rank > 0 && rank % 8 == 0 && D > 0 && D % 8 == 0 && B <= SIP_MAX_TOKENS && adapters <= SIP_MAX_ADAPTERS &&
         rank <= SIP_MAX_RANK && D <= SIP_MAX_D;
}

}  // namespace

extern "C" {

sip_status sip_embed(const void* weight, sip_dtype weight_dtype, int32_t V, int32_t D, int64_t weight_stride, const int32_t* ids,
                     int32_t N, float scale, void* out, int64_t out_stride, sip_dtype out_dtype, void* hip_stream) {
  if (!dtype_ok(weight_dtype) || !rows_ok(weight, D, weight_stride, weight_dtype)) return SIP_ERR_INVALID_ARG;
  const sip_status ok = embed_check(V, D, ids, N, out, out_stride, out_dtype);
  if (ok != SIP_OK) return ok;
  if (weight_stride > (1ll << 32)) return SIP_ERR_UNSUPPORTED;
  if (N == 0) return SIP_OK;
  sip::EmbedArgs a = embed_args(V, D, ids, N, scale, out, out_stride, out_dtype);
  a.weight = weight; a.weight_stride = weight_stride; a.weight_bf16 = weight_dtype == SIP_BF16;
  launch_embed<false>(a, static_cast<hipStream_t>(hip_stream));
  return launched();
}

sip_status sip_embed_codes(const uint8_t* codes, int64_t codes_stride, const void* scales, sip_dtype scales_dtype,
                           const uint8_t* zeros, int32_t group, int32_t V, int32_t D, const int32_t* ids, int32_t N, float scale,
                           void* out, int64_t out_stride, sip_dtype out_dtype, void* hip_stream) {
  if (!codes || !scales || !dtype_ok(scales_dtype) || V <= 0 || D <= 0) return SIP_ERR_INVALID_ARG;
  if (group != 32 && group != 64 && group != 128) return group > 0 ? SIP_ERR_UNSUPPORTED : SIP_ERR_INVALID_ARG;
  if (D % group != 0 || codes_stride < D / 2 || codes_stride % 16 != 0 || !aligned16(codes)) return SIP_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(scales) % dtype_bytes(scales_dtype) != 0) return SIP_ERR_INVALID_ARG;
  const sip_status ok = embed_check(V, D, ids, N, out, out_stride, out_dtype);
  if (ok != SIP_OK) return ok;
  if (codes_stride > (1ll << 32)) return SIP_ERR_UNSUPPORTED;
  if (N == 0) return SIP_OK;
  sip::EmbedArgs a = embed_args(V, D, ids, N, scale, out, out_stride, out_dtype);
  a.codes = codes; a.codes_stride = codes_stride; a.scales = scales; a.scales_bf16 = scales_dtype == SIP_BF16;
  a.zeros = zeros; a.group_shift = group == 32 ? 5 : group == 64 ? 6 : 7;
  launch_embed<true>(a, static_cast<hipStream_t>(hip_stream));
  return launched();
}

size_t sip_embed_workspace_bytes(int32_t N, int32_t V, int32_t D) {
  if (!matrix_shape_ok(V, D) || N < 0 || N > SIP_MAX_TOKENS) return 0;
  return embed_plan(std::max(N, 1), D).bytes;
}

sip_status sip_embed_backward(const void* grad_out, int64_t grad_out_stride, sip_dtype grad_out_dtype, const int32_t* ids, int32_t N,
                              int32_t V, int32_t D, float scale, int32_t accumulate, void* grad_weight,
                              int64_t grad_weight_stride, sip_dtype grad_weight_dtype, void* workspace, size_t workspace_bytes,
                              void* hip_stream) {
  if (V <= 0 || D <= 0 || D % 8 != 0 || N < 0 || !dtype_ok(grad_out_dtype) || !dtype_ok(grad_weight_dtype)) return SIP_ERR_INVALID_ARG;
  if (N > 0 && (!ids || !rows_ok(grad_out, D, grad_out_stride, grad_out_dtype))) return SIP_ERR_INVALID_ARG;
  if (!rows_ok(grad_weight, D, grad_weight_stride, grad_weight_dtype)) return SIP_ERR_INVALID_ARG;
  if (!matrix_shape_ok(V, D) || N > SIP_MAX_TOKENS || grad_out_stride > (1ll << 32) || grad_weight_stride > (1ll << 32))
    return SIP_ERR_UNSUPPORTED;
  if (!workspace_ok(workspace, workspace_bytes, sip_embed_workspace_bytes(N, V, D))) return SIP_ERR_WORKSPACE;
  if (N == 0 && accumulate) return SIP_OK;
  const EmbedPlan pl = embed_plan(std::max(N, 1), D);
  char* ws = static_cast<char*>(workspace);
  sip::EmbedGradArgs a{};
  a.grad = grad_out; a.grad_stride = grad_out_stride;
  a.ids = ids; a.N = N; a.V = V; a.D = D; a.scale = scale;
  a.out = grad_weight; a.out_stride = grad_weight_stride; a.out_bf16 = grad_weight_dtype == SIP_BF16;
  a.shift = embed_shift(V);
  a.buckets = N > 0 ? tiles(V, 1 << a.shift) : 0;
  a.pieces = pl.pieces;
  a.piece = pl.piece;
  a.whole = 2 * pl.piece;
  a.live = reinterpret_cast<int*>(ws + pl.live);
  a.key = reinterpret_cast<uint32_t*>(ws + pl.key);
  a.pos = reinterpret_cast<uint32_t*>(ws + pl.pos);
  a.cut = reinterpret_cast<int*>(ws + pl.cut);
  for (int i = 0; i < 2; ++i) a.spare[i] = reinterpret_cast<uint32_t*>(ws + pl.spare[i]);
  a.part = reinterpret_cast<float*>(ws + pl.part);
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if (N > 0 && embed_is_small(N, V, D, grad_weight_dtype, accumulate)) {
    auto launch = [&](auto in_add) {
      constexpr bool kAdd = decltype(in_add)::value;
      if (grad_out_dtype == SIP_BF16) hipLaunchKernelGGL((sip::embed_small_kernel<true, kAdd>), dim3(a.buckets), dim3(sip::kSortThreads), 0, stream, a);
      else hipLaunchKernelGGL((sip::embed_small_kernel<false, kAdd>), dim3(a.buckets), dim3(sip::kSortThreads), 0, stream, a);
    };
    if (accumulate) launch(std::true_type{});
    else launch(std::false_type{});
    return launched();
  }
  const long long lines = (long long)V * D * dtype_bytes(grad_weight_dtype) / 16;
  const dim3 sort_grid(a.buckets + (accumulate ? 0 : std::min(tiles(lines, sip::kSortThreads * 4), 16 * kChip)));
  if (N <= 8192) hipLaunchKernelGGL(sip::embed_sort_kernel<8192>, sort_grid, dim3(sip::kSortThreads), 0, stream, a);
  else hipLaunchKernelGGL(sip::embed_sort_kernel<16384>, sort_grid, dim3(sip::kSortThreads), 0, stream, a);
  if (N > 0) {
    const dim3 sum_grid(tiles((long long)pl.pieces * (D / 8), 256)), join_grid(tiles(pl.pieces, sip::kJoinPieces), tiles(D, sip::kJoinLanes * 8));
    auto launch = [&](auto in_add) {
      constexpr bool kAdd = decltype(in_add)::value;
      if (grad_out_dtype == SIP_BF16) hipLaunchKernelGGL((sip::embed_sum_kernel<true, kAdd>), sum_grid, dim3(256), 0, stream, a);
      else hipLaunchKernelGGL((sip::embed_sum_kernel<false, kAdd>), sum_grid, dim3(256), 0, stream, a);
      hipLaunchKernelGGL(sip::embed_join_kernel<kAdd>, join_grid, dim3(sip::kJoinThreads), 0, stream, a);
    };
    if (accumulate) launch(std::true_type{});
    else launch(std::false_type{});
  }
  return launched();
}

size_t sip_head_adapt_workspace_bytes(int32_t B, int32_t adapters, int32_t rank, int32_t D) {
  return adapt_shape_ok(B, adapters, rank, D) ? adapt_plan(B, adapters, rank).bytes : 0;
}

sip_status sip_head_adapt(const void* hidden, int32_t B, int32_t D, int64_t hidden_stride, sip_dtype hidden_dtype,
                          const void* down, const void* up, int32_t adapters, int32_t rank, const int32_t* adapter_of_row,
                          const float* scales, int32_t V, void* logits, int64_t logits_stride, sip_dtype logits_dtype,
                          void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (B <= 0 || D <= 0 || D % 8 != 0 || V <= 0 || adapters <= 0 || rank <= 0 || rank % 8 != 0 || !dtype_ok(hidden_dtype) ||
      !dtype_ok(logits_dtype))
    return SIP_ERR_INVALID_ARG;
  if (!rows_ok(hidden, D, hidden_stride, hidden_dtype) || !down || !up || !aligned16(down) || !aligned16(up) || !adapter_of_row)
    return SIP_ERR_INVALID_ARG;
  if (!logits || logits_stride < V || reinterpret_cast<uintptr_t>(logits) % dtype_bytes(logits_dtype) != 0) return SIP_ERR_INVALID_ARG;
  if (!adapt_shape_ok(B, adapters, rank, D) || V > SIP_MAX_V || hidden_stride > (1ll << 32) || logits_stride > (1ll << 32))
    return SIP_ERR_UNSUPPORTED;
  const AdaptPlan pl = adapt_plan(B, adapters, rank);
  if (!workspace_ok(workspace, workspace_bytes, pl.bytes)) return SIP_ERR_WORKSPACE;
  char* ws = static_cast<char*>(workspace);
  sip::AdaptArgs a{};
  a.hidden = hidden; a.hidden_stride = hidden_stride;
  a.B = B; a.D = D; a.V = V; a.rank = rank; a.adapters = adapters;
  a.down = static_cast<const uint16_t*>(down); a.up = static_cast<const uint16_t*>(up);
  a.adapter_of_row = adapter_of_row; a.scales = scales;
  a.logits = logits; a.logits_stride = logits_stride;
  a.count = reinterpret_cast<int*>(ws + pl.count);
  a.rows = reinterpret_cast<int*>(ws + pl.rows);
  a.batch = reinterpret_cast<int4*>(ws + pl.batch);
  a.t = reinterpret_cast<float*>(ws + pl.t);
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const bool direct = B <= sip::kAdaptDirect;
  const int batches = adapt_batches(B, adapters), steps = tiles(rank, 32);
  if (!direct) hipLaunchKernelGGL(sip::adapt_rows_kernel, dim3(1), dim3(1024), 0, stream, a);
  // Tiles of a workgroup: fewer where that leaves the chip half empty.  (The second product for 59 rows of 57 adapters of rank 8, V = 125990, 47.8 us with 16,
  // 56.0 with 8; for 224 rows of 32 of rank 64, V = 128256, 167 and 161.)
  int each = steps == 1 ? 16 : 8;
  while (each > 1 && (long long)tiles(V, sip::kUpEntries * each) * batches < 8 * kChip) each /= 2;
  a.parts = each == 1 ? adapt_parts(batches, rank, D) : 1;
  a.batches = batches;
  const dim3 down_grid(batches, tiles(rank, 16), a.parts), up_grid(tiles(tiles(V, sip::kUpEntries * each), 8) * 8 * batches);
  auto launch = [&](auto in_direct) {
    constexpr bool kDirect = decltype(in_direct)::value;
    if (hidden_dtype == SIP_BF16) hipLaunchKernelGGL((sip::adapt_down_kernel<true, kDirect>), down_grid, dim3(sip::kDownWaves * 64), 0, stream, a);
    else hipLaunchKernelGGL((sip::adapt_down_kernel<false, kDirect>), down_grid, dim3(sip::kDownWaves * 64), 0, stream, a);
    auto add = [&](auto in_steps, auto in_bf16) {
      constexpr int kSteps = decltype(in_steps)::value;
      constexpr bool kBf16 = decltype(in_bf16)::value;
      if (each == 1) hipLaunchKernelGGL((sip::adapt_up_kernel<kSteps, true, kDirect, kBf16>), up_grid, dim3(sip::kUpWaves * 64), 0, stream, a, batches, each);
      else hipLaunchKernelGGL((sip::adapt_up_kernel<kSteps, false, kDirect, kBf16>), up_grid, dim3(sip::kUpWaves * 64), 0, stream, a, batches, each);
    };
    auto add_steps = [&](auto in_bf16) {
      if (steps == 1) add(std::integral_constant<int, 1>{}, in_bf16);
      else if (steps == 2) add(std::integral_constant<int, 2>{}, in_bf16);
      else if (steps == 3) add(std::integral_constant<int, 3>{}, in_bf16);
      else add(std::integral_constant<int, 4>{}, in_bf16);
    };
    if (logits_dtype == SIP_BF16) add_steps(std::true_type{});
    else add_steps(std::false_type{});
  };
  if (direct) launch(std::true_type{});
  else launch(std::false_type{});
  return launched();
}

}  // extern "C"
