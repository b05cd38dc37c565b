// Host side of the entry points declared in include/sip_head.h: argument checks, workspace carving, launches.
#pragma once
#include <algorithm>
#include <initializer_list>

#include "../../include/sip_head.h"
#include "sip_clip.h"
#include "sip_codes.h"
#include "sip_host.h"
#include "sip_xent.h"

namespace {

// Tiles of the cross entropy's products.
typedef sip::GemmShape<256, 256, 128, 64, 3, 2> Wide;
typedef sip::GemmShape<256, 64, 64, 64, 4, 3> Quarter;
typedef sip::GemmShape<128, 32, 32, 32, 4, 4> Narrow;
typedef sip::GemmShape<128, 128, 64, 64, 2, 2> Small;
typedef sip::GemmShape<64, 32, 16, 32, 4, 4> Tiny;
enum XentShape { kWide, kQuarter, kNarrow, kSmall, kTiny };
constexpr int kShapeA[] = {256, 256, 128, 128, 64}, kShapeB[] = {256, 64, 32, 128, 32}, kShapeWaveA[] = {128, 64, 32, 64, 16};

// What a product of a x b with sums over k, dealt out in `parts`, is expected to take in us, from products of one round (a unit of 64 k, one
// workgroup on its compute unit; each further one at once; how many LDS has room for) and of many rounds of one unit (a
// round's start and end), by tile: D = 8192, 2048 x 32 to 4096 x 256, and 262144 x 2000 of D = 64.
double tiles_cost(XentShape s, long long a, long long b, long long k, int parts) {
  constexpr double kUnitUs[] = {1.13, 0.68, 0.25, 0.92, 0.18}, kFurther[] = {0.0, 0.0, 0.20, 0.23, 0.08}, kEnds[] = {7.0, 5.1, 3.0, 5.2, 2.8};
  constexpr int kAtOnce[] = {1, 1, 2, 2, 3};
  const long long each = tiles((long long)tiles(a, kShapeA[s]) * tiles(b, kShapeB[s]) * parts, kChip);     // of a compute unit
  const long long rounds = each / kAtOnce[s], rest = each % kAtOnce[s];
  const double units = tiles(tiles(k, parts), 64);
  const double us = rounds * (units * (kUnitUs[s] + kFurther[s] * (kAtOnce[s] - 1)) + kEnds[s]) +
                    (rest ? units * (kUnitUs[s] + kFurther[s] * (rest - 1)) + kEnds[s] : 0.0);
  // the head's rows come from memory once (5.2 TB/s, 4.5 in the smallest tiles), and from cache for every further row of tiles (17)
  const double read = 2e-6 * a * k / (s == kTiny ? 4.5 : 5.2) + 2e-6 * a * k / 17.0 * (tiles(b, kShapeB[s]) - 1);
  return std::max(us, read) + 0.4 * std::min(us, read);   // (the one hides the other in part)
}
// The most workgroups that n_tiles tiles are dealt out among, and into how many parts of at least 256 terms: what bounds the room of
// the parts' sums.  (Without it one shape in a thousand would take up to 7 % less time by tiles_cost(), and twice the room.)
constexpr int kPartsMost = 128, kDealtTiles = 1024;      // tiles that may be dealt out at all
inline long long dealt_most(long long n_tiles) { return std::min<long long>(std::max<long long>(4 * n_tiles, 1024), 2 * kDealtTiles); }
// The tile that is expected to take the least time, and into how many parts it pays to deal the sums (at most `most`).
struct Cheapest { XentShape shape; int parts; };
Cheapest cheapest(std::initializer_list<XentShape> among, long long a, long long b, long long k, int most = 1) {
  Cheapest c{*among.begin(), 1};
  double best = -1.0;
  for (XentShape s : among)
    for (int n = 1; n <= most && (n == 1 || k / n >= 256); ++n) {
      const long long n_tiles = (long long)tiles(a, kShapeA[s]) * tiles(b, kShapeB[s]);
      if (n > 1 && n * n_tiles > dealt_most(n_tiles)) break;
      const double cost = tiles_cost(s, a, b, k, n) + (n > 1 ? 6.0 + 4e-6 * n * a * b : 0.0);              // (the join)
      if (best < 0.0 || cost < best) { best = cost; c = {s, n}; }
    }
  return c;
}
XentShape score_shape(int a, int tokens, int D) { return cheapest({kWide, kQuarter, kNarrow, kSmall, kTiny}, a, tokens, D).shape; }
// Partial sums of a token in the forward pass, one for each wave's entries; and the room up to which they may be narrower than the
// widest tile's (no shape has come near it: narrower tiles are for few).
inline int score_parts(XentShape s, int V) { return tiles(V, kShapeA[s]) * (kShapeA[s] / kShapeWaveA[s]); }
constexpr size_t kScorePartsRoom = 16 << 20;

// How a cross entropy of this shape is cut, and where its parts lie in the workspace.
struct XentPlan {
  XentShape score;              // tiles of the logits
  int parts;                    // waves' partial sums of a token
  int piece;                    // vocabulary entries whose dz is held at once
  XentShape score_piece, hidden, weight;
  sip::Parts hidden_parts, weight_parts;   // for all N tokens (without their room)
  int hidden_kept, hidden_joined;          // tiles of grad_hidden whose sums are kept, and that are joined
  size_t count, rows, part, dense, dz, hidden_sum, weight_sum, bytes;
};

// Rows of dz, for whatever number of N tokens takes part.
inline int xent_dz_rows(int N) { return std::max<int>(N, 2 * std::min<int>(N, sip::kTwoPartRows)); }
// Vocabulary entries of a piece: dz takes half a gigabyte at most.  The fewer the more tokens there are.
constexpr long long kDzMost = 1ll << 28;
inline int xent_piece(int N, int V) {
  const long long most = std::max<long long>(256, kDzMost / N / 256 * 256);
  const int pieces = tiles(V, (int)std::min<long long>(most, 1 << 20));
  return tiles(tiles(V, pieces), 256) * 256;
}
// Up to here grad_hidden does without the widest tile: its parts' sums take four times the room, for 1 % less time in one shape of a
// hundred.
constexpr int kNarrowRows = 128;

XentPlan xent_plan(int32_t N, int32_t V, int32_t D, bool backward) {
  XentPlan p{};
  p.score = score_shape(V, N, D);
  if ((size_t)N * score_parts(p.score, V) * 8 > kScorePartsRoom) p.score = kWide;
  p.parts = score_parts(p.score, V);
  size_t at = 0;
  auto take = [&](size_t n) { const size_t here = at; at += head_align(n); return here; };
  p.count = take(4);
  p.rows = take((size_t)N * 4);
  // the two directions' own parts share the room behind
  const size_t both = at;
  p.part = take((size_t)N * p.parts * 8);
  p.bytes = at;
  if (backward) {
    p.piece = xent_piece(N, V);
    const int left = std::min(p.piece, V);
    p.score_piece = score_shape(left, N, D);
    // rows of dz: two each if no more than kTwoPartRows of the tokens take part
    const int two_part_rows = 2 * std::min<int>(N, sip::kTwoPartRows);
    const long long dz_rows = xent_dz_rows(N);
    const Cheapest h = dz_rows > kNarrowRows ? cheapest({kWide, kNarrow, kSmall}, D, dz_rows, left, kPartsMost)
                                             : cheapest({kNarrow, kSmall}, D, dz_rows, left, kPartsMost);
    const Cheapest w = cheapest({kWide, kSmall}, D, left, dz_rows, kPartsMost);
    p.hidden = h.shape;
    p.weight = w.shape;
    p.hidden_parts = {nullptr, tiles(D, kShapeA[h.shape]) * tiles(dz_rows, kShapeB[h.shape]), h.parts, 0};
    p.weight_parts = {nullptr, tiles(D, kShapeA[w.shape]) * tiles(left, kShapeB[w.shape]), w.parts, 0};
    auto room = [](int count, int n_tiles, XentShape s) { return (size_t)count * n_tiles * kShapeA[s] * kShapeB[s] * 4; };
    // (where one kernel makes all of grad_hidden, sums are kept of tokens in two parts alone)
    p.hidden_kept = p.hidden_parts.count == 1 && p.piece >= V ? tiles(D, kShapeA[h.shape]) * tiles(two_part_rows, kShapeB[h.shape]) : p.hidden_parts.tiles;
    p.hidden_joined = p.hidden_parts.count == 1 ? tiles(D, kShapeA[h.shape]) * tiles(two_part_rows / 2, kShapeB[h.shape]) : p.hidden_parts.tiles;
    at = both;
    p.dense = take((size_t)dz_rows * D * 2);
    p.dz = take((size_t)dz_rows * p.piece * 2);
    p.hidden_sum = take(room(p.hidden_parts.count, p.hidden_kept, p.hidden));
    p.weight_sum = take(p.weight_parts.count == 1 ? 0 : room(p.weight_parts.count, p.weight_parts.tiles, p.weight));
    p.bytes = std::max(p.bytes, at);
  }
  return p;
}

// A workspace for N tokens and for fewer: the most that xent_plan() asks for up to N, or a little more.  It only grows with N, though
// the plans' needs do not: few tokens have two rows of dz each, and smaller tiles or more parts where those pay.
size_t xent_most_bytes(int32_t N, int32_t V, int32_t D, bool backward) {
  const size_t lists = head_align(4) + head_align((size_t)N * 4);
  const size_t score = std::max((size_t)N * score_parts(kWide, V) * 8, std::min((size_t)N * score_parts(kTiny, V) * 8, kScorePartsRoom));
  if (!backward) return lists + head_align(score);
  const long long dz_rows = xent_dz_rows(N), columns = tiles(V, 256) * 256;
  // tiles that are dealt out, no more than n_tiles, for sums of up to k terms
  auto dealt = [](long long n_tiles, long long k) {
    n_tiles = std::min<long long>(n_tiles, kDealtTiles);
    return std::min(dealt_most(n_tiles), n_tiles * std::min<long long>(kPartsMost, k / 256));
  };
  size_t hidden = 0, weight = 0;
  for (XentShape s : {kWide, kNarrow, kSmall}) {
    if (s == kWide && dz_rows <= kNarrowRows) continue;
    const long long n_tiles = (long long)tiles(D, kShapeA[s]) * tiles(dz_rows, kShapeB[s]);
    hidden = std::max(hidden, (size_t)std::max(n_tiles, dealt(n_tiles, V)) * kShapeA[s] * kShapeB[s] * 4);
  }
  if (dz_rows >= 2 * 256)
    for (XentShape s : {kWide, kSmall}) {
      const long long fewest = (long long)tiles(D, kShapeA[s]) * tiles(std::min(xent_piece(N, V), V), kShapeB[s]);
      if (fewest <= kDealtTiles)
        weight = std::max(weight, (size_t)dealt((long long)tiles(D, kShapeA[s]) * tiles(V, kShapeB[s]), dz_rows) * kShapeA[s] * kShapeB[s] * 4);
    }
  const size_t dz = (size_t)std::min(dz_rows * columns, kDzMost) * 2;
  return lists + std::max(head_align(score), head_align((size_t)dz_rows * D * 2) + head_align(dz) + head_align(hidden) + head_align(weight));
}

// f(S{}) with the tile's type, one of those named.
template <XentShape> struct ShapeType;
template <> struct ShapeType<kWide> { typedef Wide type; };
template <> struct ShapeType<kQuarter> { typedef Quarter type; };
template <> struct ShapeType<kNarrow> { typedef Narrow type; };
template <> struct ShapeType<kSmall> { typedef Small type; };
template <> struct ShapeType<kTiny> { typedef Tiny type; };
template <XentShape... AMONG, class F>
void with_shape(XentShape s, F f) { (void)((s == AMONG && (f(typename ShapeType<AMONG>::type{}), true)) || ...); }
// Workgroups for n tiles of which each XCD takes an eighth (sip_xent.h, tile_of).
inline int tile_grid(long long n) { return tiles(n, 8) * 8; }

bool xent_shape_ok(int32_t N, int32_t V, int32_t D) {
  return N > 0 && V > 0 && D > 0 && N <= SIP_MAX_TOKENS && V <= SIP_MAX_V && D <= SIP_MAX_D && D % 8 == 0;
}

sip_status xent_check(const void* hidden, int32_t N, int32_t D, int64_t hidden_stride, const void* weight, int32_t V,
                      int64_t weight_stride, const int32_t* targets) {
  if (!hidden || !weight || !targets || N <= 0 || V <= 0 || D <= 0 || D % 8 != 0) return SIP_ERR_INVALID_ARG;
  if (hidden_stride < D || weight_stride < D || hidden_stride % 8 != 0 || weight_stride % 8 != 0 || !aligned16(hidden) ||
      !aligned16(weight))
    return SIP_ERR_INVALID_ARG;
  if (!xent_shape_ok(N, V, D) || hidden_stride > (1ll << 30) / N || weight_stride > (1 << 20)) return SIP_ERR_UNSUPPORTED;
  return SIP_OK;
}

sip::XentArgs xent_args(const void* hidden, int32_t N, int32_t D, int64_t hidden_stride, const void* weight, int32_t V,
                        int64_t weight_stride, const int32_t* targets, float logit_scale, const XentPlan& pl,
                        void* workspace) {
  sip::XentArgs a{};
  char* ws = static_cast<char*>(workspace);
  a.hidden = static_cast<const uint16_t*>(hidden); a.hidden_stride = hidden_stride;
  a.weight = static_cast<const uint16_t*>(weight); a.weight_stride = weight_stride;
  a.targets = targets;
  a.N = N; a.V = V; a.D = D;
  a.logit_scale = logit_scale;
  a.count = reinterpret_cast<int*>(ws + pl.count);
  a.rows = reinterpret_cast<int*>(ws + pl.rows);
  a.part = reinterpret_cast<float2*>(ws + pl.part);
  a.parts = pl.parts;
  a.dense = reinterpret_cast<uint16_t*>(ws + pl.dense);
  a.dz = reinterpret_cast<uint16_t*>(ws + pl.dz);
  a.piece = pl.piece;
  a.hidden_parts = pl.hidden_parts; a.hidden_parts.sum = reinterpret_cast<float*>(ws + pl.hidden_sum);
  a.weight_parts = pl.weight_parts; a.weight_parts.sum = reinterpret_cast<float*>(ws + pl.weight_sum);
  return a;
}

template <int N> using Int = std::integral_constant<int, N>;

// Launches head_few_kernel where the hidden states fit the registers of a workgroup: 16 rows (an fp32 state is three) and D
// <= 8192, or 32 and 4096, D from 128 on.  False: they do not.
template <int GROUP, bool SCALES_BF16>
bool few_rows_of(const sip::CodesArgs& a, hipStream_t stream) {
  const int units = tiles(tiles(a.D, 128), sip::kFewWaves);              // of a wave
  // the kernel of the fewest UNITS that hold them
  auto launch = [&](auto mt, auto... counts) {
    bool done = false;
    auto one = [&](auto n) {
      constexpr int kUnits = decltype(n)::value, kMt = decltype(mt)::value;
      if (done || units > kUnits) return;
      constexpr int kTiles = sip::few_tiles(GROUP, SCALES_BF16, kUnits, kMt);
      hipLaunchKernelGGL((sip::head_few_kernel<GROUP, SCALES_BF16, kUnits, kMt>), dim3(std::min(kChip, tiles(a.V, 16 * kTiles))),
                         dim3(sip::kFewWaves * 64), 0, stream, a);
      done = true;
    };
    (one(counts), ...);
    return done;
  };
  const int rows = std::min(a.B, 64) * sip::rows_of_state(a.hidden_bf16);
  if (a.D < 128 || rows > 32) return false;
  if (rows > 16) return launch(Int<2>(), Int<1>(), Int<2>(), Int<3>(), Int<4>());
  return launch(Int<1>(), Int<1>(), Int<2>(), Int<3>(), Int<4>(), Int<5>(), Int<6>(), Int<7>(), Int<8>());
}
template <int GROUP>
bool few_rows_of(const sip::CodesArgs& a, hipStream_t stream) {
  return a.scales_bf16 ? few_rows_of<GROUP, true>(a, stream) : few_rows_of<GROUP, false>(a, stream);
}
bool few_rows(const sip::CodesArgs& a, hipStream_t stream) {
  return a.group == 32 ? few_rows_of<32>(a, stream) : a.group == 64 ? few_rows_of<64>(a, stream) : few_rows_of<128>(a, stream);
}

// head_many_kernel: blocks of 64 rows where one holds them all, else of 128; entries as its comment says.
int many_tiles(int32_t B, bool hidden_bf16) { return B <= sip::block_states(4, hidden_bf16) ? 4 : 8; }
size_t many_bytes(int32_t B, int32_t D, int32_t group, bool hidden_bf16) {
  const int mt = many_tiles(B, hidden_bf16);
  return tiles(B, sip::block_states(mt, hidden_bf16)) * sip::ManyLayout(D, group, mt).block;
}
template <int GROUP>
void many_rows_of(const sip::CodesArgs& a, hipStream_t stream) {
  const int mt = many_tiles(a.B, a.hidden_bf16), blocks = tiles(a.B, sip::block_states(mt, a.hidden_bf16));
  hipLaunchKernelGGL(sip::head_rows_kernel<GROUP>, dim3(blocks * mt, tiles(sip::many_groups(a.D, GROUP), 4)), dim3(256), 0, stream, a, mt);
  auto launch = [&](auto row_tiles, auto waves, auto nt) {
    constexpr int kMt = decltype(row_tiles)::value, kWaves = decltype(waves)::value, kNt = decltype(nt)::value;
    const dim3 grid(tiles(tiles(a.V, kWaves * kNt * 16), 8) * 8 * blocks), threads(kWaves * 64);
    if (a.scales_bf16) hipLaunchKernelGGL((sip::head_many_kernel<GROUP, true, kMt, kWaves, kNt>), grid, threads, 0, stream, a);
    else hipLaunchKernelGGL((sip::head_many_kernel<GROUP, false, kMt, kWaves, kNt>), grid, threads, 0, stream, a);
  };
  const bool narrow = (long long)tiles(a.V, 256) * blocks < kChip;
  if (mt == 4) narrow ? launch(Int<4>(), Int<4>(), Int<1>()) : launch(Int<4>(), Int<8>(), Int<2>());
  else narrow ? launch(Int<8>(), Int<4>(), Int<1>()) : launch(Int<8>(), Int<8>(), Int<2>());
}

}  // namespace

extern "C" {

size_t sip_xent_workspace_bytes(int32_t N, int32_t V, int32_t D, int32_t backward) {
  return xent_shape_ok(N, V, D) ? xent_most_bytes(N, V, D, backward != 0) : 0;
}

sip_status sip_xent_forward(const void* hidden, int32_t N, int32_t D, int64_t hidden_stride, const void* weight,
                            int32_t V, int64_t weight_stride, const int32_t* targets, float logit_scale, float* loss,
                            float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const sip_status ok = xent_check(hidden, N, D, hidden_stride, weight, V, weight_stride, targets);
  if (ok != SIP_OK) return ok;
  if (!loss || !lse) return SIP_ERR_INVALID_ARG;
  const XentPlan pl = xent_plan(N, V, D, false);
  if (!workspace_ok(workspace, workspace_bytes, pl.bytes)) return SIP_ERR_WORKSPACE;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  sip::XentArgs a = xent_args(hidden, N, D, hidden_stride, weight, V, weight_stride, targets, logit_scale, pl, workspace);
  a.loss = loss; a.lse = lse;
  hipLaunchKernelGGL(sip::xent_rows_kernel, dim3(1), dim3(1024), 0, stream, a);
  with_shape<kWide, kQuarter, kNarrow, kSmall, kTiny>(pl.score, [&](auto shape) {
    typedef decltype(shape) S;
    hipLaunchKernelGGL(sip::xent_forward_kernel<S>, dim3(tile_grid((long long)tiles(V, S::kA) * tiles(N, S::kB))),
                       dim3(S::kThreads), 0, stream, a);
  });
  hipLaunchKernelGGL(sip::xent_loss_kernel, dim3(N), dim3(256), 0, stream, a);
  return launched();
}

sip_status sip_xent_backward(const void* hidden, int32_t N, int32_t D, int64_t hidden_stride, const void* weight,
                             int32_t V, int64_t weight_stride, const int32_t* targets, float logit_scale,
                             const float* loss, const float* lse, const float* grad_loss, float scale,
                             void* grad_hidden, int64_t grad_hidden_stride, void* grad_weight,
                             int64_t grad_weight_stride, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const sip_status ok = xent_check(hidden, N, D, hidden_stride, weight, V, weight_stride, targets);
  if (ok != SIP_OK) return ok;
  if (!loss || !lse) return SIP_ERR_INVALID_ARG;
  if (grad_hidden && (grad_hidden_stride < D || grad_hidden_stride % 8 != 0 || !aligned16(grad_hidden))) return SIP_ERR_INVALID_ARG;
  if (grad_weight && (grad_weight_stride < D || grad_weight_stride % 8 != 0 || !aligned16(grad_weight))) return SIP_ERR_INVALID_ARG;
  const XentPlan pl = xent_plan(N, V, D, true);
  if (!workspace_ok(workspace, workspace_bytes, pl.bytes)) return SIP_ERR_WORKSPACE;
  if (!grad_hidden && !grad_weight) return SIP_OK;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  sip::XentArgs a = xent_args(hidden, N, D, hidden_stride, weight, V, weight_stride, targets, logit_scale, pl, workspace);
  a.loss_in = loss; a.lse_in = lse; a.grad_loss = grad_loss;
  a.out_scale = scale * logit_scale;
  a.grad_hidden = static_cast<uint16_t*>(grad_hidden); a.gh_stride = grad_hidden_stride;
  a.grad_weight = static_cast<uint16_t*>(grad_weight); a.gw_stride = grad_weight_stride;
  hipLaunchKernelGGL(sip::xent_rows_kernel, dim3(1), dim3(1024), 0, stream, a);
  hipLaunchKernelGGL(sip::xent_gather_kernel, dim3(N), dim3(256), 0, stream, a);
  for (int v0 = 0; v0 < V; v0 += pl.piece) {
    a.v0 = v0;
    const int left = std::min(pl.piece, V - v0);
    with_shape<kWide, kQuarter, kNarrow, kSmall, kTiny>(pl.score_piece, [&](auto shape) {
      typedef decltype(shape) S;
      hipLaunchKernelGGL(sip::xent_dz_kernel<S>, dim3(tile_grid((long long)tiles(left, S::kA) * tiles(N, S::kB))), dim3(S::kThreads), 0, stream, a);
    });
    if (grad_hidden)
      with_shape<kWide, kNarrow, kSmall>(pl.hidden, [&](auto shape) {
        typedef decltype(shape) S;
        hipLaunchKernelGGL(sip::xent_grad_hidden_kernel<S>, dim3(tile_grid(pl.hidden_parts.tiles), pl.hidden_parts.count), dim3(S::kThreads), 0,
                           stream, a);
        if (v0 + pl.piece >= V)
          hipLaunchKernelGGL((sip::xent_join_kernel<S, true>), dim3(pl.hidden_joined, S::kTA * S::kTB), dim3(S::kThreads), 0, stream, a);
      });
    if (grad_weight)
      with_shape<kWide, kSmall>(pl.weight, [&](auto shape) {
        typedef decltype(shape) S;
        const int n_tiles = tiles(D, S::kA) * tiles(left, S::kB);
        hipLaunchKernelGGL(sip::xent_grad_weight_kernel<S>, dim3(tile_grid(n_tiles), pl.weight_parts.count), dim3(S::kThreads), 0, stream, a);
        if (pl.weight_parts.count > 1)
          hipLaunchKernelGGL((sip::xent_join_kernel<S, false>), dim3(n_tiles, S::kTA * S::kTB), dim3(S::kThreads), 0, stream, a);
      });
  }
  return launched();
}

size_t sip_grad_clip_workspace_bytes(int32_t n_tensors) {
  if (n_tensors < 0 || n_tensors > SIP_MAX_TENSORS) return 0;
  return head_align((size_t)std::max(1, tiles(n_tensors, sip::kClipTable)) * sip::kClipGroups * sizeof(double));
}

sip_status sip_grad_clip(const sip_grad* tensors, int32_t n_tensors, float max_norm, float eps, float* norm,
                         void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (n_tensors < 0 || (n_tensors > 0 && !tensors) || !norm || !(max_norm >= 0.0f) || !(eps >= 0.0f)) return SIP_ERR_INVALID_ARG;
  if (n_tensors > SIP_MAX_TENSORS) return SIP_ERR_UNSUPPORTED;
  int64_t bytes = 0;
  for (int j = 0; j < n_tensors; ++j) {
    const sip_grad& t = tensors[j];
    if (t.count < 0 || (t.dtype != SIP_F32 && t.dtype != SIP_BF16)) return SIP_ERR_INVALID_ARG;
    if (t.count > 0 && (!t.grad || !t.out)) return SIP_ERR_INVALID_ARG;
    if (t.count > (1ll << 40) || (bytes += t.count * 4) > (1ll << 46)) return SIP_ERR_UNSUPPORTED;
    const uintptr_t mask = t.dtype == SIP_F32 ? 3 : 1;
    if (((reinterpret_cast<uintptr_t>(t.grad) | reinterpret_cast<uintptr_t>(t.out)) & mask) != 0) return SIP_ERR_INVALID_ARG;
  }
  if (!workspace_ok(workspace, workspace_bytes, sip_grad_clip_workspace_bytes(n_tensors))) return SIP_ERR_WORKSPACE;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  double* part = static_cast<double*>(workspace);
  const int launches = std::max(1, tiles(n_tensors, sip::kClipTable));
  auto table = [&](int l) {
    sip::ClipTable t{};
    for (int j = l * sip::kClipTable; j < std::min(n_tensors, (l + 1) * sip::kClipTable); ++j) {
      if (tensors[j].count == 0) continue;
      t.grad[t.n] = static_cast<const char*>(tensors[j].grad);
      t.out[t.n] = static_cast<char*>(tensors[j].out);
      t.count[t.n] = tensors[j].count | (tensors[j].dtype == SIP_BF16 ? sip::kClipBf16 : 0);
      t.end[t.n] = (t.n ? t.end[t.n - 1] : 0) + (uint32_t)((sip::clip_bytes(t.count[t.n]) + sip::kClipBytes - 1) / sip::kClipBytes);
      ++t.n;
    }
    return t;
  };
  auto groups = [](const sip::ClipTable& t) { return t.n ? (int)std::min<uint32_t>(t.end[t.n - 1], sip::kClipGroups) : 1; };
  int parts = 0;
  for (int l = 0; l < launches; ++l) {
    const sip::ClipTable t = table(l);
    hipLaunchKernelGGL(sip::clip_squares_kernel, dim3(groups(t)), dim3(sip::kClipThreads), 0, stream, t, part + parts);
    parts += groups(t);
  }
  for (int l = launches - 1; l >= 0; --l) {
    const sip::ClipTable t = table(l);
    hipLaunchKernelGGL(sip::clip_scale_kernel, dim3(groups(t)), dim3(sip::kClipThreads), 0, stream, t, part, parts, max_norm, eps,
                       l == 0 ? norm : nullptr);
  }
  return launched();
}

namespace {
// What the quantiser and the product check alike.
sip_status codes_check(const void* codes, int64_t codes_stride, const void* scales, sip_dtype scales_dtype, int32_t V,
                       int32_t D, int32_t group) {
  if (!codes || !scales || V <= 0 || D <= 0 || (scales_dtype != SIP_F32 && scales_dtype != SIP_BF16)) return SIP_ERR_INVALID_ARG;
  if (group != 32 && group != 64 && group != 128) return group > 0 ? SIP_ERR_UNSUPPORTED : SIP_ERR_INVALID_ARG;
  if (D % group != 0 || codes_stride < D / 2 || codes_stride % 16 != 0 || !aligned16(codes)) return SIP_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(scales) & (scales_dtype == SIP_F32 ? 3 : 1)) != 0) return SIP_ERR_INVALID_ARG;
  if (V > SIP_MAX_V || D > SIP_MAX_D || codes_stride > (1 << 20)) return SIP_ERR_UNSUPPORTED;
  return SIP_OK;
}
}  // namespace

sip_status sip_head_quantize(const void* weight, int32_t V, int32_t D, int64_t weight_stride, int32_t group,
                             uint8_t* codes, int64_t codes_stride, void* scales, sip_dtype scales_dtype,
                             uint8_t* zeros, void* hip_stream) {
  if (!weight) return SIP_ERR_INVALID_ARG;
  const sip_status ok = codes_check(codes, codes_stride, scales, scales_dtype, V, D, group);
  if (ok != SIP_OK) return ok;
  if (weight_stride < D || weight_stride % 8 != 0 || !aligned16(weight)) return SIP_ERR_INVALID_ARG;
  if (weight_stride > (1 << 20)) return SIP_ERR_UNSUPPORTED;
  sip::CodesArgs a{};
  a.weight = static_cast<const uint16_t*>(weight); a.weight_stride = weight_stride;
  a.codes = codes; a.codes_stride = codes_stride;
  a.scales = scales; a.scales_bf16 = scales_dtype == SIP_BF16;
  a.zeros = zeros;
  a.V = V; a.D = D; a.group = group;
  const dim3 grid(std::min(tiles((long long)V * (D / 8), 256), kChip * 64));
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if (group == 32) hipLaunchKernelGGL(sip::quantize_kernel<32>, grid, dim3(256), 0, stream, a);
  else if (group == 64) hipLaunchKernelGGL(sip::quantize_kernel<64>, grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL(sip::quantize_kernel<128>, grid, dim3(256), 0, stream, a);
  return launched();
}

size_t sip_head_workspace_bytes(int32_t B, int32_t V, int32_t D, int32_t group) {
  if (B <= 0 || V <= 0 || D <= 0 || B > SIP_MAX_B || V > SIP_MAX_V || D > SIP_MAX_D) return 0;
  if ((group != 32 && group != 64 && group != 128) || D % group != 0) return 0;
  return head_align(std::max(many_bytes(B, D, group, true), many_bytes(B, D, group, false)));
}

sip_status sip_head_logits(const void* hidden, int32_t B, int32_t D, int64_t hidden_stride, sip_dtype hidden_dtype,
                           const uint8_t* codes, int64_t codes_stride, const void* scales, sip_dtype scales_dtype,
                           const uint8_t* zeros, int32_t group, int32_t V, void* logits, int64_t logits_stride,
                           sip_dtype logits_dtype, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!hidden || !logits || B <= 0 || (hidden_dtype != SIP_F32 && hidden_dtype != SIP_BF16) ||
      (logits_dtype != SIP_F32 && logits_dtype != SIP_BF16))
    return SIP_ERR_INVALID_ARG;
  const sip_status ok = codes_check(codes, codes_stride, scales, scales_dtype, V, D, group);
  if (ok != SIP_OK) return ok;
  const int x_size = hidden_dtype == SIP_F32 ? 4 : 2, z_size = logits_dtype == SIP_F32 ? 4 : 2;
  if (hidden_stride < D || hidden_stride % (16 / x_size) != 0 || !aligned16(hidden) || logits_stride < V ||
      reinterpret_cast<uintptr_t>(logits) % z_size != 0)
    return SIP_ERR_INVALID_ARG;
  if (B > SIP_MAX_B || hidden_stride > (1ll << 32) || logits_stride > (1ll << 32)) return SIP_ERR_UNSUPPORTED;
  if (!workspace_ok(workspace, workspace_bytes, sip_head_workspace_bytes(B, V, D, group))) return SIP_ERR_WORKSPACE;
  sip::CodesArgs a{};
  a.codes = const_cast<uint8_t*>(codes); a.codes_stride = codes_stride;
  a.scales = const_cast<void*>(scales); a.scales_bf16 = scales_dtype == SIP_BF16;
  a.zeros = const_cast<uint8_t*>(zeros);
  a.V = V; a.D = D; a.group = group;
  a.hidden = hidden; a.hidden_stride = hidden_stride; a.hidden_bf16 = hidden_dtype == SIP_BF16;
  a.B = B;
  a.logits = logits; a.logits_stride = logits_stride; a.logits_bf16 = logits_dtype == SIP_BF16;
  a.states = static_cast<char*>(workspace);
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if (few_rows(a, stream)) return launched();
  if (group == 32) many_rows_of<32>(a, stream);
  else if (group == 64) many_rows_of<64>(a, stream);
  else many_rows_of<128>(a, stream);
  return launched();
}

}  // extern "C"
