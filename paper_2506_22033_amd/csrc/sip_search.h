// Host side of the entry points declared in include/sip_beam.h: argument checks, workspace carving, launches.
#pragma once
#include <algorithm>

#include "../../include/sip_beam.h"
#include "sip_beam.h"
#include "sip_host.h"

namespace {

inline int beam_chunks(int32_t V, bool bf16) { return tiles(V, sip::beam_chunk(bf16)); }
bool beam_shape_ok(int32_t groups, int32_t width, int32_t V, int32_t n) {
  return groups > 0 && width > 0 && V > 0 && n > 0 && width <= SIP_MAX_BEAMS && V <= SIP_MAX_V && n <= SIP_MAX_CONTINUATIONS &&
         (int64_t)groups * width <= SIP_MAX_B;
}
static_assert(SIP_MAX_V <= 64 * sip::kBeamThreads * sip::kBeamLoads * 4, "the merging kernels: a lane a chunk");
size_t beam_part_bytes(int64_t lists) { return head_align((size_t)lists * sizeof(sip::BeamPart)); }

// Up to so many words a group's slots are moved by one workgroup, in one launch instead of two.  Kernels in us, one and two: a group of 4 beams,
// L_max = 512, 4.8 and 3.3 + 2.7; 128 groups of 4, 2048, 10.0 and 7.5 + 4.0; but 64 of 8, 4096, 16.6 and 9.5 + 4.4.
constexpr long long kGroupWords = 48 << 10;
static_assert(kGroupWords < (sip::kGroupWidth + 1) * 2 * sip::kTableSlots, "no wider groups");

}  // namespace

extern "C" {

size_t sip_beam_workspace_bytes(int32_t groups, int32_t width, int32_t V, int32_t n) {
  if (!beam_shape_ok(groups, width, V, n)) return 0;
  const int64_t lists = (int64_t)groups * width * beam_chunks(V, false);                   // (of fp32: the most)
  return beam_part_bytes(lists) + head_align((size_t)lists * n * 8);
}

sip_status sip_beam_select(const void* logits, int32_t groups, int32_t width, int32_t V, int64_t row_stride, sip_dtype dtype,
                           float logit_scale, const float* scores, const uint8_t* finished, int32_t end_token,
                           const float* rank_scale, int32_t n, int32_t* tokens, int32_t* parents, float* out_scores,
                           void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!logits || !scores || !tokens || !parents || !out_scores || groups <= 0 || width <= 0 || V <= 0 || n <= 0 || !dtype_ok(dtype))
    return SIP_ERR_INVALID_ARG;
  if (!rows_ok(logits, V, row_stride, dtype) || !(logit_scale >= 1e-30f && logit_scale <= 1e30f)) return SIP_ERR_INVALID_ARG;
  if (finished && (end_token < 0 || end_token >= V)) return SIP_ERR_INVALID_ARG;
  if (!beam_shape_ok(groups, width, V, n) || row_stride > (1ll << 32)) return SIP_ERR_UNSUPPORTED;
  if (!workspace_ok(workspace, workspace_bytes, sip_beam_workspace_bytes(groups, width, V, n))) return SIP_ERR_WORKSPACE;
  sip::BeamArgs a{};
  a.logits = logits; a.row_stride = row_stride;
  a.width = width; a.V = V; a.n = n;
  a.chunks = beam_chunks(V, dtype == SIP_BF16);
  a.chunk = sip::beam_chunk(dtype == SIP_BF16);
  const int group = dtype == SIP_BF16 ? 8 : 4;
  a.wanted = sip::beam_wanted(n, sip::kBeamThreads);
  a.wanted_last = sip::beam_wanted(n, std::min(tiles(V - (a.chunks - 1) * a.chunk, group), sip::kBeamThreads));
  a.scale = (double)logit_scale;
  a.c = (float)(a.scale * 1.4426950408889634074);
  a.scores = scores; a.finished = finished; a.rank_scale = rank_scale; a.end_token = end_token;
  a.tokens = tokens; a.parents = parents; a.out_scores = out_scores;
  const int64_t lists = (int64_t)groups * width * a.chunks;
  a.part = static_cast<sip::BeamPart*>(workspace);
  a.cand = reinterpret_cast<unsigned long long*>(static_cast<char*>(workspace) + beam_part_bytes(lists));
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if (dtype == SIP_BF16) hipLaunchKernelGGL(sip::beam_chunk_kernel<true>, dim3(lists), dim3(sip::kBeamThreads), 0, stream, a);
  else hipLaunchKernelGGL(sip::beam_chunk_kernel<false>, dim3(lists), dim3(sip::kBeamThreads), 0, stream, a);
  if (width * a.chunks * n <= sip::kMergeFew) hipLaunchKernelGGL(sip::beam_merge_few_kernel, dim3(groups), dim3(256), 0, stream, a);
  else hipLaunchKernelGGL(sip::beam_merge_kernel, dim3(groups), dim3(sip::kMergeThreads), 0, stream, a);
  return launched();
}

sip_status sip_state_reorder(void* state, size_t state_bytes, int32_t slots, int32_t L_max, int32_t groups, int32_t width,
                             const int32_t* slot_of_row, const int32_t* parents, const int32_t* tokens, void* hip_stream) {
  if (slots <= 0 || L_max <= 0 || slots > SIP_MAX_SLOTS || L_max > SIP_MAX_L || groups < 0 || width <= 0) return SIP_ERR_INVALID_ARG;
  if (groups > 0 && (!slot_of_row || !parents)) return SIP_ERR_INVALID_ARG;
  if (width > SIP_MAX_BEAMS || (int64_t)groups * width > SIP_MAX_B) return SIP_ERR_UNSUPPORTED;
  if (!workspace_ok(state, state_bytes, sip::state_total(slots, L_max))) return SIP_ERR_WORKSPACE;
  if (groups == 0) return SIP_OK;
  const sip::StateView v = sip::state_view(state, slots, L_max);
  sip::ReorderArgs a{};
  a.head = v.head; a.len = v.len; a.ndist = v.ndist; a.tokens = v.tokens; a.table = v.table;
  a.slots = slots; a.L_max = L_max; a.width = width;
  a.slot_of_row = slot_of_row; a.parents = parents; a.new_tokens = tokens;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if ((long long)width * (L_max + 2 * sip::kTableSlots) <= kGroupWords) {
    hipLaunchKernelGGL(sip::state_reorder_group_kernel, dim3(groups), dim3(sip::kGroupThreads), 0, stream, a);
    return launched();
  }
  // (groups along x: of both along it, more than a launch can have)
  if (width <= sip::kGroupWidth) {
    const dim3 grid(groups, sip::kReorderTables + tiles(L_max, sip::kReorderThreads * 4));
    hipLaunchKernelGGL(sip::state_reorder_few_kernel, grid, dim3(sip::kReorderThreads), 0, stream, a);
  } else {
    const dim3 grid(groups, sip::kReorderTableBlocks + tiles(L_max, sip::kReorderWords));
    hipLaunchKernelGGL(sip::state_reorder_kernel, grid, dim3(tiles(width, sip::kReorderEach) * 64), 0, stream, a);
  }
  hipLaunchKernelGGL(sip::state_reorder_append_kernel, dim3(groups), dim3(64), 0, stream, a);
  return launched();
}

}  // extern "C"
