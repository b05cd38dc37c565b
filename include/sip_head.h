/*
 * sip_head.h -- the vocabulary head around the sampler of sip.h: the product that makes the logits
 * from hidden states, and what trains its weights.
 *
 * A model's last step turns hidden states [N, D] into logits [N, V] by a matrix W [V, D]; sip_sample()
 * turns those into tokens.  The functions here score given tokens under W and differentiate that
 * score without ever holding the logits (sip_xent_*), bound a set of gradients by their common norm
 * (sip_grad_clip), bring W to 4 bits (sip_head_quantize), and make the logits of a decode step from
 * such weights in the form that sip_sample() takes (sip_head_logits).
 *
 * Conventions are those of sip.h: DEVICE pointers, caller-owned buffers, everything enqueued on
 * `hip_stream`, argument errors found on the host before anything is enqueued, no allocation and no
 * synchronisation.  Calls that overlap in time need workspaces of their own.  The same inputs give
 * the same output bits on every call.  Matrices are row-major with a row stride in elements; bf16
 * rows start at multiples of 16 bytes (base pointer, stride) unless said otherwise.
 */
#ifndef SIP_HEAD_H_
#define SIP_HEAD_H_

#include "sip.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SIP_MAX_D 16384        /* widest hidden state                                              */
#define SIP_MAX_TOKENS 65536   /* most tokens of one sip_xent_* call                               */
#define SIP_MAX_TENSORS 65536  /* most tensors of one sip_grad_clip() call                         */

/*
 * ---- Cross entropy of given tokens under the head, and its gradient ----------------------------
 *
 *   z[i, v] = logit_scale * sum_d hidden[i, d] * weight[v, d]
 *   lse[i]  = ln sum_v exp(z[i, v])
 *   loss[i] = lse[i] - z[i, targets[i]]            (= -log-probability of the token)
 *
 * logit_scale is 1, or the reciprocal of the temperature that the tokens were sampled with, 0 for an infinite one.  A row
 * whose target lies outside [0, V) -- a masked token -- costs nothing: loss and lse are 0, and
 * whatever its hidden state holds (NaN included) goes nowhere.  Logits are made a tile at a time from
 * bf16 operands with fp32 sums and never written; maxima and sums of exponentials are fp32, the
 * target's own logit is summed in fp64.  The loss is formed as ln(1 + sum_{v != target} exp(z_v -
 * z_target)), so that it keeps its relative accuracy for a token that is nearly certain.
 *
 *  hidden   [N, hidden_stride] bf16, N * hidden_stride up to 2^30.
 *  weight   [V, weight_stride] bf16.
 *  D        a multiple of 8.
 *  targets  [N] int32.
 *  loss,    [N] fp32.
 *  lse
 *  workspace  256-byte aligned, at least sip_xent_workspace_bytes(N, V, D, 0) bytes for
 *             sip_xent_forward(), (N, V, D, 1) for either; contents need not be kept.  What
 *             is enough for N tokens is enough for fewer of the same V and D.
 */
size_t sip_xent_workspace_bytes(int32_t N, int32_t V, int32_t D, int32_t backward);
sip_status sip_xent_forward(const void* hidden, int32_t N, int32_t D, int64_t hidden_stride, const void* weight,
                            int32_t V, int64_t weight_stride, const int32_t* targets, float logit_scale, float* loss,
                            float* lse, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Gradient of  scale * sum_i grad_loss[i] * loss[i]  with respect to hidden and weight:
 *
 *   dz[i, v]       = grad_loss[i] * (exp(z[i, v] - lse[i]) - [v = targets[i]])
 *   grad_hidden[i] = scale * logit_scale * sum_v dz[i, v] * weight[v]
 *   grad_weight[v] = scale * logit_scale * sum_i dz[i, v] * hidden[i]
 *
 *  loss, lse    what sip_xent_forward() gave for the same arguments.
 *  grad_loss    [N] fp32, NULL = all ones.
 *  grad_hidden  [N, grad_hidden_stride] bf16, NULL = not wanted; rows of masked tokens are zero.
 *  grad_weight  [V, grad_weight_stride] bf16, NULL = not wanted.  Both are overwritten.
 * The logits are made again, a piece of the vocabulary at a time; dz of a piece is held as bf16, where
 * no more than 64 tokens take part as the sum of two bf16 (without scale * logit_scale, which the fp32
 * sums are multiplied with), sums over the vocabulary and over the tokens are fp32 across pieces, and the
 * gradients are rounded once.
 */
sip_status sip_xent_backward(const void* hidden, int32_t N, int32_t D, int64_t hidden_stride, const void* weight,
                             int32_t V, int64_t weight_stride, const int32_t* targets, float logit_scale,
                             const float* loss, const float* lse, const float* grad_loss, float scale,
                             void* grad_hidden, int64_t grad_hidden_stride, void* grad_weight,
                             int64_t grad_weight_stride, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * ---- Global gradient norm, and clipping ----------------------------------------------------------
 *
 *   norm   = sqrt(sum over all elements of all tensors of g^2)
 *   out_j  = g_j * min(1, max_norm / (norm + eps))
 *
 * The table of tensors is read before the call returns (HOST array); the tensors themselves are device
 * memory, contiguous, fp32 or bf16, aligned to their element.  `out` may be `grad` itself (in place)
 * or another tensor of the same type; two entries must not overlap otherwise.  Squares are formed and
 * summed in fp64, in an order that depends only on the sizes.  A norm that is NaN makes every output
 * NaN, an infinite one makes them 0 (NaN where g is infinite); max_norm = +inf leaves the gradients as
 * they are and only measures, and so does norm + eps = 0.
 *
 *  tensors    host array of n_tensors entries; n_tensors = 0 or entries of 0 elements are allowed.
 *  norm       device fp32, one value.
 *  workspace  256-byte aligned, at least sip_grad_clip_workspace_bytes(n_tensors) bytes.
 */
typedef struct {
  const void* grad;
  void* out;
  int64_t count;                     /* elements, 0 .. 2^40; of all tensors together up to 2^44      */
  sip_dtype dtype;
} sip_grad;

size_t sip_grad_clip_workspace_bytes(int32_t n_tensors);
sip_status sip_grad_clip(const sip_grad* tensors, int32_t n_tensors, float max_norm, float eps, float* norm,
                         void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * ---- A head of 4-bit codes with group scales -----------------------------------------------------
 *
 *   w[v, d] ~ scales[v, d / group] * (q[v, d] - zeros[v, d / group]),   q in 0..15
 *
 *  codes   [V, codes_stride] bytes: byte j of a row holds q[v, 2 j] in its low and q[v, 2 j + 1] in
 *          its high half; rows start at multiples of 16 bytes.
 *  scales  [V, D / group] fp32 or bf16, contiguous.
 *  zeros   [V, D / group] bytes, contiguous, 0..15; NULL = 8 for every group.
 *  group   32, 64 or 128; D a multiple of it.
 *
 * sip_head_quantize() makes them from bf16 weights by rounding to nearest.  Per group, with lo the
 * smaller of 0 and the smallest weight and hi the larger of 0 and the largest,
 *   zeros given:  s = (hi - lo) / 15,         zero = clamp(rint(-lo / s), 0, 15)
 *   zeros NULL:   s = max(hi, -lo) / 7,       zero = 8
 * s rounded to its type (and 1 if that is 0), q = clamp(rint(w / s) + zero, 0, 15), all in fp32.  A group that
 * holds an infinity or a NaN gets that as its scale: logits made from it are not finite.
 */
sip_status sip_head_quantize(const void* weight, int32_t V, int32_t D, int64_t weight_stride, int32_t group,
                             uint8_t* codes, int64_t codes_stride, void* scales, sip_dtype scales_dtype,
                             uint8_t* zeros, void* hip_stream);

/*
 * Logits of B hidden states under such a head:
 *
 *   logits[b, v] = sum_g scales[v, g] * sum_{d in g} (q[v, d] - zeros[v, g]) * hidden[b, d]
 *
 *  hidden   [B, hidden_stride] bf16 or fp32, rows aligned to 16 bytes.  fp32 values enter with all their 24 bits.
 *  logits   [B, logits_stride] fp32 or bf16, aligned to its element; only the first V entries of a row are written.
 *           logits_stride a multiple of 16 bytes makes rows that sip_sample() takes.
 *  workspace  256-byte aligned, at least sip_head_workspace_bytes(B, V, D, group) bytes.
 * Products are exact, sums fp32, scales are applied to the fp32 sum of a group; rounded once.  A code enters as 16 + q, and what
 * that adds is taken off again: by group for up to 16 rows with D from 128 to 8192, or 32 with D up to 4096 (an fp32 state counts
 * as three), else by 256 entries, where states whose mean is far from zero lose about three bits more.  An infinity or a NaN in a
 * hidden state makes the whole of its row infinite or NaN, and other rows nothing.
 */
size_t sip_head_workspace_bytes(int32_t B, int32_t V, int32_t D, int32_t group);
sip_status sip_head_logits(const void* hidden, int32_t B, int32_t D, int64_t hidden_stride, sip_dtype hidden_dtype,
                           const uint8_t* codes, int64_t codes_stride, const void* scales, sip_dtype scales_dtype,
                           const uint8_t* zeros, int32_t group, int32_t V, void* logits, int64_t logits_stride,
                           sip_dtype logits_dtype, void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SIP_HEAD_H_ */
