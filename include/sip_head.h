/*
 * sip_head.h -- the vocabulary head around the sampler of sip.h: the product that makes the logits
 * from hidden states, and what trains its weights.
 *
 * A model's last step turns hidden states [N, D] into logits [N, V] by a matrix W [V, D]; sip_sample()
 * turns those into tokens.  The functions here score given tokens under W and differentiate that
 * score without ever holding the logits (sip_xent_*), bound a set of gradients by their common norm
 * (sip_grad_clip), bring W to 4 bits (sip_head_quantize), and make the logits of a decode step from
 * such weights in the form that sip_sample() takes (sip_head_logits), with every request's own low-rank adapter on top
 * (sip_head_adapt).  sip_embed() and its gradient are the matrix's other use, from tokens to vectors.
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
#define SIP_MAX_RANK 128       /* widest low-rank adapter                                          */
#define SIP_MAX_ADAPTERS 4096  /* most adapters of one sip_head_adapt() call                       */

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

/*
 * ---- Low-rank adapters of many requests beside the shared head ---------------------------------------
 *
 *   t[b, j]       = sum_d down[a, j, d] * hidden[b, d],   a = adapter_of_row[b]
 *   logits[b, v] += scales[a] * sum_j up[a, v, j] * t[b, j]
 *
 * in place, behind whatever made the logits.  A row whose adapter lies outside [0, adapters) is not touched, and what its
 * hidden state holds goes nowhere.
 *
 *  hidden    [B, hidden_stride] bf16 or fp32, B up to SIP_MAX_TOKENS, rows aligned to 16 bytes.
 *  down      [adapters, rank, D] bf16, up [adapters, V, rank] bf16, contiguous, aligned to 16 bytes.  An adapter of a
 *            smaller rank is filled up with zeros.
 *  rank      a multiple of 8 up to SIP_MAX_RANK; D a multiple of 8.
 *  scales    [adapters] fp32, NULL = 1.
 *  logits    [B, logits_stride] fp32 or bf16, aligned to its element; only the first V entries of a row are read or written.
 *  workspace 256-byte aligned, at least sip_head_adapt_workspace_bytes(B, adapters, rank, D) bytes.  What is enough for B
 *            rows is enough for fewer.
 * Products and sums are fp32, scales[a] * t is kept in fp32; the new logit is rounded once.  A row with an entry of t (or of scales[a] * t)
 * that is not finite or beyond the largest bf16, or with such an entry in an fp32 hidden state, has logits of NaN; other rows are not
 * affected.  An entry of `up` that is not finite makes its own logit NaN or infinite, of either sign.
 */
size_t sip_head_adapt_workspace_bytes(int32_t B, int32_t adapters, int32_t rank, int32_t D);
sip_status sip_head_adapt(const void* hidden, int32_t B, int32_t D, int64_t hidden_stride, sip_dtype hidden_dtype,
                          const void* down, const void* up, int32_t adapters, int32_t rank, const int32_t* adapter_of_row,
                          const float* scales, int32_t V, void* logits, int64_t logits_stride, sip_dtype logits_dtype,
                          void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * ---- Embedding: rows of the matrix by token, and their gradient ---------------------------------------
 *
 *   out[i] = scale * weight[ids[i]]
 *
 * in fp32, rounded once.  A token outside [0, V) -- padding -- gives a row of zeros.
 *
 *  weight  [V, weight_stride] bf16 or fp32 (sip_embed), or a head of 4-bit codes as sip_head_quantize() makes it
 *          (sip_embed_codes), which then serves both ends of a model: weight = scales * (q - zeros).
 *  D       a multiple of 8, of the group for codes.
 *  ids     [N] int32; N = 0 is allowed and does nothing.  N up to SIP_MAX_B.
 *  out     [N, out_stride] bf16 or fp32.  Rows of weight and out are aligned to 16 bytes.
 */
sip_status sip_embed(const void* weight, sip_dtype weight_dtype, int32_t V, int32_t D, int64_t weight_stride, const int32_t* ids,
                     int32_t N, float scale, void* out, int64_t out_stride, sip_dtype out_dtype, void* hip_stream);
sip_status sip_embed_codes(const uint8_t* codes, int64_t codes_stride, const void* scales, sip_dtype scales_dtype,
                           const uint8_t* zeros, int32_t group, int32_t V, int32_t D, const int32_t* ids, int32_t N, float scale,
                           void* out, int64_t out_stride, sip_dtype out_dtype, void* hip_stream);

/*
 *   grad_weight[v] = scale * sum_{i: ids[i] = v} grad_out[i]   (+ grad_weight[v] if accumulate)
 *
 * Tokens are sorted, and a row of grad_weight is the fp32 sum of its tokens' rows, scaled, added to what was there if asked for, and
 * rounded once.  The same call gives the same bits every time; calls that differ in sizes, types or `accumulate` may add up the same
 * rows in another order.  A token outside [0, V) takes no part, whatever its row of grad_out holds.  With accumulate != 0 rows of
 * grad_weight that no token names are not touched; without, they become zeros.  (A matrix that is head and embedding at once: sip_xent_backward() first, then this call with accumulate.)
 *
 *  grad_out    [N, grad_out_stride] bf16 or fp32, grad_weight [V, grad_weight_stride] bf16 or fp32; rows aligned to 16 bytes.
 *  N           0 .. SIP_MAX_TOKENS; D a multiple of 8.
 *  workspace   256-byte aligned, at least sip_embed_workspace_bytes(N, V, D) bytes.  What is enough for N tokens is enough
 *              for fewer.
 */
size_t sip_embed_workspace_bytes(int32_t N, int32_t V, int32_t D);
sip_status sip_embed_backward(const void* grad_out, int64_t grad_out_stride, sip_dtype grad_out_dtype, const int32_t* ids, int32_t N,
                              int32_t V, int32_t D, float scale, int32_t accumulate, void* grad_weight,
                              int64_t grad_weight_stride, sip_dtype grad_weight_dtype, void* workspace, size_t workspace_bytes,
                              void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SIP_HEAD_H_ */
