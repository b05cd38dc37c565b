/*
 * sip_beam.h -- beam search on the sampler's terms: the best continuations of many groups of beams from
 * their logits, and the reordering of the device-resident histories that follows.
 *
 * A request is a group of `width` beams; row g * width + k of every array is beam k of group g.
 * One step of a search is sip_beam_select() on the logits of all beams, then sip_state_reorder() with
 * its parents and tokens.
 *
 * Conventions are those of sip.h: DEVICE pointers, caller-owned buffers, everything enqueued on `hip_stream`,
 * argument errors found on the host before anything is enqueued, no allocation and no synchronisation; both
 * calls can be recorded into a graph.  The same inputs give the same output bits on every call.
 */
#ifndef SIP_BEAM_H_
#define SIP_BEAM_H_

#include "sip.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SIP_MAX_BEAMS 64           /* widest group                                    */
#define SIP_MAX_CONTINUATIONS 128  /* most continuations of a group that are selected */

/*
 * ---- Selection over beams and vocabulary --------------------------------------------------------
 *
 *   lse[k]      = ln sum_v exp(logit_scale * z[k, v])
 *   total[k, v] = scores[k] + logit_scale * z[k, v] - lse[k]
 *
 * and of the width * V continuations (k, v) of a group the n with the largest total[k, v] * rank_scale[k], in
 * descending order; of equal ones the lower beam first, of one beam's the larger logit, then the lower token.
 * Sums of exponentials are fp32 in a lane and fp64 beyond, totals are formed, scaled and compared in fp64.
 *
 *  logits      [groups * width, row_stride] fp32 or bf16, as sip_sample() takes them: base pointer and row stride
 *              multiples of 16 bytes.  Only the first V entries of a row are read; never written.  A logit of -inf is no
 *              continuation; a row that holds a NaN or +inf has none.
 *  logit_scale 1e-30 to 1e30: 1, or the reciprocal of a temperature.
 *  scores      [groups * width] fp32: the beams' log-probabilities so far.  A beam whose score is not finite
 *              (-inf: one that does not exist, as all but the first before the first step) has no
 *              continuation, and its logits are not looked at.
 *  finished    [groups * width] bytes, NULL = none.  A beam with a value other than 0 has one continuation, end_token
 *              at its unchanged score, and its logits are not looked at.
 *  end_token   in [0, V); looked at only if `finished` is given.
 *  rank_scale  [groups * width] fp32, finite and > 0, NULL = 1: what totals are multiplied with for comparison, such
 *              as a length penalty's 1 / length^a.  The scores that are returned are without it.  A beam with another
 *              value has no continuation.
 *  n           1 .. SIP_MAX_CONTINUATIONS, normally width, or 2 * width where the caller takes out those that end.
 *  tokens,     [groups, n] int32: the continuation's token, and the beam (0 .. width - 1) that it continues.
 *  parents
 *  out_scores  [groups, n] fp32: total, -inf below fp32's range (a mask's lowest value times a logit_scale above 1).  May be `scores`
 *              itself where n = width.
 *  Where a group has fewer than n continuations, the rest is token -1, parent -1, score -inf.
 *  workspace   256-byte aligned, at least sip_beam_workspace_bytes(groups, width, V, n) bytes; contents need not be kept.  What
 *              is enough is enough for fewer groups, fewer beams, a smaller vocabulary or a smaller n too.
 */
size_t sip_beam_workspace_bytes(int32_t groups, int32_t width, int32_t V, int32_t n);
sip_status sip_beam_select(const void* logits, int32_t groups, int32_t width, int32_t V, int64_t row_stride, sip_dtype dtype,
                           float logit_scale, const float* scores, const uint8_t* finished, int32_t end_token,
                           const float* rank_scale, int32_t n, int32_t* tokens, int32_t* parents, float* out_scores,
                           void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * ---- Reordering of a sampler state's histories ---------------------------------------------------
 * For every row r = g * width + k, with p = parents[r] and everything as it stands before the call: slot
 * slot_of_row[r] takes the history of slot slot_of_row[g * width + p], and tokens[r] behind it.  In place, every
 * history that changes its slot read once and written once.
 *
 *  state, state_bytes, slots, L_max  as for sip_sample_state(); the call counter stays as it is.
 *  slot_of_row [groups * width], distinct.  A value outside [0, slots) is a row without a history: it leaves no
 *              trace, and rows that continue it start empty.  Of rows of one group that name the same slot the first one's
 *              history is the slot's.
 *  parents     [groups * width], beams of the row's own group; a value outside [0, width) leaves the row's slot as it is,
 *              and its token is not appended.
 *  tokens      [groups * width], NULL = nothing is appended; nor is a negative token.  A full slot stays as it is, and the
 *              state's `overflow` grows by one.
 * Entries of a slot's token row from its new length on are left as they were.
 */
sip_status sip_state_reorder(void* state, size_t state_bytes, int32_t slots, int32_t L_max, int32_t groups, int32_t width,
                             const int32_t* slot_of_row, const int32_t* parents, const int32_t* tokens, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SIP_BEAM_H_ */
