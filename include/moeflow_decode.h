/*
 * moeflow_decode.h -- the part of libmoeflow.so that a decode step of several
 * sequences calls: one new token per sequence (row), the rows of a request
 * (its beams, or a batch behind one prompt) next to each other.
 *
 *   moe_prefix_attention  attention of every row over the prompt its group
 *                         shares and over the row's own suffix
 *   moe_layer_decode      a whole MoE layer for at most 64 tokens (Sec. 2.1)
 *   moe_beam_select       the best continuations of a request's beams
 *   moe_beam_reorder      suffix states follow their beams, in place
 *
 * The conventions of moeflow.h hold: device memory owned by the caller, row
 * major and densely packed; work enqueued on `stream` only; host validation
 * before anything is enqueued; no allocation, no synchronisation, no state kept
 * between calls. Every call may be captured into a HIP graph. Workspaces are
 * scratch of one call: calls that may overlap need their own.
 */
#ifndef MOEFLOW_DECODE_H
#define MOEFLOW_DECODE_H

#include "moeflow.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------------
 * moe_layer_decode -- a whole MoE layer (Sec. 2.1) for the T <= 64 tokens of a
 * decode step: what moe_route, moe_permute, moe_expert_ffn and moe_combine
 * compute together, without the maps and row copies between them:
 *
 *   z[t, e]   = x_t . w_router[e] (+ bias), in float64
 *   idx[t, :] = the k largest z[t, :], descending; equal ones go to the lower
 *               expert; a NaN is never chosen (fewer than k numbers: idx -1,
 *               gate 0)
 *   w[t, j]   = softmax(z[t, :])[idx[t, j]], with renormalize divided by their
 *               sum over j
 *   y[t]      = (accumulate: y[t] +) sum_{j: slot(idx) in 0..S-1} w[t, j] E(x_t)
 *               + Shared(x_t)
 *   E(x)      = w_down . a,  a = silu(w_gate . x) * (w_up . x)
 * float32 accumulation; w[t, j] * a is rounded to dtype once, as the operand of
 * the down projection, and y once.
 *
 * x [T, H], w_router [E, H], bias as for moe_route (bias_mode 0: NULL, 1: [E],
 * 2: [T, E]); w_gate, w_up [S, F, H], w_down [S, H, F]: the expert slots;
 * slot_of_expert [E] int32 (outside 0..S-1: not resident) or NULL (expert e in
 * slot e, S >= E)
 * shared_gate, shared_up [Fs, H], shared_down [H, Fs]: the always-on experts,
 *   concatenated along Fs; NULL with Fs == 0
 * y          [T, H] dtype output, may be x; no other overlap is allowed
 * topk_idx, topk_w  [T, k] outputs
 * incomplete [T] int32 output or NULL: 1 when some choice is not resident
 * workspace  moe_layer_decode_workspace bytes, 256-byte aligned
 * Results do not depend on scheduling: sums run in a fixed order.
 * Limits: 1 <= T <= 64, 1 <= k <= min(E, 32), E <= 256; H, F, Fs multiples of 8
 *   (bf16) or 4 (float32), at most 2^22, 2^24, 2^24; tensors of dtype on 16 bytes;
 *   (T*k*F + T*Fs) values below 2 GiB; else MOE_ERR_UNSUPPORTED (the four calls
 *   take such batches). Errors: MOE_ERR_ARG, MOE_ERR_WORKSPACE, MOE_ERR_HIP.
 * ---------------------------------------------------------------------- */
size_t moe_layer_decode_workspace(int64_t T, int64_t H, int64_t F, int32_t E, int32_t k,
                                  int64_t Fs, int32_t dtype);
int moe_layer_decode(const void* x, int32_t dtype, int64_t T, int64_t H, const void* w_router,
                     int32_t E, int32_t k, const float* bias, int32_t bias_mode,
                     int32_t renormalize, const void* w_gate, const void* w_up,
                     const void* w_down, int32_t S, int64_t F, const int32_t* slot_of_expert,
                     const void* shared_gate, const void* shared_up, const void* shared_down,
                     int64_t Fs, int32_t accumulate, void* y, int32_t* topk_idx, float* topk_w,
                     int32_t* incomplete, void* workspace, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------
 * moe_beam_select -- the n_out best continuations of each of B requests over
 * its K beams and V tokens:
 *
 *   c(b, v)  = scores[b] + logits[b, v] - ln sum_u exp logits[b, u]
 *   a beam with finished[b] != 0 has one continuation only: (b, eos) with
 *   c = scores[b], whatever its logits hold
 *   result   the n_out largest c, descending; equal ones lower beam first,
 *            then lower token
 *
 * A continuation counts when its c is a number above -inf: rows whose logits
 * hold a NaN or +inf, tokens of logit -inf and beams of score -inf have none.
 * Where fewer than n_out count, the places left hold parent = token = -1,
 * score = -inf, finished = 0.
 * Numerics: log-sum-exp from float32 exponentials, added in float64 beyond 32 of
 * them; c = logits + (scores - log-sum-exp) in float64, rounded to float32 once,
 * after the choice. Equal rows of equal score tie exactly.
 *
 * logits        [B, K, V] dtype (any element-aligned address)
 * scores        [B, K] float32
 * finished      [B, K] int32 or NULL (none has finished)
 * eos           the end token, 0 <= eos < V; read with finished or out_finished
 * parent        [B, n_out] int32 output: row b*K + beam that is continued
 * token         [B, n_out] int32 output
 * out_scores    [B, n_out] float32 output
 * out_finished  [B, n_out] int32 output or NULL: 1 when the parent had finished
 *               or token == eos
 * No output may overlap an input.
 * Limits: B >= 1, 1 <= K <= 32, V >= 1, K * V <= 2^25, 1 <= n_out <= 64,
 *   B * K < 2^31 / 64. Errors: MOE_ERR_ARG, MOE_ERR_UNSUPPORTED,
 *   MOE_ERR_WORKSPACE, MOE_ERR_HIP.
 * ---------------------------------------------------------------------- */
size_t moe_beam_select_workspace(int64_t B, int32_t K, int64_t V, int32_t n_out);
int moe_beam_select(const void* logits, int32_t dtype, int64_t B, int32_t K, int64_t V,
                    const float* scores, const int32_t* finished, int64_t eos, int32_t n_out,
                    int32_t* parent, int32_t* token, float* out_scores, int32_t* out_finished,
                    void* workspace, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------
 * moe_beam_reorder -- the states of the beams after moe_beam_select (K of its
 * places): in every cache and layer, row r takes over the first
 * lens[parent[r]] positions of row parent[r], all rows at once (as if from a
 * copy of the cache), in place. Rows that keep themselves and positions from
 * there on are neither read nor written.
 *
 * caches    HOST array of n_caches (1..16) DEVICE pointers (not read when
 *           S == 0), no two overlapping, each [L, B*K, S, unit_bytes]:
 *           S positions of unit_bytes opaque bytes per row and layer (keys, values)
 * parent    [B*K] int32: a row of the same request, or -1 (the row keeps its
 *           state); any other value sets *err and the row keeps its state
 * lens      [B*K] int32 positions in use per row (clipped to 0..S) or NULL (S)
 * new_lens  [B*K] int32 output or NULL: lens[parent[r]] (lens[r] where the row
 *           keeps its state); must not be lens itself
 * err       int32, set to 1 by a bad parent; the caller clears it
 * Limits: L >= 1, B >= 1, 1 <= K <= 32, S >= 0, unit_bytes >= 1, B*K < 2^31,
 *   S * unit_bytes < 2^31.
 * Errors: MOE_ERR_ARG, MOE_ERR_UNSUPPORTED, MOE_ERR_HIP.
 * ---------------------------------------------------------------------- */
int moe_beam_reorder(void* const* caches, int32_t n_caches, int64_t L, int64_t B, int32_t K,
                     int64_t S, int64_t unit_bytes, const int32_t* parent, const int32_t* lens,
                     int32_t* new_lens, int32_t* err, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MOEFLOW_DECODE_H */
