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
 * moe_prefix_attention -- softmax attention of R rows, one new token each.
 * Group g's rows group_offsets[g] .. group_offsets[g+1]-1 share the keys and
 * values of prefix g (a prompt whose beams they are, a prompt that a whole batch
 * starts with); every row r goes on with its own suffix (the tokens since, the
 * new one included):
 *
 *   s_i       = scale * q[r, h] . K_i over the keys of head h / (Hq / Hkv):
 *               k_prefix[g, 0 .. prefix_len[g]), k_suffix[r, 0 .. suffix_len[r])
 *   out[r, h] = sum_i softmax(s)_i V_i,  lse[r, h] = ln sum_i exp s_i
 * A row without any key, or whose scores are all -inf: out 0, lse -inf. Float32
 * scores, statistics and accumulation; bf16: the softmax numerators are rounded to
 * bf16 for the second product, their sum is not. Results do not depend on scheduling.
 *
 * q, out         [R, Hq, D] dtype; lse [R, Hq] float32 or NULL
 * group_offsets  [G+1] int32, non-decreasing (clipped to 0..R), or NULL: G equal
 *                groups (R a multiple of G). Rows before the first and from the
 *                last offset on belong to no group: out and lse keep what they
 *                hold there
 * k_prefix, v_prefix  [G, P, Hkv, D] dtype (may be NULL when P == 0)
 * k_suffix, v_suffix  [R, S, Hkv, D] dtype (may be NULL when S == 0)
 * prefix_len [G], suffix_len [R] int32 (clipped to 0..P, 0..S) or NULL (all).
 *                What the caches hold from a length on is not used, be it NaN
 * workspace      moe_prefix_attention_workspace bytes, 256-byte aligned (0 and
 *                NULL when P == S == 0); a size that does not fall as R, G, P or S
 *                grows: that of the largest call serves all
 * Limits: R >= 1, 1 <= G <= R, Hq a multiple of Hkv, D a multiple of 8 up to
 *   256, P, S < 2^31, Hkv * D * element size < 2^26, tensors of dtype on 16
 *   bytes, launches below 2^32 threads (R * Hkv * ceil(Hq / Hkv / 16) of some
 *   2^22), |scale| up to 2.3e38 (below 1e-37 it counts as 0). Errors: MOE_ERR_ARG,
 *   MOE_ERR_UNSUPPORTED, MOE_ERR_WORKSPACE, MOE_ERR_HIP.
 * ---------------------------------------------------------------------- */
size_t moe_prefix_attention_workspace(int64_t R, int64_t G, int32_t Hq, int32_t Hkv, int32_t D,
                                      int64_t P, int64_t S, int32_t dtype);
int moe_prefix_attention(const void* q, int32_t dtype, int64_t R, int32_t Hq, int32_t Hkv,
                         int32_t D, const int32_t* group_offsets, int64_t G, const void* k_prefix,
                         const void* v_prefix, int64_t P, const int32_t* prefix_len,
                         const void* k_suffix, const void* v_suffix, int64_t S,
                         const int32_t* suffix_len, float scale, void* out, float* lse,
                         void* workspace, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------
 * moe_layer_decode -- a whole MoE layer (Sec. 2.1) for the T <= 64 tokens of a
 * decode step: what moe_route, moe_permute, moe_expert_ffn and moe_combine
 * compute together, without the maps and row copies between them:
 *
 *   z[t, e]   = x_t . w_router[e] (+ bias), in float64
 *   idx[t, :] = the k largest z[t, :], descending; equal ones go to the lower
 *               expert; a NaN is never chosen (fewer than k numbers: idx -1,
 *               gate 0), and where no z[t, :] is above -inf (a mask that leaves
 *               nothing) nothing is: idx -1, gate 0 throughout
 *   w[t, j]   = softmax(z[t, :])[idx[t, j]] over the z[t, :] that are numbers,
 *               with renormalize divided by their sum over j; an expert of z -inf
 *               beside others has gate 0, a z of +inf makes the gates NaN
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
 * workspace  moe_layer_decode_workspace bytes, 256-byte aligned; a size that does not
 *            fall as T grows: that of the most tokens serves all
 * Results do not depend on scheduling: sums run in a fixed order.
 * Limits: T >= 1, 1 <= k <= E <= 256, as for moe_route, else MOE_ERR_ARG; T <= 64,
 *   k <= 32; H, F, Fs multiples of 8 (bf16) or 4 (float32), at most 2^22, 2^24, 2^24;
 *   tensors of dtype on 16 bytes; (T*k*F + T*Fs) values below 2 GiB; else
 *   MOE_ERR_UNSUPPORTED (the four calls take such batches). Other errors:
 *   MOE_ERR_ARG, MOE_ERR_WORKSPACE, MOE_ERR_HIP.
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
 *   result   the n_out largest c, descending; equal ones lower beam first; within
 *            a beam larger logit first, then lower token (a score so large that
 *            sums of different logits are equal does not change their order)
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
 * workspace     moe_beam_select_workspace bytes, 256-byte aligned; a size that does not
 *               fall as B, K, V or n_out grows: that of the largest call serves all
 * With n_out == K out_scores may be scores and out_finished may be finished; no
 * other output may overlap an input.
 * Limits: B >= 1, 1 <= K <= 32, V >= 1, K * V <= 2^25, 1 <= n_out <= 64,
 *   B * K < 2^31 / 64, B < 2^23. Errors: MOE_ERR_ARG, MOE_ERR_UNSUPPORTED,
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
 *           S == 0), no two overlapping (MOE_ERR_ARG), each
 *           [L, B*K, S, unit_bytes]:
 *           S positions of unit_bytes opaque bytes per row and layer (keys, values)
 * parent    [B*K] int32: a row of the same request, or -1 (the row keeps its
 *           state); any other value sets *err and the row keeps its state
 * lens      [B*K] int32 positions in use per row (clipped to 0..S) or NULL (S)
 * new_lens  [B*K] int32 output or NULL: lens[parent[r]] (lens[r] where the row
 *           keeps its state); must not be lens or parent itself
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
