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
