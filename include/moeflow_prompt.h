/*
 * moeflow_prompt.h -- the part of libmoeflow.so that a prompt passes beside the
 * MoE layers, and the tokens after it when their cache is held in 4 bits:
 *
 *   moe_prompt_attention  causal attention over packed prompts, or chunks of them
 *   moe_kv4_store         keys and values of new tokens into a cache of 4 bits
 *   moe_kv4_load          values back from it, for a prompt's next chunk
 *   moe_kv4_attention     attention of single tokens over that cache
 *   moe_token_logprobs    log-probabilities of given tokens, entropy, alternatives
 *
 * The conventions of moeflow.h hold: device memory owned by the caller; work
 * enqueued on `stream` only; host validation before anything is enqueued; no
 * allocation, no synchronisation, no state kept between calls. Arrays are row major
 * and densely packed but for the strides given below. Every call may be captured into
 * a HIP graph. Workspaces are scratch of one call: calls that may overlap need their
 * own. Outputs must not overlap inputs, workspaces or each other.
 */
#ifndef MOEFLOW_PROMPT_H
#define MOEFLOW_PROMPT_H

#include "moeflow.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------------
 * moe_prompt_attention -- causal softmax attention of B packed sequences. Sequence
 * b's queries are rows q_offsets[b] .. q_offsets[b+1]-1 of q, its keys and values
 * rows k_offsets[b] .. k_offsets[b+1]-1 of k and v. Of n queries and m keys the
 * last query is the token of the last key (a chunk of a prompt follows m - n keys
 * that are there already): query i attends to the keys 0 .. m - n + i.
 *
 *   s_j       = scale * q[i, h] . k[j, h / (Hq / Hkv)]
 *   out[i, h] = sum_j softmax(s)_j v[j, h / (Hq / Hkv)],  lse[i, h] = ln sum_j exp s_j
 * A query without any key (i < n - m), or whose scores are all -inf: out 0, lse
 * -inf. What later tokens hold does not reach earlier ones, be it NaN. An infinite
 * value of a key that a query attends to counts whatever the key's weight, also 0:
 * that dimension of out is the infinity, or NaN of a NaN or of both signs. Float32
 * scores, statistics and accumulation; bf16: the softmax numerators are rounded to
 * bf16 for the second product, their sum is not. Sums of values are held with weights
 * of at most 1 and divided by the weights' sum at the end: results are finite where the
 * sum of |v| over a query's keys is below 3.4e38; terms below 2^-118 may count as 0.
 * Results do not depend on scheduling.
 *
 * q    [N, Hq, D] dtype, tokens q_stride elements apart (at least Hq * D)
 * k, v [M, Hkv, D] dtype, tokens k_stride, v_stride elements apart (at least
 *      Hkv * D): q, k and v may lie in one buffer. May be NULL when M == 0
 * q_offsets, k_offsets  [B+1] int32, non-decreasing (clipped to 0..N, 0..M). With
 *      B == 1 NULL is (0, N), (0, M); k_offsets NULL with B > 1 is q_offsets (M == N).
 *      Rows before the first and from the last q_offset on belong to no sequence: out
 *      and lse keep what they hold there
 * out  [N, Hq, D] dtype; lse [N, Hq] float32 or NULL
 * workspace  moe_prompt_attention_workspace bytes, 256-byte aligned (may be 0); a size
 *      that does not fall as N, M or B grows: that of the largest call serves all
 * Limits: N >= 1, M >= 0, B >= 1, Hq a multiple of Hkv, D a multiple of 8 up to
 *   256, Hq <= 65536; N * Hq, B < 2^31, M <= 2^30; strides a multiple of 16 bytes, at
 *   most 2^24 elements; tensors of dtype on 16 bytes; N * Hq / 32 + B * Hkv below
 *   2^22; |scale| up to 2.3e38 (below 1e-37 it counts as 0). Outputs and workspace
 *   whose ranges meet those of inputs or each other are MOE_ERR_ARG, in this and the
 *   other calls.
 * Errors: MOE_ERR_ARG, MOE_ERR_UNSUPPORTED, MOE_ERR_WORKSPACE, MOE_ERR_HIP.
 * ---------------------------------------------------------------------- */
size_t moe_prompt_attention_workspace(int64_t N, int64_t M, int64_t B, int32_t Hq, int32_t Hkv,
                                      int32_t D, int32_t dtype);
int moe_prompt_attention(const void* q, const void* k, const void* v, int32_t dtype, int64_t N,
                         int64_t M, int64_t B, int32_t Hq, int32_t Hkv, int32_t D,
                         int64_t q_stride, int64_t k_stride, int64_t v_stride,
                         const int32_t* q_offsets, const int32_t* k_offsets, float scale, void* out,
                         float* lse, void* workspace, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------
 * A cache of 4 bits: n_slots token slots, each with Hkv heads of D channels for keys
 * and for values. 32 channels of a head are a block that shares a power of two 2^e,
 * the least with max |x| <= 7 * 2^e and e in -124..125; a channel is held as the
 * nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times 2^e (ties to the even code; larger
 * ones as 6), with its sign. No value is off by more than half of the step it lies
 * in, 2^e at most, but for those beyond 7 * 2^125, which become 6 * 2^125. A block with a
 * NaN or an infinity is NaN as a whole.
 *
 * codes  [n_slots, Hkv, D / 2] uint8: channel 2i in the lower half of byte i, 2i + 1 in
 *        the upper; bit 3 the sign, bits 0..2 the index of the value
 * scales [n_slots, Hkv, D / 32] uint8: e + 127, or 255 for a block of NaN
 * moe_kv_gather and moe_beam_reorder move such caches like any other (codes and scales
 * in calls of their own, as their bytes a position differ).
 *
 * moe_kv4_store -- tokens 0 .. N-1 of k and v into slots slots[n].
 * moe_kv4_load  -- slots slots[n] back into tokens 0 .. N-1 of k and v, dtype. Every
 *   value a block can hold is a bf16 number.
 *
 * k, v   [N, Hkv, D] dtype, tokens k_stride, v_stride elements apart (at least Hkv * D)
 * slots  [N] int32, or NULL: slot n (N <= n_slots). A token whose slot is outside
 *        0 .. n_slots-1 (padding: -1) is left out: nothing of it is written. Slots that
 *        tokens are stored to must differ, else they hold a mix of those tokens
 * Limits: N >= 1, n_slots >= 1, N * Hkv < 2^31, n_slots < 2^31, D a multiple of 32
 *   up to 256, strides a multiple of 16 bytes, at most 2^24 elements, k and v and codes
 *   on 16 bytes, N * Hkv * D < 2^34. Errors: MOE_ERR_ARG, MOE_ERR_UNSUPPORTED,
 *   MOE_ERR_HIP.
 * ---------------------------------------------------------------------- */
int moe_kv4_store(const void* k, const void* v, int32_t dtype, int64_t N, int32_t Hkv, int32_t D,
                  int64_t k_stride, int64_t v_stride, const int32_t* slots, int64_t n_slots,
                  uint8_t* k_codes, uint8_t* k_scales, uint8_t* v_codes, uint8_t* v_scales,
                  void* stream);
int moe_kv4_load(const uint8_t* k_codes, const uint8_t* k_scales, const uint8_t* v_codes,
                 const uint8_t* v_scales, int64_t n_slots, const int32_t* slots, int64_t N,
                 int32_t Hkv, int32_t D, int32_t dtype, int64_t k_stride, int64_t v_stride, void* k,
                 void* v, void* stream);

/* ------------------------------------------------------------------------
 * moe_kv4_attention -- softmax attention of R rows, one token each, over a cache of
 * C rows of S slots. Row r reads the first lens[r] slots of cache row cache_row[r]
 * (rows may share one):
 *
 *   s_i       = scale * q[r, h] . K_i of head h / (Hq / Hkv)
 *   out[r, h] = sum_i softmax(s)_i V_i,  lse[r, h] = ln sum_i exp s_i
 * A row without any key, or whose scores are all -inf: out 0, lse -inf. A block of NaN
 * of a key that a row reads counts whatever the key's weight. Float32 scores, statistics
 * and accumulation; with float32 q products are of 24 bits, with bf16 the softmax
 * numerators are rounded to bf16 for the second product, their sum is not. Large values
 * as for moe_prompt_attention (one key of 6 * 2^125 is held); terms below 2^-100 may lose
 * bits, below 2^-115 may count as 0. Results do not depend on scheduling. lse joins the
 * result with that over other keys (moe_prefix_attention).
 *
 * q, out     [R, Hq, D] dtype; lse [R, Hq] float32 or NULL
 * k_codes .. v_scales  [C, S, Hkv, D / 2], [C, S, Hkv, D / 32] as above
 * cache_row  [R] int32 or NULL (row r, R <= C); outside 0..C-1: no keys
 * lens       [R] int32 (clipped to 0..S) or NULL (S). What a cache holds from a length
 *            on is not used
 * workspace  moe_kv4_attention_workspace bytes, 256-byte aligned; a size that does
 *            not fall as R or S grows: that of the largest call serves all
 * Limits: R, C, S >= 1, Hq a multiple of Hkv, D a multiple of 32 up to 256; R * Hq,
 *   C, S < 2^31, Hkv * D < 2^24, q, out and codes on 16 bytes, scales on 4,
 *   R * Hkv * ceil(Hq / Hkv / 16) below 2^22, |scale| as for moe_prompt_attention.
 *   Errors: MOE_ERR_ARG, MOE_ERR_UNSUPPORTED, MOE_ERR_WORKSPACE, MOE_ERR_HIP.
 * ---------------------------------------------------------------------- */
size_t moe_kv4_attention_workspace(int64_t R, int64_t S, int32_t Hq, int32_t Hkv, int32_t D);
int moe_kv4_attention(const void* q, int32_t dtype, int64_t R, int32_t Hq, int32_t Hkv, int32_t D,
                      const uint8_t* k_codes, const uint8_t* k_scales, const uint8_t* v_codes,
                      const uint8_t* v_scales, int64_t C, int64_t S, const int32_t* cache_row,
                      const int32_t* lens, float scale, void* out, float* lse, void* workspace,
                      size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------------
 * moe_token_logprobs -- of R rows of logits over V tokens:
 *
 *   logprobs[r, j]  = z[r, tokens[r, j]] - ln sum_v exp z[r, v]
 *   entropy[r]      = - sum_v p_v ln p_v,  p = softmax(z[r])
 *   top_tokens[r]   = the n_top tokens of the largest logits, descending; equal ones
 *                     lower token first; top_logprobs[r] theirs
 * A token outside 0..V-1 (padding) has -inf. Logits of -inf are masked: probability
 * 0, no share of the entropy, never a top token. Where fewer than n_top are left, the
 * places hold -1 and -inf. A row of nothing but -inf: logprobs -inf, entropy 0. A row
 * with a NaN or +inf: logprobs (of tokens in 0..V-1) and entropy NaN, top_tokens -1,
 * top_logprobs -inf.
 * Numerics: float32 exponentials of differences to a reference that no logit exceeds by
 * more than 8, summed in float64 beyond 32 of them, the best logit's terms apart where
 * they are most of the sum. A log-probability is off by at most 2^-15 of the
 * best token's own, the entropy by at most 2^-13 of itself, beside the rounding to
 * float32: no log-probability is above 0, no entropy below, and both are 0 where one
 * token has all.
 *
 * logits  [R, V] dtype, rows `stride` elements apart (at least V), any
 *         element-aligned address
 * tokens  [R, m] int32 (NULL when m == 0); logprobs [R, m] float32
 * entropy [R] float32 or NULL
 * top_tokens [R, n_top] int32, top_logprobs [R, n_top] float32 (NULL when n_top == 0)
 * workspace  none is needed: the size is 0, and what is given is not used
 * Limits: R, V >= 1, m >= 0, 0 <= n_top <= 64, V <= 2^24, R < 2^22, R * m < 2^31,
 *   stride < 2^31; one output at least (m, entropy or n_top).
 * Errors: MOE_ERR_ARG, MOE_ERR_UNSUPPORTED, MOE_ERR_HIP.
 * ---------------------------------------------------------------------- */
size_t moe_token_logprobs_workspace(int64_t R, int64_t V, int64_t m, int32_t n_top);
int moe_token_logprobs(const void* logits, int32_t dtype, int64_t R, int64_t V, int64_t stride,
                       const int32_t* tokens, int64_t m, int32_t n_top, float* logprobs,
                       float* entropy, int32_t* top_tokens, float* top_logprobs, void* workspace,
                       size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MOEFLOW_PROMPT_H */
