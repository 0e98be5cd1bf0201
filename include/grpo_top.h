/*
 * grpo_top.h -- what a row of logits says about a token: the log-prob of a given one, the policy's entropy and its
 * likeliest alternatives with their log-probs, and the gradient of the three (libgrpo, gfx950).
 *
 * Of a row z_0 .. z_(V-1) at temperature tau, over its words, those with z > -1e8 (as everywhere in this library, a
 * lower logit is a masked word):
 *   log p_v = z_v / tau - log sum exp(z / tau),   H = -sum p log p,
 *   alternatives: the n words of largest z, the lowest index first among equal ones (-0 equals 0).
 *
 * Conventions (streams, errors, device pointers) are those of grpo.h.
 */
#ifndef GRPO_TOP_H_
#define GRPO_TOP_H_

#include "grpo_sampling.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The most alternatives of a call, and the largest vocabulary. */
#define GRPO_TOP_MAX 64
#define GRPO_TOP_MAX_V 4194304

/* What a row's distribution comes to, for the backward call: log p_v = (z_v - max) / temperature - log_sum. */
typedef struct {
  double log_sum;    /* log sum exp((z - max) / tau); NaN for a row with a NaN, +inf or a temperature out of range,
                        -inf for one without words                                   */
  float max;         /* max z over the words, -inf without any                       */
  float entropy;     /* H                                                            */
  float temperature; /* tau                                                          */
  float logp;        /* the action's log-prob, a word's no lower than -FLT_MAX       */
} grpo_top_row;

/* Bytes of device workspace grpo_token_logp_top needs: 0 for many or short rows (ws may then be NULL), and for invalid
 * sizes. */
size_t grpo_token_logp_top_workspace_bytes(int64_t T, int64_t V, int32_t n);

/*
 * Log-prob, entropy and alternatives of each row.
 *   logits       device [T, ld] of `dtype`, columns >= V unread
 *   0 <= T < 2^31, 1 <= V <= GRPO_TOP_MAX_V, V <= ld, 0 <= n <= GRPO_TOP_MAX
 *   temperature  device fp32 [T], a value for each row, or NULL and temperature_all for all: 1e-6 .. 1e6
 *   actions      device int32 [T]
 *   logp         device fp32 [T] or NULL: log p of the action; -inf for a masked word and below fp32's range; 0 where the
 *                action is outside [0, V) (GRPO_FLAG_ACTION)
 *   entropy      device fp32 [T] or NULL
 *   top_ids      device int32 [T, n] or NULL, -1 past a row's last word
 *   top_logp     device fp32 [T, n] or NULL, -inf past a row's last word
 *   rows         device grpo_top_row [T] or NULL, 8-byte aligned: what the backward call takes
 *   error_flags  device int32 [1] or NULL, overwritten
 *   ws, ws_bytes device workspace of at least grpo_token_logp_top_workspace_bytes(T, V, n), 16-byte aligned; calls that
 *                may overlap (on two streams, in two graphs) need one each
 * A row with a NaN or +inf (GRPO_FLAG_NONFINITE), or with its own temperature out of range (GRPO_FLAG_SETTING): log-prob,
 * entropy and alternatives' log-probs NaN, alternatives -1.  A row without words (GRPO_FLAG_NONFINITE): entropy 0, no
 * alternatives, the log-prob of an action in [0, V) -inf.
 * Each row is read once, but for the few words that may be alternatives; a row whose large words repeat more often than a list
 * of 1,024 holds (256 for rows of one wave) is read up to 16 (bf16) or 32 (fp32) times more.  Sums run in fp32 over at most 32 words, in fp64
 * beyond; the same inputs give the same bits.  Log-probs are at most 0, entropies at least 0.
 * Errors: GRPO_ERR_ARG (a required pointer NULL, temperature_all out of range), GRPO_ERR_SHAPE, GRPO_ERR_DTYPE,
 *   GRPO_ERR_ALIGN (logits and arrays to their element, ws to 16), GRPO_ERR_WORKSPACE, GRPO_ERR_HIP.
 */
int grpo_token_logp_top(const void* logits, int32_t dtype, int64_t T, int64_t V, int64_t ld, const float* temperature,
                        float temperature_all, const int32_t* actions, int32_t n, float* logp, float* entropy,
                        int32_t* top_ids, float* top_logp, grpo_top_row* rows, int32_t* error_flags, void* ws,
                        size_t ws_bytes, hipStream_t s);

/*
 * The gradient of sum_t dlogp_t log p(a_t) + dentropy_t H_t + sum_j dtop_tj log p(id_tj):
 *   dlogits_v = (c_v - p_v (C + dentropy (log p_v + H))) / tau  on the words, 0 elsewhere,
 *   c_v = dlogp [v = a] + sum_j dtop_j [v = id_j],  C = sum c.
 *   logits, actions, top_ids, rows: as grpo_token_logp_top took and gave them
 *   dlogp        device fp32 [T] or NULL; not looked at where the action is outside [0, V) or masked
 *   dentropy     device fp32 [T] or NULL
 *   dtop         device fp32 [T, n] or NULL; not looked at where the id is outside [0, V)
 *   dlogits      device [T, ld] of `dtype`; columns >= V are not written; may be `logits` itself, and otherwise shares
 *                no element with it (rows of the two may lie in turn)
 * A row with a NaN or +inf, or its temperature out of range, has NaN throughout; a row without words zeros.
 * Errors: GRPO_ERR_ARG (a required pointer NULL, dlogits over part of logits), GRPO_ERR_SHAPE, GRPO_ERR_DTYPE,
 *   GRPO_ERR_ALIGN, GRPO_ERR_HIP.
 */
int grpo_token_logp_top_bwd(const void* logits, int32_t dtype, int64_t T, int64_t V, int64_t ld,
                            const int32_t* actions, int32_t n, const int32_t* top_ids, const grpo_top_row* rows,
                            const float* dlogp, const float* dentropy, const float* dtop, void* dlogits,
                            hipStream_t s);

#ifdef __cplusplus
}
#endif

#endif /* GRPO_TOP_H_ */
