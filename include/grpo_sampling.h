/*
 * grpo_sampling.h -- the policy as a rollout samples from it: actions drawn from
 * a row's logits under temperature, top-k, top-p and min-p, the log-prob of a
 * given action under that distribution, and its gradient (libgrpo, gfx950).
 *
 * The sampling distribution of a row z_0 .. z_(V-1) at temperature tau:
 *   words that take part   those with z > -1e8 (as everywhere in this library, a lower
 *                          logit is a masked word), ordered by z from the largest down,
 *                          equal ones by their index from the lowest up
 *   top_k  = k > 0         the first k of them remain
 *   top_p  = p < 1         of these, with weights w = exp((z - max z) / tau), the
 *                          shortest prefix whose weights sum to at least p of the
 *                          remaining words' sum (never less than one word)
 *   min_p  > 0             of these, the ones with w >= min_p
 *   tau    = 0             the first word alone, with log-prob 0
 * What is kept is a prefix of the order: P(a) = w_a / S, S the sum over the kept words.
 * Which words are kept, and which one is drawn, is decided on weights and sums in fp64.
 *
 * Conventions (streams, errors, device pointers) are those of grpo.h.
 */
#ifndef GRPO_SAMPLING_H_
#define GRPO_SAMPLING_H_

#include "grpo.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A further bit of error_flags: a row's setting is out of its range, or its u outside [0, 1).  That row's outputs are
 * those of a row with a NaN. */
#define GRPO_FLAG_SETTING 8

/* The largest vocabulary these entry points take (2^22). */
#define GRPO_SAMPLING_MAX_V 4194304

/* The settings of a call: for each, a device array [T] with one value for each row, or NULL and one value for all. */
typedef struct {
  const float* temperature; /* device [T] or NULL                                  */
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  float temperature_all;    /* 0, or 1e-6 .. 1e6                                   */
  int32_t top_k_all;        /* <= 0: off                                           */
  float top_p_all;          /* 0 .. 1, 1: off                                      */
  float min_p_all;          /* 0 .. 1, 0: off                                      */
} grpo_sampling;

/* What a row's distribution comes to: word v is kept where z_v > threshold, or z_v = threshold and v <= tie. */
typedef struct {
  double sum;        /* S; NaN for a row with a NaN, +inf or a setting out of range  */
  float max;         /* max z                                                        */
  float threshold;   /* +inf where nothing is kept                                   */
  int32_t tie;
  int32_t n_kept;    /* the number of kept words                                     */
  float temperature; /* tau                                                          */
  float logp;        /* the action's log-prob                                        */
} grpo_sampling_row;

/* Bytes of device workspace grpo_sample and grpo_sampled_logp need: 0 from 192 rows on or up to 16,384 words (ws may then
 * be NULL), and for invalid sizes. */
size_t grpo_sampling_workspace_bytes(int64_t T, int64_t V);

/*
 * Draws one action per row: the first kept word a, by index, with sum_(v <= a, kept) w_v > u S (the last kept word of
 * non-zero weight where rounding leaves none).
 *   logits       device [T, ld] of `dtype`, columns >= V unread
 *   0 <= T < 2^31, 1 <= V <= GRPO_SAMPLING_MAX_V, V <= ld
 *   par          host struct (above)
 *   u            device fp32 [T], uniform random numbers in [0, 1)
 *   actions      device int32 [T]
 *   logp         device fp32 [T] or NULL: log P(a), what the loss takes as behave_logp of rollouts at temperature 1
 *                with nothing cut off
 *   n_kept       device int32 [T] or NULL
 *   error_flags  device int32 [1] or NULL, overwritten
 *   ws, ws_bytes device workspace of at least grpo_sampling_workspace_bytes(T, V), 16-byte aligned; calls that may
 *                overlap (on two streams, in two graphs) need one each
 * A row with a NaN or +inf: action -1, log-prob NaN, n_kept 0, GRPO_FLAG_NONFINITE.  A row with nothing above -1e8:
 * action -1, log-prob -inf, n_kept 0, GRPO_FLAG_NONFINITE.  The same inputs give the same bits.
 * Errors: GRPO_ERR_ARG (a required pointer NULL, an `_all` value out of range), GRPO_ERR_SHAPE, GRPO_ERR_DTYPE,
 *   GRPO_ERR_ALIGN (logits and arrays to their element, ws to 16), GRPO_ERR_WORKSPACE, GRPO_ERR_HIP.
 */
int grpo_sample(const void* logits, int32_t dtype, int64_t T, int64_t V, int64_t ld, const grpo_sampling* par,
                const float* u, int32_t* actions, float* logp, int32_t* n_kept, int32_t* error_flags, void* ws,
                size_t ws_bytes, hipStream_t s);

/*
 * The log-prob of given actions under the sampling distribution.
 *   actions      device int32 [T]
 *   logp         device fp32 [T] or NULL: log P(a_t); -inf for a word that is not kept; 0 where a_t is outside [0, V)
 *                (GRPO_FLAG_ACTION)
 *   n_kept       device int32 [T] or NULL
 *   rows         device grpo_sampling_row [T] or NULL, 8-byte aligned: what the backward call takes
 *   other arguments, rows without a distribution and errors as grpo_sample (u is not needed)
 */
int grpo_sampled_logp(const void* logits, int32_t dtype, int64_t T, int64_t V, int64_t ld, const grpo_sampling* par,
                      const int32_t* actions, float* logp, int32_t* n_kept, grpo_sampling_row* rows,
                      int32_t* error_flags, void* ws, size_t ws_bytes, hipStream_t s);

/*
 * Its gradient: dlogits_v = dlogp_t / tau_t ([v = a_t] - [v kept] P(v)).  The kept set is a constant of the derivative.
 * A row whose action is not kept or out of range, or whose temperature is 0, has no gradient (zeros, whatever dlogp);
 * a row with a NaN or +inf has NaN throughout.
 *   rows         device [T], from grpo_sampled_logp on the same logits and actions
 *   dlogp        device fp32 [T]
 *   dlogits      device [T, ld] of `dtype`; columns >= V are not written; may be `logits` itself, and otherwise shares
 *                no element with it (rows of the two may lie in turn)
 * Errors: GRPO_ERR_ARG (a pointer NULL, dlogits over part of logits), GRPO_ERR_SHAPE, GRPO_ERR_DTYPE, GRPO_ERR_ALIGN,
 *   GRPO_ERR_HIP.
 */
int grpo_sampled_logp_bwd(const void* logits, int32_t dtype, int64_t T, int64_t V, int64_t ld,
                          const int32_t* actions, const grpo_sampling_row* rows, const float* dlogp, void* dlogits,
                          hipStream_t s);

#ifdef __cplusplus
}
#endif

#endif /* GRPO_SAMPLING_H_ */
