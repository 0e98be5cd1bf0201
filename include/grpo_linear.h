/*
 * grpo_linear.h -- a product with bias, activation and residual in its epilogue, and its gradient: the policy's logits
 * from hidden states, where they are wanted themselves, and the small blocks in front of a head (libgrpo, gfx950).
 *
 *   z = x W + bias,   y = act(z) + residual,
 *   dz = dy act'(z),  dx = dz W^T,  dW = x^T dz,  dbias = sum over the rows of dz.
 *
 * x, W and dx are bf16, sums are fp32 (on the matrix cores), every result is rounded once.  Conventions (streams, errors,
 * device pointers) are those of grpo.h.
 */
#ifndef GRPO_LINEAR_H_
#define GRPO_LINEAR_H_

#include "grpo.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  GRPO_ACT_NONE = 0,
  GRPO_ACT_RELU = 1,      /* max(z, 0); derivative 0 at 0                                      */
  GRPO_ACT_GELU = 2,      /* z (1 + erf(z / sqrt 2)) / 2                                       */
  GRPO_ACT_GELU_TANH = 3, /* z (1 + tanh(sqrt(2 / pi) (z + 0.044715 z^3))) / 2                 */
  GRPO_ACT_SILU = 4       /* z / (1 + e^-z)                                                    */
} grpo_act;

/* The operator and its inputs. */
typedef struct {
  int64_t M, K, N;    /* 0 <= M, 1 <= K, N; each <= 8,388,352                                  */
  const void* x;      /* device bf16 [M, K], rows ldx elements apart                           */
  int64_t ldx;
  const void* w;      /* device bf16 [K, N], or with w_out_in [N, K], rows ldw elements apart  */
  int64_t ldw;
  int32_t w_out_in;   /* 0 or 1                                                                */
  int32_t act;        /* grpo_act                                                              */
  const void* bias;   /* device [N] of bias_dtype, or NULL; the backward call does not read it */
  int32_t bias_dtype; /* GRPO_F32 or GRPO_BF16, where bias or dbias is given                   */
} grpo_linear_op;

/* Bytes of device workspace grpo_linear needs, which go by the sizes and by how x and W lie (aligned to 16 bytes, rows of
 * multiples of 8 elements, or not); 0 for none and for an invalid operator. */
size_t grpo_linear_workspace_bytes(const grpo_linear_op* op);

/*
 * y = act(x W + bias) + residual.
 *   op           host struct (above)
 *   residual     device [M, N] of y's type, rows ldr apart, or NULL; may be y itself (ldr = ldy)
 *   y            device [M, N] of y_dtype (GRPO_F32 or GRPO_BF16), rows ldy apart; shares no element with x, w or bias, nor
 *                with a residual that is not y itself (rows of two operands may lie in turn)
 *   z            device fp32 [M, N], contiguous, or NULL: z, which the backward call takes unless act is GRPO_ACT_NONE; shares
 *                no element with another operand
 *   ws, ws_bytes device workspace of at least grpo_linear_workspace_bytes(op), 16-byte aligned; calls that may overlap (on
 *                two streams, in two graphs) need one each
 * The same inputs give the same bits.
 * Errors: GRPO_ERR_ARG (NULL pointer, act or w_out_in unknown, operands that share elements), GRPO_ERR_SHAPE (a size outside
 *   its range, rows closer than their length), GRPO_ERR_DTYPE, GRPO_ERR_ALIGN (a pointer not aligned to its element),
 *   GRPO_ERR_WORKSPACE, GRPO_ERR_HIP.
 */
int grpo_linear(const grpo_linear_op* op, const void* residual, int64_t ldr, void* y, int64_t ldy, int32_t y_dtype,
                float* z, void* ws, size_t ws_bytes, hipStream_t s);

/* What the backward call writes; each may be NULL. */
typedef struct {
  void* dx;              /* device bf16 [M, K], contiguous                                            */
  void* dw;              /* device [K, N], or with w_out_in [N, K], contiguous                        */
  void* dbias;           /* device [N] of op->bias_dtype                                              */
  int32_t dw_dtype;      /* GRPO_F32 or GRPO_BF16                                                     */
  int32_t accumulate_dw; /* 1 (fp32 dw alone): dw += x^T dz                                           */
} grpo_linear_grads;

/* Bytes of device workspace grpo_linear_bwd needs for these arguments. */
size_t grpo_linear_bwd_workspace_bytes(const grpo_linear_op* op, const void* dy, int64_t lddy, int32_t dy_dtype,
                                       const grpo_linear_grads* grads);

/*
 * The gradients.  dz is formed in fp32 and rounded to bf16 for the two products (an error of half a step in each term of
 * sums over N or M); dbias is summed from dz as it is before that.
 *   op           as the forward call took it
 *   dy           device [M, N] of dy_dtype (GRPO_F32 or GRPO_BF16), rows lddy apart
 *   z            device fp32 [M, N]: what grpo_linear stored; NULL where act is GRPO_ACT_NONE
 *   grads        host struct (above); its arrays share no element with one another or with an input that the call reads
 *                (dy; z; x for dw; w for dx)
 *   ws, ws_bytes device workspace of at least grpo_linear_bwd_workspace_bytes(...), as above
 * With M = 0 dw and dbias are zeros (dw as it was with accumulate_dw).
 * Errors: as grpo_linear, and GRPO_ERR_ARG for z NULL with an activation, or accumulate_dw with a bf16 dw.
 */
int grpo_linear_bwd(const grpo_linear_op* op, const void* dy, int64_t lddy, int32_t dy_dtype, const float* z,
                    const grpo_linear_grads* grads, void* ws, size_t ws_bytes, hipStream_t s);

#ifdef __cplusplus
}
#endif

#endif /* GRPO_LINEAR_H_ */
