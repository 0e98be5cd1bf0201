/*
 * grpo_clip.h -- the gradients' common norm and their clipping to it, the last
 * step of an update before the optimizer (libgrpo, gfx950).
 *
 *   norm = sqrt( sum over all tensors of sum g^2 ),
 *   f = min(1, max_norm / (norm + GRPO_CLIP_EPS)),   out = f g.
 *
 * The tensors are described once, in a table that the caller builds on the host
 * and copies to the device, and every later call takes them together: one launch
 * for the norm and one for the clipping, whatever their number.  Conventions
 * (streams, errors, device pointers) are those of grpo.h.
 */
#ifndef GRPO_CLIP_H_
#define GRPO_CLIP_H_

#include "grpo.h"

#ifdef __cplusplus
extern "C" {
#endif

#define GRPO_CLIP_EPS 1e-6

/* Slots of the sum of squares that grpo_grad_sumsq writes and grpo_grad_clip adds up. */
#define GRPO_GRAD_PARTIALS 2048

/* A gradient and where its clipped values go.  Both are contiguous, aligned to their element size. */
typedef struct {
  void* data;        /* device, n elements of `dtype`                                          */
  void* out;         /* device, n elements of `out_dtype`; `data` itself = in place            */
  int64_t n;         /* 0 <= n < 2^40                                                          */
  int32_t dtype;     /* GRPO_F32 or GRPO_BF16                                                  */
  int32_t out_dtype; /* GRPO_F32 or GRPO_BF16; `dtype` where out = data                        */
} grpo_grad;

/* What the host has to know of a table. */
typedef struct {
  int32_t n;        /* tensors in it                                      */
  int32_t in_place; /* 1 where every out is its data                      */
  int64_t units;    /* pieces of work, each of at most 8192 elements      */
  int64_t bytes;    /* of all data                                        */
} grpo_grad_layout;

/* Bytes of the table of n tensors, 0 for n < 0 or n > 2^20. */
size_t grpo_grad_table_bytes(int32_t n);

/*
 * Builds the table of `n` tensors in host memory; touches no device.  The caller copies `table_bytes` bytes of it to
 * the device (8-byte aligned there) before the first call that takes it, and keeps the layout.
 *   grads        host [n]
 *   table        host, at least grpo_grad_table_bytes(n) bytes, 8-byte aligned
 *   layout       host (written)
 * Errors: GRPO_ERR_ARG (NULL pointer; data or out NULL with n > 0; out = data with another type), GRPO_ERR_SHAPE (n
 *   outside 0 .. 2^20, a size outside its range, more than 2^31 - 1 units; an out that overlaps another tensor's data or
 *   out, or its own data without being it), GRPO_ERR_DTYPE, GRPO_ERR_ALIGN, GRPO_ERR_WORKSPACE (table_bytes).
 *   Gradients may overlap one another where they are only read; each then counts.
 */
int grpo_grad_table(const grpo_grad* grads, int32_t n, void* table, size_t table_bytes, grpo_grad_layout* layout);

/*
 * The sum of squares of all gradients, in GRPO_GRAD_PARTIALS slots whose sum it is (summed in fp64, in an order that the
 * sizes alone give: bitwise reproducible).  Devices that hold different gradients of one model add their slots (an
 * all-reduce over the 2048 numbers) before each clips its own.
 *   layout       host; table device: as grpo_grad_table built them
 *   partials     device fp64 [GRPO_GRAD_PARTIALS] (written)
 * Errors: GRPO_ERR_ARG, GRPO_ERR_ALIGN (table or partials not 8-byte aligned), GRPO_ERR_HIP.
 */
int grpo_grad_sumsq(const grpo_grad_layout* layout, const void* table, double* partials, hipStream_t s);

/*
 * The norm from the slots, and every gradient times f, formed in fp32 and rounded once to its out's type.
 *   max_norm     >= 0 (+inf: nothing is scaled)
 *   norm_out     device fp32 [1] or NULL: the norm (+inf beyond fp32's range: f is formed from the fp64 norm)
 *   error_flags  device int32 [1] or NULL: overwritten with GRPO_FLAG_NONFINITE when the norm is not finite
 * A norm that is not finite leaves f at 1: the gradients are as they were, and norm_out says that the step is to be
 * skipped.  Where f = 1, gradients clipped in place are not touched.
 * Errors: GRPO_ERR_ARG (NULL pointer, max_norm < 0 or NaN), GRPO_ERR_ALIGN, GRPO_ERR_HIP.
 */
int grpo_grad_clip(const grpo_grad_layout* layout, const void* table, const double* partials, double max_norm,
                   float* norm_out, int32_t* error_flags, hipStream_t s);

#ifdef __cplusplus
}
#endif

#endif /* GRPO_CLIP_H_ */
