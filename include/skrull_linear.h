/*
 * skrull_linear.h -- C ABI of the product of packed rows and a weight with what follows it in a block: bias, activation, gate and residual, forward and
 * backward.
 *
 * For rows x [rows, inputs], a weight w [n, inputs] and a bias b [n] (absent: 0), with f the activation,
 *     z = x w^T + b,     y = f(z) + residual                                          n = outputs
 *     gated:             y = f(z_1) * z_2 + residual, z_1 and z_2 the two halves of z  n = 2 outputs
 * and for a gradient dy, with dz = dy * f'(z) (gated: dy * z_2 * f'(z_1) and dy * f(z_1)):
 *     dx = dz w,     dw = dz^T x,     db = sum over rows of dz       (and the residual's gradient is dy)
 * Everything but the operands of products is held in fp32, and y, dx, dw and db are rounded once; what the backward reads of z is rounded to bf16 by the
 * forward, and dz before the products that it goes into.  Sums are taken in an order that the sizes alone decide: results are bit-reproducible.
 *
 * f is one of: z; max(z, 0) (f' = 0 at 0); z P(z) with P(z) the normal distribution's share below z; z / (1 + e^-z).
 *
 * Tensors are caller-owned DEVICE memory, bf16 and 16-byte aligned.  Rows of x, residual, y and dy begin `stride` elements apart, a multiple of 8; everything else is
 * contiguous.  Values are to be finite; a NaN in z gives one in y, and in dz wherever that depends on z (f = z without a gate: dz is dy).
 */
#ifndef SKRULL_LINEAR_H
#define SKRULL_LINEAR_H

#include <stddef.h>
#include <stdint.h>

#include "skrull_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SKRULL_LINEAR_NONE 0
#define SKRULL_LINEAR_RELU 1
#define SKRULL_LINEAR_GELU 2
#define SKRULL_LINEAR_SILU 3

typedef struct {
    int64_t rows;        /* 0..2^24; with no rows nothing but dw and db is written, as zeros                 */
    int32_t inputs;      /* a multiple of 8 from 8 to 65,536                                                 */
    int32_t outputs;     /* likewise; gated: (outputs + 256) * inputs below 2^30                             */
    int32_t activation;  /* SKRULL_LINEAR_*                                                                  */
    int32_t gated;       /* 0 or 1: of the first half of z, times the second                                 */
    int64_t x_stride, residual_stride, y_stride, dy_stride;  /* multiples of 8 from the width to 2^20; those of a call's tensors are read */
} skrull_linear_t;

/* Device scratch that skrull_linear_fwd or (`backward` not 0) skrull_linear_bwd asks for with these sizes, in bytes; -1 where a value is outside the limits. */
int64_t skrull_linear_workspace(const skrull_linear_t *p, int backward);

/*
 * Forward.  b and residual may be NULL.  z [rows, n], what the backward needs of an activation or a gate, may be NULL.  y may be the residual itself, with the same
 * stride; nothing else that is written may overlap anything.  `workspace`: at least skrull_linear_workspace bytes, 16-byte aligned (may be
 * NULL where that is 0); contents on entry are ignored.  Only enqueues on `hip_stream`; allocates nothing, may be captured.  Calls that may overlap need a
 * workspace each.
 * SKRULL_EINVAL: a null or misaligned pointer, a value outside the limits.
 */
int skrull_linear_fwd(const skrull_linear_t *p, const void *x, const void *w, const void *b, const void *residual, void *y, void *z,
                      void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Backward, given x, w, dy and the forward's z (NULL with SKRULL_LINEAR_NONE that is not gated).  dx, dw and db may be NULL where they are not wanted.  Otherwise as the
 * forward.
 */
int skrull_linear_bwd(const skrull_linear_t *p, const void *x, const void *w, const void *z, const void *dy, void *dx, void *dw, void *db,
                      void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SKRULL_LINEAR_H */
