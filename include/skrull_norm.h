/*
 * skrull_norm.h -- C ABI of the norm of packed rows, forward and backward: layer norm, and its form
 * without a mean (root mean square).
 *
 * For a row x of `cols` elements, with w the weight and b the bias (absent, or of SKRULL_NORM_LAYER):
 *     m    = sum x / cols                      (SKRULL_NORM_RMS: 0)
 *     rstd = 1 / sqrt(sum (x - m)^2 / cols + eps)
 *     h    = (x - m) * rstd,     y = h * w + b
 * and for a gradient dy, with g = dy * w:
 *     dx = rstd * (g - mean(g) - h * mean(g * h))   (SKRULL_NORM_RMS: without mean(g))
 *     dw = sum over rows of dy * h,   db = sum over rows of dy
 * All sums are held in fp32, in an order that the sizes alone decide: results are bit-reproducible.  y and dx are
 * rounded once to the type of x, dw and db to the type of w.
 *
 * Tensors are caller-owned DEVICE memory, x, y, dy and dx of one type (`type`), w, b, dw and db of one
 * (`weight_type`).  Rows of a tensor begin `stride` elements apart and are contiguous within; rows of any alignment, width and stride are taken.
 */
#ifndef SKRULL_NORM_H
#define SKRULL_NORM_H

#include <stddef.h>
#include <stdint.h>

#include "skrull_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SKRULL_NORM_RMS   0
#define SKRULL_NORM_LAYER 1

#define SKRULL_TYPE_BF16 0
#define SKRULL_TYPE_FP32 1

#define SKRULL_NORM_MAX_COLS 8192

typedef struct {
    int64_t rows;         /* 0..2^31-1; with no rows nothing but dw and db is written, as zeros */
    int32_t cols;         /* 1..SKRULL_NORM_MAX_COLS                                         */
    int32_t kind;         /* SKRULL_NORM_RMS or SKRULL_NORM_LAYER                            */
    int32_t type;         /* of x, y, dy, dx                                                 */
    int32_t weight_type;  /* of w, b, dw, db                                                 */
    float   eps;          /* finite, >= 0                                                    */
    int64_t x_stride, y_stride, dy_stride, dx_stride;  /* elements, at least cols; those of a call's tensors are read */
} skrull_norm_t;

/*
 * Forward.  b may be NULL.  mean (which may be NULL, and is not written, with SKRULL_NORM_RMS) and rstd, [rows] fp32, are what the backward
 * needs; both may be NULL.  y may be x itself with the same stride, or must not overlap it.  Only enqueues on `hip_stream`; allocates nothing, may be captured.
 * SKRULL_EINVAL: a null pointer, a pointer that is not a multiple of its type's size, a value outside the limits.
 */
int skrull_norm_fwd(const skrull_norm_t *p, const void *x, const void *w, const void *b, void *y, float *mean, float *rstd, void *hip_stream);

/* Device scratch that skrull_norm_bwd asks for with these sizes, in bytes; 0 where a value is outside the limits. */
int64_t skrull_norm_workspace(const skrull_norm_t *p);

/*
 * Backward, given x, w, dy and the forward's mean (ignored with SKRULL_NORM_RMS) and rstd.  dw and db may be NULL where they are not
 * wanted.  dx may be dy itself (or x) with the same stride, or must overlap neither.  `workspace`: at least
 * skrull_norm_workspace bytes, 16-byte aligned (may be NULL where neither dw nor db is wanted); contents on entry are ignored.
 * Only enqueues on `hip_stream`; allocates nothing, may be captured.  Calls that may overlap need a workspace each.
 */
int skrull_norm_bwd(const skrull_norm_t *p, const void *x, const void *w, const float *mean, const float *rstd, const void *dy,
                    void *dx, void *dw, void *db, void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SKRULL_NORM_H */
