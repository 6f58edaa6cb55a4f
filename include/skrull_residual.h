/*
 * skrull_residual.h -- C ABI of the residual stream between two blocks, forward and backward: a block's output z, itself normed
 * and gated where the model does that, added to the scaled stream r, and the norm of the sum for the next block.
 *
 * For a row of `cols` elements, with norm(x) = (x - m) * rstd the norm of skrull_norm.h (of one `kind` and `eps` for both):
 *     n     = norm(z) * post_w + post_b     (post_w NULL: z itself)
 *     r_out = scale * r + gate * n          (gate [cols], NULL: 1)
 *     y     = norm(r_out) * w + b
 * and for gradients d_r_out of the stream and dy, with h1 = norm(z) (z, without post_w) and h2 = norm(r_out):
 *     g2 = dy * w,     e  = d_r_out + rstd2 * (g2 - mean(g2) - h2 * mean(g2 * h2))     (SKRULL_NORM_RMS: without mean(g2))
 *     dr = scale * e,  dn = gate * e,  dz = rstd1 * (g1 - mean(g1) - h1 * mean(g1 * h1)) with g1 = dn * post_w   (dz = dn without post_w)
 * and, summed over rows,
 *     dw = dy * h2,  db = dy,  dgate = e * n,  dpost_w = dn * h1,  dpost_b = dn.
 * y is formed from the sum before that is rounded to r_out; the backward forms it anew from r and z.  All sums are held in fp32, in an
 * order that the sizes alone decide: results are bit-reproducible, and each is rounded once, to its tensor's type.
 *
 * Tensors are caller-owned DEVICE memory: z, y and their gradients of one type, r, r_out and theirs of another (or the same), vectors and
 * theirs of one.  Rows of a tensor begin `stride` elements apart and are contiguous within; rows of any alignment, width and stride are taken.
 */
#ifndef SKRULL_RESIDUAL_H
#define SKRULL_RESIDUAL_H

#include <stddef.h>
#include <stdint.h>

#include "skrull_norm.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    int64_t rows;          /* 0..2^31-1; with no rows nothing but the vectors' gradients is written, as zeros */
    int32_t cols;          /* 1..SKRULL_NORM_MAX_COLS                                                         */
    int32_t kind;          /* SKRULL_NORM_RMS or SKRULL_NORM_LAYER                                            */
    int32_t type;          /* of z, y, dy, dz: SKRULL_TYPE_BF16 or _FP32                                      */
    int32_t residual_type; /* of r, r_out, d_r_out, dr: `type` or SKRULL_TYPE_FP32                            */
    int32_t weight_type;   /* of w, b, post_w, post_b, gate and their gradients                               */
    float   eps;           /* finite, >= 0                                                                    */
    float   scale;         /* finite                                                                          */
    int64_t r_stride, z_stride, r_out_stride, y_stride;     /* elements, at least cols; those of a call's tensors are read */
    int64_t d_r_out_stride, dy_stride, dr_stride, dz_stride;
} skrull_residual_t;

/*
 * Forward.  b, post_w, post_b (only with post_w) and gate may be NULL; there are no biases with SKRULL_NORM_RMS.  stats, [4][rows] fp32 (mean and rstd of z's norm,
 * mean and rstd of the sum's), is what the backward needs, and may be NULL; rows of it that the kind or a missing post_w leaves out
 * are not written.  r_out may be r itself and y may be z itself, with the same stride; nothing else that is written may overlap anything.  Only
 * enqueues on `hip_stream`; allocates nothing, may be captured.
 * SKRULL_EINVAL: a null pointer, a pointer that is not a multiple of its type's size, a value outside the limits.
 */
int skrull_residual_fwd(const skrull_residual_t *p, const void *r, const void *z, const void *w, const void *b, const void *post_w,
                        const void *post_b, const void *gate, void *r_out, void *y, float *stats, void *hip_stream);

/* Device scratch that skrull_residual_bwd asks for with these sizes, in bytes; 0 where a value is outside the limits. */
int64_t skrull_residual_workspace(const skrull_residual_t *p);

/*
 * Backward, given the forward's inputs and stats.  d_r_out or dy may be NULL: no gradient comes that way.  Any of the vectors' gradients may be NULL
 * where it is not wanted.  dr and dz must overlap nothing.  `workspace`: at least skrull_residual_workspace bytes, 16-byte aligned (may be NULL
 * where no vector's gradient is wanted); contents on entry are ignored.  Only enqueues on `hip_stream`; allocates nothing, may be
 * captured.  Calls that may overlap need a workspace each.
 */
int skrull_residual_bwd(const skrull_residual_t *p, const void *r, const void *z, const void *w, const void *post_w, const void *post_b,
                        const void *gate, const float *stats, const void *d_r_out, const void *dy, void *dr, void *dz, void *dw, void *db,
                        void *dpost_w, void *dpost_b, void *dgate, void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SKRULL_RESIDUAL_H */
