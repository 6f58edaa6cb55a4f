/*
 * skrull_loss.h -- C ABI of the loss at the end of a training step over packed rows: softmax cross entropy
 * of the rows' products with the vocabulary's weight, and its gradients, without keeping the logits.
 *
 * For row t with hidden values x_t, target c_t and the weight's rows w_v, v < vocab:
 *     z_v = x_t . w_v,   lse_t = log sum_v exp(z_v),   loss_t = lse_t - z_{c_t}
 * and for a gradient d_t of loss_t (rows may be weighed as the program likes: by sequence, by token):
 *     dz_v = d_t (exp(z_v - lse_t) - [v = c_t]),   dx_t = sum_v dz_v w_v,   dw_v = sum_t dz_v x_t
 * A row whose target is negative has none (a prompt's tokens, padding): its loss and lse are 0, its dx is 0, it adds nothing to dw,
 * whatever its values are (infinities and NaN too), and no product is formed for it.  A target of vocab or more gives that
 * row a loss of NaN and gradients of NaN.
 *
 * The products run on the matrix cores in bf16 with fp32 sums; logits stay in fp32 registers.  The backward
 * forms them again, in pieces of the vocabulary that fit the workspace, and rounds dz to bf16 (by 2^-8 relative to
 * its value at most, as x and w are; where up to 128 rows have a target, to the sum of two bf16, by 2^-16) for the two products with w and x.
 * dx and dw are summed in fp32 and rounded to bf16 once.
 * No sum depends on the order in which workgroups run: results are bit-reproducible.
 *
 * Tensors are caller-owned DEVICE memory: x bf16 [rows, hidden], row t x_stride elements after row t - 1; w bf16 [vocab, hidden]
 * contiguous, 16-byte aligned; target int64 [rows]; loss, lse, d_loss fp32 [rows]; dx bf16 [rows, hidden] and dw bf16
 * [vocab, hidden] contiguous, 16-byte aligned.
 */
#ifndef SKRULL_LOSS_H
#define SKRULL_LOSS_H

#include <stddef.h>
#include <stdint.h>

#include "skrull_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    int64_t rows;      /* 0..2^24; with no rows nothing but dw is written, as zeros             */
    int32_t hidden;    /* a multiple of 8, 8..65536                                             */
    int32_t vocab;     /* 1..2^22                                                               */
    int64_t x_stride;  /* elements, at least hidden                                             */
} skrull_loss_t;

/* Device scratch in bytes that skrull_loss_fwd (backward = 0) or skrull_loss_bwd (1) asks for with these sizes; 0 where a value is
 * outside the limits. */
int64_t skrull_loss_workspace(const skrull_loss_t *p, int backward);

/*
 * loss and lse of every row.  `workspace`: at least skrull_loss_workspace(p, 0) bytes, 16-byte aligned; contents on entry
 * are ignored, nothing in it is needed afterwards.  Only enqueues on `hip_stream`; allocates nothing, may be captured.  Calls that
 * may overlap need a workspace each.
 * SKRULL_EINVAL: a null or misaligned pointer, a value outside the limits, a workspace that is too small.
 */
int skrull_loss_fwd(const skrull_loss_t *p, const void *x, const void *w, const int64_t *target, float *loss, float *lse,
                    void *workspace, size_t workspace_bytes, void *hip_stream);

/* dx and dw, given the forward's lse; either may be NULL where it is not wanted.  dx may lie where x does (all of x is read before); dx and dw overlap
 * neither w nor each other.  As skrull_loss_fwd otherwise, with skrull_loss_workspace(p, 1) bytes. */
int skrull_loss_bwd(const skrull_loss_t *p, const void *x, const void *w, const int64_t *target, const float *lse, const float *d_loss,
                    void *dx, void *dw, void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SKRULL_LOSS_H */
