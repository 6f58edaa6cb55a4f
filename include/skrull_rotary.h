/*
 * skrull_rotary.h -- C ABI of the rotary positions of a micro-batch's packed rows: Q and K are turned
 * by the positions that the plan's sequences, slices and chunks give their rows, before
 * skrull_attn_fwd; their gradients are turned back after skrull_attn_bwd.
 *
 * A row at position p of its sequence has, in every head, pairs (a, b) of elements that become
 *     a' = amplitude * (a cos t - b sin t),   b' = amplitude * (a sin t + b cos t),   t = p * f_i
 * for pair i of rotary_dim / 2 (inverse: sin has the other sign, which is the transposed map, as a gradient
 * needs it).  Elements from rotary_dim on stay as they are.  Pair i is elements
 *   SKRULL_ROTARY_HALF         i and i + rotary_dim / 2
 *   SKRULL_ROTARY_INTERLEAVED  2 i and 2 i + 1
 * and its frequency, in radians per position, base^(-2 i / rotary_dim), for contexts longer than the model was made for scaled:
 *   SKRULL_ROTARY_PLAIN   as it is
 *   SKRULL_ROTARY_LINEAR  f_i / factor
 *   SKRULL_ROTARY_NTK     with the base times factor^(r / (r - 2)), r = rotary_dim: the first pair keeps its frequency, the
 *                         last one's is divided by factor
 *   SKRULL_ROTARY_PARTS   by the turns n_i = original_length * f_i / (2 pi) that the pair makes in the original length:
 *                         f_i * (g + (1 - g) / factor) with g = (n_i - low_turns) / (high_turns - low_turns) within 0 and 1
 * The angle's whole turns are taken off in 64 bits (an angle of 131,072 radians has steps of 0.008 in 32), its sine and cosine
 * and the products are formed in 32 bits, the result is rounded to bf16 once.
 */
#ifndef SKRULL_ROTARY_H
#define SKRULL_ROTARY_H

#include <stdint.h>

#include "skrull_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SKRULL_ROTARY_HALF        0
#define SKRULL_ROTARY_INTERLEAVED 1

#define SKRULL_ROTARY_PLAIN  0
#define SKRULL_ROTARY_LINEAR 1
#define SKRULL_ROTARY_NTK    2
#define SKRULL_ROTARY_PARTS  3

typedef struct {
    int32_t head_dim;         /* 64 or 128, the plan's                                             */
    int32_t rotary_dim;       /* elements that are turned: a multiple of 16, 16..head_dim          */
    int32_t layout;           /* SKRULL_ROTARY_HALF or _INTERLEAVED                                */
    int32_t scaling;          /* SKRULL_ROTARY_PLAIN, _LINEAR, _NTK or _PARTS                      */
    double  base;             /* finite, > 1                                                       */
    double  factor;           /* finite, >= 1; 1 with _PLAIN                                       */
    double  original_length;  /* _PARTS: finite, > 0                                               */
    double  low_turns, high_turns; /* _PARTS: finite, 0 <= low_turns < high_turns                  */
    double  amplitude;        /* finite, > 0; 1 for none                                           */
} skrull_rotary_t;

/* Which rows of the micro-batch a tensor holds. */
#define SKRULL_ROWS_Q 0  /* total_q rows: this rank's own tokens (Q, and K before the ranks exchange it)   */
#define SKRULL_ROWS_K 1  /* total_k rows: the gathered prefixes, positions 0..kv_len-1 of each             */

/* One tensor: `rows` of the plan's, each with `heads` heads of head_dim contiguous bf16.  Row r begins `stride` elements after row
 * r - 1, so a tensor may be part of the rows of a larger one (a projection's Q, K and V side by side). */
typedef struct {
    const void *in;     /* DEVICE, 16-byte aligned                                                 */
    void       *out;    /* DEVICE, 16-byte aligned; `in` itself, with the same stride, or memory that does not overlap it */
    int64_t     in_stride, out_stride; /* elements: multiples of 8, at least heads * head_dim       */
    int32_t     heads;  /* 1..4096                                                                 */
    int32_t     rows;   /* SKRULL_ROWS_Q or SKRULL_ROWS_K                                          */
} skrull_rotary_tensor_t;

/* Whether `rotary` is within the limits above: SKRULL_OK or SKRULL_EINVAL (skrull_attn_strerror names the field). */
int skrull_rotary_check(const skrull_rotary_t *rotary);

/*
 * Turn one or two tensors of `plan`'s rows (`second` may be NULL); neither's `out` may hold elements of the other one's tensors.
 * Bytes between the rows of `out` stay as they were.  Only enqueues one kernel on `hip_stream`; allocates nothing, may be captured.
 * Calls may overlap where their tensors do not.
 * SKRULL_EINVAL: a null pointer, a value outside the limits above, rotary->head_dim other than the plan's, `out` that overlaps `in`
 * otherwise, or the current device not the one the plan was made on.
 */
int skrull_rotary(const skrull_attn_plan_t *plan, const skrull_rotary_t *rotary, const skrull_rotary_tensor_t *first,
                  const skrull_rotary_tensor_t *second, int inverse, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SKRULL_ROTARY_H */
