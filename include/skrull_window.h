/*
 * skrull_window.h -- C ABI of attention to a window of keys: packed varlen causal attention as skrull_attn.h has it, on the same plans, where a
 * query sees only the last keys before it and, if asked for, the first ones of its sequence (sinks).
 *
 * The key at position j of a sequence is visible to the query at position p of it if
 *     j <= p  and  (p - j < window  or  j < sinks).
 * Positions are the plan's: of whole sequences and of a rank's slices of distributed ones, whose K and V are the gathered prefixes from position 0 on.
 * O, LSE and the gradients are those of skrull_attn_fwd and skrull_attn_bwd over the visible keys.  The gradient of a key that
 * no query of this rank sees is zero, and is written.  Work and traffic are those of the visible keys, up to tiles of 64.
 *
 * Layouts, types and limits of the tensors are skrull_attn.h's.  A window of at least the longest sequence gives skrull_attn_fwd's results, up to
 * roundings.  Values are to be finite: an infinity or NaN in a hidden key of a tile that also has visible ones may reach a row, as in skrull_attn_fwd.
 */
#ifndef SKRULL_WINDOW_H
#define SKRULL_WINDOW_H

#include <stddef.h>
#include <stdint.h>

#include "skrull_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    int32_t window;  /* keys that a query sees up to its own, >= 1                      */
    int32_t sinks;   /* first keys of its sequence that it sees besides (if any), >= 0  */
} skrull_window_t;

/*
 * Forward: O [total_q, Hq, d] bf16 and LSE [Hq, total_q] fp32, as skrull_attn_fwd.  O and LSE must not overlap Q, K, V or each other.  Only enqueues on
 * `hip_stream`; allocates nothing, may be captured.
 * SKRULL_EINVAL: a null pointer, one that is not 16-byte aligned, a value outside the limits, a plan of another device.
 */
int skrull_window_fwd(const skrull_attn_plan_t *plan, const skrull_window_t *window, const void *q, const void *k, const void *v, void *o,
                      float *lse, void *hip_stream);

/* Device scratch that skrull_window_bwd asks for, in bytes; 0 where the plan is null or a value is outside the limits. */
int64_t skrull_window_workspace(const skrull_attn_plan_t *plan, const skrull_window_t *window);

/*
 * Backward, given the forward's inputs, O and LSE: dQ, dK and dV, every row of them, which must overlap no input and not each other.  `workspace`: at least
 * skrull_window_workspace bytes, 16-byte aligned; contents on entry are ignored.  Only enqueues on `hip_stream`; allocates nothing, may
 * be captured.  Calls that may overlap need a workspace each.
 */
int skrull_window_bwd(const skrull_attn_plan_t *plan, const skrull_window_t *window, const void *q, const void *k, const void *v, const void *o,
                      const float *lse, const void *d_o, void *dq, void *dk, void *dv, void *workspace, size_t workspace_bytes,
                      void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SKRULL_WINDOW_H */
