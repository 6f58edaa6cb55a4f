// Internal declarations of the operators around attention (rotary.hip, norm.hip, loss.hip).
#pragma once

#include "common.h"

// api.hip
// The calling thread's error text (skrull_attn_strerror appends it); returns SKRULL_EINVAL.
__attribute__((format(printf, 1, 2))) int refuse(const char *format, ...);
int launch_failed(hipError_t e, const char *what);
// Compute units of the current device, or the code of why there is none that can be used.  Looked up once per device.
int current_device(int *compute_units);
// SKRULL_EINVAL where the plan was made on another device.
int plan_on_current_device(const skrull_attn_plan_t *plan);

inline bool aligned_to(const void *p, uintptr_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

// Whether [a, a + a_bytes) and [b, b + b_bytes) have a byte in common.
inline bool overlap(const void *a, int64_t a_bytes, const void *b, int64_t b_bytes)
{
    return (uintptr_t)a < (uintptr_t)b + (uintptr_t)b_bytes && (uintptr_t)b < (uintptr_t)a + (uintptr_t)a_bytes;
}
