// Entry points of attention to a window of keys (include/skrull_window.h): checks, and the launches of fwd.hip and bwd.hip with a window.
#include "ops.h"
#include "skrull_window.h"

namespace {

struct Span {
    const char *name;
    const void *at;
    int64_t bytes;
};
int check_spans(const Span *in, int n_in, const Span *out, int n_out)
{
    for (int i = 0; i < n_in + n_out; ++i) {
        const Span &s = i < n_in ? in[i] : out[i - n_in];
        if (!s.at || !aligned_to(s.at, 16)) return refuse("window: %s is null or misaligned", s.name);
    }
    for (int i = 0; i < n_out; ++i) {
        for (int j = 0; j < n_in; ++j)
            if (overlap(out[i].at, out[i].bytes, in[j].at, in[j].bytes)) return refuse("window: %s overlaps %s", out[i].name, in[j].name);
        for (int j = 0; j < i; ++j)
            if (overlap(out[i].at, out[i].bytes, out[j].at, out[j].bytes)) return refuse("window: %s overlaps %s", out[i].name, out[j].name);
    }
    return SKRULL_OK;
}

int check(const skrull_attn_plan_t *plan, const skrull_window_t *window)
{
    if (!plan || !window) return refuse("window: null pointer");
    if (window->window < 1) return refuse("window: a window of %d keys", window->window);
    if (window->sinks < 0) return refuse("window: %d sinks", window->sinks);
    return SKRULL_OK;
}

// What a launch needs to know.  Where every key is visible, nothing: those of the plain attention do the same with less.
struct Keys {
    KeyWindow window;
    bool all;
    // (positions are below 2^26, so that no sum of a position and one of these passes 32 bits)
    Keys(const skrull_attn_plan_t *plan, const skrull_window_t *w)
        : window{w->window < 1 << 30 ? w->window : 1 << 30, w->sinks < 1 << 30 ? w->sinks : 1 << 30}, all(w->window >= plan->longest_seq || w->sinks >= plan->longest_seq)
    {
    }
    const KeyWindow *get() const { return all ? nullptr : &window; }
};

struct Sizes {
    int64_t q, k, lse;
    explicit Sizes(const skrull_attn_plan_t *p)
        : q((int64_t)p->total_q * p->Hq * p->d * 2), k((int64_t)p->total_k * p->Hkv * p->d * 2), lse((int64_t)p->total_q * p->Hq * 4)
    {
    }
};

}  // namespace

extern "C" {

int skrull_window_fwd(const skrull_attn_plan_t *plan, const skrull_window_t *window, const void *q, const void *k, const void *v, void *o,
                      float *lse, void *hip_stream)
{
    if (int rc = check(plan, window)) return rc;
    const Sizes n(plan);
    const Span in[] = {{"q", q, n.q}, {"k", k, n.k}, {"v", v, n.k}}, out[] = {{"o", o, n.q}, {"lse", lse, n.lse}};
    if (int rc = check_spans(in, 3, out, 2)) return rc;
    if (int rc = plan_on_current_device(plan)) return rc;
    const Keys keys(plan, window);
    const hipError_t e = launch_fwd(plan, q, k, v, o, lse, (hipStream_t)hip_stream, nullptr, keys.get());
    return e == hipSuccess ? SKRULL_OK : launch_failed(e, "window launch");
}

int64_t skrull_window_workspace(const skrull_attn_plan_t *plan, const skrull_window_t *window)
{
    skrull_attn_plan_info_t info;
    if (check(plan, window) != SKRULL_OK || skrull_attn_plan_info(plan, &info) != SKRULL_OK) return 0;
    const Keys keys(plan, window);
    return keys.all ? info.bwd_workspace_bytes : window_workspace(plan, &keys.window);
}

int skrull_window_bwd(const skrull_attn_plan_t *plan, const skrull_window_t *window, const void *q, const void *k, const void *v, const void *o,
                      const float *lse, const void *d_o, void *dq, void *dk, void *dv, void *workspace, size_t workspace_bytes,
                      void *hip_stream)
{
    if (int rc = check(plan, window)) return rc;
    const int64_t bytes = skrull_window_workspace(plan, window);
    if ((int64_t)workspace_bytes < bytes) return refuse("window: workspace below %lld bytes", (long long)bytes);
    const Sizes n(plan);
    const Span in[] = {{"q", q, n.q}, {"k", k, n.k}, {"v", v, n.k}, {"o", o, n.q}, {"lse", lse, n.lse}, {"d_o", d_o, n.q}};
    const Span out[] = {{"dq", dq, n.q}, {"dk", dk, n.k}, {"dv", dv, n.k}, {"workspace", workspace, bytes}};
    if (int rc = check_spans(in, 6, out, 4)) return rc;
    if (int rc = plan_on_current_device(plan)) return rc;
    const Keys keys(plan, window);
    const hipError_t e = launch_bwd(plan, q, k, v, o, lse, d_o, dq, dk, dv, (float *)workspace, (hipStream_t)hip_stream, nullptr, nullptr, keys.get());
    return e == hipSuccess ? SKRULL_OK : launch_failed(e, "window launch");
}

}  // extern "C"
