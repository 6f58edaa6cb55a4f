// The differentiable calls of the package (autograd.py) in native code: checks, output tensors and bookkeeping around
// skrull_attn_fwd and skrull_attn_bwd.  A pass of 932 tokens, 4/4 heads of 64, forward and gradients, takes the GPU 34 us;
// written in Python the calls around it kept the host busy for 50 us in a process whose threads run close to each other and
// 107 in one where they do not (the backward runs in a thread of the autograd engine, and every Python object it touches
// moves between the two).  36 and 70 this way; torch's own a + b and its gradient take 30 and 42.

#include <Python.h>

#include <ATen/ATen.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <memory>

#include "skrull_attn.h"
#include "skrull_loss.h"
#include "skrull_norm.h"
#include "skrull_rotary.h"

namespace {

using torch::autograd::AutogradContext;
using torch::autograd::Variable;
using torch::autograd::variable_list;

PyObject *g_check = nullptr;  // binding._check: raises what an error code stands for

// A binding.Plan, kept by the graph.  Its handle is read when it is needed: the program may destroy the plan before.
struct PlanObject {
    PyObject *plan;
    explicit PlanObject(PyObject *p) : plan(p) { Py_INCREF(p); }
    ~PlanObject()
    {
        if (!Py_IsInitialized()) return;
        const PyGILState_STATE gil = PyGILState_Ensure();
        Py_DECREF(plan);
        PyGILState_Release(gil);
    }
    PlanObject(const PlanObject &) = delete;
    PlanObject &operator=(const PlanObject &) = delete;
};

// The handle of a plan, null for one that is destroyed.  With the GIL held.
const skrull_attn_plan_t *handle_of(PyObject *plan)
{
    PyObject *handle = PyObject_GetAttrString(plan, "handle");
    if (!handle) throw python_error();
    void *p = nullptr;
    if (handle != Py_None) {
        PyObject *value = PyObject_GetAttrString(handle, "value");  // (a ctypes.c_void_p)
        if (value && value != Py_None) p = PyLong_AsVoidPtr(value);
        Py_XDECREF(value);
    }
    Py_DECREF(handle);
    if (PyErr_Occurred()) throw python_error();
    return (const skrull_attn_plan_t *)p;
}

void check(int rc)
{
    if (rc == SKRULL_OK) return;
    const PyGILState_STATE gil = PyGILState_Ensure();
    PyObject *r = PyObject_CallFunction(g_check, "i", rc);
    Py_XDECREF(r);
    python_error error;
    error.persist();
    PyGILState_Release(gil);
    throw error;
}

void *current_stream() { return (void *)c10::hip::getCurrentHIPStream().stream(); }

struct Attention : torch::autograd::Function<Attention> {
    static Variable forward(AutogradContext *ctx, const Variable &q, const Variable &k, const Variable &v, const std::shared_ptr<PlanObject> &plan,
                            const skrull_attn_plan_t *handle, int64_t q_heads, int64_t total_q)
    {
        at::Tensor o = at::empty_like(q), lse = at::empty({q_heads, total_q}, q.options().dtype(at::kFloat));
        check(skrull_attn_fwd(handle, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), (float *)lse.data_ptr(), current_stream()));
        ctx->saved_data["plan"] = c10::IValue::make_capsule(c10::make_intrusive<Holder>(plan));
        ctx->save_for_backward({q, k, v, o, lse});
        return o;
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        const variable_list saved = ctx->get_saved_variables();
        const at::Tensor &q = saved[0], &k = saved[1], &v = saved[2], &o = saved[3], &lse = saved[4];
        const auto holder = c10::static_intrusive_pointer_cast<Holder>(ctx->saved_data["plan"].toCapsule());
        const skrull_attn_plan_t *handle;
        {
            const PyGILState_STATE gil = PyGILState_Ensure();
            try {
                handle = handle_of(holder->plan->plan);
            } catch (python_error &e) {
                e.persist();
                PyGILState_Release(gil);
                throw;
            }
            PyGILState_Release(gil);
        }
        skrull_attn_plan_info_t info;
        check(skrull_attn_plan_info(handle, &info));
        const at::Tensor d_o = grads[0].contiguous();
        at::Tensor dq = at::empty_like(q), dk = at::empty_like(k), dv = at::empty_like(v);
        const int64_t bytes = std::max<int64_t>(info.bwd_workspace_bytes, 16);
        at::Tensor ws = at::empty({bytes}, q.options().dtype(at::kByte));
        check(skrull_attn_bwd(handle, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), (const float *)lse.data_ptr(), d_o.data_ptr(),
                              dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), ws.data_ptr(), (size_t)bytes, current_stream()));
        return {dq, dk, dv, at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor()};
    }
    struct Holder : torch::CustomClassHolder {
        std::shared_ptr<PlanObject> plan;
        explicit Holder(std::shared_ptr<PlanObject> p) : plan(std::move(p)) {}
    };
};

// attention(q, k, v, plan, total_q, total_k, q_heads, kv_heads, head_dim)
PyObject *attention(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 9 || !THPVariable_Check(args[0]) || !THPVariable_Check(args[1]) || !THPVariable_Check(args[2])) {
        PyErr_SetString(PyExc_TypeError, "attention(q, k, v, plan, total_q, total_k, q_heads, kv_heads, head_dim)");
        return nullptr;
    }
    const at::Tensor &q = THPVariable_Unpack(args[0]), &k = THPVariable_Unpack(args[1]), &v = THPVariable_Unpack(args[2]);
    int64_t size[5];
    for (int i = 0; i < 5; ++i) size[i] = PyLong_AsLongLong(args[4 + i]);
    if (PyErr_Occurred()) return nullptr;
    for (const at::Tensor *t : {&q, &k, &v})
        if (!t->is_cuda() || t->scalar_type() != at::kBFloat16 || !t->is_contiguous()) {
            PyErr_SetString(PyExc_ValueError, "q, k, v must be contiguous bf16 CUDA tensors");
            return nullptr;
        }
    const int64_t q_shape[3] = {size[0], size[2], size[4]}, k_shape[3] = {size[1], size[3], size[4]};
    if (q.sizes() != at::IntArrayRef(q_shape, 3) || k.sizes() != at::IntArrayRef(k_shape, 3) || v.sizes() != k.sizes()) {
        PyErr_SetString(PyExc_ValueError, "tensor shapes do not match the plan");
        return nullptr;
    }
    const skrull_attn_plan_t *handle = handle_of(args[3]);
    auto plan = std::make_shared<PlanObject>(args[3]);
    at::Tensor o;
    {
        pybind11::gil_scoped_release no_gil;
        o = Attention::apply(q, k, v, plan, handle, size[2], size[0]);
    }
    return THPVariable_Wrap(std::move(o));
    END_HANDLE_TH_ERRORS
}

// ---- rotary positions, norm, loss.  A call whose tensors are not as the library takes them returns None: the Function in autograd.py then brings
// them into that form, or raises. ----

struct PlanHolder : torch::CustomClassHolder {
    std::shared_ptr<PlanObject> plan;
    explicit PlanHolder(std::shared_ptr<PlanObject> p) : plan(std::move(p)) {}
};

// Whether `t` is on the current GPU.
bool here(const at::Tensor &t) { return t.is_cuda() && t.get_device() == c10::hip::current_device(); }
bool is_bf16(const at::Tensor &t) { return t.scalar_type() == at::kBFloat16; }
// The library's number of a type, -1 for one that it does not take.
int type_of(const at::Tensor &t)
{
    return t.scalar_type() == at::kBFloat16 ? SKRULL_TYPE_BF16 : t.scalar_type() == at::kFloat ? SKRULL_TYPE_FP32 : -1;
}
// Rows of contiguous elements, each at or behind the end of the one before.
bool is_rows(const at::Tensor &t) { return t.dim() == 2 && t.size(1) > 0 && (t.stride(1) == 1 || t.size(1) == 1) && (t.stride(0) >= t.size(1) || t.size(0) < 2); }
int64_t row_stride(const at::Tensor &t) { return t.size(0) > 1 ? t.stride(0) : t.size(1); }
void *address(const at::Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }
at::Tensor bytes_like(const at::Tensor &t, int64_t n) { return at::empty({std::max<int64_t>(n, 16)}, t.options().dtype(at::kByte)); }

// Whether a call of these has to be kept for a backward pass.  (One that has not is made without a Function around it.)
bool differentiable(std::initializer_list<const at::Tensor *> inputs)
{
    return at::GradMode::is_enabled() && std::any_of(inputs.begin(), inputs.end(), [](const at::Tensor *t) { return t->defined() && t->requires_grad(); });
}

// A gradient that is asked for with create_graph cannot be differentiated again.  `varies`: whether it depends on inputs that need gradients, so that it is
// no constant where the gradients that come in are.
variable_list once(const variable_list &grads, variable_list out, bool varies = false)
{
    if (!at::GradMode::is_enabled()) return out;
    if (!varies && !std::any_of(grads.begin(), grads.end(), [](const at::Tensor &g) { return g.defined() && g.requires_grad(); })) return out;
    const auto error = std::make_shared<torch::autograd::DelayedError>("the gradients of this operator cannot be differentiated again", (int)out.size());
    variable_list given;
    for (const at::Tensor &t : out) given.push_back(t.defined() ? t.detach().requires_grad_() : t);
    return (*error)(std::move(given));
}

// A node of its own and not a Function, whose tables and wrappers a small norm waits for (932 x 896, forward and gradients, 14 us of the GPU: 57 us of the host, 61
// as a Function).
struct Norm : torch::autograd::Node {
    torch::autograd::SavedVariable x, w;
    at::Tensor stats;
    int64_t kind = 0;
    bool bias = false;

    static at::Tensor forward(const at::Tensor &x, const at::Tensor &w, const at::Tensor &b, double eps, int64_t kind)
    {
        const std::shared_ptr<Norm> node(new Norm, torch::autograd::deleteNode);
        node->set_next_edges(torch::autograd::collect_next_edges(x, w, b));
        node->stats = at::empty({2, x.size(0)}, x.options().dtype(at::kFloat));
        at::Tensor y = run(x, w, address(b), eps, kind, (float *)node->stats.data_ptr());
        node->x = torch::autograd::SavedVariable(x, false);
        node->w = torch::autograd::SavedVariable(w, false);
        node->kind = kind;
        node->bias = b.defined();
        torch::autograd::set_history(y, node);
        return y;
    }
    variable_list apply(variable_list &&grads) override
    {
        std::lock_guard<std::mutex> lock(mutex_);
        const at::Tensor x = this->x.unpack(), w = this->w.unpack();
        variable_list out(3);
        if (!grads[0].defined()) return out;
        const at::Tensor dy = is_rows(grads[0]) ? grads[0] : grads[0].contiguous();
        at::Tensor dx = at::empty(x.sizes(), x.options()), ws;
        if (task_should_compute_output(1)) out[1] = at::empty_like(w);
        if (bias && task_should_compute_output(2)) out[2] = at::empty_like(w);
        skrull_norm_t p = sizes(x, w, 0.0f, kind);
        p.dy_stride = row_stride(dy);
        p.dx_stride = x.size(1);
        const int64_t bytes = out[1].defined() || out[2].defined() ? skrull_norm_workspace(&p) : 0;
        if (bytes) ws = bytes_like(x, bytes);
        const float *mean = (const float *)stats.data_ptr();
        check(skrull_norm_bwd(&p, x.data_ptr(), w.data_ptr(), mean, mean + x.size(0), dy.data_ptr(), dx.data_ptr(), address(out[1]), address(out[2]), address(ws), (size_t)bytes,
                              current_stream()));
        if (task_should_compute_output(0)) out[0] = std::move(dx);
        return once(grads, std::move(out), x.requires_grad());   // (without x's, dx is not asked for, and dw and db depend on no weight)
    }
    void release_variables() override
    {
        std::lock_guard<std::mutex> lock(mutex_);
        x.reset_data();
        w.reset_data();
        stats.reset();
    }
    static at::Tensor run(const at::Tensor &x, const at::Tensor &w, const void *b, double eps, int64_t kind, float *stats)
    {
        at::Tensor y = at::empty(x.sizes(), x.options());
        skrull_norm_t p = sizes(x, w, (float)eps, kind);
        p.y_stride = x.size(1);
        check(skrull_norm_fwd(&p, x.data_ptr(), w.data_ptr(), b, y.data_ptr(), stats, stats ? stats + x.size(0) : nullptr, current_stream()));
        return y;
    }
    static skrull_norm_t sizes(const at::Tensor &x, const at::Tensor &w, float eps, int64_t kind)
    {
        skrull_norm_t p = {};
        p.rows = x.size(0);
        p.cols = (int32_t)x.size(1);
        p.kind = (int32_t)kind;
        p.type = type_of(x);
        p.weight_type = type_of(w);
        p.eps = eps;
        p.x_stride = row_stride(x);
        return p;
    }
};

struct CrossEntropy : torch::autograd::Function<CrossEntropy> {
    static Variable forward(AutogradContext *ctx, const Variable &x, const Variable &w, const Variable &target)
    {
        const at::Tensor lse = at::empty({x.size(0)}, x.options().dtype(at::kFloat));
        at::Tensor loss = run(x, w, target, lse);
        ctx->save_for_backward({x, w, target, lse});
        return loss;
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        const variable_list saved = ctx->get_saved_variables();
        const at::Tensor &x = saved[0], &w = saved[1], &target = saved[2], &lse = saved[3];
        const at::Tensor d = grads[0].contiguous();
        at::Tensor dx, dw;
        if (ctx->needs_input_grad(0)) dx = at::empty(x.sizes(), x.options());
        if (ctx->needs_input_grad(1)) dw = at::empty_like(w);
        const skrull_loss_t p = sizes(x, w);
        const int64_t bytes = skrull_loss_workspace(&p, 1);
        const at::Tensor ws = bytes_like(x, bytes);
        check(skrull_loss_bwd(&p, x.data_ptr(), w.data_ptr(), (const int64_t *)target.data_ptr(), (const float *)lse.data_ptr(), (const float *)d.data_ptr(), address(dx), address(dw),
                              ws.data_ptr(), (size_t)bytes, current_stream()));
        return once(grads, {dx, dw, at::Tensor()}, true);
    }
    static at::Tensor run(const at::Tensor &x, const at::Tensor &w, const at::Tensor &target, const at::Tensor &lse)
    {
        at::Tensor loss = at::empty_like(lse);
        const skrull_loss_t p = sizes(x, w);
        const int64_t bytes = skrull_loss_workspace(&p, 0);
        const at::Tensor ws = bytes_like(x, bytes);
        check(skrull_loss_fwd(&p, x.data_ptr(), w.data_ptr(), (const int64_t *)target.data_ptr(), (float *)loss.data_ptr(), (float *)lse.data_ptr(), ws.data_ptr(), (size_t)bytes,
                              current_stream()));
        return loss;
    }
    static skrull_loss_t sizes(const at::Tensor &x, const at::Tensor &w)
    {
        return skrull_loss_t{x.size(0), (int32_t)x.size(1), (int32_t)w.size(0), row_stride(x)};
    }
};

// [rows, heads, head_dim] as skrull_rotary takes it
bool is_heads(const at::Tensor &t)
{
    return t.dim() == 3 && t.stride(2) == 1 && (t.size(1) == 1 || t.stride(1) == t.size(2)) && (t.size(0) < 2 || (t.stride(0) >= t.size(1) * t.size(2) && t.stride(0) % 8 == 0)) &&
           (uintptr_t)t.data_ptr() % 16 == 0;
}

struct Rotary : torch::autograd::Function<Rotary> {
    static variable_list forward(AutogradContext *ctx, const Variable &q, const Variable &k, const std::shared_ptr<PlanObject> &plan, const skrull_attn_plan_t *handle,
                                 const std::string &rotary, int64_t k_rows)
    {
        ctx->saved_data["plan"] = c10::IValue::make_capsule(c10::make_intrusive<PlanHolder>(plan));
        ctx->saved_data["rotary"] = rotary;
        ctx->saved_data["k_rows"] = k_rows;
        return turn(handle, rotary, q, k, k_rows, 0);
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        const auto holder = c10::static_intrusive_pointer_cast<PlanHolder>(ctx->saved_data["plan"].toCapsule());
        const skrull_attn_plan_t *handle;
        {
            const PyGILState_STATE gil = PyGILState_Ensure();
            try {
                handle = handle_of(holder->plan->plan);
            } catch (python_error &e) {
                e.persist();
                PyGILState_Release(gil);
                throw;
            }
            PyGILState_Release(gil);
        }
        // (cloned and not made contiguous, which a part of a flat buffer is already, at whatever address)
        const auto taken = [](const at::Tensor &t) { return is_heads(t) ? t : t.clone(at::MemoryFormat::Contiguous); };
        const at::Tensor dq = taken(grads[0]), dk = taken(grads[1]);
        variable_list out = turn(handle, ctx->saved_data["rotary"].toStringRef(), dq, dk, ctx->saved_data["k_rows"].toInt(), 1);
        return once(grads, {out[0], out[1], at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor()});
    }
    static variable_list turn(const skrull_attn_plan_t *handle, const std::string &rotary, const at::Tensor &q, const at::Tensor &k, int64_t k_rows, int inverse)
    {
        variable_list out = {at::empty(q.sizes(), q.options()), at::empty(k.sizes(), k.options())};
        const skrull_rotary_tensor_t t[2] = {tensor(q, out[0], SKRULL_ROWS_Q), tensor(k, out[1], k_rows)};
        check(skrull_rotary(handle, (const skrull_rotary_t *)rotary.data(), &t[0], &t[1], inverse, current_stream()));
        return out;
    }
    static skrull_rotary_tensor_t tensor(const at::Tensor &in, const at::Tensor &out, int64_t rows)
    {
        const int64_t width = in.size(1) * in.size(2);
        const bool many = in.size(0) > 1;   // (a single row's stride says nothing)
        return skrull_rotary_tensor_t{in.data_ptr(), out.data_ptr(), many ? in.stride(0) : width, many ? out.stride(0) : width, (int32_t)in.size(1), (int32_t)rows};
    }
};

// While a graph is captured, a backward pass that reaches a leaf through a node which an eager graph keeps alive waits for that node's own
// stream, which is not captured: the process ends there.  So such a call is refused before it records anything.
void refuse_captured(std::initializer_list<const at::Tensor *> inputs)
{
    const c10::hip::HIPStream stream = c10::hip::getCurrentHIPStream();
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(stream.stream(), &capture) != hipSuccess || capture == hipStreamCaptureStatusNone || !at::GradMode::is_enabled()) return;
    for (const at::Tensor *t : inputs) {
        if (!t->defined() || !t->requires_grad() || !t->is_leaf()) continue;
        const auto node = torch::autograd::impl::try_get_grad_accumulator(*t);
        if (!node) continue;
        const auto other = node->stream();
        TORCH_CHECK_VALUE(!other || *other == stream.unwrap(),
                          "a graph made outside this capture is alive and has the same leaf: release it (its outputs) before a backward pass is captured");
    }
}

#define SKRULL_TENSOR(i) THPVariable_Unpack(args[i])

// norm(x, weight, bias or None, eps, kind)
PyObject *norm(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    TORCH_CHECK_TYPE(n == 5 && THPVariable_Check(args[0]) && THPVariable_Check(args[1]) && (args[2] == Py_None || THPVariable_Check(args[2])), "norm(x, weight, bias, eps, kind)");
    const at::Tensor &x = SKRULL_TENSOR(0), &w = SKRULL_TENSOR(1), b = args[2] == Py_None ? at::Tensor() : SKRULL_TENSOR(2);
    const double eps = PyFloat_AsDouble(args[3]);
    const int64_t kind = PyLong_AsLongLong(args[4]);
    if (PyErr_Occurred()) return nullptr;
    if (!here(x) || !here(w) || !is_rows(x) || x.size(1) > SKRULL_NORM_MAX_COLS || type_of(x) < 0 || type_of(w) < 0 || w.dim() != 1 || w.size(0) != x.size(1) || !w.is_contiguous() ||
        (b.defined() && (!here(b) || b.scalar_type() != w.scalar_type() || b.dim() != 1 || b.size(0) != x.size(1) || !b.is_contiguous())))
        Py_RETURN_NONE;
    at::Tensor y;
    {
        pybind11::gil_scoped_release no_gil;
        if (differentiable({&x, &w, &b})) {
            refuse_captured({&x, &w, &b});
            y = Norm::forward(x, w, b, eps, kind);
        } else {
            y = Norm::run(x, w, address(b), eps, kind, nullptr);
        }
    }
    return THPVariable_Wrap(std::move(y));
    END_HANDLE_TH_ERRORS
}

// cross_entropy(x, weight, target)
PyObject *cross_entropy(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    TORCH_CHECK_TYPE(n == 3 && THPVariable_Check(args[0]) && THPVariable_Check(args[1]) && THPVariable_Check(args[2]), "cross_entropy(x, weight, target)");
    const at::Tensor &x = SKRULL_TENSOR(0), &w = SKRULL_TENSOR(1), &target = SKRULL_TENSOR(2);
    if (!here(x) || !here(w) || !here(target) || !is_rows(x) || !is_bf16(x) || !is_bf16(w) || w.dim() != 2 || w.size(1) != x.size(1) || !w.is_contiguous() || w.size(0) > INT32_MAX ||
        x.size(1) > INT32_MAX || target.scalar_type() != at::kLong || target.dim() != 1 || target.size(0) != x.size(0) || !target.is_contiguous())
        Py_RETURN_NONE;
    at::Tensor loss;
    {
        pybind11::gil_scoped_release no_gil;
        if (differentiable({&x, &w})) {
            refuse_captured({&x, &w});
            loss = CrossEntropy::apply(x, w, target);
        } else {
            loss = CrossEntropy::run(x, w, target, at::empty({x.size(0)}, x.options().dtype(at::kFloat)));
        }
    }
    return THPVariable_Wrap(std::move(loss));
    END_HANDLE_TH_ERRORS
}

// rotary(q, k, plan, address of the skrull_rotary_t, k_rows)
PyObject *rotary(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    TORCH_CHECK_TYPE(n == 5 && THPVariable_Check(args[0]) && THPVariable_Check(args[1]), "rotary(q, k, plan, rotary, k_rows)");
    const at::Tensor &q = SKRULL_TENSOR(0), &k = SKRULL_TENSOR(1);
    const void *given = PyLong_AsVoidPtr(args[3]);
    const int64_t k_rows = PyLong_AsLongLong(args[4]);
    if (PyErr_Occurred()) return nullptr;
    const skrull_attn_plan_t *handle = handle_of(args[2]);
    skrull_attn_plan_info_t info;
    if (skrull_attn_plan_info(handle, &info) != SKRULL_OK || (k_rows != SKRULL_ROWS_Q && k_rows != SKRULL_ROWS_K)) Py_RETURN_NONE;
    if (!here(q) || !here(k) || !is_bf16(q) || !is_bf16(k) || !is_heads(q) || !is_heads(k) || q.size(0) != info.total_q ||
        k.size(0) != (k_rows == SKRULL_ROWS_Q ? info.total_q : info.total_k) || q.size(2) != info.head_dim || k.size(2) != info.head_dim)
        Py_RETURN_NONE;
    const std::string copy((const char *)given, sizeof(skrull_rotary_t));
    variable_list out;
    if (differentiable({&q, &k})) {
        auto plan = std::make_shared<PlanObject>(args[2]);
        pybind11::gil_scoped_release no_gil;
        refuse_captured({&q, &k});
        out = Rotary::apply(q, k, plan, handle, copy, k_rows);
    } else {
        pybind11::gil_scoped_release no_gil;
        out = Rotary::turn(handle, copy, q, k, k_rows, 0);
    }
    PyObject *both = PyTuple_New(2);
    if (!both) throw python_error();
    for (int i = 0; i < 2; ++i) PyTuple_SET_ITEM(both, i, THPVariable_Wrap(std::move(out[i])));
    return both;
    END_HANDLE_TH_ERRORS
}

// turn(plan, address of the skrull_rotary_t, q, k, q_out, k_out, inverse, k_rows, stream or None): binding.skrull_rotary, False where that has
// to look at the tensors itself.
PyObject *turn(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    TORCH_CHECK_TYPE(n == 9, "turn(plan, rotary, q, k, q_out, k_out, inverse, k_rows, stream)");
    const void *rotary = PyLong_AsVoidPtr(args[1]);
    const int inverse = PyObject_IsTrue(args[6]);
    const int64_t k_rows = PyLong_AsLongLong(args[7]);
    void *stream = args[8] == Py_None ? nullptr : PyLong_AsVoidPtr(args[8]);
    if (PyErr_Occurred()) return nullptr;
    const skrull_attn_plan_t *handle = handle_of(args[0]);
    skrull_attn_plan_info_t info;
    if (skrull_attn_plan_info(handle, &info) != SKRULL_OK || (k_rows != SKRULL_ROWS_Q && k_rows != SKRULL_ROWS_K)) Py_RETURN_FALSE;
    skrull_rotary_tensor_t t[2];
    int count = 0;
    for (int i = 0; i < 2; ++i) {
        if (args[2 + i] == Py_None) continue;
        if (!THPVariable_CheckExact(args[2 + i]) || !THPVariable_CheckExact(args[4 + i])) Py_RETURN_FALSE;
        const at::Tensor &in = SKRULL_TENSOR(2 + i), &out = SKRULL_TENSOR(4 + i);
        const int64_t rows = i ? k_rows : SKRULL_ROWS_Q;
        if (!here(in) || !here(out) || !is_bf16(in) || !is_bf16(out) || !is_heads(in) || !is_heads(out) || in.sizes() != out.sizes() || in.size(2) != info.head_dim ||
            in.size(0) != (rows == SKRULL_ROWS_Q ? info.total_q : info.total_k))
            Py_RETURN_FALSE;
        t[count++] = Rotary::tensor(in, out, rows);
    }
    if (!count) Py_RETURN_FALSE;
    {
        pybind11::gil_scoped_release no_gil;
        check(skrull_rotary(handle, (const skrull_rotary_t *)rotary, &t[0], count > 1 ? &t[1] : nullptr, inverse, args[8] == Py_None ? current_stream() : stream));
    }
    Py_RETURN_TRUE;
    END_HANDLE_TH_ERRORS
}

// refuse_captured(tensors): the same for calls that take the Function in autograd.py
PyObject *refuse_captured_of(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    for (Py_ssize_t i = 0; i < n; ++i)
        if (THPVariable_Check(args[i])) refuse_captured({&SKRULL_TENSOR(i)});
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

PyObject *set_check(PyObject *, PyObject *f)
{
    Py_INCREF(f);
    Py_XSETREF(g_check, f);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"attention", (PyCFunction)(void (*)())attention, METH_FASTCALL, "the differentiable call"},
                         {"norm", (PyCFunction)(void (*)())norm, METH_FASTCALL, "the differentiable norm"},
                         {"cross_entropy", (PyCFunction)(void (*)())cross_entropy, METH_FASTCALL, "the differentiable loss"},
                         {"rotary", (PyCFunction)(void (*)())rotary, METH_FASTCALL, "the differentiable rotary positions"},
                         {"turn", (PyCFunction)(void (*)())turn, METH_FASTCALL, "binding.skrull_rotary"},
                         {"refuse_captured", (PyCFunction)(void (*)())refuse_captured_of, METH_FASTCALL, "refuses leaves that an eager graph has"},
                         {"set_check", set_check, METH_O, "the callable that raises what an error code stands for"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_autograd", "autograd of skrull_attn", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__autograd() { return PyModule_Create(&module); }
