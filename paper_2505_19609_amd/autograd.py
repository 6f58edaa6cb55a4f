"""torch.autograd wrappers around the library's forwards and backwards (attention, rotary positions, norm, loss), for callers that
train with PyTorch: argument marshalling and bookkeeping only, every step of the
operators runs in the HIP kernels behind the C ABI.  The marshalling is native code where
nothing watches the call from Python, else the Functions below: the same checks, outputs and errors."""
from __future__ import annotations

import ctypes
import sys
import warnings

import torch
from torch.autograd.function import once_differentiable

from . import binding as B


class _SkrullAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, plan):
        if not (q.is_cuda and q.dtype == torch.bfloat16 and q.is_contiguous() and k.is_contiguous()
                and v.is_contiguous() and k.dtype == torch.bfloat16 and v.dtype == torch.bfloat16):
            raise ValueError("q, k, v must be contiguous bf16 CUDA tensors")
        if q.shape != (plan.total_q, plan.num_q_heads, plan.head_dim) or \
                k.shape != (plan.total_k, plan.num_kv_heads, plan.head_dim) or v.shape != k.shape:
            raise ValueError("tensor shapes do not match the plan")
        o = torch.empty_like(q)
        lse = torch.empty((plan.num_q_heads, plan.total_q), dtype=torch.float32, device=q.device)
        B.skrull_attn_fwd(plan, q, k, v, o, lse)
        ctx.plan = plan
        ctx.save_for_backward(q, k, v, o, lse)
        return o

    @staticmethod
    def backward(ctx, d_o):
        q, k, v, o, lse = ctx.saved_tensors
        plan = ctx.plan
        d_o = d_o.contiguous()
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        ws = torch.empty(max(int(plan.bwd_workspace_bytes), 16), dtype=torch.uint8, device=q.device)
        B.skrull_attn_bwd(plan, q, k, v, o, lse, d_o, dq, dk, dv, ws)
        return dq, dk, dv, None


def _watched():
    """Whether something follows torch's calls from Python (a trace, a functorch transform, forward-mode
    gradients, a mode, a compiler), which has to see the Function above."""
    try:
        return (torch._C._get_tracing_state() is not None or torch._C._functorch.peek_interpreter_stack() is not None
                or torch.autograd.forward_ad._current_level >= 0 or torch._C._len_torch_dispatch_stack() > 0
                or torch._C._len_torch_function_stack() > 0 or torch.compiler.is_compiling())
    except AttributeError:   # (most of these are private to torch)
        return True


_native = None   # the same in native code; False where that cannot be loaded


def _load_native():
    """csrc/autograd.cpp, built in-tree with the library against the torch of that build.  The library's kernels are called either
    way: without this module, or with one for another torch, by the Function above."""
    global _native
    B.lib()
    try:
        from . import _autograd
    except ImportError as e:
        warnings.warn(f"paper_2505_19609_amd/_autograd.so cannot be loaded ({e}): calls of skrull_attention take the host "
                      "longer; build it with python -m paper_2505_19609_amd.build", RuntimeWarning, stacklevel=3)
        _native = False
    else:
        _autograd.set_check(B._check)
        _native = _autograd.attention
    return _native


_TENSORS = (torch.Tensor, torch.nn.Parameter)


def skrull_attention(q, k, v, plan):
    """O = packed varlen causal attention of the micro-batch `plan` describes
    (a binding.Plan); differentiable with respect to q, k, v."""
    if type(q) in _TENSORS and type(k) in _TENSORS and type(v) in _TENSORS and type(plan) is B.Plan and not _watched():
        native = _load_native() if _native is None else _native
        if native:
            i = plan.info
            return native(q, k, v, plan, i.total_q, i.total_k, i.num_q_heads, i.num_kv_heads, i.head_dim)
    return _SkrullAttention.apply(q, k, v, plan)


# ---- rotary positions, norm, loss: the same way ---------------------------------------------------------------------

_KINDS = {"layer": B.NORM_LAYER, "rms": B.NORM_RMS}


def _module():
    """The native module, or None where it cannot be loaded."""
    if _native is None:
        _load_native()
    return sys.modules.get(__package__ + "._autograd") if _native else None


def _native_for(*tensors):
    """The native module for a call that nothing watches from Python, else None."""
    return _module() if all(type(t) in _TENSORS or t is None for t in tensors) and not _watched() else None


def _refuse_captured(*tensors):
    if any(t is not None and t.is_cuda for t in tensors) and torch.cuda.is_current_stream_capturing():
        module = _module()
        if module is not None:
            module.refuse_captured(*tensors)


def _once(varies):
    """once_differentiable, also where the gradients that come in need none: `varies(ctx)` says whether the ones that go out depend on inputs that do, and
    then they must not pass for constants."""
    def decorate(backward):
        refused = once_differentiable(backward)

        def wrapped(ctx, *grads):
            if torch.is_grad_enabled() and not any(g.requires_grad for g in grads) and varies(ctx):
                grads = [g.detach().requires_grad_() for g in grads]
            return refused(ctx, *grads)
        return wrapped
    return decorate


def _workspace(n, device):
    return torch.empty(max(int(n), 16), dtype=torch.uint8, device=device)


class _SkrullRotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, plan, rotary, k_rows):
        ctx.plan, ctx.rotary, ctx.k_rows = plan, B.Rotary.from_buffer_copy(rotary), k_rows   # (the program may change its own)
        out = [torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k)]
        B.skrull_rotary(plan, rotary, q, k, *out, k_rows=k_rows)
        return tuple(out)

    @staticmethod
    @once_differentiable
    def backward(ctx, dq, dk):
        given = [_rows_of_heads(t) for t in (dq, dk)]
        out = [torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in given]
        B.skrull_rotary(ctx.plan, ctx.rotary, *given, *out, inverse=True, k_rows=ctx.k_rows)
        return out[0], out[1], None, None, None


def _rows_of_heads(t):
    """`t` [rows, heads, head_dim] as the library takes it: strides as they are where it can."""
    if t.dim() != 3:
        raise ValueError("q and k must be [rows, heads, head_dim]")
    heads, d = t.shape[1:]
    fits = t.stride(2) == 1 and (heads == 1 or t.stride(1) == d) and t.data_ptr() % 16 == 0 and \
        (t.shape[0] < 2 or (t.stride(0) >= heads * d and t.stride(0) % 8 == 0))
    return t if fits else t.clone(memory_format=torch.contiguous_format)


def skrull_rotary(q, k, plan, rotary, k_rows=B.ROWS_K):
    """q and k turned by the positions of the rows of `plan` (a binding.Plan); differentiable.  `rotary`: from
    binding.skrull_rotary_init.  k holds the gathered prefixes, or with k_rows=binding.ROWS_Q this rank's own tokens.
    q and k may be parts of one projection's rows; what comes back is contiguous, as skrull_attention takes it."""
    module = _native_for(q, k) if type(plan) is B.Plan and type(rotary) is B.Rotary else None
    out = module.rotary(q, k, plan, ctypes.addressof(rotary), k_rows) if module is not None else None
    if out is None:
        _refuse_captured(q, k)
        out = _SkrullRotary.apply(_rows_of_heads(q), _rows_of_heads(k), plan, rotary, k_rows)
    return out


class _SkrullNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, kind):
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        mean, rstd = torch.empty((2, x.shape[0]), dtype=torch.float32, device=x.device)
        B.skrull_norm_fwd(x, weight, bias, y, mean, rstd, eps, kind)
        ctx.kind, ctx.bias = kind, bias is not None
        ctx.save_for_backward(x, weight, mean, rstd)
        return y

    @staticmethod
    @_once(lambda ctx: ctx.needs_input_grad[0])   # (without x's, dx is not asked for, and dw and db depend on no weight)
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        dy = _rows(dy)
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        need_w, need_b = ctx.needs_input_grad[1], ctx.bias and ctx.needs_input_grad[2]
        dw = torch.empty_like(weight) if need_w else None
        db = torch.empty_like(weight) if need_b else None
        ws = _workspace(B.skrull_norm_workspace(x, weight, ctx.kind), x.device) if need_w or need_b else None
        B.skrull_norm_bwd(x, weight, mean, rstd, dy, dx, dw, db, ws, ctx.kind)
        return dx, dw, db, None, None


def _rows(t):
    """`t` [rows, cols] with contiguous rows, one behind the other."""
    return t if t.dim() != 2 or (t.stride(1) == 1 and (t.stride(0) >= t.shape[1] or t.shape[0] < 2)) else t.contiguous()


def skrull_norm(x, weight, bias=None, eps=1e-5, kind="layer"):
    """The norm of the rows of x [rows, cols] (bf16 or fp32) with weight and bias [cols]: "layer", or "rms" without mean and
    bias; differentiable with respect to x, weight and bias."""
    if kind not in _KINDS:
        raise ValueError(f"kind must be one of {sorted(_KINDS)}")
    if x.dim() != 2:
        raise ValueError("x must be [rows, cols]")
    module = _native_for(x, weight, bias)
    y = module.norm(x, weight, bias, eps, _KINDS[kind]) if module is not None else None
    if y is None:
        _refuse_captured(x, weight, bias)
        y = _SkrullNorm.apply(_rows(x), weight.contiguous(), None if bias is None else bias.contiguous(), eps, _KINDS[kind])
    return y


class _SkrullCrossEntropy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, target):
        loss, lse = (torch.empty(x.shape[0], dtype=torch.float32, device=x.device) for _ in range(2))
        B.skrull_loss_fwd(x, weight, target, loss, lse, _workspace(B.skrull_loss_workspace(x, weight, False), x.device))
        ctx.save_for_backward(x, weight, target, lse)
        return loss

    @staticmethod
    @_once(lambda ctx: True)
    def backward(ctx, d_loss):
        x, weight, target, lse = ctx.saved_tensors
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device) if ctx.needs_input_grad[0] else None
        dw = torch.empty_like(weight) if ctx.needs_input_grad[1] else None
        B.skrull_loss_bwd(x, weight, target, lse, d_loss.contiguous(), dx, dw,
                          _workspace(B.skrull_loss_workspace(x, weight, True), x.device))
        return dx, dw, None


def skrull_cross_entropy(x, weight, target):
    """The softmax cross entropy of each row of x [rows, hidden] times the vocabulary's weight [vocab, hidden] against
    target [rows] (int64; a negative one: the row has none, and a loss of 0), fp32 [rows], without keeping the logits;
    differentiable with respect to x and weight."""
    module = _native_for(x, weight, target)
    loss = module.cross_entropy(x, weight, target) if module is not None else None
    if loss is None:
        _refuse_captured(x, weight)
        loss = _SkrullCrossEntropy.apply(_rows(x), weight.contiguous(), target.contiguous())
    return loss
