"""The operators that a block is made of (attention to a window, the residual stream, products) without a GPU: symbols, struct layouts and what the
entry points refuse."""
import ctypes
import math
import os
import re

import pytest
import torch

from paper_2505_19609_amd import autograd as A
from paper_2505_19609_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ONE = 1 << 20   # an address that is aligned and never read: the call fails first
HEADERS = ("skrull_window.h", "skrull_residual.h", "skrull_linear.h")


def test_library_exports_every_declared_operator():
    header = "".join(open(os.path.join(ROOT, "include", f)).read() for f in HEADERS)
    declared = set(re.findall(r"\b(skrull_(?:window|residual|linear)(?:_[a-z]+)*)\s*\(", header))
    assert declared == set(B.BLOCK_SYMBOLS)
    for name in declared:
        assert getattr(B.lib(), name) is not None


def test_argument_counts_match_headers():
    """What ctypes is told of each call is what the header declares."""
    for f in HEADERS:
        header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", f)).read(), flags=re.S)
        for name, args in re.findall(r"\b(skrull_[a-z_]+)\s*\(([^)]*)\)\s*;", header):
            assert len(getattr(B.lib(), name).argtypes) == len(args.split(",")), name


def test_struct_layouts_match_headers():
    assert ctypes.sizeof(B.Linear) == 8 + 4 * 4 + 4 * 8
    assert ctypes.sizeof(B.Window) == 2 * 4
    assert ctypes.sizeof(B.Residual) == 8 + 7 * 4 + 4 + 8 * 8   # (scale and its padding)


# ---- the residual stream --------------------------------------------------------------------------------------------

STRIDES = ("r_stride", "z_stride", "r_out_stride", "y_stride", "d_r_out_stride", "dy_stride", "dr_stride", "dz_stride")


def _residual(**kw):
    p = dict(rows=4, cols=64, kind=B.NORM_LAYER, type=B.TYPE_BF16, residual_type=B.TYPE_BF16, weight_type=B.TYPE_BF16, eps=1e-5, scale=1.0, **{s: 64 for s in STRIDES})
    p.update(kw)
    return B.Residual(**p)


def _fwd(p, b=None, **kw):
    a = dict(r=ONE, z=2 * ONE, w=3 * ONE, b=b, post_w=None, post_b=None, gate=None, r_out=4 * ONE, y=5 * ONE, stats=6 * ONE)
    a.update(kw)
    return B.lib().skrull_residual_fwd(ctypes.byref(p), *a.values(), None)


def _bwd(p, workspace_bytes=1 << 30, **kw):
    a = dict(r=ONE, z=2 * ONE, w=3 * ONE, post_w=None, post_b=None, gate=None, stats=6 * ONE, d_r_out=7 * ONE, dy=8 * ONE, dr=9 * ONE, dz=10 * ONE, dw=11 * ONE, db=None,
             dpost_w=None, dpost_b=None, dgate=None, workspace=20 * ONE)
    a.update(kw)
    return B.lib().skrull_residual_bwd(ctypes.byref(p), *a.values(), workspace_bytes, None)


WIDE = {s: 8193 for s in STRIDES}
BAD = [dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(cols=8193, **WIDE), dict(kind=2), dict(type=2), dict(residual_type=2),
       dict(type=B.TYPE_FP32, residual_type=B.TYPE_BF16), dict(weight_type=-1), dict(eps=-1.0), dict(eps=math.nan), dict(scale=math.inf), dict(scale=math.nan),
       dict(r_stride=63), dict(z_stride=-64)]


@pytest.mark.parametrize("kw", BAD + [dict(r_out_stride=63), dict(y_stride=1 << 62)])
def test_residual_fwd_refuses(kw):
    assert _fwd(_residual(**kw)) == B.SKRULL_EINVAL
    assert "residual" in B.skrull_attn_strerror(B.SKRULL_EINVAL)


@pytest.mark.parametrize("kw", BAD + [dict(d_r_out_stride=63), dict(dy_stride=0), dict(dr_stride=63), dict(dz_stride=63)])
def test_residual_bwd_refuses(kw):
    assert _bwd(_residual(**kw)) == B.SKRULL_EINVAL
    assert "residual" in B.skrull_attn_strerror(B.SKRULL_EINVAL)


@pytest.mark.parametrize("kw", [dict(r=None), dict(z=None), dict(w=None), dict(r_out=None), dict(y=None), dict(r=ONE + 1), dict(w=3 * ONE + 1), dict(stats=6 * ONE + 2),
                                dict(post_b=ONE), dict(r_out=ONE + 128), dict(y=2 * ONE + 2), dict(r_out=2 * ONE), dict(y=ONE), dict(y=4 * ONE), dict(gate=ONE + 1)])
def test_residual_fwd_refuses_pointers(kw):
    assert _fwd(_residual(), **kw) == B.SKRULL_EINVAL


@pytest.mark.parametrize("kw", [dict(r=None), dict(z=None), dict(w=None), dict(stats=None), dict(dr=None), dict(dz=None), dict(workspace=None), dict(workspace=20 * ONE + 8), dict(workspace_bytes=64),
                                dict(post_b=ONE), dict(dpost_w=ONE), dict(dpost_b=ONE), dict(dw=ONE + 1), dict(dr=7 * ONE), dict(dz=8 * ONE), dict(dz=9 * ONE + 2), dict(dr=ONE), dict(dz=2 * ONE)])
def test_residual_bwd_refuses_pointers(kw):
    assert _bwd(_residual(), **kw) == B.SKRULL_EINVAL


def test_residual_refuses_biases_without_a_mean():
    p = _residual(kind=B.NORM_RMS)
    assert _fwd(p, b=ONE) == _fwd(p, post_w=ONE, post_b=ONE) == B.SKRULL_EINVAL
    assert _bwd(p, db=ONE) == _bwd(p, post_w=ONE, post_b=ONE) == _bwd(p, post_w=ONE, dpost_b=ONE) == B.SKRULL_EINVAL


def test_residual_workspace():
    assert B.lib().skrull_residual_workspace(ctypes.byref(_residual(cols=0))) == 0
    assert B.lib().skrull_residual_workspace(ctypes.byref(_residual())) >= 4 * 64 * 4
    # (bounded however many rows there are)
    assert B.lib().skrull_residual_workspace(ctypes.byref(_residual(rows=(1 << 31) - 1, cols=8192, **{s: 8192 for s in STRIDES}))) <= 64 << 20


def test_residual_wrappers_refuse():
    r, z, w = torch.zeros(4, 64), torch.zeros(4, 64), torch.zeros(64)
    with pytest.raises(ValueError, match="kind"):
        A.skrull_residual_norm(r, z, w, kind="batch")
    with pytest.raises(ValueError, match="rows, cols"):
        A.skrull_residual_norm(r[0], z, w)
    with pytest.raises(B.SkrullError, match="current GPU"):
        A.skrull_residual_norm(r, z, w)


# ---- attention to a window ------------------------------------------------------------------------------------------

def test_window_refuses_null():
    w = B.Window(4, 0)
    lib = B.lib()
    assert lib.skrull_window_fwd(None, ctypes.byref(w), *[ONE] * 5, None) == B.SKRULL_EINVAL
    assert "window" in B.skrull_attn_strerror(B.SKRULL_EINVAL)
    assert lib.skrull_window_bwd(None, ctypes.byref(w), *[ONE] * 10, 1 << 30, None) == B.SKRULL_EINVAL
    assert lib.skrull_window_workspace(None, ctypes.byref(w)) == 0
    assert lib.skrull_window_fwd(ONE, None, *[ONE] * 5, None) == lib.skrull_window_bwd(ONE, None, *[ONE] * 10, 1 << 30, None) == B.SKRULL_EINVAL


@pytest.mark.parametrize("window,sinks", [(0, 0), (-1, 0), (4, -1)])
def test_window_refuses_values(window, sinks):
    """(the plan is not looked at before)"""
    w = B.Window(window, sinks)
    lib = B.lib()
    assert lib.skrull_window_fwd(ONE, ctypes.byref(w), *[ONE] * 5, None) == B.SKRULL_EINVAL
    assert lib.skrull_window_bwd(ONE, ctypes.byref(w), *[ONE] * 10, 1 << 30, None) == B.SKRULL_EINVAL
    assert lib.skrull_window_workspace(ONE, ctypes.byref(w)) == 0


def test_window_wrappers_refuse():
    q = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    info = B.PlanInfo(total_q=4, total_k=4, num_q_heads=2, num_kv_heads=2, head_dim=64)
    plan = B.Plan(None, info)
    lse = torch.zeros(2, 4)
    with pytest.raises(B.SkrullError, match="current GPU"):
        A.skrull_window_attention(q, q, q, plan, 4)
    for value in (1 << 31, -(1 << 31) - 1):
        with pytest.raises(B.SkrullError, match="window"):
            B._window_of(value, 0)
        with pytest.raises(B.SkrullError, match="sinks"):
            B._window_of(1, value)
    with pytest.raises(B.SkrullError, match="contiguous bf16"):
        B._heads(plan, (q.float(),))
    with pytest.raises(B.SkrullError, match="contiguous bf16"):
        B._heads(plan, (), (q[:3],))
    with pytest.raises(B.SkrullError, match="contiguous bf16"):
        B._heads(plan, (torch.zeros(4, 4, 64, dtype=torch.bfloat16)[:, ::2],))
    with pytest.raises(B.SkrullError, match="lse"):
        B._lse(plan, lse.t())


# ---- products -------------------------------------------------------------------------------------------------------

def _linear(**kw):
    p = dict(rows=16, inputs=64, outputs=128, activation=B.LINEAR_NONE, gated=0, x_stride=64, residual_stride=128, y_stride=128, dy_stride=128)
    p.update(kw)
    return B.Linear(**p)


def _linear_fwd(p, workspace_bytes=1 << 30, **kw):
    a = dict(x=ONE, w=2 * ONE, b=3 * ONE, residual=4 * ONE, y=5 * ONE, z=6 * ONE, workspace=40 * ONE)
    a.update(kw)
    return B.lib().skrull_linear_fwd(ctypes.byref(p), *a.values(), workspace_bytes, None)


def _linear_bwd(p, workspace_bytes=1 << 30, **kw):
    a = dict(x=ONE, w=2 * ONE, z=3 * ONE, dy=4 * ONE, dx=5 * ONE, dw=6 * ONE, db=7 * ONE, workspace=40 * ONE)
    a.update(kw)
    return B.lib().skrull_linear_bwd(ctypes.byref(p), *a.values(), workspace_bytes, None)


BAD_LINEAR = [dict(rows=-1), dict(rows=(1 << 24) + 1), dict(inputs=0), dict(inputs=60), dict(inputs=65544, x_stride=65544), dict(outputs=4), dict(outputs=132), dict(outputs=1 << 17),
              dict(activation=4), dict(activation=-1), dict(gated=2), dict(gated=1, outputs=32768, inputs=32768, x_stride=32768, y_stride=32768, dy_stride=32768, residual_stride=32768),
              dict(x_stride=56), dict(x_stride=68), dict(x_stride=(1 << 20) + 8)]


@pytest.mark.parametrize("kw", BAD_LINEAR + [dict(y_stride=120), dict(y_stride=132), dict(residual_stride=64)])
def test_linear_fwd_refuses(kw):
    assert _linear_fwd(_linear(**kw)) == B.SKRULL_EINVAL
    assert "linear" in B.skrull_attn_strerror(B.SKRULL_EINVAL)


@pytest.mark.parametrize("kw", BAD_LINEAR + [dict(dy_stride=120), dict(dy_stride=129)])
def test_linear_bwd_refuses(kw):
    assert _linear_bwd(_linear(**kw)) == B.SKRULL_EINVAL
    assert "linear" in B.skrull_attn_strerror(B.SKRULL_EINVAL)


@pytest.mark.parametrize("kw", [dict(x=None), dict(w=None), dict(y=None), dict(x=ONE + 2), dict(w=2 * ONE + 8), dict(b=3 * ONE + 2), dict(residual=4 * ONE + 8), dict(y=5 * ONE + 4), dict(z=6 * ONE + 2),
                                dict(y=ONE), dict(y=2 * ONE + 16), dict(y=4 * ONE + 16), dict(z=5 * ONE), dict(z=4 * ONE), dict(y=3 * ONE)])
def test_linear_fwd_refuses_pointers(kw):
    assert _linear_fwd(_linear(), **kw) == B.SKRULL_EINVAL


@pytest.mark.parametrize("kw", [dict(x=None), dict(w=None), dict(dy=None), dict(dx=5 * ONE + 8), dict(dw=6 * ONE + 2), dict(db=7 * ONE + 4), dict(workspace=None), dict(workspace=40 * ONE + 8),
                                dict(workspace_bytes=16), dict(dx=ONE), dict(dw=2 * ONE), dict(dx=4 * ONE), dict(dw=5 * ONE + 16), dict(db=6 * ONE), dict(dw=40 * ONE)])
def test_linear_bwd_refuses_pointers(kw):
    assert _linear_bwd(_linear(), **kw) == B.SKRULL_EINVAL


def test_linear_backward_of_an_activation_needs_z():
    assert _linear_bwd(_linear(activation=B.LINEAR_SILU), z=None) == _linear_bwd(_linear(gated=1), z=None) == B.SKRULL_EINVAL


def test_linear_workspace():
    size = lambda backward, **kw: B.lib().skrull_linear_workspace(ctypes.byref(_linear(**kw)), backward)  # noqa: E731
    assert size(0, inputs=4) == size(1, activation=9) == -1
    assert size(0, rows=0) == 0 and size(1, rows=0) >= 0
    big = dict(rows=32768, inputs=4096, outputs=4096)
    assert size(0, **big) == 0                                                     # (a tile for every compute unit)
    assert size(1, activation=B.LINEAR_GELU, **big) >= 32768 * 4096 * 2            # dz
    assert size(1, **big) < 64 << 20


def test_linear_wrappers_refuse():
    x, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(128, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="activation"):
        A.skrull_linear(x, w, activation="tanh")
    with pytest.raises(ValueError, match="rows, inputs"):
        A.skrull_linear(x[0], w)
    with pytest.raises(B.SkrullError, match="weight"):
        B._linear_of(x, w[:, :32], 0, False)
    with pytest.raises(B.SkrullError, match="gated"):
        B._linear_of(x, w[:127], 0, True)
    with pytest.raises(B.SkrullError, match="y must be"):
        B._linear_of(x, w, 0, True, y=torch.zeros(4, 128, dtype=torch.bfloat16))
    with pytest.raises(B.SkrullError, match="current GPU"):
        B.skrull_linear_fwd(x, w, None, None, x, None, None)
