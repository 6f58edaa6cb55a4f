"""Rotary positions, norm and loss without a GPU: symbols, struct layouts and what the entry points refuse."""
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


def test_library_exports_every_declared_operator():
    header = "".join(open(os.path.join(ROOT, "include", f)).read() for f in ("skrull_rotary.h", "skrull_norm.h", "skrull_loss.h"))
    declared = set(re.findall(r"\b(skrull_(?:rotary|norm|loss)(?:_[a-z]+)*)\s*\(", header))
    assert declared == set(B.OPERATOR_SYMBOLS)
    for name in declared:
        assert getattr(B.lib(), name) is not None


def test_struct_layouts_match_headers():
    assert ctypes.sizeof(B.Rotary) == 4 * 4 + 6 * 8
    assert ctypes.sizeof(B.RotaryTensor) == 4 * 8 + 2 * 4
    assert ctypes.sizeof(B.Norm) == 8 + 4 * 4 + 8 + 4 * 8   # (eps and its padding)
    assert ctypes.sizeof(B.Loss) == 8 + 2 * 4 + 8


@pytest.mark.parametrize("kw", [
    dict(head_dim=96), dict(rotary_dim=8), dict(rotary_dim=0), dict(rotary_dim=72), dict(rotary_dim=144), dict(layout=2), dict(layout=-1), dict(scaling=4), dict(scaling=-1),
    dict(base=1.0), dict(base=math.inf), dict(base=math.nan), dict(factor=2.0), dict(scaling=B.ROTARY_LINEAR, factor=0.5),
    dict(scaling=B.ROTARY_NTK, factor=math.nan), dict(amplitude=0.0), dict(amplitude=math.inf),
    dict(scaling=B.ROTARY_PARTS, factor=2.0), dict(scaling=B.ROTARY_PARTS, factor=2.0, original_length=8192),
    dict(scaling=B.ROTARY_PARTS, factor=2.0, original_length=8192, low_turns=4, high_turns=1),
    dict(scaling=B.ROTARY_PARTS, factor=2.0, original_length=-1, low_turns=1, high_turns=4)])
def test_rotary_init_refuses(kw):
    with pytest.raises(B.SkrullError, match="rotary") as e:
        B.skrull_rotary_init(**{"head_dim": 128, **kw})
    assert e.value.code == B.SKRULL_EINVAL


def test_rotary_init_takes():
    assert B.skrull_rotary_init(64).rotary_dim == 64
    assert B.skrull_rotary_init(128, 48, B.ROTARY_INTERLEAVED, 5e5, B.ROTARY_PARTS, 8.0, 8192, 0, 32, 1.2).scaling == B.ROTARY_PARTS


def test_rotary_refuses_null():
    r = B.skrull_rotary_init(64)
    t = B.RotaryTensor(ONE, ONE, 64, 64, 1, B.ROWS_Q)
    assert B.lib().skrull_rotary(None, ctypes.byref(r), ctypes.byref(t), None, 0, None) == B.SKRULL_EINVAL
    assert B.lib().skrull_rotary_check(None) == B.SKRULL_EINVAL


def _norm(**kw):
    p = dict(rows=4, cols=64, kind=B.NORM_LAYER, type=B.TYPE_BF16, weight_type=B.TYPE_BF16, eps=1e-5, x_stride=64, y_stride=64, dy_stride=64,
             dx_stride=64)
    p.update(kw)
    return B.Norm(**p)


BAD_NORMS = [dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(cols=8193, x_stride=8193, y_stride=8193, dy_stride=8193, dx_stride=8193),
             dict(kind=2), dict(type=2), dict(weight_type=-1), dict(eps=-1.0), dict(eps=math.nan), dict(x_stride=63)]


@pytest.mark.parametrize("kw", BAD_NORMS + [dict(y_stride=63)])
def test_norm_fwd_refuses(kw):
    # (two tensors a page apart: they would not overlap)
    assert B.lib().skrull_norm_fwd(ctypes.byref(_norm(**kw)), ONE, 2 * ONE, None, 3 * ONE, None, None, None) == B.SKRULL_EINVAL
    assert "norm" in B.skrull_attn_strerror(B.SKRULL_EINVAL)


@pytest.mark.parametrize("kw", BAD_NORMS + [dict(dy_stride=63), dict(dx_stride=63)])
def test_norm_bwd_refuses(kw):
    args = [ONE, 2 * ONE, 3 * ONE, 4 * ONE, 5 * ONE, 6 * ONE, 7 * ONE, 8 * ONE, 9 * ONE, 1 << 30, None]
    assert B.lib().skrull_norm_bwd(ctypes.byref(_norm(**kw)), *args) == B.SKRULL_EINVAL


@pytest.mark.parametrize("at,value", [(0, None), (0, ONE + 1), (1, None), (3, None), (3, ONE + 64), (4, 5 * ONE + 2)])
def test_norm_fwd_refuses_pointers(at, value):
    args = [ONE, 2 * ONE, None, 3 * ONE, 5 * ONE, 6 * ONE, None]
    args[at] = value
    assert B.lib().skrull_norm_fwd(ctypes.byref(_norm()), *args) == B.SKRULL_EINVAL


@pytest.mark.parametrize("at,value", [(0, None), (1, None), (2, None), (3, None), (4, None), (5, None), (5, ONE + 64), (5, 5 * ONE + 128), (8, None), (8, ONE + 8), (9, 100)])
def test_norm_bwd_refuses_pointers(at, value):
    args = [ONE, 2 * ONE, 3 * ONE, 4 * ONE, 5 * ONE, 6 * ONE, 7 * ONE, 8 * ONE, 9 * ONE, 1 << 30, None]
    args[at] = value
    assert B.lib().skrull_norm_bwd(ctypes.byref(_norm()), *args) == B.SKRULL_EINVAL


def test_norm_without_a_mean_has_no_bias():
    p = _norm(kind=B.NORM_RMS)
    assert B.lib().skrull_norm_fwd(ctypes.byref(p), ONE, 2 * ONE, 4 * ONE, 3 * ONE, None, None, None) == B.SKRULL_EINVAL
    args = [ONE, 2 * ONE, None, 4 * ONE, 5 * ONE, 6 * ONE, 7 * ONE, 8 * ONE, 9 * ONE, 1 << 30, None]
    assert B.lib().skrull_norm_bwd(ctypes.byref(p), *args) == B.SKRULL_EINVAL


def _loss(**kw):
    p = dict(rows=4, hidden=64, vocab=100, x_stride=64)
    p.update(kw)
    return B.Loss(**p)


BAD_LOSSES = [dict(rows=-1), dict(rows=(1 << 24) + 1), dict(hidden=0), dict(hidden=60), dict(hidden=65544, x_stride=65544), dict(vocab=0), dict(vocab=(1 << 22) + 1),
              dict(x_stride=63)]


@pytest.mark.parametrize("kw", BAD_LOSSES)
def test_loss_refuses(kw):
    p = ctypes.byref(_loss(**kw))
    assert B.lib().skrull_loss_workspace(p, 0) == 0 and B.lib().skrull_loss_workspace(p, 1) == 0
    assert B.lib().skrull_loss_fwd(p, *[ONE] * 6, 1 << 40, None) == B.SKRULL_EINVAL
    assert B.lib().skrull_loss_bwd(p, *[ONE] * 8, 1 << 40, None) == B.SKRULL_EINVAL
    assert "loss" in B.skrull_attn_strerror(B.SKRULL_EINVAL)


@pytest.mark.parametrize("at,value", [(0, None), (0, ONE + 1), (1, None), (1, ONE + 8), (2, None), (2, ONE + 4), (3, None), (3, ONE + 2), (4, None), (5, None), (5, ONE + 8), (6, 1000)])
def test_loss_fwd_refuses_pointers(at, value):
    args = [ONE] * 6 + [1 << 40, None]
    args[at] = value
    assert B.lib().skrull_loss_fwd(ctypes.byref(_loss()), *args) == B.SKRULL_EINVAL


@pytest.mark.parametrize("at,value", [(0, None), (1, None), (1, ONE + 8), (2, None), (3, None), (4, None), (5, ONE + 8), (6, ONE + 8), (7, None), (8, 1000)])
def test_loss_bwd_refuses_pointers(at, value):
    args = [ONE + (i << 32) for i in range(8)] + [1 << 40, None]
    args[at] = value
    assert B.lib().skrull_loss_bwd(ctypes.byref(_loss()), *args) == B.SKRULL_EINVAL


@pytest.mark.parametrize("at,other,by", [(6, 1, 0), (6, 1, 100 * 64 * 2 - 16), (5, 1, 16), (5, 6, 100 * 64 * 2 - 16), (5, 6, 16 - 4 * 64 * 2)])
def test_loss_bwd_refuses_overlaps(at, other, by):
    args = [ONE + (i << 32) for i in range(8)] + [1 << 40, None]
    args[at] = args[other] + by
    assert B.lib().skrull_loss_bwd(ctypes.byref(_loss()), *args) == B.SKRULL_EINVAL
    assert "overlaps" in B.skrull_attn_strerror(B.SKRULL_EINVAL)


def test_loss_workspace_is_bounded():
    """dz is kept a piece of the vocabulary at a time, 2 GiB at most, however many rows and words there are."""
    x, w = torch.empty(1 << 20, 64, dtype=torch.bfloat16, device="meta"), torch.empty(1 << 20, 64, dtype=torch.bfloat16, device="meta")
    rows = (1 << 20) * 64
    assert B.skrull_loss_workspace(x, w, True) < (2 << 30) + 2 * rows + 4 * rows + (1 << 26)
    with pytest.raises(B.SkrullError, match="hidden"):
        B.skrull_loss_workspace(x[:, :60], w[:, :60].contiguous(), True)


def test_tensors_that_are_not_on_the_gpu_are_refused():
    x, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(64, dtype=torch.bfloat16)
    plan = B.Plan(None, B.PlanInfo(total_q=4, total_k=4, num_q_heads=1, num_kv_heads=1, head_dim=64))
    heads = x.view(4, 1, 64)
    for call in (lambda: A.skrull_norm(x, w), lambda: A.skrull_cross_entropy(x, x, torch.zeros(4, dtype=torch.int64)),
                 lambda: A.skrull_rotary(heads, heads, plan, B.skrull_rotary_init(64))):
        with pytest.raises(B.SkrullError, match="not on the current GPU"):
            call()


def test_the_wrappers_refuse_kinds_and_shapes():
    x, w = torch.zeros(4, 64), torch.zeros(64)
    with pytest.raises(ValueError, match="kind"):
        A.skrull_norm(x, w, kind="batch")
    with pytest.raises(ValueError, match="rows"):
        A.skrull_norm(x[0], w)


@pytest.mark.parametrize("call", [
    lambda x, w: B._norm_of(x, w, 1e-5, 0, y=x[:2]), lambda x, w: B._norm_of(x, w, 1e-5, 0, y=x.float()), lambda x, w: B._norm_of(x.t(), w, 1e-5, 0),
    lambda x, w: B._norm_of(x.half(), w, 1e-5, 0), lambda x, w: B._norm_of(x, w.half(), 1e-5, 0), lambda x, w: B._vector(w, 63, torch.bfloat16, "w"),
    lambda x, w: B._loss_of(x.float(), x, None), lambda x, w: B._loss_of(x, x[:, :32], None), lambda x, w: B._loss_of(x, x.t(), None),
    lambda x, w: B._loss_of(x, x, torch.zeros(4, dtype=torch.int32)), lambda x, w: B._loss_of(x, x, torch.zeros(5, dtype=torch.int64)),
    lambda x, w: B._loss_of(x.t(), x, None), lambda x, w: B._loss_of(x[0], x, None)])
def test_shapes_types_and_strides_are_checked(call):
    with pytest.raises(B.SkrullError):
        call(torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(64, dtype=torch.bfloat16))


def test_rotary_tensors_are_checked():
    plan = B.Plan(None, B.PlanInfo(total_q=4, total_k=6, num_q_heads=2, num_kv_heads=1, head_dim=64))
    q = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    k = torch.zeros(6, 1, 64, dtype=torch.bfloat16)
    assert B._rotary_tensor(plan.info, q, q, B.ROWS_Q).in_stride == 128
    assert B._rotary_tensor(plan.info, k, k, B.ROWS_K).heads == 1
    for x, out, rows in ((q, q, B.ROWS_K), (q, k, B.ROWS_Q), (q.float(), q, B.ROWS_Q), (q[:, :, :32], q, B.ROWS_Q),
                         (q.transpose(0, 1), q, B.ROWS_Q), (torch.zeros(4, 64, 2, dtype=torch.bfloat16).transpose(1, 2), q, B.ROWS_Q)):
        with pytest.raises(B.SkrullError):
            B._rotary_tensor(plan.info, x, out, rows)
