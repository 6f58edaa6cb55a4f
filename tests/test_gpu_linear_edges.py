"""Products on the GPU at the edges of what their entry points take."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("inputs,outputs,activation,gated", [(4096, 6144, "none", False), (3584, 14336, "silu", True)])
@pytest.mark.parametrize("watched", [False, True])
def test_no_rows_of_a_wide_weight(monkeypatch, inputs, outputs, activation, gated, watched):
    """An empty micro-batch through a weight whose gradient has more than a round of tiles and a few left over: gradients of zero, by both paths."""
    from paper_2505_19609_amd import autograd as A
    monkeypatch.setattr(A, "_watched", lambda: watched)
    n = outputs * (1 + gated)
    x, w, b, r = (torch.zeros(s, dtype=torch.bfloat16, device="cuda", requires_grad=True) for s in ((0, inputs), (n, inputs), (n,), (0, outputs)))
    y = A.skrull_linear(x, w, b, r, activation, gated)
    assert y.shape == (0, outputs)
    dx, dw, db, dr = torch.autograd.grad(y, (x, w, b, r), torch.zeros_like(y))
    assert dx.shape == x.shape and dr.shape == r.shape and dw.shape == w.shape and db.shape == b.shape
    assert (dw == 0).all() and (db == 0).all()


def test_no_rows_write_whole_gradients():
    from paper_2505_19609_amd import binding as B
    from gpu_util import guarded, margins_intact
    x, w, dy = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((0, 4096), (6144, 4096), (0, 6144)))
    bufs = {s: guarded(s, torch.bfloat16, float("nan")) for s in ((6144, 4096), (6144,))}
    (_, dw), (_, db) = bufs.values()
    B.skrull_linear_bwd(x, w, None, dy, None, dw, db, None)
    assert (dw == 0).all() and (db == 0).all() and all(margins_intact(v[0]) for v in bufs.values())


@pytest.mark.parametrize("rows,inputs,outputs", [(70, 72, 136), (1500, 520, 264)])
@pytest.mark.parametrize("activation,gated", [("relu", False), ("gelu", False), ("silu", False), ("none", True), ("relu", True), ("gelu", True), ("silu", True)])
def test_gradients_of_rows_that_are_not_finite(rows, inputs, outputs, activation, gated):
    """A row whose z is NaN has a dx of NaN, and so have dw and db, which are sums over it; the other rows' dx is what it is beside any values there."""
    from paper_2505_19609_amd.autograd import skrull_linear
    gen = torch.Generator(device="cuda").manual_seed(rows)
    n = outputs * (1 + gated)
    x, w, b, dy = ((torch.randn(s, generator=gen, device="cuda") * scale).to(torch.bfloat16)
                   for s, scale in (((rows, inputs), 1.0), ((n, inputs), inputs ** -0.5), ((n,), 0.5), ((rows, outputs), 1.0)))
    bad = torch.tensor([0, 33, rows - 1], device="cuda")
    good = torch.ones(rows, dtype=torch.bool, device="cuda")
    good[bad] = False

    def gradients():
        leaves = [t.detach().clone().requires_grad_() for t in (x, w, b)]
        return torch.autograd.grad(skrull_linear(*leaves, None, activation, gated), leaves, dy)
    want = gradients()
    assert all(torch.isfinite(t).all() for t in want)
    x[bad, inputs - 1] = float("nan")
    dx, dw, db = gradients()
    assert torch.isnan(dx[bad]).all() and torch.isnan(dw).all() and torch.isnan(db).all()
    assert torch.equal(dx[good], want[0][good])


@pytest.mark.parametrize("rows,inputs,outputs,activation,gated,stride", [(33, 16312, 65536, "silu", True, 16312), (40, 65536, 65536, "gelu", False, 65536), (1500, 520, 264, "silu", True, 1 << 20)])
def test_widths_and_strides_at_their_limits(rows, inputs, outputs, activation, gated, stride):
    """The widest weights, where a gate's second half begins almost 2^31 bytes behind the first, and rows 2^20 elements apart: y and dw at a sample of columns, dx whole, within test_gpu_linear.py's
    bounds.  (dx's reference adds up pieces of 4,096 columns, whose bound counts 4,096 sums each: more than there are in all, since a product adds 32 columns at once.)"""
    from paper_2505_19609_amd.autograd import skrull_linear
    from test_gpu_linear import _check, _reference
    gen = torch.Generator(device="cuda").manual_seed(outputs)
    n = outputs * (1 + gated)
    wide = torch.full((rows, stride), float("nan"), dtype=torch.bfloat16, device="cuda")
    x = wide[:, :inputs].normal_(generator=gen).requires_grad_()
    w = torch.empty(n, inputs, dtype=torch.bfloat16, device="cuda").normal_(generator=gen).mul_(inputs ** -0.5).requires_grad_()
    dy = torch.empty(rows, outputs, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    y = skrull_linear(x, w, None, None, activation, gated)
    dx, dw = torch.autograd.grad(y, (x, w), dy)

    def reference(cols):
        at = torch.cat((cols, outputs + cols)) if gated else cols
        return at, _reference(x, w.detach()[at], None, None, dy[:, cols], activation, gated)
    at, want = reference(torch.tensor([0, 1, 255, 256, outputs // 2, outputs - 9, outputs - 1], device="cuda"))
    _check({"y": y.detach()[:, at[:7]], "dw": dw[at]}, want, "sample")
    exact, error = torch.zeros(2, rows, inputs, dtype=torch.float64, device="cuda")
    for first in range(0, outputs, 4096):
        value, off = reference(torch.arange(first, min(first + 4096, outputs), device="cuda"))[1]["dx"]
        exact += value
        error += off
    _check({"dx": dx}, {"dx": (exact, error)}, "dx")
    torch.cuda.empty_cache()
