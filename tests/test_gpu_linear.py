"""Products with bias, activation, gate and residual on the GPU against plain implementations in 64 bits.

Tolerances are bounds, not observations: a rounding to bf16 is off by at most 2^-8 of the value, one of fp32 by 2^-24, and a sum of n fp32 terms by at
most n 2^-24 of the sum of their magnitudes.  The kernels round z (for the backward) and dz (for its products) to bf16; everything else is fp32
until the results are rounded.  Activations and their slopes are within 1e-5 of their size (exponentials of arguments up to 80, whose rounding is 2^-24 of
them, and a fit within 1.5e-6)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, FP32, TINY, ACT = 2.0 ** -8, 2.0 ** -24, 1e-30, 1e-5


def _randn(gen, *shape, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(torch.bfloat16)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _share(z):
    return 0.5 * torch.special.erfc(-z / math.sqrt(2.0))


# f, f' and bounds of |f'| and |f''|
ACTIVATIONS = {
    "none": (lambda z: z, torch.ones_like, 1.0, 0.0),
    "relu": (lambda z: z.clamp(min=0.0), lambda z: (z > 0.0).double(), 1.0, 0.0),
    "gelu": (lambda z: z * _share(z), lambda z: _share(z) + z * (-0.5 * z * z).exp() / math.sqrt(2.0 * math.pi), 1.13, 0.8),
    "silu": (lambda z: z * torch.sigmoid(z), lambda z: torch.sigmoid(z) * (1.0 + z * (1.0 - torch.sigmoid(z))), 1.1, 0.5),
}


def _reference(x, w, b, add, dy, activation, gated):
    """{name: (value, error)}: of each result in 64 bits, and what the kernels' arithmetic may be off before the last rounding"""
    x, w, b, add, dy = (None if t is None else t.detach().double() for t in (x, w, b, add, dy))
    f, slope, steepest, bend = ACTIVATIONS[activation]
    rows, inputs = x.shape
    size = x.abs() @ w.abs().t()
    z, ez = x @ w.t(), (inputs + 8) * FP32 * size
    if b is not None:
        z, ez = z + b, ez + 2 * FP32 * (size + b.abs())
    halves = z.chunk(2, 1) if gated else (z,)
    errors = ez.chunk(2, 1) if gated else (ez,)
    y = f(halves[0])
    ey = steepest * errors[0] + ACT * y.abs() if activation != "none" else errors[0]
    if gated:
        y, ey = y * halves[1], ey * halves[1].abs() + y.abs() * errors[1] + ey * errors[1] + FP32 * (y * halves[1]).abs()
    if add is not None:
        y, ey = y + add, ey + 2 * FP32 * (y.abs() + add.abs())
    out = {"y": (y, ey)}
    if dy is None:
        return out
    kept = [e + BF16 * (h.abs() + e) for h, e in zip(halves, errors)]        # of z as the backward reads it
    s = slope(halves[0])
    es = bend * kept[0] + (ACT * (1.0 + halves[0].abs()) if activation in ("gelu", "silu") else 0.0)
    if activation == "relu":
        es = (halves[0].abs() <= errors[0]).double()                         # (the sign of z is not known there)
    if gated:
        value = f(halves[0])
        ev = steepest * kept[0] + ACT * value.abs()
        dz = torch.cat((dy * halves[1] * s, dy * value), 1)
        e = torch.cat((dy.abs() * (halves[1].abs() * es + kept[1] * (s.abs() + es)), dy.abs() * ev), 1) + 4 * FP32 * dz.abs()
    else:
        dz, e = dy * s, dy.abs() * es + 2 * FP32 * (dy * s).abs()
    plain = activation == "none" and not gated
    rounded = 0.0 * e if plain else e + BF16 * (dz.abs() + e)
    n = w.shape[0]
    out["dx"] = (dz @ w, (rounded + (n + 8) * FP32 * dz.abs()) @ w.abs())
    out["dw"] = (dz.t() @ x, (rounded + (rows + 64) * FP32 * dz.abs()).t() @ x.abs())
    out["db"] = (dz.sum(0), (e + (rows + 64) * FP32 * dz.abs()).sum(0))
    return out


def _check(got, want, what):
    for name, value in got.items():
        exact, error = want[name]
        assert value.shape == exact.shape and torch.isfinite(value).all(), (what, name)
        tolerance = 1.02 * error + BF16 * (exact.abs() + error) + TINY
        excess = ((value.double() - exact).abs() - tolerance).max().item()
        assert excess <= 0.0, (what, name, excess, (value.double() - exact).abs().max().item())


def _inputs(gen, rows, inputs, outputs, bias, gated, add):
    n = outputs * (2 if gated else 1)
    return (_randn(gen, rows, inputs), _randn(gen, n, inputs, scale=1.5 * inputs ** -0.5), _randn(gen, n, scale=0.5) if bias else None,
            _randn(gen, rows, outputs) if add else None, _randn(gen, rows, outputs))


SIZES = [(1, 8, 8), (1, 64, 128), (2, 72, 64), (37, 896, 1152), (64, 136, 264), (65, 512, 120), (130, 904, 1160), (300, 64, 2048), (257, 1032, 8), (1001, 200, 520), (50, 4096, 64), (700, 2048, 96),
         (513, 256, 512)]
KINDS = [("none", False), ("relu", False), ("gelu", False), ("silu", False), ("silu", True), ("gelu", True), ("relu", True), ("none", True)]


@pytest.mark.parametrize("rows,inputs,outputs", SIZES)
@pytest.mark.parametrize("activation,gated", KINDS)
@pytest.mark.parametrize("bias,add", [(False, False), (True, True)])
def test_linear(rows, inputs, outputs, activation, gated, bias, add):
    from paper_2505_19609_amd.autograd import skrull_linear
    x, w, b, r, dy = _inputs(_gen(rows * 13 + inputs + outputs), rows, inputs, outputs, bias, gated, add)
    leaves = {n: t.requires_grad_() for n, t in (("dx", x), ("dw", w), ("db", b), ("add", r)) if t is not None}
    y = skrull_linear(x, w, b, r, activation, gated)
    grads = dict(zip(leaves, torch.autograd.grad(y, list(leaves.values()), dy)))
    if add:
        assert torch.equal(grads.pop("add"), dy)
    _check({"y": y.detach(), **grads}, _reference(x, w, b, r, dy, activation, gated), (activation, gated))


@pytest.mark.parametrize("rows,inputs,outputs", [(5000, 136, 72), (3000, 64, 8), (20, 16384, 128), (8192, 512, 256)])
@pytest.mark.parametrize("activation,gated", [("none", False), ("gelu", False), ("silu", True)])
def test_linear_of_long_contractions(rows, inputs, outputs, activation, gated):
    """Few tiles and many steps: the contraction in parts."""
    from paper_2505_19609_amd.autograd import skrull_linear
    x, w, b, _, dy = _inputs(_gen(rows), rows, inputs, outputs, True, gated, False)
    leaves = [t.requires_grad_() for t in (x, w, b)]
    y = skrull_linear(*leaves, None, activation, gated)
    got = dict(zip(("dx", "dw", "db"), torch.autograd.grad(y, leaves, dy)), y=y.detach())
    _check(got, _reference(x, w, b, None, dy, activation, gated), (activation, gated))


@pytest.mark.parametrize("rows,inputs,outputs,activation,gated", [(4400, 4104, 4104, "none", False), (4400, 4104, 4104, "gelu", False), (4400, 4104, 2056, "silu", True), (4352, 1024, 4096, "relu", False)])
def test_linear_of_a_round_of_tiles_and_some(rows, inputs, outputs, activation, gated):
    """Some tiles more than there are units, the last ones in parts where they have many steps; workspaces hold NaN before, and their margins stay."""
    from paper_2505_19609_amd import binding as B
    from gpu_util import guarded, margins_intact
    act = {"none": B.LINEAR_NONE, "relu": B.LINEAR_RELU, "gelu": B.LINEAR_GELU, "silu": B.LINEAR_SILU}[activation]
    x, w, b, r, dy = _inputs(_gen(rows + inputs), rows, inputs, outputs, True, gated, True)
    n = w.shape[0]
    sizes = [B.skrull_linear_workspace(x, w, k, act, gated) for k in (False, True)]
    assert sizes[0] > 0 or inputs < 4096    # (a few steps are not worth it)
    ws = [guarded((max(16, s),), torch.uint8, 0xFF) for s in sizes]
    shapes = {"y": (rows, outputs), "dx": (rows, inputs), "dw": (n, inputs), "db": (n,)}
    bufs = {name: guarded(s, torch.bfloat16, float("nan")) for name, s in shapes.items()}
    t = {name: v[1] for name, v in bufs.items()}
    z = torch.empty(rows, n, dtype=torch.bfloat16, device="cuda") if act or gated else None
    B.skrull_linear_fwd(x, w, b, r, t["y"], z, ws[0][1], act, gated)
    B.skrull_linear_bwd(x, w, z, dy, t["dx"], t["dw"], t["db"], ws[1][1], act, gated)
    assert all(margins_intact(v[0]) for v in (*bufs.values(), *ws))
    _check(t, _reference(x, w, b, r, dy, activation, gated), (activation, gated))


def _padded(t, pad, fill=float("nan")):
    wide = torch.full((t.shape[0], t.shape[1] + pad), fill, dtype=t.dtype, device=t.device)
    view = wide[:, :t.shape[1]]
    view.copy_(t)
    return wide, view


@pytest.mark.parametrize("rows,inputs,outputs", [(37, 72, 120), (300, 136, 264), (1500, 520, 64)])
@pytest.mark.parametrize("activation,gated", [("none", False), ("gelu", False), ("silu", True)])
def test_linear_strides_and_in_place(rows, inputs, outputs, activation, gated):
    """Rows inside wider ones that hold NaN beside them: what contiguous rows give, to the same bits, and nothing beside them is touched; y in the place of the
    residual and without z is the same bits too.  Workspaces hold NaN before."""
    from paper_2505_19609_amd import binding as B
    x, w, b, r, dy = _inputs(_gen(rows), rows, inputs, outputs, True, gated, True)
    act, n = {"none": B.LINEAR_NONE, "gelu": B.LINEAR_GELU, "silu": B.LINEAR_SILU}[activation], w.shape[0]

    def scratch(backward):
        return torch.full((max(16, B.skrull_linear_workspace(x, w, backward, act, gated)),), 0xFF, dtype=torch.uint8, device="cuda")

    def both(x, r, dy, y, z):
        B.skrull_linear_fwd(x, w, b, r, y, z, scratch(False), act, gated)
        grads = [torch.full(s, float("nan"), dtype=torch.bfloat16, device="cuda") for s in ((rows, inputs), (n, inputs), (n,))]
        B.skrull_linear_bwd(x, w, z if act or gated else None, dy, *grads, scratch(True), act, gated)
        return [y, *grads]
    z = torch.full((rows, n), float("nan"), dtype=torch.bfloat16, device="cuda")
    want = both(x, r, dy, torch.empty_like(r), z)
    assert torch.isfinite(z).all()
    wides, views = zip(*(_padded(t, 24) for t in (x, r, dy, torch.zeros_like(r))))
    got = both(*views, torch.empty_like(z))
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    assert all(torch.isnan(t[:, -24:]).all() for t in wides)
    again = r.clone()
    B.skrull_linear_fwd(x, w, b, again, again, None, scratch(False), act, gated)
    assert torch.equal(again, want[0])


def test_linear_nothing_beside_the_results_is_written():
    from paper_2505_19609_amd import binding as B
    from gpu_util import guarded, margins_intact
    for rows, inputs, outputs, gated in ((37, 72, 120, True), (300, 136, 264, False), (1, 8, 8, False), (2000, 520, 72, True)):
        x, w, b, r, dy = _inputs(_gen(rows), rows, inputs, outputs, True, gated, True)
        n = w.shape[0]
        shapes = {"y": (rows, outputs), "z": (rows, n), "dx": (rows, inputs), "dw": (n, inputs), "db": (n,)}
        bufs = {name: guarded(s, torch.bfloat16, float("nan")) for name, s in shapes.items()}
        ws = [guarded((max(16, B.skrull_linear_workspace(x, w, k, B.LINEAR_SILU, gated)),), torch.uint8, 0xFF) for k in (False, True)]
        t = {name: v[1] for name, v in bufs.items()}
        B.skrull_linear_fwd(x, w, b, r, t["y"], t["z"], ws[0][1], B.LINEAR_SILU, gated)
        B.skrull_linear_bwd(x, w, t["z"], dy, t["dx"], t["dw"], t["db"], ws[1][1], B.LINEAR_SILU, gated)
        assert all(margins_intact(v[0]) for v in (*bufs.values(), *ws))
        assert all(torch.isfinite(v).all() for v in t.values())


def test_linear_without_rows():
    from paper_2505_19609_amd.autograd import skrull_linear
    x, w, b = (torch.zeros(s, dtype=torch.bfloat16, device="cuda", requires_grad=True) for s in ((0, 64), (128, 64), (128,)))
    for activation, gated in (("none", False), ("silu", True)):
        y = skrull_linear(x, w, b, None, activation, gated)
        grads = torch.autograd.grad(y, (x, w, b), torch.zeros_like(y))
        assert y.shape == (0, 64 if gated else 128) and grads[0].shape == (0, 64) and all((g == 0).all() for g in grads[1:])


def test_linear_backward_for_some_of_its_inputs():
    from paper_2505_19609_amd.autograd import skrull_linear
    given = _inputs(_gen(3), 200, 264, 136, True, True, True)
    want = None
    for need in ((1, 1, 1, 1), (1, 0, 0, 0), (0, 1, 0, 0), (0, 0, 1, 0), (0, 0, 0, 1), (0, 1, 1, 0)):
        leaves = [t.clone().requires_grad_(bool(n)) for t, n in zip(given, need)]
        grads = torch.autograd.grad(skrull_linear(*leaves, "gelu", True), [t for t in leaves if t.requires_grad], given[4])
        want = want or grads
        assert all(torch.equal(g, want[i]) for g, i in zip(grads, [i for i in range(4) if need[i]]))


def test_linear_gradients_of_a_sum_and_of_transposed_rows():
    """Gradients that come in expanded (a sum's) or transposed, and rows that are transposed: as contiguous ones."""
    from paper_2505_19609_amd.autograd import skrull_linear
    x, w, b, _, dy = _inputs(_gen(4), 96, 72, 64, True, False, False)
    x, w = x.requires_grad_(), w.requires_grad_()
    y = skrull_linear(x, w, b, None, "silu")
    for given in (torch.ones((), dtype=torch.bfloat16, device="cuda").expand(96, 64), dy.t().contiguous().t()):
        got = torch.autograd.grad(y, (x, w), given, retain_graph=True)
        want = torch.autograd.grad(y, (x, w), given.contiguous(), retain_graph=True)
        assert all(torch.equal(a, c) for a, c in zip(got, want))
    assert torch.equal(skrull_linear(x.detach().t().contiguous().t(), w, b, None, "silu"), y)


@pytest.mark.parametrize("activation,gated", [("gelu", False), ("silu", True)])
def test_linear_gradient_against_differences(activation, gated):
    """The change of the 64-bit result along the gradient is what the gradient says, up to its roundings."""
    from paper_2505_19609_amd.autograd import skrull_linear
    x, w, b, r, dy = _inputs(_gen(5), 60, 72, 40, True, gated, True)
    leaves = [t.requires_grad_() for t in (x, w, b, r)]
    grads = torch.autograd.grad(skrull_linear(*leaves, activation, gated), leaves, dy)

    def value(step):
        moved = [t.detach().double() + step * g.double() for t, g in zip(leaves, grads)]
        return (_reference(*moved, None, activation, gated)["y"][0] * dy.double()).sum().item()
    step = 1e-6
    slope, square = (value(step) - value(-step)) / (2 * step), sum(g.double().square().sum().item() for g in grads)
    # (grads = exact + error: slope - square = -(grads . error), and |error| is some 2^-8 of |grads| for z, dz and the results each)
    assert abs(slope - square) <= 4 * BF16 * square


@pytest.mark.parametrize("activation", ["gelu", "silu"])
def test_linear_activations_far_out(activation):
    """Activations of z from -90 to 90 and zero: within their bounds, tails included."""
    from paper_2505_19609_amd.autograd import skrull_linear
    x = torch.eye(64, dtype=torch.bfloat16, device="cuda")
    w = torch.cat((torch.linspace(-90, 90, 4096, device="cuda"), torch.linspace(-6, 6, 4096, device="cuda"))).to(torch.bfloat16).view(128, 64).contiguous()
    w[0, 0] = 0.0
    dy = torch.ones(64, 128, dtype=torch.bfloat16, device="cuda")
    leaves = [x.requires_grad_(), w.requires_grad_()]
    y = skrull_linear(*leaves, None, None, activation)
    f, slope = ACTIVATIONS[activation][:2]
    z = w.detach().double().t()        # (exact: a product with ones and zeros)
    want = f(z)
    # relative to the result also where that is tiny: exponentials of -z^2 / 2 or -|z| whose argument has a rounding of 2^-24 of it; a share of z below fp32's normal
    # numbers, 2^-126, is 0, which is |z| 2^-126 of the result and (1 + |z|) 2^-126 of the slope
    argument = 0.5 * z * z if activation == "gelu" else z.abs()
    bound = (BF16 + ACT + 4 * FP32 * argument) * want.abs() + (1 + z.abs()) * 2.0 ** -126
    assert ((y.double() - want).abs() <= bound).all()
    dw = torch.autograd.grad(y, leaves[1], dy)[0].double().t()      # = slope of each z
    want = slope(z)
    # z as stored is z itself here; dz is rounded, and so is dw
    assert ((dw - want).abs() <= 2 * BF16 * want.abs() + ACT * (1 + z.abs()) * want.abs().clamp(min=2.0 ** -20) + (1 + z.abs()) * 2.0 ** -126).all()


def test_linear_captured_and_replayed_and_on_other_streams():
    from paper_2505_19609_amd.autograd import skrull_linear
    given = _inputs(_gen(6), 1500, 520, 264, True, True, True)
    leaves, dy = [t.requires_grad_() for t in given[:4]], given[4]

    def step():
        y = skrull_linear(*leaves, "silu", True)
        return [y.detach(), *torch.autograd.grad(y, leaves, dy)]
    want = step()
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(2):
        runs = []
        for st in streams:
            with torch.cuda.stream(st):
                runs.append(step())
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for r in runs for a, b in zip(r, want))
    runs = want = None
    side = streams[0]
    with torch.cuda.stream(side):
        step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        captured = step()
    for rep in range(3):
        with torch.no_grad():
            for t, v in zip(given, _inputs(_gen(20 + rep), 1500, 520, 264, True, True, True)):
                t.copy_(v)
        for t in captured[:4]:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, want)), rep


def test_linear_offsets_past_32_bits():
    """x, dx of 2.3 GB and y of 4.6: a sample of rows, and the gradient of the weight."""
    from paper_2505_19609_amd.autograd import skrull_linear
    gen = _gen(7)
    rows, inputs, outputs = 140000, 8192, 16384
    w = _randn(gen, outputs, inputs, scale=inputs ** -0.5)
    x = torch.empty(rows, inputs, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    dy = torch.zeros(rows, outputs, dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 1, 63, 65535, 65536, 131071, 131072, 139999], device="cuda")
    dy[at] = _randn(gen, len(at), outputs)
    x.requires_grad_()
    w.requires_grad_()
    y = skrull_linear(x, w, None, None, "silu")
    dx, dw = torch.autograd.grad(y, (x, w), dy)
    want = _reference(x.detach()[at], w, None, None, dy[at], "silu", False)
    _check({"y": y.detach()[at], "dx": dx[at], "dw": dw}, want, "sample")   # (rows without a gradient add nothing to dw)
    other = torch.ones(rows, dtype=torch.bool, device="cuda")
    other[at] = False
    assert (dx[other] == 0).all()


@pytest.mark.parametrize("rows,inputs,outputs", [(70, 72, 136), (1500, 520, 264)])
@pytest.mark.parametrize("activation,gated", KINDS)
def test_linear_rows_that_are_not_finite(rows, inputs, outputs, activation, gated):
    """A row with a NaN gives a row of NaN, and the others what they give beside any values there."""
    from paper_2505_19609_amd.autograd import skrull_linear
    x, w, b, r, _ = _inputs(_gen(12), rows, inputs, outputs, True, gated, True)
    want = skrull_linear(x, w, b, r, activation, gated)
    bad = torch.tensor([0, 33, rows - 1], device="cuda")
    x[bad, inputs - 1] = float("nan")
    got = skrull_linear(x, w, b, r, activation, gated)
    assert torch.isnan(got[bad]).all()
    good = torch.ones(rows, dtype=torch.bool, device="cuda")
    good[bad] = False
    assert torch.equal(got[good], want[good])
