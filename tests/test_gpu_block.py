"""What a block is made of besides its attention, rotary positions and loss, on the GPU against plain implementations in 64 bits: the residual stream
between two blocks.

Tolerances are bounds, not observations: a rounding to bf16 is off by at most 2^-8 of the value (half a step is 2^-9 of the next power of two), one
of fp32 by 2^-24, and a sum of n fp32 terms by at most n 2^-24 of the sum of their magnitudes; TINY covers results below bf16's normal numbers."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, FP32, TINY = 2.0 ** -8, 2.0 ** -24, 1e-30
TYPES = {torch.bfloat16: BF16, torch.float32: FP32}


def _randn(gen, *shape, dtype=torch.bfloat16, scale=1.0, mean=0.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale + mean).to(dtype)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _within(got, want, error, what):
    """`error`: of the result before it is rounded to its type"""
    assert got.shape == want.shape, what
    assert torch.isfinite(got).all(), what
    tolerance = error * 1.05 + TYPES[got.dtype] * (want.abs() + error) + TINY   # (5 %: products of two errors)
    excess = ((got.double() - want).abs() - tolerance).max().item() if want.numel() else 0.0
    assert excess <= 0.0, (what, excess, (got.double() - want).abs().max().item())


def _padded(t, pad=24, fill=float("nan")):
    """The rows of `t` inside wider ones: (the wider tensor, a view that equals t)."""
    wide = torch.full((t.shape[0], t.shape[1] + pad), fill, dtype=t.dtype, device=t.device)
    view = wide[:, :t.shape[1]]
    view.copy_(t)
    return wide, view


# ---- the residual stream between two blocks -------------------------------------------------------------------------

# roundings of a sum over a row: 8 values of a lane, 6 across a wavefront, 16 across wavefronts, and a few of the formula
ROW = 64 * FP32


def _mean(t):
    return t.mean(1, keepdim=True)


def _normed(x, ex, eps, layer):
    """The normed x, 1 / its deviation, and the errors of both (the second one relative), given x's."""
    mean = _mean(x) if layer else torch.zeros_like(x[:, :1])
    rstd = 1 / (_mean((x - mean).square()) + eps).sqrt()
    h = (x - mean) * rstd
    e = ex + ROW * x.abs() + (_mean(ex) + ROW * _mean(x.abs()) if layer else 0.0)   # of x less its mean
    relative = ROW + rstd * _mean(h.abs() * e)
    return h, rstd, rstd * e + h.abs() * relative, relative


def _norm_back(g, eg, h, eh, rstd, relative, layer):
    m, size = _mean(g * h), _mean((g * h).abs())
    em = _mean(g.abs() * eh + h.abs() * eg) + ROW * size
    d, ed = g - h * m, eg + eh * m.abs() + h.abs() * em + ROW * (g.abs() + h.abs() * size)
    if layer:
        d, ed = d - _mean(g), ed + _mean(eg) + ROW * _mean(g.abs())
    return d * rstd, ed * rstd + relative * (d * rstd).abs()


def _residual_in_64_bits(r, z, w, b, pw, pb, gate, scale, d_r, dy, eps, layer):
    """{name: (value, error)}: of each result in 64 bits, and what an evaluation in 32 bits may be off"""
    r, z, w, b, pw, pb, gate, d_r, dy = (None if t is None else t.detach().double() for t in (r, z, w, b, pw, pb, gate, d_r, dy))
    zero, rows = torch.zeros_like(z), len(z)
    one, none = torch.ones_like(w), torch.zeros_like(w)
    g, b1, b2 = (d if t is None else t for t, d in ((gate, one), (pb, none), (b, none)))
    w1 = one if pw is None else pw
    h1, rstd1, eh1, rel1 = (z, None, zero, None) if pw is None else _normed(z, zero, eps, layer)
    n = h1 * w1 + b1
    en = w1.abs() * eh1 + 4 * FP32 * ((h1 * w1).abs() + b1.abs())
    x = scale * r + g * n
    ex = g.abs() * en + 4 * FP32 * ((scale * r).abs() + g.abs() * ((h1 * w1).abs() + b1.abs()))
    h2, rstd2, eh2, rel2 = _normed(x, ex, eps, layer)
    out = {"r": (x, ex), "y": (h2 * w + b2, w.abs() * eh2 + 4 * FP32 * ((h2 * w).abs() + b2.abs()))}
    if d_r is None and dy is None:
        return out
    e, ee = (zero, zero) if dy is None else _norm_back(dy * w, FP32 * (dy * w).abs(), h2, eh2, rstd2, rel2, layer)
    if d_r is not None:
        e, ee = e + d_r, ee + 2 * FP32 * (e.abs() + d_r.abs())
    if dy is None:
        dy = zero
    out["dr"] = (scale * e, abs(scale) * ee + 2 * FP32 * (scale * e).abs())
    g1, eg1 = e * g * w1, (g * w1).abs() * (ee + 4 * FP32 * e.abs())
    out["dz"] = (g1, eg1) if pw is None else _norm_back(g1, eg1, h1, eh1, rstd1, rel1, layer)
    sums = (rows + 64) * FP32
    E1, eE1 = (e * h1).sum(0), (h1.abs() * ee + e.abs() * eh1 + sums * (e * h1).abs()).sum(0)
    E0, eE0 = e.sum(0), (ee + sums * e.abs()).sum(0)
    out.update(dw=((dy * h2).sum(0), (dy.abs() * eh2 + sums * (dy * h2).abs()).sum(0)), db=(dy.sum(0), sums * dy.abs().sum(0)),
               dpw=(g * E1, g.abs() * eE1 + 2 * FP32 * (g * E1).abs()), dpb=(g * E0, g.abs() * eE0 + 2 * FP32 * (g * E0).abs()),
               dgate=(w1 * E1 + b1 * E0, w1.abs() * eE1 + b1.abs() * eE0 + 4 * FP32 * ((w1 * E1).abs() + (b1 * E0).abs())))
    return out


RESIDUAL_SHAPES = [(1, 1), (1, 64), (3, 7), (5, 8), (3, 9), (5, 896), (64, 512), (33, 513), (2, 1024), (130, 1025), (9, 2048), (700, 3584), (17, 4096), (6, 4097), (3, 8192), (600, 8190),
                   (5000, 104)]
NAMES = ("r", "z", "w", "b", "pw", "pb", "gate")


def _residual_inputs(gen, rows, cols, t, rt, wt, b, pw, pb, gate):
    r = (_randn(gen, rows, cols, dtype=torch.float32) * _randn(gen, rows, 1, dtype=torch.float32).exp() + 2.0).to(rt)
    vectors = [_randn(gen, cols, dtype=wt, scale=0.3, mean=m) if there else None for m, there in ((1.0, True), (0.0, b), (1.0, pw), (0.0, pb), (0.5, gate))]
    return [r, _randn(gen, rows, cols, dtype=t, mean=0.5), *vectors]


@pytest.mark.parametrize("rows,cols", RESIDUAL_SHAPES)
@pytest.mark.parametrize("kind,b,pw,pb,gate", [("rms", 0, 0, 0, 0), ("rms", 0, 1, 0, 1), ("layer", 1, 1, 1, 1), ("layer", 0, 0, 0, 1), ("layer", 1, 1, 0, 0)])
@pytest.mark.parametrize("t,rt,wt", [(torch.bfloat16, torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32, torch.float32), (torch.float32, torch.float32, torch.bfloat16)])
def test_residual_norm(rows, cols, kind, b, pw, pb, gate, t, rt, wt):
    from paper_2505_19609_amd.autograd import skrull_residual_norm
    gen = _gen(rows * 10007 + cols)
    given = [None if v is None else v.requires_grad_() for v in _residual_inputs(gen, rows, cols, t, rt, wt, b, pw, pb, gate)]
    d_r, dy = _randn(gen, rows, cols, dtype=rt), _randn(gen, rows, cols, dtype=t)
    eps, scale = 1e-3, 0.75
    out = skrull_residual_norm(*given, scale, eps, kind)
    assert out[0].dtype == rt and out[1].dtype == t
    wanted = {n: v for n, v in zip(NAMES, given) if v is not None}
    grads = torch.autograd.grad(out, list(wanted.values()), (d_r, dy))
    got = {"r": out[0].detach(), "y": out[1].detach(), **{"d" + n: g for n, g in zip(wanted, grads)}}
    want = _residual_in_64_bits(*given, scale, d_r, dy, eps, kind == "layer")
    for name, value in got.items():
        _within(value, *want[name], name)


@pytest.mark.parametrize("which", [0, 1])
@pytest.mark.parametrize("cols", [77, 896, 8192])
def test_residual_norm_with_one_gradient(which, cols):
    """Only the stream's gradient, or only the normed rows': the other one's is as if it were zero, the same bits."""
    from paper_2505_19609_amd.autograd import skrull_residual_norm
    gen = _gen(cols)
    given = [v.requires_grad_() for v in _residual_inputs(gen, 37, cols, torch.bfloat16, torch.float32, torch.bfloat16, 1, 1, 1, 1)]
    d = [_randn(gen, 37, cols, dtype=torch.float32), _randn(gen, 37, cols)]
    out = skrull_residual_norm(*given)
    used = [n for i, n in enumerate(given) if not (which == 0 and i in (2, 3))]
    got = torch.autograd.grad(out[which], used, d[which], retain_graph=True)
    want = torch.autograd.grad(out, used, [v if i == which else torch.zeros_like(v) for i, v in enumerate(d)])
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("cols,pad", [(896, 8), (896, 3), (4096, 24), (1001, 7), (5, 2)])
def test_residual_strides_and_in_place(cols, pad):
    """Rows inside wider ones, aligned and not: what contiguous rows give, to the same bits, and nothing beside them is touched; the new stream in the
    place of the old one and y in the place of z are the same bits too, and stats may be left out."""
    from paper_2505_19609_amd import binding as B
    gen, rows = _gen(cols + pad), 41
    r, z, *vectors = _residual_inputs(gen, rows, cols, torch.bfloat16, torch.bfloat16, torch.bfloat16, 1, 1, 1, 1)
    d_r, dy = _randn(gen, rows, cols), _randn(gen, rows, cols)

    def both(r, z, d_r, dy, r_out, y, dr, dz):
        stats = torch.empty(4, rows, device="cuda")
        grads = [torch.full_like(v, float("nan")) for v in vectors]
        B.skrull_residual_fwd(r, z, *vectors, r_out, y, stats, 1.25, 1e-5, B.NORM_LAYER)
        ws = torch.full((B.skrull_residual_workspace(r, z, vectors[0], B.NORM_LAYER),), 0xFF, dtype=torch.uint8, device="cuda")
        w, _, pw, pb, gate = vectors
        B.skrull_residual_bwd(r, z, w, pw, pb, gate, stats, d_r, dy, dr, dz, *grads, ws, 1.25, B.NORM_LAYER)
        return [r_out, y, dr, dz, *grads]

    fresh = [torch.empty_like(r) for _ in range(4)]
    want = both(r, z, d_r, dy, *fresh)
    wides, views = zip(*(_padded(t, pad, 5.0) for t in (r, z, d_r, dy, r, r, r, r)))
    got = both(*views)
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    assert all((t[:, cols:] == 5).all() for t in wides)
    r2, z2 = r.clone(), z.clone()
    B.skrull_residual_fwd(r2, z2, *vectors, r2, z2, None, 1.25, 1e-5, B.NORM_LAYER)
    assert torch.equal(r2, want[0]) and torch.equal(z2, want[1])


@pytest.mark.parametrize("cols", [136, 4096])
def test_residual_of_rows_far_apart(cols):
    """Rows 2^31 elements and more apart: the bits of contiguous ones."""
    from paper_2505_19609_amd import binding as B
    gen = _gen(cols)
    r, z, *vectors = _residual_inputs(gen, 3, cols, torch.bfloat16, torch.bfloat16, torch.bfloat16, 1, 1, 1, 1)
    d_r, dy = _randn(gen, 3, cols), _randn(gen, 3, cols)
    w, _, pw, pb, gate = vectors
    far = lambda t: torch.empty(2 * ((1 << 31) + 8) + cols, dtype=t.dtype, device="cuda").as_strided((3, cols), ((1 << 31) + 8, 1)).copy_(t)   # noqa: E731
    results = []
    for place in (torch.Tensor.clone, far):
        R, Z, DR, DY, *out = [place(t) for t in (r, z, d_r, dy, r, z, r, z)]
        stats, grads = torch.empty(4, 3, device="cuda"), [torch.empty_like(v) for v in vectors]
        B.skrull_residual_fwd(R, Z, *vectors, out[0], out[1], stats, 1.25, 1e-5, B.NORM_LAYER)
        ws = torch.empty(B.skrull_residual_workspace(R, Z, w, B.NORM_LAYER), dtype=torch.uint8, device="cuda")
        B.skrull_residual_bwd(R, Z, w, pw, pb, gate, stats, DR, DY, out[2], out[3], *grads, ws, 1.25, B.NORM_LAYER)
        results.append([t.contiguous() for t in out] + grads)
        del R, Z, DR, DY, out
    assert all(torch.equal(a, c) for a, c in zip(*results))
    torch.cuda.empty_cache()


def test_residual_without_rows_and_with_a_row_of_infinities():
    from paper_2505_19609_amd.autograd import skrull_residual_norm
    vectors = [torch.ones(96, device="cuda", requires_grad=True) for _ in range(5)]
    r, z = (torch.empty(0, 96, device="cuda", requires_grad=True) for _ in range(2))
    out = skrull_residual_norm(r, z, *vectors)
    grads = torch.autograd.grad(out, (r, z, *vectors), [torch.empty(0, 96, device="cuda")] * 2)
    assert all(t.shape == (0, 96) for t in (*out, *grads[:2])) and all((g == 0).all() for g in grads[2:])
    r, z = torch.ones(5, 96, device="cuda"), torch.ones(5, 96, device="cuda")
    r[2, 3] = math.inf
    r[3], z[3] = -1.0, 0.5
    stream, y = skrull_residual_norm(r, z, vectors[0], eps=0.25, kind="rms")
    assert stream[2, 3] == math.inf and torch.isnan(y[2, 3]) and torch.isfinite(y[[0, 1, 3, 4]]).all()   # (a row's own trouble stays its own)
    assert torch.equal(y[0], y[4]) and (stream[3] == -0.5).all()


def test_residual_backward_for_some_of_its_inputs():
    from paper_2505_19609_amd.autograd import skrull_residual_norm
    gen = _gen(78)
    given = _residual_inputs(gen, 40, 640, torch.bfloat16, torch.bfloat16, torch.float32, 1, 1, 1, 1)
    d = _randn(gen, 40, 640), _randn(gen, 40, 640)
    want = None
    for need in ((1,) * 7, (1, 1, 0, 0, 0, 0, 0), (0, 0, 1, 0, 0, 0, 0), (0, 0, 0, 1, 0, 0, 1), (0, 1, 0, 0, 1, 0, 0), (0, 0, 0, 0, 0, 1, 0)):
        leaves = [t.clone().requires_grad_(bool(n)) for t, n in zip(given, need)]
        grads = torch.autograd.grad(skrull_residual_norm(*leaves), [t for t in leaves if t.requires_grad], d)
        want = want or grads
        assert all(torch.equal(g, want[i]) for g, i in zip(grads, [i for i in range(7) if need[i]]))


def test_residual_gradient_against_differences():
    """The change of both results along the gradient is what the gradient says (differences of the 64-bit form)."""
    from paper_2505_19609_amd.autograd import skrull_residual_norm
    gen = _gen(5)
    given = [t.requires_grad_() for t in _residual_inputs(gen, 9, 96, *[torch.float32] * 3, 1, 1, 1, 1)]
    d = [_randn(gen, 9, 96, dtype=torch.float32) for _ in range(2)]
    grads = torch.autograd.grad(skrull_residual_norm(*given, 0.75, 1e-3), given, d)

    def value(step):
        out = _residual_in_64_bits(*[t.detach().double() + step * g.double() for t, g in zip(given, grads)], 0.75, None, None, 1e-3, True)
        return sum((out[n][0] * v.double()).sum().item() for n, v in zip("ry", d))
    step = 1e-6
    slope = (value(step) - value(-step)) / (2 * step)
    square = sum(g.double().square().sum().item() for g in grads)
    # (the gradients' own errors, some 2^-20 of them, and the differences' third derivatives and roundings)
    assert abs(slope - square) <= 1e-4 * square


# ---- the wrappers, of all of a block's operators --------------------------------------------------------------------

def _calls():
    """Differentiable calls: (inputs, call)."""
    from paper_2505_19609_amd import autograd as A
    from paper_2505_19609_amd import binding as B
    gen = _gen(71)
    plan = B.skrull_attn_plan([700, 129, 640, 64], [1, 1, 2, 1], [0, 0, 1, 0], 4, 2, 64, 0.125, shard_cut=[0, 0, 1, 0])
    q, k, v = _randn(gen, plan.total_q, 4, 64), _randn(gen, plan.total_k, 2, 64), _randn(gen, plan.total_k, 2, 64)
    stream = _residual_inputs(gen, 50, 264, *[torch.bfloat16] * 3, 1, 1, 1, 1)
    x, w, b, r = _randn(gen, 50, 264), _randn(gen, 128, 264, scale=0.1), _randn(gen, 128), _randn(gen, 50, 64)
    return [((q, k, v), lambda q, k, v: A.skrull_window_attention(q, k, v, plan, 90, 5)),
            (stream, lambda *t: A.skrull_residual_norm(*t, 1.5, 1e-4)),
            ([t.float() for t in stream[:3]], lambda r, z, w: A.skrull_residual_norm(r, z, w, kind="rms")),
            ((x, w, b, r), lambda x, w, b, r: A.skrull_linear(x, w, b, r, "gelu", True)),
            ((x, w), lambda x, w: A.skrull_linear(x, w)),
            ((x, w, b), lambda x, w, b: A.skrull_linear(x, w, b, None, "silu"))]


CALLS = range(6)


def _tuple(out):
    return out if isinstance(out, tuple) else (out,)


@pytest.mark.parametrize("i", CALLS)
def test_native_calls_and_functions_give_the_same_bits(monkeypatch, i):
    from paper_2505_19609_amd import autograd as A
    inputs, call = _calls()[i]
    results = []
    for watched in (False, True):
        monkeypatch.setattr(A, "_watched", lambda: watched)
        given = [t.clone().requires_grad_() for t in inputs]
        out = _tuple(call(*given))
        gen = _gen(72)
        d = [_randn(gen, *o.shape, dtype=o.dtype) for o in out]
        results.append([o.detach() for o in out] + list(torch.autograd.grad(out, given, d)))
        assert all(("Skrull" in type(o.grad_fn).__name__) == watched for o in out)
        with torch.no_grad():   # (and what a call without gradients gives)
            plain = _tuple(call(*inputs))
        assert all(torch.equal(a, b) and a.grad_fn is None for a, b in zip(plain, results[-1]))
    assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("watched", [False, True])
@pytest.mark.parametrize("i", CALLS)
def test_gradients_are_not_differentiated_again(monkeypatch, i, watched):
    from paper_2505_19609_amd import autograd as A
    monkeypatch.setattr(A, "_watched", lambda: watched)
    inputs, call = _calls()[i]
    for varies in (True, False):
        given = [t.clone().requires_grad_() for t in inputs]
        out = _tuple(call(*given))
        d = [torch.ones_like(o).requires_grad_(varies) for o in out]
        grads = torch.autograd.grad(out, given, d, create_graph=True)
        with pytest.raises(RuntimeError, match="differentiate"):
            torch.autograd.grad(grads[0].float().sum(), d if varies else given)


@pytest.mark.parametrize("watched", [False, True])
@pytest.mark.parametrize("i", CALLS)
def test_a_graph_is_freed_by_its_backward_pass_and_sees_changed_inputs(monkeypatch, i, watched):
    from paper_2505_19609_amd import autograd as A
    monkeypatch.setattr(A, "_watched", lambda: watched)
    inputs, call = _calls()[i]

    def outputs():
        given = [t.clone().requires_grad_() for t in inputs]
        out = _tuple(call(*given))
        return given, out, [torch.ones_like(o) for o in out]

    given, out, d = outputs()
    first = torch.autograd.grad(out, given, d, retain_graph=True)
    assert all(torch.equal(a, b) for a, b in zip(first, torch.autograd.grad(out, given, d)))
    with pytest.raises(RuntimeError, match="second time"):
        torch.autograd.grad(out, given, d)
    given, out, d = outputs()
    with torch.no_grad():
        given[1].mul_(2)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad(out, given, d)
    given, out, d = outputs()
    del given
    out[0].sum().backward()      # (leaves that only the graph holds)


@pytest.mark.parametrize("watched", [False, True])
@pytest.mark.parametrize("i", CALLS)
def test_a_captured_call_is_refused_while_an_eager_graph_has_its_leaves(monkeypatch, i, watched):
    from paper_2505_19609_amd import autograd as A
    inputs, call = _calls()[i]
    given = [t.clone().requires_grad_() for t in inputs]
    eager = call(*given)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    monkeypatch.setattr(A, "_watched", lambda: watched)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        given[0].detach().add(1)     # (something to capture)
        with pytest.raises(ValueError, match="outside this capture"):
            call(*given)
        with torch.no_grad():
            call(*given)             # (without gradients there is nothing to refuse)
    torch.cuda.synchronize()
    del eager


@pytest.mark.parametrize("i", CALLS)
def test_captured_training_calls(i):
    """Forward and gradients through autograd, captured: replays give the eager bits, on new values too."""
    inputs, call = _calls()[i]
    given = [t.clone().requires_grad_() for t in inputs]
    gen = _gen(73)

    def step():
        out = _tuple(call(*given))
        return [o.detach() for o in out] + list(torch.autograd.grad(out, given, d))

    with torch.no_grad():
        d = [_randn(gen, *o.shape, dtype=o.dtype) for o in _tuple(call(*given))]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        captured = step()
    for rep in range(3):
        with torch.no_grad():
            for t in given:
                t.copy_(_randn(gen, *t.shape, dtype=t.dtype))
        for t in captured:
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, want)), rep


@pytest.mark.parametrize("i", CALLS)
def test_calls_on_other_streams(i):
    """Three at a time, on streams of their own."""
    inputs, call = _calls()[i]
    given = [t.clone().requires_grad_() for t in inputs]

    def step():
        out = _tuple(call(*given))
        return [o.detach() for o in out] + list(torch.autograd.grad(out, given, [torch.ones_like(o) for o in out]))
    want = step()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(3):
        runs = []
        for st in streams:
            with torch.cuda.stream(st):
                runs.append(step())
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for r in runs for a, b in zip(r, want))


def test_wrappers_refuse_alike():
    """Calls that the native module hands back and the Functions refuse."""
    from paper_2505_19609_amd import autograd as A
    from paper_2505_19609_amd import binding as B
    z = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    w = torch.zeros(64, dtype=torch.bfloat16, device="cuda")
    plan = B.skrull_attn_plan([4], [1], [0], 2, 2, 64, 0.125)
    q = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    wide = torch.zeros(64, 64, dtype=torch.bfloat16, device="cuda")
    for call in (lambda: A.skrull_residual_norm(z, z.float(), w), lambda: A.skrull_residual_norm(z, z, w.float(), w), lambda: A.skrull_residual_norm(z[:3], z, w),
                 lambda: A.skrull_residual_norm(z, z, w, w, kind="rms"), lambda: A.skrull_residual_norm(z, z, w, post_bias=w), lambda: A.skrull_residual_norm(z, z, w, eps=-1.0),
                 lambda: A.skrull_residual_norm(z, z, w, scale=math.nan), lambda: A.skrull_residual_norm(z.half(), z.half(), w),
                 lambda: A.skrull_window_attention(q, q, q, plan, 0), lambda: A.skrull_window_attention(q, q, q, plan, 1, -1), lambda: A.skrull_window_attention(q, q, q[:3], plan, 1),
                 lambda: A.skrull_window_attention(q, q, q.float(), plan, 1), lambda: A.skrull_window_attention(q, q, q, plan, 1 << 31), lambda: A.skrull_window_attention(q, q, q, plan, 1, 1 << 40),
                 lambda: A.skrull_linear(z, wide[:, :60]), lambda: A.skrull_linear(z[:, :60], wide[:, :60].contiguous()), lambda: A.skrull_linear(z, wide[:60]),
                 lambda: A.skrull_linear(z, wide, w[:32]), lambda: A.skrull_linear(z, wide, None, z[:, :32]), lambda: A.skrull_linear(z, wide[:33], gated=True), lambda: A.skrull_linear(z.float(), wide),
                 lambda: A.skrull_linear(z, wide, w.float())):
        with pytest.raises(B.SkrullError):
            call()
    assert A.skrull_window_attention(q, q, q, plan, 1).shape == q.shape
    plan.destroy()
    with pytest.raises(B.SkrullError):
        A.skrull_window_attention(q, q, q, plan, 1)


# ---- all of them together, with the other operators -----------------------------------------------------------------

_LENGTHS, _WINDOW, _SINKS = (37, 200, 1, 410), 100, 3


def _block_case(seed=5, heads=(4, 2), d=64, hidden=264, middle=360, vocab=500):
    from paper_2505_19609_amd import binding as B
    gen, n = _gen(seed), (heads[0] + 2 * heads[1]) * d
    plan = B.skrull_attn_plan(list(_LENGTHS), [1] * len(_LENGTHS), [0] * len(_LENGTHS), heads[0], heads[1], d, d ** -0.5)
    one = lambda: 1 + _randn(gen, hidden, scale=0.2)   # noqa: E731
    leaves = {"r": _randn(gen, plan.total_q, hidden), "z": _randn(gen, plan.total_q, hidden), "w1": one(), "post": one(), "gate": 0.5 * one(),
              "wqkv": _randn(gen, n, hidden, scale=hidden ** -0.5), "bqkv": _randn(gen, n, scale=0.2), "wo": _randn(gen, hidden, heads[0] * d, scale=(heads[0] * d) ** -0.5),
              "w2": one(), "b2": _randn(gen, hidden, scale=0.1), "wgu": _randn(gen, 2 * middle, hidden, scale=hidden ** -0.5),
              "wd": _randn(gen, hidden, middle, scale=middle ** -0.5), "bd": _randn(gen, hidden, scale=0.2), "w3": one(), "vocab": _randn(gen, vocab, hidden, scale=1.5 * hidden ** -0.5)}
    target = torch.randint(0, vocab, (plan.total_q,), generator=gen, device="cuda")
    target[::17] = -1
    return plan, B.skrull_rotary_init(d, base=1e4), heads, d, {n: t.detach().requires_grad_() for n, t in leaves.items()}, target


def _block(plan, rotary, heads, d, p, target):
    """The stream, a block of windowed attention and a gated one of products, and the loss."""
    from paper_2505_19609_amd.autograd import skrull_cross_entropy, skrull_linear, skrull_norm, skrull_residual_norm, skrull_rotary, skrull_window_attention
    hq, hkv = heads
    r, y = skrull_residual_norm(p["r"], p["z"], p["w1"], None, p["post"], None, p["gate"], 1.0, 1e-5, "rms")
    q, k, v = (t.unflatten(1, (-1, d)) for t in skrull_linear(y, p["wqkv"], p["bqkv"]).split([hq * d, hkv * d, hkv * d], 1))
    q, k = skrull_rotary(q, k, plan, rotary)
    o = skrull_window_attention(q, k, v, plan, _WINDOW, _SINKS)
    r, y = skrull_residual_norm(r, skrull_linear(o.flatten(1), p["wo"]), p["w2"], p["b2"])
    r = skrull_linear(skrull_linear(y, p["wgu"], None, None, "silu", True), p["wd"], p["bd"], r)
    return skrull_cross_entropy(skrull_norm(r, p["w3"], None, 1e-5, "rms"), p["vocab"], target)


def _block_in_64_bits(heads, d, p, target):
    hq, hkv = heads
    rms = lambda t: t * (t.square().mean(1, keepdim=True) + 1e-5).rsqrt()   # noqa: E731
    r = p["r"] + p["gate"] * rms(p["z"]) * p["post"]
    q, k, v = (t.unflatten(1, (-1, d)) for t in ((rms(r) * p["w1"]) @ p["wqkv"].t() + p["bqkv"]).split([hq * d, hkv * d, hkv * d], 1))
    pos = torch.cat([torch.arange(n) for n in _LENGTHS]).cuda()
    seq = torch.repeat_interleave(torch.arange(len(_LENGTHS)), torch.tensor(_LENGTHS)).cuda()
    angle = (pos[:, None].double() * 1e4 ** (-torch.arange(d // 2, device="cuda").double() * 2 / d))[:, None]
    turn = lambda t: torch.cat((t[..., :d // 2] * angle.cos() - t[..., d // 2:] * angle.sin(), t[..., :d // 2] * angle.sin() + t[..., d // 2:] * angle.cos()), -1)   # noqa: E731
    q, k = turn(q), turn(k)
    far = pos[:, None] - pos[None]
    seen = (seq[:, None] == seq[None]) & (far >= 0) & ((far < _WINDOW) | (pos[None] < _SINKS))
    o = [(q[:, h] @ k[:, h * hkv // hq].t() * d ** -0.5).masked_fill(~seen, -math.inf).softmax(1) @ v[:, h * hkv // hq] for h in range(hq)]
    r = r + torch.cat(o, 1) @ p["wo"].t()
    y = (r - r.mean(1, keepdim=True)) / (r.var(1, unbiased=False, keepdim=True) + 1e-5).sqrt() * p["w2"] + p["b2"]
    a, b = (y @ p["wgu"].t()).chunk(2, 1)
    r = r + (a * torch.sigmoid(a) * b) @ p["wd"].t() + p["bd"]
    return torch.nn.functional.cross_entropy((rms(r) * p["w3"]) @ p["vocab"].t(), target.clamp(min=0), reduction="none") * (target >= 0)


def test_block_against_64_bits():
    plan, rotary, heads, d, p, target = _block_case()
    weight = torch.rand(len(target), generator=_gen(6), device="cuda")
    loss = _block(plan, rotary, heads, d, p, target)
    grads = torch.autograd.grad((loss * weight).sum(), list(p.values()))
    exact = {n: t.detach().double().requires_grad_() for n, t in p.items()}
    want = _block_in_64_bits(heads, d, exact, target)
    wanted = torch.autograd.grad((want * weight).sum(), list(exact.values()))
    # Thirteen tensors are rounded to bf16 on the way there (two streams, three normed rows, qkv, the turned ones, probabilities, o, three products' rows, the last stream) and
    # as many on the way back, each by 2^-8 of its values at most: their errors in 2-norm add to at most 26 * 2^-8 = 10 % of a gradient's, and of the loss 13 * 2^-8.
    assert ((loss.double() - want).norm() / want.norm()).item() <= 13 * BF16
    for name, a, b in zip(p, grads, wanted):
        assert ((a.double() - b).norm() / b.norm()).item() <= 26 * BF16, name
    plan.destroy()


def test_block_by_native_calls_and_by_functions_gives_the_same_bits(monkeypatch):
    from paper_2505_19609_amd import autograd as A
    plan, rotary, heads, d, p, target = _block_case(seed=8)

    def run():
        loss = _block(plan, rotary, heads, d, p, target)
        return [loss.detach(), *torch.autograd.grad(loss.sum(), list(p.values()))]
    native = run()
    monkeypatch.setattr(A, "_native_for", lambda *t: None)
    assert all(torch.equal(a, b) for a, b in zip(native, run()))
    plan.destroy()


def test_block_captured_and_replayed():
    plan, rotary, heads, d, p, target = _block_case(seed=7)
    gen = _gen(9)
    weight = torch.rand(len(target), generator=gen, device="cuda")

    def step():
        loss = _block(plan, rotary, heads, d, p, target)
        return [loss.detach(), *torch.autograd.grad(loss, list(p.values()), weight)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        captured = step()
    for rep in range(4):
        if rep >= 2:
            with torch.no_grad():
                for name in ("r", "z", "wqkv", "gate"):
                    p[name].mul_(0.9)
                target.copy_(target.roll(3))
        for t in captured:
            t.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, want)), rep
    plan.destroy()
