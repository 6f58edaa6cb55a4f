"""Attention to a window of keys and the first keys of a sequence on the GPU against a plain implementation in 64 bits.

Tolerances are bounds, not observations.  A rounding to bf16 is off by at most 2^-8 of the value, one to fp16 by 2^-11 (2^-25 near zero), one of
fp32 by 2^-24, and a sum of n fp32 terms by at most n 2^-24 of the sum of their magnitudes.  The kernels round the probabilities to bf16 before the
product with V or dO, to fp16 before that with dP - D, and dS to bf16; everything else is fp32 until the results are rounded."""
import itertools

import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = 2.0 ** -8, 2.0 ** -11, 2.0 ** -24


def _slices(seq_len, degree, index, cut):
    """(first position, end, first row of Q, first row of K) of every slice of queries, rows of Q, rows of K"""
    out, q, k = [], 0, 0
    for s, n, r, z in zip(seq_len, degree, index, cut):
        chunks, end = n * (1 + z), 0
        for i in ([r, 2 * n - 1 - r] if z else [r]):
            begin, end = i * s // chunks, (i + 1) * s // chunks
            out.append((begin, end, q, k))
            q += end - begin
        k += end
    return out, q, k


def _reference(shape, q, k, v, d_o, scale, window, sinks):
    """{name: (value, error)} of O, LSE, dQ, dK, dV in 64 bits, and what the kernels' arithmetic may be off before the last rounding"""
    q, k, v, d_o = (t.double() for t in (q, k, v, d_o))
    hq, hkv, d = q.shape[1], k.shape[1], q.shape[2]
    g = hq // hkv
    names = {"o": q, "dq": q, "dk": k, "dv": k}
    out = {n: [torch.zeros_like(t), torch.zeros_like(t)] for n, t in names.items()}
    out["lse"] = [torch.zeros(hq, len(q), dtype=torch.float64, device=q.device) for _ in range(2)]
    for begin, end, q0, k0 in _slices(*shape)[0]:
        n = end
        if end == begin:
            continue
        qs, do = (t[q0:q0 + end - begin].transpose(0, 1) for t in (q, d_o))                              # [Hq, rows, d]
        ks, vs = (t[k0:k0 + n].transpose(0, 1).repeat_interleave(g, 0) for t in (k, v))                  # [Hq, keys, d]
        i, j = torch.arange(begin, end, device=q.device)[:, None], torch.arange(n, device=q.device)[None, :]
        seen = (j <= i) & ((i - j < window) | (j < sinks))
        s = (qs @ ks.transpose(1, 2)) * scale
        es = ((d + 8) * FP32 * scale) * (qs.abs() @ ks.abs().transpose(1, 2))
        s = torch.where(seen, s, -torch.inf)
        es = torch.where(seen, es, 0.0).amax(-1, keepdim=True)                                           # of a row's scores
        lse = torch.logsumexp(s, -1, keepdim=True)
        p = (s - lse).exp()
        sums = (seen.sum(-1, keepdim=True) + 16) * FP32
        elem = es + sums + 8 * FP32 * (1 + lse.abs())                                                     # of LSE, and relative of p
        o = p @ vs
        eo = (BF16 + 2 * elem) * (p @ vs.abs())
        total = eo + BF16 * (o.abs() + eo)
        dp = do @ vs.transpose(1, 2)
        edp = ((d + 8) * FP32) * (do.abs() @ vs.abs().transpose(1, 2))
        D = (do * o).sum(-1, keepdim=True)
        eD = (do.abs() * total).sum(-1, keepdim=True) + (d + 8) * FP32 * (do * o).abs().sum(-1, keepdim=True)
        ds = p * (dp - D)
        # (FP16's smallest step: a probability below 2^-14 may be off by 2^-25)
        eds = p * (2 * elem * (dp - D).abs() + edp + eD) + (BF16 + FP16) * 1.02 * ds.abs() + torch.where(seen, 2.0 ** -25 * (dp - D).abs(), 0.0)
        eds = eds * (1 + BF16)
        rows = (n + 64) * FP32
        at = slice(q0, q0 + end - begin)

        def put(name, where, value, error):
            out[name][0][where] += value
            out[name][1][where] += error

        def group(t):   # sum over the heads of a group, [keys, Hkv, d]
            return t.view(hkv, g, n, d).sum(1).transpose(0, 1)
        put("o", at, o.transpose(0, 1), eo.transpose(0, 1))
        out["lse"][0][:, at], out["lse"][1][:, at] = lse[..., 0], elem[..., 0]
        put("dq", at, scale * (ds @ ks).transpose(0, 1), scale * ((eds + rows * ds.abs()) @ ks.abs()).transpose(0, 1))
        put("dk", slice(k0, k0 + n), scale * group(ds.transpose(1, 2) @ qs), scale * group((eds + rows * ds.abs()).transpose(1, 2) @ qs.abs()))
        put("dv", slice(k0, k0 + n), group(p.transpose(1, 2) @ do), group((p * (BF16 + 2 * elem + rows)).transpose(1, 2) @ do.abs()))
    return out


def _check(got, want, what):
    for name, value in got.items():
        exact, error = want[name]
        assert value.shape == exact.shape and torch.isfinite(value).all(), (what, name)
        tolerance = 1.02 * error + (FP32 if name == "lse" else BF16) * (exact.abs() + error) + 1e-30
        excess = ((value.double() - exact).abs() - tolerance).max().item()
        assert excess <= 0.0, (what, name, excess, (value.double() - exact).abs().max().item())


def _inputs(plan, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    sizes = {"q": (plan.total_q, plan.num_q_heads), "k": (plan.total_k, plan.num_kv_heads), "v": (plan.total_k, plan.num_kv_heads), "do": (plan.total_q, plan.num_q_heads)}
    return {n: torch.randn(*s, plan.head_dim, generator=gen, device="cuda").to(torch.bfloat16) for n, s in sizes.items()}


def _run(plan, x, window, sinks, stream=None):
    """Forward and backward through the binding, in buffers that hold NaN before"""
    from paper_2505_19609_amd import binding as B
    o, dq = (torch.full_like(x["q"], float("nan")) for _ in range(2))
    dk, dv = (torch.full_like(x["k"], float("nan")) for _ in range(2))
    lse = torch.full((plan.num_q_heads, plan.total_q), float("nan"), device="cuda")
    B.skrull_window_fwd(plan, x["q"], x["k"], x["v"], o, lse, window, sinks, stream=stream)
    ws = torch.full((B.skrull_window_workspace(plan, window, sinks),), 0xFF, dtype=torch.uint8, device="cuda")
    B.skrull_window_bwd(plan, x["q"], x["k"], x["v"], o, lse, x["do"], dq, dk, dv, ws, window, sinks, stream=stream)
    return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


def _plan(shape, heads, d, **kw):
    from paper_2505_19609_amd import binding as B
    return B.skrull_attn_plan(*shape[:3], heads[0], heads[1], d, d ** -0.5, shard_cut=shape[3], **kw)


def _whole(*lengths):
    return list(lengths), [1] * len(lengths), [0] * len(lengths), [0] * len(lengths)


SHAPES = {
    "one": _whole(1),
    "short": _whole(1, 2, 31, 32, 33, 64, 65, 5),
    "mixed": _whole(700, 129, 64, 1, 300, 97),
    "long": _whole(1500),
    "slices": ([900, 120, 1000], [3, 1, 4], [1, 0, 3], [0, 0, 0]),
    "chunks": ([1400, 77, 640], [4, 1, 2], [1, 0, 0], [1, 0, 1]),   # two chunks far apart; one sequence; chunks that nearly meet
    "last": ([2000], [8], [7], [1]),                                # the first and the last chunk
}
HEADS = [((4, 4), 64), ((14, 2), 64), ((8, 2), 128), ((3, 1), 128)]
WINDOWS = [(1, 0), (1, 1), (7, 0), (32, 4), (33, 0), (64, 1), (65, 64), (100, 33), (128, 0), (200, 130), (333, 4), (600, 500), (5000, 0), (5000, 3), (2, 5000), ((1 << 31) - 1, (1 << 31) - 1)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("heads,d", HEADS)
@pytest.mark.parametrize("rows", [0, 128, 256])
def test_window_against_64_bits(shape, heads, d, rows):
    if rows and shape in ("one", "slices"):
        pytest.skip("the plan's own choice covers these")
    plan = _plan(SHAPES[shape], heads, d, wg_query_rows=rows)
    x = _inputs(plan, len(shape) + d)
    for window, sinks in WINDOWS:
        got = _run(plan, x, window, sinks)
        _check(got, _reference(SHAPES[shape], x["q"], x["k"], x["v"], x["do"], d ** -0.5, window, sinks), (window, sinks))
    plan.destroy()


@pytest.mark.parametrize("block_n,head_split", [(64, 0), (128, 1), (192, 0), (256, 2), (192, 7), (64, 7)])
@pytest.mark.parametrize("shape", ["mixed", "chunks", "long"])
def test_window_with_other_blocks(shape, block_n, head_split):
    plan = _plan(SHAPES[shape], (14, 2), 64, block_n=block_n, head_split=head_split)
    x = _inputs(plan, block_n)
    for window, sinks in ((50, 0), (90, 5), (300, 70)):
        _check(_run(plan, x, window, sinks), _reference(SHAPES[shape], x["q"], x["k"], x["v"], x["do"], 64 ** -0.5, window, sinks), (window, sinks))
    plan.destroy()


_CHUNKS = ([24000, 300, 16000], [4, 1, 2], [1, 0, 0], [1, 0, 1])


@pytest.mark.parametrize("shape,heads,d,pieces", [(_whole(4200, 40, 3000, 300), (7, 1), 64, False), (_whole(2100, 700, 1900), (8, 1), 128, False),
                                                  (([9000, 300, 6000], [4, 1, 2], [1, 0, 0], [1, 0, 1]), (4, 2), 64, False), (([6000, 2500], [2, 3], [1, 2], [0, 1]), (8, 2), 128, False),
                                                  (_whole(8000, 200, 6000), (8, 2), 64, True), (_whole(12000, 300), (8, 2), 128, True), (_CHUNKS, (8, 2), 64, True), (_CHUNKS, (8, 2), 128, True),
                                                  (_whole(*[2048] * 16), (16, 2), 64, True), (_whole(*[2048 - 70 * i for i in range(16)]), (32, 4), 64, True)])
def test_window_sinks_of_long_sequences(shape, heads, d, pieces):
    """Queries far behind the sinks' own windows, of several sequences and chunks; `pieces`: they are many enough to be taken by themselves.  The workspace between margins."""
    from paper_2505_19609_amd import binding as B
    from gpu_util import guarded, margins_intact
    plan = _plan(shape, heads, d)
    x = _inputs(plan, 17)
    assert (B.skrull_window_workspace(plan, 100, 4) > B.skrull_window_workspace(plan, 100, 0)) == pieces   # (for the pieces' sums)
    for window, sinks in ((100, 4), (300, 128), (64, 65), (20, 129), (1000, 1)):
        buf, ws = guarded((B.skrull_window_workspace(plan, window, sinks),), torch.uint8, 0xFF)
        o, lse = torch.empty_like(x["q"]), torch.empty(heads[0], plan.total_q, device="cuda")
        B.skrull_window_fwd(plan, x["q"], x["k"], x["v"], o, lse, window, sinks)
        dq, dk, dv = torch.full_like(o, float("nan")), *(torch.full_like(x["k"], float("nan")) for _ in range(2))
        B.skrull_window_bwd(plan, x["q"], x["k"], x["v"], o, lse, x["do"], dq, dk, dv, ws, window, sinks)
        assert margins_intact(buf)
        _check({"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}, _reference(shape, x["q"], x["k"], x["v"], x["do"], d ** -0.5, window, sinks), (window, sinks))
        torch.cuda.empty_cache()
    plan.destroy()


def test_window_workgroups_of_twelve():
    """A micro-batch of short sequences at head_dim 64, for which the plan takes workgroups of 12 wavefronts."""
    shape = _whole(*[200 + 37 * i % 300 for i in range(64)])
    plan = _plan(shape, (14, 2), 64)
    assert plan.info.fwd_waves == 12 and plan.info.dq_waves == 12
    x = _inputs(plan, 3)
    for window, sinks in ((64, 4), (150, 0)):
        _check(_run(plan, x, window, sinks), _reference(shape, x["q"], x["k"], x["v"], x["do"], 64 ** -0.5, window, sinks), (window, sinks))
    plan.destroy()


@pytest.mark.parametrize("heads,d", [((4, 4), 64), ((14, 2), 64), ((8, 2), 128)])
def test_whole_window_is_attention(heads, d):
    """A window of the whole sequence, or sinks that are: what skrull_attn_fwd gives, up to the roundings of a row's sum of 700 probabilities (of the same
    values, so LSE is off by 2 (700 + 24) 2^-24 and a few roundings of its own) and, of O, the last one."""
    from paper_2505_19609_amd import binding as B
    shape = SHAPES["mixed"]
    plan = _plan(shape, heads, d)
    x = _inputs(plan, d)
    o, lse = torch.empty_like(x["q"]), torch.empty(heads[0], plan.total_q, device="cuda")
    B.skrull_attn_fwd(plan, x["q"], x["k"], x["v"], o, lse)
    sums = 2 * (700 + 24) * FP32
    for window, sinks in ((700, 0), (1, 700)):
        got = _run(plan, x, window, sinks)
        assert ((got["lse"] - lse).abs() <= sums + 8 * FP32 * (1 + lse.abs())).all()
        assert ((got["o"].double() - o.double()).abs() <= 2 * BF16 * o.double().abs() + sums * x["v"].abs().max()).all()
    plan.destroy()


def test_window_of_one_key_is_v():
    plan = _plan(SHAPES["mixed"], (8, 2), 128)
    x = _inputs(plan, 9)
    got = _run(plan, x, 1, 0)
    assert torch.equal(got["o"], x["v"].repeat_interleave(4, 1))
    plan.destroy()


def test_far_window_of_a_long_sequence():
    """One rank's chunks of a long sequence: keys between the sinks, the chunks' windows and their ends are not looked at, but for two tiles beside them (they
    hold NaN), and have gradients of zero."""
    shape = ([40000, 60], [8, 1], [3, 0], [1, 0])
    plan = _plan(shape, (4, 2), 128)
    x = _inputs(plan, 11)
    window, sinks = 1000, 70
    slices, _, _ = _slices(*shape)
    unseen = torch.ones(plan.total_k, dtype=torch.bool, device="cuda")
    for begin, end, _, k0 in slices:
        unseen[k0:k0 + min(sinks + 128, end)] = False
        unseen[k0 + max(0, begin - window - 128):k0 + end + 128] = False
    assert unseen.sum() > 15000
    plain = {n: t.clone() for n, t in x.items()}
    for n in "kv":
        plain[n][unseen] = 0.0
        x[n][unseen] = float("nan")
    got, again = _run(plan, x, window, sinks), _run(plan, plain, window, sinks)
    for n in got:
        assert torch.equal(got[n], again[n]), n
    assert (got["dk"][unseen] == 0).all() and (got["dv"][unseen] == 0).all()
    # a sample of rows against 64 bits
    for begin, end, q0, k0 in slices:
        for i in {begin, (begin + end) // 2, end - 1}:
            j = torch.arange(i + 1, device="cuda")
            j = j[(i - j < window) | (j < sinks)]
            for h in range(4):
                s = plain["k"][k0 + j, h // 2].double() @ plain["q"][q0 + i - begin, h].double() * 128 ** -0.5
                p = torch.softmax(s, 0)
                v = plain["v"][k0 + j, h // 2].double()
                error = (BF16 + 1e-4) * (p @ v.abs())
                assert ((got["o"][q0 + i - begin, h].double() - p @ v).abs() <= error + BF16 * ((p @ v).abs() + error)).all()
    plan.destroy()


@pytest.mark.parametrize("shape", [_whole(3000, 500, 77, 1200), _whole(8000, 500, 77)])
def test_window_results_are_the_same_bits_each_time_and_on_other_streams(shape):
    plan = _plan(shape, (14, 2), 64)
    x = _inputs(plan, 21)
    want = _run(plan, x, 400, 4)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(3):
        runs = []
        for st in streams:
            with torch.cuda.stream(st):
                runs.append(_run(plan, x, 400, 4))
        torch.cuda.synchronize()
        assert all(torch.equal(r[n], want[n]) for r in runs for n in want)
        # calls with and without a window by turns share the plan's queues
        from paper_2505_19609_amd.autograd import skrull_attention
        skrull_attention(x["q"], x["k"], x["v"], plan)
        assert all(torch.equal(t, want[n]) for n, t in _run(plan, x, 400, 4).items())
    plan.destroy()


@pytest.mark.parametrize("shape,heads,d,pieces", [(_whole(900, 60, 2000), (8, 2), 128, False), (_whole(8000, 200, 6000), (8, 2), 64, True)])
def test_window_captured_and_replayed(shape, heads, d, pieces):
    """Forward and gradients through autograd in a graph: every replay is the eager result, on new values too.  `pieces`: as above."""
    from paper_2505_19609_amd import binding as B
    from paper_2505_19609_amd.autograd import skrull_window_attention
    plan = _plan(shape, heads, d)
    x = _inputs(plan, 31)
    leaves = [x[n].requires_grad_() for n in "qkv"]

    def step():
        o = skrull_window_attention(*leaves, plan, 100, 4)
        return [o.detach(), *torch.autograd.grad(o, leaves, x["do"])]
    assert (B.skrull_window_workspace(plan, 100, 4) > B.skrull_window_workspace(plan, 100, 0)) == pieces
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        captured = step()
    for rep in range(4):
        with torch.no_grad():
            for n, t in _inputs(plan, 40 + rep).items():
                x[n].copy_(t)
        for t in captured:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, want)), rep
    plan.destroy()


def test_window_gradient_against_differences():
    """The change of the 64-bit results along the gradient is what the gradient says, up to its roundings."""
    from paper_2505_19609_amd.autograd import skrull_window_attention
    shape = SHAPES["chunks"]
    plan = _plan(shape, (4, 2), 64)
    x = _inputs(plan, 51)
    leaves = [x[n].requires_grad_() for n in "qkv"]
    grads = torch.autograd.grad(skrull_window_attention(*leaves, plan, 90, 5), leaves, x["do"])

    def value(step):
        moved = [t.detach().double() + step * g.double() for t, g in zip(leaves, grads)]
        return (_reference(shape, *moved, x["do"], 64 ** -0.5, 90, 5)["o"][0] * x["do"].double()).sum().item()
    step = 1e-5
    slope, square = (value(step) - value(-step)) / (2 * step), sum(g.double().square().sum().item() for g in grads)
    # grads = exact + error, so slope - square = -(grads . error): at most |grads| |error|, and |error| is some 2^-8 of |grads| for P, dS, O and the results each
    assert abs(slope - square) <= 4 * BF16 * square
    plan.destroy()


@pytest.mark.parametrize("q_scale", [30.0, 0.0])
def test_window_scores_far_apart_or_equal(q_scale):
    """Scores of some hundreds: rows whose first key in view is far below the later ones, and the reverse; and scores that are all equal."""
    shape = SHAPES["mixed"]
    plan = _plan(shape, (8, 2), 128)
    x = _inputs(plan, 61)
    x["q"] = (x["q"].float() * q_scale).to(torch.bfloat16)
    for window, sinks in itertools.product((40, 200), (0, 3)):
        _check(_run(plan, x, window, sinks), _reference(shape, x["q"], x["k"], x["v"], x["do"], 128 ** -0.5, window, sinks), (window, sinks))
    plan.destroy()


def test_window_refuses_on_the_gpu():
    """Tensors that overlap or are misaligned, and a workspace that is too small: refused before anything runs."""
    from paper_2505_19609_amd import binding as B
    plan = _plan(_whole(40, 24), (4, 2), 64)
    x = _inputs(plan, 1)
    o, lse = torch.full_like(x["q"], 7.0), torch.full((4, 64), 7.0, device="cuda")
    ws = torch.zeros(B.skrull_window_workspace(plan, 8), dtype=torch.uint8, device="cuda")
    dq, dk, dv = torch.full_like(o, 7.0), torch.full_like(x["k"], 7.0), torch.full_like(x["k"], 7.0)
    odd = torch.zeros(o.numel() + 8, dtype=torch.bfloat16, device="cuda")[1:1 + o.numel()].view(o.shape)
    for args in ((x["q"], x["k"], x["v"], x["q"], lse, 8), (x["q"], x["k"], x["v"], odd, lse, 8), (x["q"], x["k"], x["k"].float(), o, lse, 8), (x["q"], x["k"], x["v"], o, lse, 0),
                 (x["q"], x["k"], x["v"], o, lse[:, :32], 8), (x["q"], x["k"], x["v"], o, lse, 8, -1)):
        with pytest.raises(B.SkrullError):
            B.skrull_window_fwd(plan, *args)
    for args in ((dq, dk, dk, ws), (x["do"], dk, dv, ws), (dq, dk, dv, ws[:-16]), (dq, dk, x["k"], ws), (dq, dq, dv, ws), (dq, dk, dv, ws[::2])):
        with pytest.raises(B.SkrullError):
            B.skrull_window_bwd(plan, x["q"], x["k"], x["v"], o, lse, x["do"], *args, 8)
    torch.cuda.synchronize()
    assert all((t == 7.0).all() for t in (o, lse, dq, dk, dv))
    plan.destroy()
