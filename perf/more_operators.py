"""The performance cases of what a transformer block is made of around the operators of perf/operators.py, on a micro-batch's packed rows:
attention over a sliding window, the residual stream between two blocks with its norms, and the products with their epilogues.

A case is one operator over one rank's rows:

  ``window``    causal attention of a plan's rows to the ``window`` last keys and the first ``sinks`` ones of their sequence.  Lengths are a
                log-normal mix of whole sequences after ``long_count`` long ones, whole or cut over ``cp`` ranks, this one being ``rank``
  ``residual``  the residual stream times ``scale`` plus a block's output (normed itself: ``post``; times a ``gate`` a column), and the norm
                of that for the next block
  ``linear``    rows times a weight, with ``bias``, ``activation`` (``gated``: of one half of the columns, times the other) and ``add``, a residual

each forward alone or (``train``) with all gradients.  ``own`` false: the plain forms, elementary operations in 32 bits; true: the library's kernels.
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-5


def _window(heads, median, sigma, lo, hi, tokens, length_seed, window, sinks, train, long_len=0, long_count=0, cp=1, rank=0, two_chunks=False, name=None):
    hq, hkv, d = heads
    c = {"op": "window", "q_heads": hq, "kv_heads": hkv, "head_dim": d, "median": median, "sigma": sigma, "lo": lo, "hi": hi, "tokens": tokens,
         "length_seed": length_seed, "long_len": long_len, "long_count": long_count, "cp": cp, "rank": rank, "two_chunks": two_chunks,
         "window": window, "sinks": sinks, "train": train}
    return {"name": name, **c} if name else c


def _residual(kind, rows, cols, dtype, residual_dtype, weight_dtype, bias, post, gate, scale, train, name=None):
    c = {"op": "residual", "kind": kind, "rows": rows, "cols": cols, "dtype": dtype, "residual_dtype": residual_dtype, "weight_dtype": weight_dtype,
         "bias": bias, "post": post, "gate": gate, "scale": scale, "train": train}
    return {"name": name, **c} if name else c


def _linear(rows, inputs, outputs, bias, activation, gated, add, train, name=None):
    c = {"op": "linear", "rows": rows, "inputs": inputs, "outputs": outputs, "bias": bias, "activation": activation, "gated": gated, "add": add,
         "train": train}
    return {"name": name, **c} if name else c


QWEN_05B = (14, 2, 64)   # query heads, key / value heads, head_dim
QWEN_7B = (28, 4, 128)
LLAMA_8B = (32, 8, 128)


def listed():
    return [
        # the smallest call: the repository's 4-head test model, a handful of short sequences
        _window((4, 4, 64), 200, 1.0, 16, 511, 932, 1, 128, 4, True, name="window_tiny"),
        # a full bucket of the 0.5B model: short sequences that the window mostly covers, long ones that it cuts
        _window(QWEN_05B, 300, 1.1, 16, 8192, 26624, 11, 1024, 0, True, name="window_qwen05b_26k"),
        # the headline micro-batch, one long sequence and short ones, with a few first tokens that stay visible
        _window(LLAMA_8B, 800, 0.8, 32, 4096, 8192, 3, 4096, 4, True, 24576, 1, name="window_llama8b_32k"),
        # a rank's two chunks of a 131,072-token sequence and the keys before them, a wide window: the largest
        _window(QWEN_7B, 1000, 0.8, 64, 4096, 8192, 4, 8192, 64, True, 131072, 1, 8, 3, True, name="window_qwen7b_shard"),
        # a small micro-batch of the 0.5B model: latency
        _residual("rms", 932, 896, "bf16", "bf16", "bf16", False, False, False, 1.0, True, name="residual_qwen05b_tiny"),
        # a full bucket (13K tokens) of the 7B model: norms on both sides of the block, a learned gate, the stream in fp32
        _residual("rms", 13312, 3584, "bf16", "fp32", "bf16", False, True, True, 1.0, True, name="residual_qwen7b_13k"),
        # the headline micro-batch's rows as layer norms with everything, the stream scaled up before each block's output is added
        _residual("layer", 32768, 4096, "bf16", "bf16", "fp32", True, True, True, 1.5, True, name="residual_llama8b_32k"),
        # rows of a width that no vector of 16 bytes divides, forward alone
        _residual("layer", 7013, 1001, "bf16", "bf16", "fp32", True, False, True, 1.0, False, name="residual_odd_fwd"),
        # the projection of Q, K and V of a few rows of the 0.5B model: latency
        _linear(37, 896, 1152, True, "none", False, False, True, name="linear_qwen05b_tiny"),
        # sizes that no tile divides, everything in the epilogue
        _linear(1001, 904, 1160, True, "gelu", False, True, True, name="linear_odd"),
        # a full bucket (13K tokens) of the 7B model into a gated block four times as wide: the largest
        _linear(13312, 3584, 14336, False, "silu", True, False, True, name="linear_qwen7b_13k_gated"),
        # the headline micro-batch's rows back out of such a block, added to the stream: evaluation, forward alone
        _linear(32768, 16384, 4096, False, "none", False, True, False, name="linear_llama8b_32k_down"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["window", "residual", "linear"])
    if op == "window":
        heads = rng.choice([(4, 4, 64), QWEN_05B, (16, 16, 64), QWEN_7B, LLAMA_8B])
        tokens = log_int(300, 24576)
        long_len, count, cp, rank, two = 0, 0, 1, 0, False
        if rng.random() < 0.5:
            count, cp = 1, rng.choice([1, 2, 4, 8])
            long_len = log_int(2048, min(65536, 8192 * cp))
            rank, two = rng.randrange(cp), cp > 1 and rng.random() < 0.7
        # (no more pairs of a query and a key than the largest listed case has)
        most = 24576 * 8192 * QWEN_7B[0] * QWEN_7B[2] // ((tokens + long_len // cp) * heads[0] * heads[2])
        return _window(heads, log_int(100, 3000), round(rng.uniform(0.4, 1.1), 2), rng.randint(1, 64), rng.choice([511, 4096, 8192]), tokens,
                       rng.randrange(1 << 30), min(log_int(8, 16384), most), rng.choice([0, 0, 1, 4, rng.randint(1, 300)]), rng.random() < 0.7,
                       long_len, count, cp, rank, two)
    if op == "residual":
        kind, dtype = rng.choice(["rms", "layer"]), rng.choice(["bf16", "bf16", "fp32"])
        cols = rng.choice([log_int(64, 8192), 8 * log_int(16, 1024)])
        stream = rng.choice([dtype, "fp32"])
        most = 32768 * 4096 * 2 // (cols * sum(1 if t == "bf16" else 2 for t in (dtype, stream)))
        return _residual(kind, min(log_int(1, 32768), most), cols, dtype, stream, rng.choice([dtype, "fp32"]),
                         kind == "layer" and rng.random() < 0.7, rng.random() < 0.6, rng.random() < 0.5, rng.choice([1.0, 1.0, 0.8, 2.5]),
                         rng.random() < 0.7)
    gated = rng.random() < 0.3
    inputs, outputs = 8 * log_int(8, 2048), 8 * log_int(8, 1792 if gated else 2048)
    rows = min(log_int(1, 32768), 13312 * 3584 * 28672 // (inputs * outputs * (2 if gated else 1)))
    return _linear(max(1, rows), inputs, outputs, rng.random() < 0.5, rng.choice(["relu", "gelu", "silu"] if gated else ["none", "none", "relu", "gelu", "silu"]),
                   gated, rng.random() < 0.3, rng.random() < 0.7)


_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ---- inputs -----------------------------------------------------------------------------------------------------

def _micro_batch(case):
    """(lengths, degrees, indices, cuts) of a window case."""
    rng = np.random.Generator(np.random.PCG64(case["length_seed"]))
    S = [case["long_len"]] * case["long_count"]
    cut = [int(case["two_chunks"])] * len(S)
    degree, index = [case["cp"]] * len(S), [case["rank"]] * len(S)
    left = case["tokens"]
    while left > 0:
        s = int(np.clip(round(float(np.exp(rng.normal(np.log(case["median"]), case["sigma"])))), case["lo"], case["hi"]))
        s = min(s, left)
        S, cut, degree, index = S + [s], cut + [0], degree + [1], index + [0]
        left -= s
    return S, degree, index, cut


def _slices(case):
    """(positions of the queries: from, to; first row of Q; first row of K) of every slice, and the rows of Q and of K."""
    out, rows_q, rows_k = [], 0, 0
    for s, n, r, z in zip(*_micro_batch(case)):
        chunks, end = n * (2 if z else 1), 0
        for i in ([r, 2 * n - 1 - r] if z else [r]):
            begin, end = i * s // chunks, (i + 1) * s // chunks
            out.append((begin, end, rows_q, rows_k))
            rows_q += end - begin
        rows_k += end
    return out, rows_q, rows_k


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape, dtype=torch.bfloat16, scale=1.0, mean=0.0):
        return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * scale + mean).to(dtype)

    if case["op"] == "window":
        hq, hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
        _, nq, nk = _slices(case)
        return {"q": normal(nq, hq, d), "k": normal(nk, hkv, d), "v": normal(nk, hkv, d), "d_o": normal(nq, hq, d)}
    rows = case["rows"]
    if case["op"] == "residual":
        cols, t, rt, wt = case["cols"], _TYPES[case["dtype"]], _TYPES[case["residual_dtype"]], _TYPES[case["weight_dtype"]]
        # (the stream: rows with a scale of their own and an offset)
        r = (normal(rows, cols, dtype=torch.float32) * normal(rows, 1, dtype=torch.float32).exp() +
             normal(rows, 1, dtype=torch.float32, scale=0.5)).to(rt)
        weight, post = normal(cols, dtype=wt, scale=0.2, mean=1.0), normal(cols, dtype=wt, scale=0.2, mean=1.0)
        bias, post_bias = normal(cols, dtype=wt, scale=0.1), normal(cols, dtype=wt, scale=0.1)
        gate = normal(cols, dtype=wt, scale=0.2, mean=0.5)
        return {"r": r, "z": normal(rows, cols, dtype=t), "w": weight, "b": bias if case["bias"] else None, "post_w": post if case["post"] else None,
                "post_b": post_bias if case["post"] and case["bias"] else None, "gate": gate if case["gate"] else None,
                "d_r": normal(rows, cols, dtype=rt), "d_y": normal(rows, cols, dtype=t)}
    n = case["outputs"] * (2 if case["gated"] else 1)
    return {"x": normal(rows, case["inputs"]), "w": normal(n, case["inputs"], scale=case["inputs"] ** -0.5),
            "b": normal(n, scale=0.3) if case["bias"] else None, "add": normal(rows, case["outputs"]) if case["add"] else None,
            "d_y": normal(rows, case["outputs"])}


_LEAVES = {"window": ("q", "k", "v"), "residual": ("r", "z", "w", "b", "post_w", "post_b", "gate"), "linear": ("x", "w", "b", "add")}


def prepare(case, seed):
    st = {"case": case, **_inputs(case, seed)}
    if case["train"]:
        for n in _LEAVES[case["op"]]:
            if st[n] is not None:
                st[n].requires_grad_()
    if case["op"] == "window" and own:
        from paper_2505_19609_amd import binding as B
        S, N, R, Z = _micro_batch(case)
        st["plan"] = B.skrull_attn_plan(S, N, R, case["q_heads"], case["kv_heads"], case["head_dim"], case["head_dim"] ** -0.5, shard_cut=Z)
    return st


# ---- the library's kernels --------------------------------------------------------------------------------------

def _run_own(st):
    from paper_2505_19609_amd import autograd as A
    case = st["case"]
    if case["op"] == "window":
        out, given = {"o": A.skrull_window_attention(st["q"], st["k"], st["v"], st["plan"], case["window"], case["sinks"])}, [st["d_o"]]
    elif case["op"] == "residual":
        r, y = A.skrull_residual_norm(st["r"], st["z"], st["w"], st["b"], st["post_w"], st["post_b"], st["gate"], case["scale"], EPS, case["kind"])
        out, given = {"r": r, "y": y}, [st["d_r"], st["d_y"]]
    else:
        out, given = {"y": A.skrull_linear(st["x"], st["w"], st["b"], st["add"], case["activation"], case["gated"])}, [st["d_y"]]
    if not case["train"]:
        return out
    leaves = [n for n in _LEAVES[case["op"]] if st[n] is not None]
    grads = torch.autograd.grad(list(out.values()), [st[n] for n in leaves], given)
    return {**{n: t.detach() for n, t in out.items()}, **{"d" + n: g for n, g in zip(leaves, grads)}}


# ---- the plain forms --------------------------------------------------------------------------------------------

@torch.no_grad()
def _plain_window(st):
    case = st["case"]
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    g, window, sinks, scale = hq // hkv, case["window"], case["sinks"], case["head_dim"] ** -0.5
    q, k, v, d_o = st["q"], st["k"], st["v"], st["d_o"]
    out = {"o": torch.empty_like(q)}
    if case["train"]:
        dq, dk, dv = torch.empty_like(q), *(torch.zeros(t.shape, dtype=torch.float32, device="cuda") for t in (k, v))

    def heads(t):   # [rows, heads, d] -> [KV heads, rows * heads of a group, d], 32 bits
        return t.float().view(len(t), hkv, -1, d).permute(1, 0, 2, 3).reshape(hkv, -1, d)

    def rows(t, like):
        return t.view(hkv, len(like), g, d).permute(1, 0, 2, 3).reshape(like.shape).to(like.dtype)

    # (a block of queries at a time, against the keys that one of them sees: all scores at once would be many GB)
    for begin, end, q0, k0 in _slices(case)[0]:
        for p in range(begin, end, 512):
            e = min(p + 512, end)
            first = max(0, p - window + 1)
            early = min(sinks, first)   # (first keys that are not among the others)
            at_q = slice(q0 + p - begin, q0 + e - begin)
            keys = [slice(k0, k0 + early), slice(k0 + first, k0 + e)]
            position = torch.cat((torch.arange(early, device="cuda"), torch.arange(first, e, device="cuda")))
            qs, ks, vs = heads(q[at_q]), heads(torch.cat([k[s] for s in keys])), heads(torch.cat([v[s] for s in keys]))
            mine = torch.arange(p, e, device="cuda").repeat_interleave(g)[:, None]
            hidden = (position > mine) | ((position <= mine - window) & (position >= sinks))
            s = (qs @ ks.transpose(1, 2) * scale).masked_fill_(hidden, -math.inf)
            s = (s - s.amax(-1, keepdim=True)).exp_()
            s /= s.sum(-1, keepdim=True)
            o = s @ vs
            out["o"][at_q] = rows(o, q[at_q])
            if case["train"]:
                do = heads(d_o[at_q])
                ds = s * (do @ vs.transpose(1, 2) - (do * o).sum(-1, keepdim=True))
                dq[at_q] = rows(ds @ ks * scale, q[at_q])
                for t, add in ((dk, ds.transpose(1, 2) @ qs * scale), (dv, s.transpose(1, 2) @ do)):
                    add = add.transpose(0, 1)
                    t[keys[0]] += add[:early]
                    t[keys[1]] += add[early:]
    if case["train"]:
        out.update(dq=dq, dk=dk.to(k.dtype), dv=dv.to(v.dtype))
    return out


def _normed(x, layer):
    """(x - its mean) times 1 / its deviation, and that factor."""
    if layer:
        x = x - x.mean(-1, keepdim=True)
    rstd = ((x * x).mean(-1, keepdim=True) + EPS).rsqrt()
    return x * rstd, rstd


def _norm_back(g, h, rstd, layer):
    d = g - h * (g * h).mean(-1, keepdim=True)
    return (d - g.mean(-1, keepdim=True) if layer else d) * rstd


@torch.no_grad()
def _plain_residual(st):
    case = st["case"]
    layer = case["kind"] == "layer"
    f = {n: st[n].float() if st[n] is not None else None for n in (*_LEAVES["residual"], "d_r", "d_y")}
    n = f["z"]
    if case["post"]:
        h1, rstd1 = _normed(n, layer)
        n = h1 * f["post_w"] + (f["post_b"] if case["bias"] else 0.0)
    r = f["r"] * case["scale"] + (n * f["gate"] if case["gate"] else n)
    h2, rstd2 = _normed(r, layer)
    out = {"r": r.to(st["r"].dtype), "y": (h2 * f["w"] + (f["b"] if case["bias"] else 0.0)).to(st["z"].dtype)}
    if not case["train"]:
        return out
    e = f["d_r"] + _norm_back(f["d_y"] * f["w"], h2, rstd2, layer)
    dn = e * f["gate"] if case["gate"] else e
    grads = {"r": e * case["scale"], "z": _norm_back(dn * f["post_w"], h1, rstd1, layer) if case["post"] else dn, "w": (f["d_y"] * h2).sum(0)}
    if case["bias"]:
        grads["b"] = f["d_y"].sum(0)
    if case["post"]:
        grads["post_w"] = (dn * h1).sum(0)
        if case["bias"]:
            grads["post_b"] = dn.sum(0)
    if case["gate"]:
        grads["gate"] = (e * n).sum(0)
    return {**out, **{"d" + name: t.to(st[name].dtype) for name, t in grads.items()}}


def _phi(z):
    """The normal distribution's share below z."""
    return 0.5 * (1.0 + torch.erf(z * 0.5 ** 0.5))


_ACTIVATIONS = {   # and their derivatives
    "none": (lambda z: z, torch.ones_like),
    "relu": (lambda z: z.clamp(min=0.0), lambda z: (z > 0.0).to(z.dtype)),
    "gelu": (lambda z: z * _phi(z), lambda z: _phi(z) + z * (-0.5 * z * z).exp() * (2.0 * math.pi) ** -0.5),
    "silu": (lambda z: z * torch.sigmoid(z), lambda z: torch.sigmoid(z) * (1.0 + z * (1.0 - torch.sigmoid(z)))),
}


@torch.no_grad()
def _plain_linear(st):
    case = st["case"]
    act, slope = _ACTIVATIONS[case["activation"]]
    x, w = st["x"].float(), st["w"].float()
    z = x @ w.t()
    if case["bias"]:
        z += st["b"].float()
    n = case["outputs"]
    y = act(z[:, :n]) * z[:, n:] if case["gated"] else act(z)
    if case["add"]:
        y = y + st["add"].float()
    out = {"y": y.to(torch.bfloat16)}
    if case["train"]:
        dz = st["d_y"].float()
        dz = torch.cat((dz * z[:, n:] * slope(z[:, :n]), dz * act(z[:, :n])), 1) if case["gated"] else dz * slope(z)
        out.update(dx=(dz @ w).to(torch.bfloat16), dw=(dz.t() @ x).to(torch.bfloat16))
        if case["bias"]:
            out["db"] = dz.sum(0).to(torch.bfloat16)
        if case["add"]:
            out["dadd"] = st["d_y"]
    return out


def run(state):
    if own:
        return _run_own(state)
    return {"window": _plain_window, "residual": _plain_residual, "linear": _plain_linear}[state["case"]["op"]](state)


# ---- what a pass cannot do without ------------------------------------------------------------------------------

def work(case):
    times = 3 if case["train"] else 1
    if case["op"] == "window":
        slices, nq, nk = _slices(case)
        pairs = 0
        for begin, end, _, _ in slices:
            p = np.arange(begin, end, dtype=np.int64)
            seen = np.minimum(p + 1, case["window"])
            pairs += int((seen + np.minimum(case["sinks"], p + 1 - seen)).sum())
        hq, hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
        # (a shard's keys before every window need not be read; their gradients, zeros, are written)
        used = min(nk, sum(min(end, end - begin + case["window"] + case["sinks"]) for begin, end, _, _ in slices))
        forward = 4 * nq * hq * d + 4 * used * hkv * d
        return {"bytes": forward + (8 * nq * hq * d + 4 * used * hkv * d + 4 * nk * hkv * d if case["train"] else 0),
                "flops": pairs * d * hq * (14 if case["train"] else 4)}
    if case["op"] == "residual":
        n, size, stream = case["rows"] * case["cols"], 2 if case["dtype"] == "bf16" else 4, 2 if case["residual_dtype"] == "bf16" else 4
        vectors = (1 + case["post"]) * (1 + case["bias"]) + case["gate"]
        w = case["cols"] * (2 if case["weight_dtype"] == "bf16" else 4) * vectors
        # r, z -> r, y; then (r or the new one), z, their gradients -> gradients of r and z
        return {"bytes": (2 * n * (size + stream)) + (3 * n * (size + stream) + w if case["train"] else 0) + w,
                "flops": n * (16 if case["post"] else 9) * (3 if case["train"] else 1)}
    n, k, rows = case["outputs"] * (2 if case["gated"] else 1), case["inputs"], case["rows"]
    y = rows * case["outputs"]
    return {"bytes": 2 * (rows * k + n * k + n * case["bias"] + y * (1 + case["add"])) + (2 * (2 * rows * k + 2 * n * k + y) if case["train"] else 0),
            "flops": 2 * rows * n * k * times}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------

def _with_gradients(case, given, forward):
    """`forward` of the inputs in 64 bits, and its gradients as torch derives them."""
    names = [n for n in _LEAVES[case["op"]] if given[n] is not None]
    leaves = {n: given[n].double().requires_grad_(case["train"]) for n in names}
    with torch.set_grad_enabled(case["train"]):
        out = forward({n: leaves.get(n) for n in _LEAVES[case["op"]]})
    result = {n: t.detach() for n, t in out.items()}
    if case["train"]:
        grads = torch.autograd.grad(list(out.values()), list(leaves.values()), [given["d_" + n].double() for n in out])
        result.update({"d" + n: t for n, t in zip(names, grads)})
    return result


def exact(case, seed):
    given = _inputs(case, seed)
    if case["op"] == "window":
        result = {"o": torch.empty(given["q"].shape, dtype=torch.float64, device="cuda")}
        if case["train"]:
            result.update({"d" + n: torch.zeros(given[n].shape, dtype=torch.float64, device="cuda") for n in "qkv"})
        g = case["q_heads"] // case["kv_heads"]
        for begin, end, q0, k0 in _slices(case)[0]:
            for p in torch.arange(begin, end, device="cuda").split(256):
                j = torch.arange(int(p[-1]) + 1, device="cuda")
                j = j[(j < case["sinks"]) | (j > p[0] - case["window"])]   # keys that the first of these queries or a later one sees
                distance = p[:, None] - j
                seen = (distance >= 0) & ((distance < case["window"]) | (j < case["sinks"]))
                rows, keys = q0 + p - begin, k0 + j
                for h in range(case["kv_heads"]):
                    mine = slice(h * g, (h + 1) * g)
                    q, k, v = (t.double().requires_grad_(case["train"]) for t in (given["q"][rows, mine], given["k"][keys, h], given["v"][keys, h]))
                    with torch.set_grad_enabled(case["train"]):
                        z = torch.where(seen, q.transpose(0, 1) @ k.t() / math.sqrt(case["head_dim"]), -math.inf)
                        o = (torch.softmax(z, -1) @ v).transpose(0, 1)
                    result["o"][rows, mine] = o.detach()
                    if case["train"]:
                        grads = torch.autograd.grad(o, (q, k, v), given["d_o"][rows, mine].double())
                        result["dq"][rows, mine] = grads[0]
                        result["dk"][keys, h] += grads[1]
                        result["dv"][keys, h] += grads[2]
        return result
    if case["op"] == "residual":
        def norm(x, w, b):
            if case["kind"] == "layer":
                x = x - x.sum(-1, keepdim=True) / case["cols"]
            y = x / (x.square().sum(-1, keepdim=True) / case["cols"] + EPS).sqrt() * w
            return y if b is None else y + b

        def forward(t):
            n = t["z"] if t["post_w"] is None else norm(t["z"], t["post_w"], t["post_b"])
            r = case["scale"] * t["r"] + (n if t["gate"] is None else t["gate"] * n)
            return {"r": r, "y": norm(r, t["w"], t["b"])}
        return _with_gradients(case, given, forward)

    def forward(t):
        z = t["x"] @ t["w"].t()
        z = z if t["b"] is None else z + t["b"]
        z, times = z.chunk(2, 1) if case["gated"] else (z, 1.0)
        if case["activation"] == "relu":
            z = torch.where(z > 0.0, z, 0.0)
        elif case["activation"] == "gelu":
            z = z * torch.special.erfc(-z / math.sqrt(2.0)) / 2.0
        elif case["activation"] == "silu":
            z = z / (1.0 + torch.exp(-z))
        z = z * times
        return {"y": z if t["add"] is None else z + t["add"]}
    return _with_gradients(case, given, forward)
