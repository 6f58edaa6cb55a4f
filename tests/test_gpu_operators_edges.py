"""Rotary positions, norm and loss where test_gpu_operators.py does not reach: logits far from zero, weights of infinities beside rows that fill
a tile, gradients that come in unaligned, gradients of gradients, and the loops, pieces and tiles that larger calls take.  The 64-bit forms and their
tolerances are that file's."""
import math

import pytest
import torch

from test_gpu_operators import (BF16, FP32, SHAPES, TINY, _calls, _check_loss, _gen, _loss_case, _loss_in_64_bits, _norm_in_64_bits, _plan,
                                _randn, _within)

pytestmark = pytest.mark.gpu


# ---- loss: an offset that all logits of a row have --------------------------------------------------------------------

# Tiles of 64 words x 64 rows, 256 x 64, x 128 and x 256; a last strip (of 32 words in the first, of 128 in the others) of 1 to 12 words, so that some of
# its lanes have none; fewer strips than the 64 that share a row's sums, and more.
OFFSET_SIZES = [(3, 64, 5), (37, 64, 300), (1000, 64, 129), (64, 72, 4099), (500, 136, 4099), (9000, 64, 129), (100, 64, 70019), (1100, 200, 19971), (33100, 64, 130)]


@pytest.mark.parametrize("offset", [-100.0, -1000.0, 1000.0])
@pytest.mark.parametrize("rows,hidden,vocab", OFFSET_SIZES)
def test_loss_of_logits_with_a_common_offset(rows, hidden, vocab, offset):
    """Softmax does not see it: x has a component along a direction that all words share."""
    x, w, target, d = _loss_case(rows, hidden, vocab, 0.25)
    target[0] = vocab - 1
    x[:, 0], w[:, 0] = offset / 8, 8.0
    _check_loss(x, w, target, d)


@pytest.mark.parametrize("offset", [-3e10, 3e10, -1e20, 1e20, -1e30, 1e30])
@pytest.mark.parametrize("rows,hidden,vocab", [(37, 64, 300), (500, 136, 4099), (100, 64, 70019), (1100, 200, 19971)])
def test_loss_of_finite_logits_is_finite(rows, hidden, vocab, offset):
    """Of any size: what is left of such a row's differences is within fp32's spacing, which is the bounds' too."""
    x, w, target, d = _loss_case(rows, hidden, vocab, 0.25)
    x[:, 0], w[:, 0] = offset / 8, 8.0
    _check_loss(x, w, target, d)


@pytest.mark.parametrize("offset", [-100.0, 100.0])
@pytest.mark.parametrize("rows,hidden,vocab", [(37, 64, 300), (500, 136, 4099), (1100, 200, 19971)])
def test_loss_of_strips_whose_words_are_all_masked(rows, hidden, vocab, offset):
    """128 words of minus infinity, and the last ones: what the words without them give."""
    from paper_2505_19609_amd.autograd import skrull_cross_entropy
    x, w, target, d = _loss_case(rows, hidden, vocab, 0.25)
    x[:, 0], w[:, 0], x[:, 1] = offset / 8, 8.0, 1.0
    masked = torch.zeros(vocab, dtype=torch.bool, device="cuda")
    masked[128:256] = True
    masked[vocab - vocab % 64:] = True
    kept = torch.nonzero(~masked)[:, 0]
    target = torch.where(target < 0, target, kept[target % len(kept)])
    want = _loss_in_64_bits(x, w[kept], torch.where(target < 0, target, (torch.cumsum(~masked, 0) - 1)[target.clamp(min=0)]), d)
    w[masked, 1] = -math.inf
    x.requires_grad_(), w.requires_grad_()
    loss = skrull_cross_entropy(x, w, target)
    dx, dw = torch.autograd.grad(loss, (x, w), d)
    columns = torch.arange(hidden, device="cuda") != 1     # (0 times infinity there, by the formula too)
    for name, got, part in (("loss", loss.detach(), lambda t: t), ("dx", dx[:, columns], lambda t: t[:, columns]), ("dw", dw[kept], lambda t: t)):
        exact, error = (part(t) for t in want[name])
        _within(got, exact, error + (BF16 if got.dtype == torch.bfloat16 else FP32) * (exact.abs() + error) + TINY, name)
    assert (dw[masked] == 0).all()


# ---- loss: rows that fill a tile ---------------------------------------------------------------------------------------

@pytest.mark.parametrize("targets", [1, 3, 31, 32, 65, 128, 130, 200, 256])
@pytest.mark.parametrize("rows,hidden,vocab", [(300, 64, 500), (1100, 72, 19971)])
def test_loss_gradients_of_a_masked_word_at_any_number_of_rows(rows, hidden, vocab, targets):
    """A word of minus infinity has a gradient of zero, however many rows fill the last tile."""
    from paper_2505_19609_amd.autograd import skrull_cross_entropy
    x, w, target, d = _loss_case(rows, hidden, vocab, 0.0)
    x[:, 0] = 1.0
    target[target == 7] = 8
    target[targets:] = -1
    kept = torch.arange(vocab, device="cuda") != 7
    want = _loss_in_64_bits(x, w[kept], target - (target > 7).long(), d)
    w[7, 0] = -math.inf
    x.requires_grad_(), w.requires_grad_()
    loss = skrull_cross_entropy(x, w, target)
    dx, dw = torch.autograd.grad(loss, (x, w), d)
    assert (dw[7] == 0).all()
    for name, got, part in (("loss", loss.detach(), lambda t: t), ("dx", dx[:, 1:], lambda t: t[:, 1:]), ("dw", dw[kept], lambda t: t)):
        exact, error = (part(t) for t in want[name])
        _within(got, exact, error + (BF16 if got.dtype == torch.bfloat16 else FP32) * (exact.abs() + error) + TINY, name)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("rows,hidden,vocab", [(1, 64, 500), (300, 64, 500), (1100, 72, 19971)])
def test_loss_without_a_target_adds_nothing_whatever_the_weight_holds(rows, hidden, vocab, bad):
    from paper_2505_19609_amd.autograd import skrull_cross_entropy
    x, w, target, d = _loss_case(rows, hidden, vocab, 0.0)
    w[7, 3], w[vocab - 1] = bad, bad
    x.requires_grad_(), w.requires_grad_()
    loss = skrull_cross_entropy(x, w, torch.full_like(target, -1))
    dx, dw = torch.autograd.grad(loss, (x, w), d)
    assert (loss == 0).all() and (dx == 0).all() and (dw == 0).all()


# ---- autograd ----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("watched", [False, True])
def test_rotary_takes_gradients_of_any_alignment(monkeypatch, watched):
    """Gradients that are parts of a flat buffer, 2 bytes off."""
    from paper_2505_19609_amd import autograd as A
    monkeypatch.setattr(A, "_watched", lambda: watched)
    (q, k), call = _calls()[0]
    given = [t.clone().requires_grad_() for t in (q, k)]
    out = call(*given)
    d = [_randn(_gen(5), *o.shape) for o in out]
    want = torch.autograd.grad(out, given, d, retain_graph=True)
    flat = torch.empty(1 + sum(t.numel() for t in d), dtype=torch.bfloat16, device="cuda")
    parts = [p.view(t.shape) for p, t in zip(flat[1:].split([t.numel() for t in d]), d)]
    for p, t in zip(parts, d):
        p.copy_(t)
        assert p.is_contiguous() and p.data_ptr() % 16 != 0
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(out, given, parts), want))


@pytest.mark.parametrize("watched", [False, True])
@pytest.mark.parametrize("i", [1, 2, 4])
def test_gradients_of_gradients_are_refused_and_not_left_out(monkeypatch, i, watched):
    """The norm's and the loss's gradients depend on their inputs, whether the gradient that comes in needs one or not: a penalty on them cannot
    be differentiated, and must not pass for a constant."""
    from paper_2505_19609_amd import autograd as A
    monkeypatch.setattr(A, "_watched", lambda: watched)
    inputs, call = _calls()[i]
    given = [t.clone().requires_grad_() for t in inputs]
    out = call(*given)
    grads = torch.autograd.grad(out, given, torch.ones_like(out), create_graph=True)
    with pytest.raises(RuntimeError, match="differentiate"):
        (out.float().sum() + grads[0].float().square().sum()).backward()


@pytest.mark.parametrize("watched", [False, True])
def test_gradients_that_depend_on_nothing_are_constants(monkeypatch, watched):
    """Rotary's gradients depend on the ones that come in alone; so do the norm's of weight and bias where x is given."""
    from paper_2505_19609_amd import autograd as A
    monkeypatch.setattr(A, "_watched", lambda: watched)
    calls = _calls()
    (q, k), call = calls[0]
    given = [t.clone().requires_grad_() for t in (q, k)]
    out = call(*given)
    d = [torch.ones_like(o) for o in out]
    want = torch.autograd.grad(out, given, d, retain_graph=True)
    grads = torch.autograd.grad(out, given, d, create_graph=True)
    (out[0].float().sum() + out[1].float().sum() + grads[0].float().sum()).backward()
    assert all(torch.equal(t.grad, g) for t, g in zip(given, want))
    (x, w, b), call = calls[1]
    w, b = w.clone().requires_grad_(), b.clone().requires_grad_()
    y = call(x, w, b)
    want = torch.autograd.grad(y, (w, b), torch.ones_like(y), retain_graph=True)
    grads = torch.autograd.grad(y, (w, b), torch.ones_like(y), create_graph=True)
    (y.float().sum() + grads[0].float().square().sum()).backward()
    assert torch.equal(w.grad, want[0]) and torch.equal(b.grad, want[1])


@pytest.mark.parametrize("watched", [False, True])
def test_rotary_turns_back_by_what_it_was_called_with(monkeypatch, watched):
    """The frequencies of the forward, also where the program has changed its struct since."""
    from paper_2505_19609_amd import autograd as A
    from paper_2505_19609_amd import binding as B
    monkeypatch.setattr(A, "_watched", lambda: watched)
    gen = _gen(6)
    plan, rotary = _plan(SHAPES[3], (4, 2), 64), B.skrull_rotary_init(64)
    q, k = (_randn(gen, n, h, 64).requires_grad_() for n, h in ((plan.total_q, 4), (plan.total_k, 2)))
    out = A.skrull_rotary(q, k, plan, rotary)
    d = [_randn(gen, *o.shape) for o in out]
    want = torch.autograd.grad(out, (q, k), d, retain_graph=True)
    rotary.base = 5e5
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(out, (q, k), d), want))
    plan.destroy()


# ---- norm: several rows to a wavefront or workgroup --------------------------------------------------------------------

# Each of the six forms (lanes of a row, pieces of a lane, narrow rows) with three rows and more to every wavefront or workgroup of the forward and the
# backward, and an uneven end.
LOOPED = [(13001, 5), (13000, 136), (9001, 1001), (3100, 1032), (3100, 4096), (1600, 8192)]


@pytest.mark.parametrize("rows,cols", LOOPED)
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("t", [torch.bfloat16, torch.float32])
def test_norm_of_several_rows_to_a_workgroup(rows, cols, kind, t):
    from paper_2505_19609_amd import binding as B
    gen = _gen(rows + cols)
    layer = kind == "layer"
    x = (_randn(gen, rows, cols, dtype=torch.float32) * _randn(gen, rows, 1, dtype=torch.float32).exp() + 3.0).to(t)
    w = (_randn(gen, cols, dtype=torch.float32, scale=0.3) + 1.0).to(t)
    b = _randn(gen, cols, dtype=t) if layer else None
    dy = _randn(gen, rows, cols, dtype=t)
    eps, number = 1e-3, B.NORM_LAYER if layer else B.NORM_RMS
    mean, rstd = torch.empty((2, rows), device="cuda")

    def both(x, given_x, y, dy, dx):
        dw, db = torch.empty_like(w), torch.empty_like(w) if layer else None
        B.skrull_norm_fwd(x, w, b, y, mean, rstd, eps, number)
        y = y.clone()
        ws = torch.full((B.skrull_norm_workspace(x, w, number),), 0xFF, dtype=torch.uint8, device="cuda")
        B.skrull_norm_bwd(given_x, w, mean, rstd, dy, dx, dw, db, ws, number)
        return {"y": y, "dx": dx.clone(), "dw": dw, **({"db": db} if layer else {})}

    got = both(x, x, torch.empty_like(x), dy, torch.empty_like(x))
    want = _norm_in_64_bits(x, w, b, dy, eps, layer)
    for name, value in got.items():
        exact, error = want[name]
        _within(value, exact, error * 1.01 + (BF16 if t == torch.bfloat16 else FP32) * (exact.abs() + error) + TINY, name)
    del want
    # y in the place of x, dx in the place of dy, then of x: the same bits
    place = x.clone()
    again = both(place, x, place, dy, dy)
    assert all(torch.equal(again[n], got[n]) for n in got)
    dy = _randn(gen, rows, cols, dtype=t)
    want = both(x, x, place, dy, torch.empty_like(x))
    again = both(x, x, place, dy, x)
    assert all(torch.equal(again[n], want[n]) for n in want)


# ---- loss: what larger calls take --------------------------------------------------------------------------------------

@pytest.mark.parametrize("rows", [33001, 70001])
def test_loss_of_more_than_64_rows_to_a_gathering_workgroup(rows):
    """A workgroup gathers rows / 512 rows, 64 at a time."""
    x, w, target, d = _loss_case(rows, 64, 96, 0.3)
    target[1000:9000] = -1
    target[20000:30000:2] = -5
    loss, dx, _ = _check_loss(x, w, target, d)
    assert (loss[target < 0] == 0).all() and (dx[target < 0] == 0).all()


def test_loss_of_several_tiles_to_a_workgroup():
    """Tiles of 256 x 256, more of them than workgroups, several steps each and the last one ragged: loads run ahead across the ends of tiles."""
    _check_loss(*_loss_case(1100, 200, 20003, 0.1))
    _check_loss(*_loss_case(2300, 328, 20003, 0.0))


def _pieces(rows, vocab, hidden):
    """The rule for the backward's pieces of the vocabulary (csrc/loss.hip: Piece), where all rows have a target: tiles of 256 words of an even cut, of the
    other one, and whether that is taken."""
    row_tiles, words, h_tiles = -(-rows // 256), -(-vocab // 256), -(-hidden // 256)
    room = min(row_tiles * 256 * (min(words * 256, 1 << 20) + 64), max(1 << 30, row_tiles * 256 * 320))
    most = min(max((room // (row_tiles * 256) - 64) // 256, 1), 4096)
    count = -(-words // most)
    even, whole, h = -(-words // count), 256, h_tiles
    while whole > 1 and h % 2 == 0:
        whole, h = whole // 2, h // 2
    other = most // whole * whole

    def rounds(tiles):
        return words // tiles * -(-tiles * h_tiles // 256) + -(-(words % tiles) * h_tiles // 256)
    return even, other, count > 1 and most >= whole and -(-words // other) <= count and rounds(other) < rounds(even)


def test_loss_in_pieces_that_make_whole_rounds_of_tiles():
    """Two pieces of unequal size, 384 tiles of words and 163, with more than one tile of hidden values."""
    rows, hidden, vocab = 8192, 264, 140003
    assert _pieces(rows, vocab, hidden) == (274, 384, True)
    x, w, target, d = _loss_case(rows, hidden, vocab, 0.0)
    border = 384 * 256
    target[:6] = torch.tensor([0, border - 1, border, border + 1, vocab - 2, vocab - 1], device="cuda")
    parts = [_loss_in_64_bits(x[i:i + 1024], w, target[i:i + 1024], d[i:i + 1024]) for i in range(0, rows, 1024)]
    want = {n: tuple(torch.cat([p[n][k] for p in parts]) for k in (0, 1)) for n in ("loss", "dx")}
    # (a sum over all rows has rows + 64 roundings, not the 1,024 + 64 of a part's bound, each of at most 2^-24 of the sum of |dz x|, and |dz| <= |d| (p + [target]))
    want["dw"] = tuple(sum(p["dw"][k] for p in parts) for k in (0, 1))
    p_at_most = torch.zeros(vocab, hidden, dtype=torch.float64, device="cuda")
    for i in range(0, rows, 1024):
        p = (x[i:i + 1024].double() @ w.double().t()).softmax(1)
        p[torch.arange(1024, device="cuda"), target[i:i + 1024]] += 1.0
        p_at_most += (p * d[i:i + 1024, None].double().abs()).t() @ x[i:i + 1024].double().abs()
    want["dw"] = (want["dw"][0], want["dw"][1] + (rows + 64) * FP32 * p_at_most)
    _check_loss(x, w, target, d, want)


@pytest.mark.parametrize("rows,offset", [(5, 0.0), (5, -200.0), (70, 0.0)])
def test_loss_of_few_rows_in_pieces(rows, offset):
    """More than 2^20 words: two pieces, dz in two bf16, parts of dX added to over the pieces, the second one with fewer steps than parts."""
    hidden, vocab = 24, (1 << 20) + 777
    assert _pieces(rows, vocab, hidden) == (2050, 4096, True)
    x, w, target, d = _loss_case(rows, hidden, vocab, 0.0)
    if offset:
        x[:, 0], w[:, 0] = offset / 8, 8.0
    target[:5] = torch.tensor([0, (1 << 20) - 1, 1 << 20, vocab - 1, vocab - 10], device="cuda")
    _check_loss(x, w, target, d)


def test_loss_of_a_short_last_tile_with_few_rows_and_a_target_in_it():
    """The last word alone in its tile, strip and step, as target and not."""
    for vocab in (257, 4097, 65537):
        x, w, target, d = _loss_case(97, 64, vocab, 0.2)
        target[:3] = torch.tensor([vocab - 1, vocab - 2, 0], device="cuda")
        _check_loss(x, w, target, d)
