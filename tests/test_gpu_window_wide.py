"""Windows of 4,096 keys and more that hide keys, on the GPU: the walks of dK/dV that wide windows take, by whole and by shared items, with and without pieces for what sees the sinks from far
behind them; and workgroups of other numbers of rows on slices.  References and tolerances are those of test_gpu_window.py."""
import pytest
import torch

from test_gpu_window import HEADS, WINDOWS, SHAPES, _check, _inputs, _plan, _reference, _run, _whole

pytestmark = pytest.mark.gpu

# (a walk of that many tiles of 64 queries times heads times head_dim is turned: see `turned` in bwd.hip)
TURNED = (4 << 20) // (4 * 64)


def _by_heads(shape, x, scale, window, sinks):
    """_reference, one query head at a time: all of them at once would be hundreds of GB.  (dK and dV are sums over a group's heads in 64 bits, and so are their errors; with up to 16
    heads that are products of 16 rows added up, as many sums as a head has rows, which is what the bound counts for each.)"""
    hq, hkv = x["q"].shape[1], x["k"].shape[1]
    g = hq // hkv
    assert g <= 16
    heads = [_reference(shape, x["q"][:, h:h + 1], x["k"][:, h // g:h // g + 1], x["v"][:, h // g:h // g + 1], x["do"][:, h:h + 1], scale, window, sinks) for h in range(hq)]

    def joined(name, i):
        if name in ("dk", "dv"):
            return torch.cat([sum(r[name][i] for r in heads[c * g:(c + 1) * g]) for c in range(hkv)], 1)
        return torch.cat([r[name][i] for r in heads], 0 if name == "lse" else 1)
    return {name: (joined(name, 0), joined(name, 1)) for name in heads[0]}


def _walked(g, head_split):
    """Query heads that one workgroup of an item walks over: its share of them, or a piece of the walk over all."""
    return g // head_split if g % head_split == 0 else g


@pytest.mark.parametrize("window,sinks", [(4096, 0), (5000, 4), (4100, 130)])
@pytest.mark.parametrize("heads,d,head_split", [((8, 1), 64, 1), ((7, 1), 64, 1), ((7, 1), 64, 3), ((4, 1), 128, 1), ((8, 2), 128, 1), ((8, 2), 128, 3), ((16, 2), 128, 2), ((3, 1), 128, 2)])
def test_wide_windows(heads, d, head_split, window, sinks):
    """Long sequences whose first keys are out of the last queries' windows, and one that its window covers.  The walk of an item, or of a workgroup's share of it, is long enough to be turned,
    and begins at different tiles for different blocks of keys."""
    assert (window // 64 + 1) * _walked(heads[0] // heads[1], head_split) * d > TURNED
    shape = _whole(9000, 300, 7777, 4000)
    plan = _plan(shape, heads, d, head_split=head_split)
    x = _inputs(plan, window + d)
    _check(_run(plan, x, window, sinks), _by_heads(shape, x, d ** -0.5, window, sinks), (window, sinks))
    torch.cuda.empty_cache()
    plan.destroy()


@pytest.mark.parametrize("heads,d,tokens,head_split", [((8, 1), 64, 20000, 1), ((8, 1), 64, 20000, 3), ((8, 1), 128, 14000, 1), ((8, 1), 128, 14000, 3)])
def test_wide_windows_with_pieces_for_sinks(heads, d, tokens, head_split):
    """Sequences so long that the sinks' far queries are taken in pieces, beside turned walks."""
    from paper_2505_19609_amd import binding as B
    window, sinks = 4096, 70
    assert (window // 64 + 1) * _walked(heads[0], head_split) * d > TURNED
    shape = _whole(tokens, 100)
    plan = _plan(shape, heads, d, head_split=head_split)
    assert B.skrull_window_workspace(plan, window, sinks) > B.skrull_window_workspace(plan, window, 0)
    x = _inputs(plan, tokens)
    _check(_run(plan, x, window, sinks), _by_heads(shape, x, d ** -0.5, window, sinks), (window, sinks))
    torch.cuda.empty_cache()
    plan.destroy()


@pytest.mark.parametrize("heads,d", [((8, 1), 64), ((8, 2), 128)])
@pytest.mark.parametrize("shape", [([30000, 500], [3, 1], [2, 0], [0, 0]), ([40000, 700, 16000], [4, 1, 2], [3, 0, 0], [1, 0, 1])])
def test_wide_windows_of_slices(shape, heads, d):
    """A rank's slices and two-chunk cuts: items of one segment and of two that share their prefix."""
    plan = _plan(shape, heads, d)
    x = _inputs(plan, d)
    for window, sinks in ((4096, 0), (4500, 5)):
        _check(_run(plan, x, window, sinks), _by_heads(shape, x, d ** -0.5, window, sinks), (window, sinks))
        torch.cuda.empty_cache()
    plan.destroy()


def test_wide_windows_give_the_same_bits_each_time():
    plan = _plan(_whole(9000, 300, 7777), (8, 2), 128)
    x = _inputs(plan, 5)
    want = _run(plan, x, 4096, 4)
    for _ in range(3):
        assert all(torch.equal(t, want[n]) for n, t in _run(plan, x, 4096, 4).items())
    plan.destroy()


@pytest.mark.parametrize("heads,d", HEADS)
@pytest.mark.parametrize("rows", [128, 256])
def test_slices_with_other_workgroups(heads, d, rows):
    """Queries that do not begin at position 0, in workgroups of 4 and of 8 wavefronts."""
    plan = _plan(SHAPES["slices"], heads, d, wg_query_rows=rows)
    x = _inputs(plan, rows + d)
    for window, sinks in WINDOWS:
        _check(_run(plan, x, window, sinks), _reference(SHAPES["slices"], x["q"], x["k"], x["v"], x["do"], d ** -0.5, window, sinks), (window, sinks))
    plan.destroy()
