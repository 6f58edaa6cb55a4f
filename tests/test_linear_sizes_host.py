"""The sizes of products that their entry points work out on the host, from no rows to the most, without a GPU."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# Every width of a few and of many tiles, of whole and of broken rounds of them; run by itself, so that a signal fails a test and does not end them all.
SWEEP = """
import ctypes, itertools, sys
from paper_2505_19609_amd import binding as B
size = B.lib().skrull_linear_workspace
widths = [8, 64, 136, 896, 1152, 2048, 3584, 4096, 4864, 6144, 8192, 14336, 18944, 28672, 65536]
for rows in map(int, sys.argv[1:]):
    for inputs, outputs, gated, activation in itertools.product(widths, widths, (0, 1), (B.LINEAR_NONE, B.LINEAR_SILU)):
        if gated and (outputs + 256) * inputs >= 1 << 30:
            continue
        p = B.Linear(rows, inputs, outputs, activation, gated, inputs, outputs, outputs, outputs)
        n = outputs * (1 + gated)
        dz = 0 if activation == B.LINEAR_NONE and not gated else rows * n * 2
        forward, backward = (size(ctypes.byref(p), k) for k in (0, 1))
        # the parts' sums: 128 MB at most (those of a tail are of fewer tiles than make a round)
        assert 0 <= forward <= 128 << 20, (rows, inputs, outputs, gated, forward)
        assert rows > 0 or forward == 0
        assert dz + 4 * n <= backward <= dz + 4 * n * 2048 + (129 << 20), (rows, inputs, outputs, gated, backward)
print("swept")
"""


@pytest.mark.parametrize("rows", [0, 1, 2, 37, 64, 65, 1001, 4500, 13312, 1 << 17, 1 << 24])
def test_workspace_of_any_sizes(rows):
    done = subprocess.run([sys.executable, "-c", SWEEP, str(rows)], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "swept" in done.stdout, (done.returncode, done.stderr[-2000:])


# A backward of no rows: dW has more than a round of tiles, with a few left over.  (No address is looked at where there is nothing to write, and there is no GPU to write with.)
NO_ROWS = """
import ctypes
from paper_2505_19609_amd import binding as B
for inputs, outputs, gated in ((3584, 14336, 1), (4096, 14336, 0), (3584, 18944, 0), (4096, 6144, 0), (64, 128, 0)):
    p = B.Linear(0, inputs, outputs, B.LINEAR_NONE, gated, inputs, outputs, outputs, outputs)
    assert B.lib().skrull_linear_fwd(ctypes.byref(p), *[None] * 7, 0, None) == 0
    assert B.lib().skrull_linear_bwd(ctypes.byref(p), *[None] * 8, 0, None) == 0
    # (a dw at a bad address is refused as it is with rows)
    assert B.lib().skrull_linear_bwd(ctypes.byref(p), None, None, None, None, None, 8, None, None, 0, None) == B.SKRULL_EINVAL
print("done")
"""


def test_calls_without_rows():
    done = subprocess.run([sys.executable, "-c", NO_ROWS], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "done" in done.stdout, (done.returncode, done.stderr[-2000:])
