"""The loss's products read their results by inline assembly too: the distance to the matrix instruction that the compiler does not
keep there is in the source.  The checks of test_mfma_waits_host.py on its assembly."""
import os

import pytest

from paper_2505_19609_amd import build
from test_mfma_waits_host import _assembly, _kernels, _too_early, needed, pytestmark  # noqa: F401


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    return _kernels(_assembly(os.path.join(build.CSRC, "loss.hip"), tmp_path_factory.mktemp("loss") / "loss.s"))


def test_no_instruction_reads_a_matrix_result_early(kernels, needed):  # noqa: F811
    assert len(kernels) == 12
    for name, code in kernels.items():
        assert not _too_early(code, needed), name


def test_a_result_is_read_where_the_check_looks(kernels):
    """The check sees accumulator registers: every product kernel reads its 16 NA NB of them by v_accvgpr_read after the loop."""
    for name, code in kernels.items():
        ops = [c[0] for c in code if not isinstance(c, str)]
        last = max(i for i, op in enumerate(ops) if op.startswith("v_mfma"))
        assert ops.count("v_accvgpr_read_b32") >= 16, name
        assert last < len(ops) - 1
