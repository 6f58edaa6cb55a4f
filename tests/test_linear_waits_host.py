"""The products of linear.hip read their results by inline assembly, as the loss's do: the checks of test_mfma_waits_host.py on its assembly."""
import os

import pytest

from paper_2505_19609_amd import build
from test_mfma_waits_host import _assembly, _kernels, _too_early, needed, pytestmark  # noqa: F401


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    return _kernels(_assembly(os.path.join(build.CSRC, "linear.hip"), tmp_path_factory.mktemp("linear") / "linear.s"))


def test_no_instruction_reads_a_matrix_result_early(kernels, needed):  # noqa: F811
    products = {name: code for name, code in kernels.items() if "product" in name}
    assert len(products) >= 18
    for name, code in products.items():
        assert not _too_early(code, needed), name
        ops = [c[0] for c in code if not isinstance(c, str)]
        assert ops.count("v_accvgpr_read_b32") >= 16, name   # (the check sees the accumulators read)
