"""Registers of the kernels of the norms around a block: nothing goes to scratch where a thread has one chunk of a row."""
import pytest

from tests import test_isa_checks as T
from tests.test_isa_learn import metadata

pytestmark = T.pytestmark


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    return metadata(T.assembly("ll_norm", tmp_path_factory.mktemp("isa")))


def clean(m):
    return m["scratch"] == 0 and m["spill"] == 0


# workgroups of up to 512 threads may have 256 registers, of up to 1024 only 128; three gates, with and without gamma_y
@pytest.mark.parametrize("kernel,count,registers", [("ll_block_norm_sums_kernel", 1, 256), ("ll_block_norm_kernelILi1ELi512E", 2, 256), ("ll_block_norm_kernelILi2ELi512E", 2, 256),
                                                    ("ll_block_norm_kernelILi2ELi1024E", 2, 128), ("ll_block_norm_grad_kernelILi1ELi512E", 6, 256),
                                                    ("ll_block_norm_grad_kernelILi1ELi1024E", 6, 128)])
def test_up_to_8192_columns_and_forward(kernels, kernel, count, registers):
    found = {n: m for n, m in kernels.items() if kernel in n}
    assert len(found) == count, sorted(kernels)
    for name, m in found.items():
        assert m["vgpr"] <= registers and clean(m), (name, m)


def test_the_gradient_of_wider_rows(kernels):
    """Two chunks a thread of 1024: some forms keep part of a row in scratch, never the plainest (no gate, no gamma_y), and none more than this."""
    found = {n: m for n, m in kernels.items() if "ll_block_norm_grad_kernelILi2E" in n}
    assert len(found) == 6, sorted(kernels)
    for name, m in found.items():
        assert m["vgpr"] <= 128 and m["scratch"] <= (0 if "ELb0ELi0E" in name else 184), (name, m)
