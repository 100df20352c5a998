"""Matmuls in 8-bit integers and moves of tokens where a launch's extents end: against exact integer sums and 64 bits."""
import pytest

from test_gpu_i8_kernels import check_product
from test_operator_ranges import ONE_ROW

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n,k,experts", ONE_ROW)
def test_blocks_of_one_row(m, n, k, experts):
    check_product(m, n, k, False, experts)
