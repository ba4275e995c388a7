"""More refusals of the 8-bit calls, without a GPU."""
import pytest

import paper_2608_05483_b200 as P
from test_w8_host import _gemm


@pytest.mark.parametrize("value", [-1, 2, 1 << 20])
def test_product_takes_weights_ready_as_a_truth_value(value):
    assert _gemm(weights_ready=value) == _gemm(weights_ready=value, m=0) == P.ERR_INVALID_ARG
    assert _gemm(weights_ready=1, m=0) == _gemm(weights_ready=0, m=0) == P.OK
