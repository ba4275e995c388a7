"""More refusals of the 8-bit calls, without a GPU."""
import pytest

import paper_2608_05483_b200 as P
from test_w8_host import _gemm


@pytest.mark.parametrize("value", [-1, 2, 1 << 20])
def test_product_takes_weights_ready_as_a_truth_value(value):
    assert _gemm(weights_ready=value) == _gemm(weights_ready=value, m=0) == P.ERR_INVALID_ARG
    assert _gemm(weights_ready=1, m=0) == _gemm(weights_ready=0, m=0) == P.OK


@pytest.mark.parametrize("kw", [dict(wait_cycles=-1), dict(test_hook=2), dict(test_hook=-1), dict(test_hook=P.HOOK_WITHHOLD_RELEASE),
                                dict(test_hook=P.HOOK_WITHHOLD_RELEASE, wait_cycles=P.HOOK_MAX_CYCLES + 1)])
def test_product_refuses_limits_and_hooks(kw):
    assert _gemm(**kw) == _gemm(m=0, **kw) == P.ERR_INVALID_ARG


def test_product_takes_limits_and_a_hook_with_a_short_one():
    assert _gemm(m=0, wait_cycles=1) == _gemm(m=0, wait_cycles=1 << 40) == P.OK
    assert _gemm(m=0, wait_cycles=P.HOOK_MAX_CYCLES, test_hook=P.HOOK_WITHHOLD_RELEASE) == P.OK


def test_product_refuses_more_tiles_than_it_can_number():
    rows, cols = 128 << 14, 64 << 14                     # 2^28 tiles
    kw = dict(m=rows, n=(0, cols), out_stride=(0, cols))
    assert _gemm(n_weights=1, **kw) == P.ERR_UNSUPPORTED
    assert _gemm(**kw) == P.ERR_UNSUPPORTED
    assert _gemm(n_weights=1, m=1 << 30, n=(0, 1 << 30), out_stride=(0, 1 << 30)) == P.ERR_UNSUPPORTED


def test_status_needs_a_place_to_go():
    assert P.load().plora_gemm_fp8_status(0, None) == P.ERR_INVALID_ARG
