"""The give-up paths of the 8-bit product's bounded waits, without stalling the GPU.

A test hook makes one warp of every CTA keep its accumulators, so the products' wait for one runs out after a limit of about
two milliseconds.  Every copy that was asked for lands, the products issued complete, and the kernel returns.  Looked at: the
status word, that nothing around the outputs was written, and that the next ordinary calls are right.
"""
import pytest
import torch

import paper_2608_05483_b200 as P
from test_gpu_w8 import _check_product, _gen, _guarded, _matrix8

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LIMIT = 4_000_000        # SM clock cycles: about 2 ms

# m, k, columns: clusters that split K, narrow tiles, single CTAs, pairs with narrow and wide tiles, several tiles per pair.  A CTA has
# more than four blocks of K in each (a cluster of eight: 64 blocks, eight to a CTA).
FORMS = [(1, 8192, (4096, 1024)), (5, 8192, (64,)), (60, 8192, (13824,)), (128, 8192, (2048,)), (300, 8192, (1024, 320)), (1111, 4176, (2056,)),
         (2500, 2048, (5120,))]


def _withheld(x, xs, w, ws, out, status):
    n = out.shape[1]
    a = P.GemmFp8Args(P.INPUT_FP32, x.shape[0], x.shape[1], 1)
    a.n[0], a.x_stride, a.w_stride[0], a.out_stride[0] = n, x.stride(0), w.stride(0), out.stride(0)
    a.x, a.x_scale, a.w[0], a.w_scale[0], a.out[0] = x.data_ptr(), xs.data_ptr(), w.data_ptr(), ws.data_ptr(), out.data_ptr()
    a.status = None if status is None else status.data_ptr()
    a.wait_cycles, a.test_hook = LIMIT, P.HOOK_WITHHOLD_RELEASE
    assert P.plora_gemm_fp8(a, torch.cuda.current_stream().cuda_stream) == P.OK


@pytest.mark.parametrize("m,k,ns", FORMS)
def test_a_wait_that_runs_out_is_reported_and_survivable(m, k, ns):
    g = _gen(m + k)
    x, xs = _matrix8(g, m, k, 1)
    ws = [_matrix8(g, n, k, 128) for n in ns]
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    for w, s in ws:
        out, intact = _guarded(m, w.shape[0], torch.float32, 3)
        _withheld(x, xs, w, s, out, status)
        torch.cuda.synchronize()
        assert int(status) == P.ERR_TIMEOUT
        intact()
        status.zero_()
    # two in a row and an ordinary call right behind them: it starts under the second one's wind-down
    w, s = ws[0]
    out, intact = _guarded(m, w.shape[0], torch.float32, 3)
    _withheld(x, xs, w, s, out, status)
    _withheld(x, xs, w, s, out, status)
    good = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = P.gemm_fp8(x, xs, [w for w, _ in ws], [s for _, s in ws], status=good)
    torch.cuda.synchronize()
    assert int(status) == P.ERR_TIMEOUT and int(good) == 0
    intact()
    for o, (w, s) in zip(got, ws):
        _check_product(o, x, xs, w, s)


def test_the_hook_alone_changes_nothing_where_no_wait_needs_the_warp():
    """Up to four blocks of K fit in a CTA's accumulators: nobody waits, and the result is right."""
    g = _gen(5)
    x, xs = _matrix8(g, 20, 128, 1)
    w, s = _matrix8(g, 100, 128, 128)
    out, status = torch.empty((20, 100), device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    _withheld(x, xs, w, s, out, status)
    torch.cuda.synchronize()
    assert int(status) == 0
    _check_product(out, x, xs, w, s)


@pytest.mark.parametrize("m,k,ns", FORMS)
def test_a_short_limit_alone_changes_nothing(m, k, ns):
    g = _gen(m + k + 1)
    x, xs = _matrix8(g, m, k, 1)
    ws = [_matrix8(g, n, k, 128) for n in ns]
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    args = (x, xs, [w for w, _ in ws], [s for _, s in ws])
    got = P.gemm_fp8(*args, status=status, wait_cycles=P.HOOK_MAX_CYCLES)
    want = P.gemm_fp8(*args)
    torch.cuda.synchronize()
    assert int(status) == 0 and all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_call_without_a_status_word_leaves_it_to_the_device():
    g = _gen(6)
    x, xs = _matrix8(g, 300, 8192, 1)
    w, s = _matrix8(g, 1024, 8192, 128)
    P.gemm_fp8_status()
    assert P.gemm_fp8_status() == P.OK
    out, intact = _guarded(300, 1024, torch.float32, 3)
    _withheld(x, xs, w, s, out, None)
    good = P.gemm_fp8(x, xs, w, s)                    # the word is sticky
    assert P.gemm_fp8_status() == P.ERR_TIMEOUT
    assert P.gemm_fp8_status(torch.device(DEV)) == P.OK
    intact()
    _check_product(good, x, xs, w, s)
    # a call with a word of its own reports there and nowhere else
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    _withheld(x, xs, w, s, out, status)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert P.gemm_fp8_status(stream=side) == P.OK and int(status) == P.ERR_TIMEOUT
