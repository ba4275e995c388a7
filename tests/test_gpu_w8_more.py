"""More of the 8-bit calls on the GPU, against 64-bit references; tolerances as in test_gpu_w8.py unless said otherwise."""
import pytest
import torch

import paper_2608_05483_b200 as P
from test_gpu_w8 import _check8, _check16, _check_product, _gen, _matrix8, _norm_ref, _randn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, HALF, F32, F8 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn


@pytest.mark.parametrize("n,d", [(640, 4168), (777, 5120), (1000, 4096), (600, 8192), (1300, 4096)])
def test_norm_of_fp32_rows_and_an_fp32_residual(n, d):
    """Batches about the number of rows that fit at one time: right, and a row's bits do not depend on the batch."""
    g = _gen(n + d)
    x, res, w = _randn(g, n, d), _randn(g, n, d) * 3.0, (_randn(g, d) * 0.3 + 1.0).to(BF)
    a = P.rms_norm(x, w, residual=res, residual_out=torch.empty_like(res), out_type=BF, fp8=True)
    h, v = _norm_ref(x, w, 1e-5, res, 0.0)
    _check16(a.y, v)
    _check8(a.q, a.scale, v)
    assert torch.equal(a.residual, h.float())
    for rows in (slice(0, 3), slice(n - 2, n)):
        b = P.rms_norm(x[rows], w, residual=res[rows], residual_out=torch.empty_like(res[rows]), out_type=BF, fp8=True)
        assert torch.equal(a.y[rows], b.y) and torch.equal(a.q[rows].float(), b.q.float()) and torch.equal(a.scale[rows], b.scale)


@pytest.mark.parametrize("m", [70, 300])
def test_product_of_operands_beyond_32_bits(m):
    """x and w whose rows lie so far apart that the last ones begin more than 2^32 bytes in."""
    g = _gen(m)
    k, n = 400, 200
    x, xs = _matrix8(g, m, k, 1)
    w, ws = _matrix8(g, n, k, 128)
    far = {}
    for name, t in (("x", x), ("w", w)):
        stride = (1 << 32) // (t.shape[0] - 1) // 16 * 16 + 64
        store = torch.empty((t.shape[0] - 1) * stride + k, dtype=torch.uint8, device=DEV)
        assert (t.shape[0] - 1) * stride > 1 << 32
        far[name] = store.view(F8).as_strided(t.shape, (stride, 1))
        far[name].copy_(t)
    out = P.gemm_fp8(far["x"], xs, far["w"], ws)
    _check_product(out, x, xs, w, ws)
    assert torch.equal(out, P.gemm_fp8(x, xs, w, ws))


def _all_exponents(g, *shape):
    """e4m3 values of uniformly distributed bits (no NaN)."""
    b = torch.randint(0, 256, shape, generator=g, device=DEV, dtype=torch.int32).to(torch.uint8)
    return torch.where((b & 127) == 127, b & 128, b).view(F8)


def _cancelling(g, x, w):
    """The largest products there are, in pairs that cancel, among what is there."""
    k = x.shape[1]
    if k > 1:
        at = torch.randperm(k, generator=g, device=DEV)[:2 * (k // 16) or 2]
        x.view(torch.uint8)[:, at] = 0x7e                      # 448
        w.view(torch.uint8)[:, at] = 0x7e
        w.view(torch.uint8)[:, at[::2]] = 0xfe                 # -448


@pytest.mark.parametrize("m,n", [(16, 70), (300, 200)])
@pytest.mark.parametrize("k", [1, 16, 32, 100, 128])
@pytest.mark.parametrize("cancel", [False, True])
def test_sum_of_one_block(m, n, k, cancel):
    """One block, scales of one: what the tensor cores add up.  An instruction adds 32 products to the sum so far; each of the 33 is
    aligned to the largest of them and cut 24 bits below it, so it is off by less than 2^-24 of that one: 132 of them in four instructions,
    and the largest is a product or a partial sum."""
    g = _gen(m + k)
    x, w = _all_exponents(g, m, -(-k // 16) * 16)[:, :k], _all_exponents(g, n, -(-k // 16) * 16)[:, :k]
    if cancel:
        _cancelling(g, x, w)
    one = torch.ones((1, 1), device=DEV)
    out = P.gemm_fp8(x, one.expand(m, 1).contiguous(), w, one.expand(-(-n // 128), 1).contiguous())
    a, b = x.double(), w.double()
    want, most = torch.zeros((m, n), dtype=torch.float64, device=DEV), torch.zeros((m, n), dtype=torch.float64, device=DEV)
    for c in range(0, k, 32):
        p = a[:, None, c:c + 32] * b[None, :, c:c + 32]
        want = want + p.sum(2)
        most = torch.maximum(most, torch.maximum(p.abs().amax(2), want.abs()))
    off = (out.double() - want).abs()
    assert (off <= 132 * 2.0 ** -24 * most).all(), float((off / most.clamp(min=1e-30)).max())
