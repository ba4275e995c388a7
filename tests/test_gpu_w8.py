"""The 8-bit calls on the GPU (norm, gated activation, weights, product), against 64-bit references.

Tolerances.  A rounding to a 16-bit type is off by at most u = eps / 2 of the value.  fp32 arithmetic in front of it: the norm's sum is
taken over at most 32 terms per thread, 5 + 5 shuffle steps and the square root, division and products behind it, some
50 roundings of 2^-24; the activations' exponential and division are good to a few 2^-22: FP32 = 2^-18 covers both.
e4m3 has three bits behind the leading one: half a step is 2^-4 of the value, or 2^-10 of the scale below its normal range
(2^-6).  A product's error: each block's sum (128 exact products, fp32 accumulators), one scaling and one addition to the fp32 sum, so at
most (blocks + 160) roundings of 2^-24 of the sum of the magnitudes.
"""
import math

import pytest
import torch

import paper_2608_05483_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, HALF, F32, F8 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn
U = {BF: 2.0 ** -8, HALF: 2.0 ** -11, F32: 2.0 ** -24}
TINY = {BF: 2.0 ** -133, HALF: 2.0 ** -25, F32: 2.0 ** -149}      # half a step below the normal range
FP32 = 2.0 ** -18
LEAST = 2.0 ** -126


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _guarded(n, d, dtype, extra, offset=0):
    """A tensor [n, d] inside a buffer of 64s: (view, check that nothing around it was written)."""
    width = d + extra
    buf = torch.full(((n + 2) * width + offset,), 64.0, device=DEV).to(dtype)
    view = buf[offset:].view(n + 2, width)[1:n + 1, :d]

    def intact():
        b = buf.float()
        keep = torch.ones_like(b, dtype=torch.bool)
        keep[offset:].view(n + 2, width)[1:n + 1, :d] = False
        assert (b[keep] == 64.0).all(), "written outside the output"
    return view, intact


def _check16(y, v):
    assert ((y.double() - v).abs() <= (U[y.dtype] + FP32) * v.abs() + TINY[y.dtype]).all()


def _check8(q, scale, v):
    """q and scale stand for v [n, d], a scale per 128 columns."""
    n, d = v.shape
    nb = -(-d // 128)
    top = torch.stack([v[:, a:a + 128].abs().amax(1) for a in range(0, d, 128)], 1)
    want = (top / 448.0).clamp(min=LEAST)
    assert scale.shape == (n, nb) and ((scale.double() - want).abs() <= FP32 * want).all()
    s = scale.double().repeat_interleave(128, 1)[:, :d]
    off = (q.double() * s - v).abs()
    assert (off <= torch.maximum(2.0 ** -4 * v.abs(), 2.0 ** -10 * s) * (1 + 2.0 ** -9)).all(), float((off / s).max())


# ---- norm ---------------------------------------------------------------------------------------
def _norm_ref(x, weight, eps, residual, offset):
    h = x.double() if residual is None else (x.float() + residual.float()).double()
    f = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    return h, h * f * ((1.0 if weight is None else weight.double()) + offset)


NORM = [
    # n, d, x, type, residual, weight, offset, extra columns of a row, first element off alignment
    (1, 4096, F32, BF, BF, BF, 0.0, 0, 0), (3, 4096, BF, BF, F32, F32, 0.0, 8, 0), (700, 1024, HALF, HALF, HALF, HALF, 1.0, 0, 0),
    (5, 1, F32, HALF, None, None, 0.0, 3, 0), (9, 7, BF, BF, BF, BF, 0.0, 0, 0), (8, 8, F32, BF, F32, F32, 0.0, 0, 0),
    (33, 120, HALF, HALF, F32, HALF, 1.0, 8, 0), (17, 128, F32, BF, BF, BF, 0.0, 0, 0), (17, 136, F32, HALF, None, HALF, 0.0, 8, 0),
    (20, 256, BF, BF, BF, F32, 0.0, 0, 0), (20, 264, BF, BF, BF, BF, 0.0, 8, 0), (11, 1000, F32, HALF, HALF, F32, 0.0, 0, 0),
    (11, 1032, HALF, HALF, F32, HALF, 0.0, 8, 0), (300, 4099, F32, BF, BF, BF, 0.0, 0, 0), (297, 4168, HALF, HALF, F32, HALF, 1.0, 0, 0),
    (2, 5120, F32, BF, BF, BF, 0.0, 8, 1), (400, 5120, F32, BF, BF, BF, 0.0, 0, 0), (299, 8192, BF, BF, BF, BF, 0.0, 0, 0),
    (2, 8200, F32, HALF, HALF, HALF, 0.0, 0, 0), (301, 8200, F32, BF, F32, BF, 0.0, 0, 0), (2, 16384, BF, BF, BF, BF, 0.0, 0, 0),
    (1, 32768, F32, BF, F32, F32, 0.0, 0, 0), (3, 32761, HALF, HALF, None, HALF, 0.0, 3, 0),
]


@pytest.mark.parametrize("n,d,xt,t,rt,wt,offset,extra,shift", NORM)
def test_norm(n, d, xt, t, rt, wt, offset, extra, shift):
    g = _gen(n * 131 + d)
    loud = torch.exp(_randn(g, d))
    x, _ = _guarded(n, d, xt, extra, shift)
    x.copy_(_randn(g, n, d) * loud)
    weight = None if wt is None else (_randn(g, d) * 0.3 + 1.0 - offset).to(wt)
    res = res_out = None
    if rt is not None:
        res, _ = _guarded(n, d, rt, extra, shift)
        res.copy_(_randn(g, n, d) * loud * 3.0)
        res_out, res_intact = _guarded(n, d, rt, extra + 8)
    y, y_intact = _guarded(n, d, t, extra, shift)
    pad = -d % 16 + 16
    q, q_intact = _guarded(n, d, F8, pad)
    scale = torch.zeros((n, -(-d // 128)), device=DEV)
    h, v = _norm_ref(x, weight, 1e-5, res, offset)
    got = P.rms_norm(x, weight, 1e-5, residual=res, residual_out=res_out, offset=offset, y=y, q=q, scale=scale)
    torch.cuda.synchronize()
    assert got.y is y and got.q is q and got.scale is scale and got.residual is res_out
    _check16(y, v)
    _check8(q, scale, v)
    y_intact(), q_intact()
    if rt is not None:
        assert torch.equal(res_out, h.float().to(rt))
        res_intact()
    # buffers of the call's own, one output at a time, and in place
    only8 = P.rms_norm(x, weight, 1e-5, residual=None if res is None else res.clone(), offset=offset, out_type=None, fp8=True)
    if rt is not None or xt is not F32 or (wt is not None and wt is not F32) or t is BF:
        assert torch.equal(only8.q.float(), q.float()) and torch.equal(only8.scale, scale) and only8.y is None
    res2 = None if res is None else res.clone()
    only16 = P.rms_norm(x, weight, 1e-5, residual=res2, offset=offset, out_type=t)
    assert torch.equal(only16.y, y) and only16.q is None
    if rt is not None:
        assert only16.residual is res2 and torch.equal(res2, res_out)
    if xt is t:
        P.rms_norm(x, weight, 1e-5, residual=res, residual_out=res_out, offset=offset, y=x)
        assert torch.equal(x, y)


def test_norm_rows_do_not_depend_on_the_batch():
    g = _gen(1)
    for d in (512, 4096, 8192):
        x, w = _randn(g, 700, d), _randn(g, d).to(BF)
        a, b = P.rms_norm(x, w, out_type=BF, fp8=True), P.rms_norm(x[5:6], w, out_type=BF, fp8=True)
        assert torch.equal(a.y[5:6], b.y) and torch.equal(a.q[5:6].float(), b.q.float()) and torch.equal(a.scale[5:6], b.scale)


def test_norm_rows_do_not_depend_on_the_round_they_fit_in():
    """Batches of some 600 to 1200 fp32 rows take a form with fewer registers: the same bits."""
    g = _gen(2)
    for n, d, res_type in ((777, 5120, BF), (1000, 4096, BF), (640, 4168, F32)):
        x, w, res = _randn(g, n, d), _randn(g, d).to(BF), _randn(g, n, d).to(res_type)
        a = P.rms_norm(x, w, residual=res, residual_out=torch.empty_like(res), out_type=BF, fp8=True)
        for rows in (slice(0, 3), slice(n - 2, n)):
            b = P.rms_norm(x[rows], w, residual=res[rows], residual_out=torch.empty_like(res[rows]), out_type=BF, fp8=True)
            assert torch.equal(a.y[rows], b.y) and torch.equal(a.q[rows].float(), b.q.float()) and torch.equal(a.scale[rows], b.scale)
            assert torch.equal(a.residual[rows], b.residual)


def test_norm_of_zeros_infinities_and_nan():
    x = torch.randn((6, 384), device=DEV)
    x[0] = 0.0
    x[1, 5] = math.inf
    x[2, 300] = math.nan
    x[3, :128] = 0.0
    x[4] *= 1e-42
    got = P.rms_norm(x, eps=1e-5, out_type=BF, fp8=True)
    _, v = _norm_ref(x, None, 1e-5, None, 0.0)
    ok = [0, 3, 5]
    _check16(got.y[ok], v[ok])
    _check8(got.q[ok], got.scale[ok], v[ok])
    assert (got.scale[0] == LEAST).all() and (got.q[0].float() == 0).all() and got.scale[3, 0] == LEAST
    assert got.y[1, 5].isnan() and (got.y[1, :5] == 0).all() and (got.y[1, 6:] == 0).all()     # inf * rsqrt(inf)
    assert got.y[2].isnan().all() and got.scale[2].isnan().all() and got.q[2].float().isnan().all()
    assert got.scale[1, 0].isnan() and (got.scale[1, 1:] == LEAST).all()
    assert got.scale[4].isfinite().all() and (got.scale[4] >= LEAST).all()
    zero = P.rms_norm(x[:1], eps=0.0, out_type=BF)
    assert zero.y.isnan().all()                                                              # 0 * rsqrt(0)


def test_norm_residual_only_and_empty():
    x, res = torch.randn((3, 64), device=DEV), torch.randn((3, 64), device=DEV).to(BF)
    want = (x + res.float()).to(BF)
    got = P.rms_norm(x, residual=res)
    assert got.y is None and got.q is None and torch.equal(res, want)
    none = P.rms_norm(x[:0], out_type=BF, fp8=True)
    assert none.y.shape == (0, 64) and none.q.shape == (0, 64) and none.scale.shape == (0, 1)
    with pytest.raises(ValueError):
        P.rms_norm(x)
    with pytest.raises(ValueError):
        P.rms_norm(x.to(BF), residual=res.to(HALF), out_type=BF)
    with pytest.raises(ValueError):
        P.rms_norm(x, out_type=F32)
    with pytest.raises(P.PloraError):
        P.rms_norm(torch.zeros((1, 32769), device=DEV), out_type=BF)


# ---- activation ------------------------------------------------------------------------------------
def _act_ref(gate, up, act):
    v = gate.double()
    if act == "silu":
        v = v * torch.sigmoid(v)
    elif act == "gelu":
        # v / 2 (1 + tanh z), written so that nothing cancels: tanh z is -1 in 64 bits from z = -19 on
        v = v * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3))
    return v if up is None else v * up.double()


ACT = [
    # n, d, in, type, act, gated, parts of one row, shift
    (1, 11008, F32, BF, "silu", True, False, 0), (3, 13824, BF, BF, "silu", True, True, 0), (257, 1000, HALF, HALF, "gelu", True, True, 0),
    (65, 136, F32, HALF, "gelu", False, False, 0), (700, 8, BF, BF, "silu", True, True, 0), (5, 1, F32, BF, "silu", True, False, 0),
    (9, 127, HALF, HALF, "none", False, False, 0), (9, 129, BF, BF, "none", True, True, 0), (130, 8192, BF, BF, "none", False, False, 0),
    (2, 40000, F32, HALF, "silu", True, False, 0), (4, 256, F32, BF, "gelu", True, True, 1), (33, 2056, HALF, HALF, "silu", False, True, 0),
]


@pytest.mark.parametrize("n,d,xt,t,act,gated,fused,shift", ACT)
def test_act(n, d, xt, t, act, gated, fused, shift):
    g = _gen(n * 17 + d)
    row, _ = _guarded(n, 2 * d, xt, 0, shift)
    row.copy_(_randn(g, n, 2 * d) * 3.0)
    gate, up = (row[:, :d], row[:, d:]) if fused else (row[:, :d].contiguous(), row[:, d:].contiguous())
    up = up if gated else None
    y, y_intact = _guarded(n, d, t, 8, shift)
    q, q_intact = _guarded(n, d, F8, -d % 16 + 16)
    scale = torch.zeros((n, -(-d // 128)), device=DEV)
    P.gated_act(gate, up, act=act, y=y, q=q, scale=scale)
    v = _act_ref(gate, up, act)
    # act is v / (1 + e^-w), w = 2 z for gelu: w has up to four roundings, so e^-w is off by 2^-22 |w|.  A quotient whose divisor
    # passes 2^126 is zero: |v| < 2^7 there.
    w = gate.double().abs()
    w = 1.6 * w + 0.0714 * w ** 3 if act == "gelu" else w
    least = TINY[t] + 2.0 ** -119 * (1.0 if up is None else up.double().abs())
    assert ((y.double() - v).abs() <= (U[t] + FP32 + 2.0 ** -22 * w) * v.abs() + least).all()
    _check8(q, scale, v)
    y_intact(), q_intact()
    own = P.gated_act(gate, up, act=act, out_type=t, fp8=True)
    assert torch.equal(own.y, y) and torch.equal(own.q.float(), q.float()) and torch.equal(own.scale, scale)


def test_act_of_far_values():
    x = torch.tensor([[-math.inf, -1e30, -200.0, -90.0, -0.0, 0.0, 90.0, 1e30, math.inf, math.nan]], device=DEV)
    y = P.gated_act(x, act="silu", out_type=BF).y[0].float()
    assert y[0].isnan() and (y[1:6] == 0).sum() >= 4 and y[1:6].abs().max() < 1e-30 and y[6] == 90.0
    assert y[7] == torch.tensor(1e30).to(BF).float() and y[8] == math.inf and y[9].isnan()
    y = P.gated_act(x, act="gelu", out_type=BF).y[0].float()
    assert y[1:6].abs().max() == 0 and y[6] == 90.0 and y[8] == math.inf and y[9].isnan()


# ---- weights ------------------------------------------------------------------------------------------
@pytest.mark.parametrize("n,k,t", [(1, 1, F32), (128, 128, BF), (129, 257, HALF), (300, 1000, BF), (2056, 4176, F32), (64, 8, BF)])
def test_quant_weight(n, k, t):
    w = _randn(_gen(n + k), n, k + 5).to(t)[:, :k]
    q, scale = P.quant_weight(w)
    v = w.double()
    assert q.shape == (n, k) and q.stride(0) % 16 == 0 and scale.shape == (-(-n // 128), -(-k // 128))
    for i in range(0, n, 128):
        for j in range(0, k, 128):
            top = v[i:i + 128, j:j + 128].abs().max()
            assert abs(float(scale[i // 128, j // 128]) - float(top) / 448.0) <= 2.0 ** -23 * float(top) / 448.0 + 1e-37
    s = scale.double().repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :k]
    assert ((q.double() * s - v).abs() <= torch.maximum(2.0 ** -4 * v.abs(), 2.0 ** -10 * s) * (1 + 2.0 ** -9)).all()


def test_quant_weight_of_zeros_and_nan():
    w = torch.zeros((256, 256), device=DEV)
    w[200, 10] = math.nan
    q, scale = P.quant_weight(w)
    assert (scale[0] == LEAST).all() and scale[1, 0].isnan() and scale[1, 1] == LEAST
    assert (q[:128].float() == 0).all() and q[128:, :128].float().isnan().all() and (q[128:, 128:].float() == 0).all()


# ---- product ------------------------------------------------------------------------------------------
def _matrix8(g, rows, cols, per_rows, pad=0):
    """A random 8-bit matrix; NaN in the bytes behind its columns."""
    q, _ = _guarded(rows, cols, F8, -cols % 16 + pad)
    q.as_strided((rows, q.stride(0)), (q.stride(0), 1)).fill_(math.nan)
    q.copy_((_randn(g, rows, cols) * 60.0).clamp(-448, 448).to(F8))
    scale = torch.exp(_randn(g, -(-rows // per_rows), -(-cols // 128))) * 0.01
    return q, scale


def _values(q, scale, per_rows):
    rows, cols = q.shape
    return q.double() * scale.double().repeat_interleave(per_rows, 0)[:rows].repeat_interleave(128, 1)[:, :cols]


def _check_product(out, x, xs, w, ws):
    a, b = _values(x, xs, 1), _values(w, ws, 128)
    want, size = a @ b.T, a.abs() @ b.abs().T
    tol = (xs.shape[1] + 160) * 2.0 ** -24 * size + U[out.dtype] * want.abs() + TINY[out.dtype]
    bad = (out.double() - want).abs() > tol
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[0].tolist(), float(((out.double() - want).abs() / tol).max()))


PRODUCT = [
    # m, k, columns of the weights, out
    (1, 4096, (4096, 1024, 1024), F32), (1, 1, (1,), F32), (1, 16, (8,), BF), (2, 100, (130, 1), F32), (7, 128, (64,), HALF),
    (8, 129, (65, 63, 64, 1), F32), (9, 1000, (200,), BF), (31, 512, (256,), F32), (33, 640, (1000, 24), HALF), (64, 5120, (1000,), F32),
    (64, 13824, (128,), F32), (127, 272, (257,), BF), (128, 2048, (512, 512), F32), (129, 2048, (512, 512), F32), (129, 16, (16,), F32),
    (200, 300, (1, 300, 129), BF), (255, 1024, (700,), HALF), (256, 4096, (256,), F32), (257, 128, (2056,), F32), (300, 4176, (4096, 1024), BF),
    (512, 13824, (640,), F32), (777, 656, (1000, 1000, 1000, 1000), F32), (1111, 4176, (2056,), BF), (2500, 1024, (5120,), F32),
    (5000, 256, (2048, 264), HALF),
]


@pytest.mark.parametrize("m,k,ns,t", PRODUCT)
def test_product(m, k, ns, t):
    g = _gen(m * 7 + k)
    x, xs = _matrix8(g, m, k, 1, 16 if m % 2 else 0)
    ws = [_matrix8(g, n, k, 128, 16 * (i % 2)) for i, n in enumerate(ns)]
    outs = [_guarded(m, n, t, 0 if n % 16 == 0 and i != 1 else 3, i == 1) for i, n in enumerate(ns)]
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = P.gemm_fp8(x, xs, [w for w, _ in ws], [s for _, s in ws], out=[o for o, _ in outs], status=status)
    torch.cuda.synchronize()
    assert int(status) == 0 and all(a is b for a, (b, _) in zip(got, outs))
    for (o, intact), (w, s) in zip(outs, ws):
        _check_product(o, x, xs, w, s)
        intact()
    # one by one, with buffers of the call's own: the same sums
    one = P.gemm_fp8(x, xs, ws[0][0], ws[0][1], out_type=t)
    _check_product(one, x, xs, *ws[0])
    again = P.gemm_fp8(x, xs, ws[0][0], ws[0][1], out_type=t)
    assert torch.equal(one, again)


# Sizes at which the call takes its different forms: tiles of 64 to 256 columns of single CTAs or of pairs, K in one part or several.
FORMS = [
    (1, 23, (22,)), (77, 2382, (3817,)), (1, 5305, (3035,)), (16, 3485, (3372,)), (90, 1175, (36,)), (33, 2234, (23,)), (59, 2573, (32,)),
    (2, 2892, (51,)), (7, 42, (2946, 84, 4683, 3467)), (5, 3119, (433, 1416)), (128, 1920, (448, 1536)), (64, 4493, (314, 4234, 194)),
    (302, 166, (123, 2550, 4414, 323)), (64, 1000, (13824, 13824)), (773, 1843, (1224, 3343)), (788, 401, (1441, 1189, 2121)),
    (334, 26, (29,)), (405, 242, (2522,)), (1474, 1888, (215, 1054)), (426, 102, (1541, 3977, 294)), (941, 237, (39, 2537, 160, 274)),
    (1001, 400, (1911, 2011)), (797, 1774, (4386,)),
]


@pytest.mark.parametrize("m,k,ns", FORMS)
def test_product_in_all_forms(m, k, ns):
    g = _gen(m + k)
    x, xs = _matrix8(g, m, k, 1)
    ws = [_matrix8(g, n, k, 128) for n in ns]
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    outs = P.gemm_fp8(x, xs, [w for w, _ in ws], [s for _, s in ws], out_type=(F32, BF, HALF)[(m + k) % 3], status=status)
    assert int(status) == 0
    for o, (w, s) in zip(outs, ws):
        _check_product(o, x, xs, w, s)


def test_offsets_beyond_32_bits():
    """Outputs of more than 2^31 elements, inputs of more than 2^31 bytes; looked at where they begin and end."""
    g = _gen(9)
    m, n = 66000, 33000
    x, xs = _matrix8(g, m, 128, 1)
    w, ws = _matrix8(g, n, 128, 128)
    out = P.gemm_fp8(x, xs, w, ws, out_type=BF)
    rows = [0, 1, m // 2, m - 2, m - 1]
    _check_product(out[rows], x[rows], xs[rows], w, ws)
    del out
    n, d = 70000, 32768
    x = torch.empty((n, d), dtype=BF, device=DEV)
    for a in range(0, n, 10000):
        x[a:a + 10000] = _randn(g, 10000, d).to(BF)
    rows = [0, n // 2, n - 1]
    norm = P.rms_norm(x, eps=1e-5, out_type=BF, fp8=True)
    v = _norm_ref(x[rows], None, 1e-5, None, 0.0)[1]
    _check16(norm.y[rows], v)
    _check8(norm.q[rows], norm.scale[rows], v)
    act = P.gated_act(x, norm.y, fp8=True)
    _check8(act.q[rows], act.scale[rows], _act_ref(x[rows], norm.y[rows], "silu"))


def test_product_keeps_rows_and_columns_apart():
    """A NaN or an infinite scale stays in its row, or its 128 columns."""
    for m in (5, 300):
        g = _gen(m)
        x, xs = _matrix8(g, m, 512, 1)
        w, ws = _matrix8(g, 400, 512, 128)
        clean = P.gemm_fp8(x, xs, w, ws)
        x[3, 100] = math.nan
        ws[1, 2] = math.inf
        out = P.gemm_fp8(x, xs, w, ws)
        assert out[3].isnan().all() and not out[:, 128:256].isfinite().any()
        keep = torch.ones_like(out, dtype=torch.bool)
        keep[3] = False
        keep[:, 128:256] = False
        assert torch.equal(out[keep], clean[keep])


def test_product_empty_and_refused():
    g = _gen(3)
    x, xs = _matrix8(g, 4, 64, 1)
    w, ws = _matrix8(g, 32, 64, 128)
    assert P.gemm_fp8(x[:0], xs[:0], w, ws).shape == (0, 32)
    for bad in (lambda: P.gemm_fp8(x, xs, w[:, :48], ws), lambda: P.gemm_fp8(x, xs[:, :0], w, ws), lambda: P.gemm_fp8(x.float(), xs, w, ws),
                lambda: P.gemm_fp8(x, xs, [w, w], [ws]), lambda: P.gemm_fp8(x, xs, w, ws, out_type=torch.float64),
                lambda: P.gemm_fp8(x, xs, w, ws, out=torch.empty((4, 31), device=DEV)),
                lambda: P.gemm_fp8(x, xs, [w] * 5, [ws] * 5), lambda: P.gemm_fp8(x, xs.half(), w, ws)):
        with pytest.raises(ValueError):
            bad()


# ---- streams, graphs, and the calls together ---------------------------------------------------------------
def _layer(g, n, d, h):
    x, res = _randn(g, n, d), _randn(g, n, d).to(BF)
    weight = (_randn(g, d) * 0.2 + 1.0).to(BF)
    gate, up, down = (P.quant_weight(_randn(g, o, i) * i ** -0.5) for o, i in ((h, d), (h, d), (d, h)))
    return x, res, weight, gate, up, down


def _ffn(x, res, weight, gate, up, down, stream=None):
    a = P.rms_norm(x, weight, 1e-5, residual=res, residual_out=torch.empty_like(res), fp8=True, out_type=BF, stream=stream)
    yg, yu = P.gemm_fp8(a.q, a.scale, [gate[0], up[0]], [gate[1], up[1]], stream=stream)
    b = P.gated_act(yg, yu, fp8=True, stream=stream)
    return a.y, a.residual, P.gemm_fp8(b.q, b.scale, *down, stream=stream)


@pytest.mark.parametrize("n", [1, 40, 300])
def test_ffn_chain(n):
    """norm -> gate and up -> activation -> down, on what each call gives, against 64 bits step by step; on another stream and in a
    graph the same bits."""
    g = _gen(n)
    args = _layer(g, n, 1024, 1536)
    x, res, weight, gate, up, down = args
    y, r, out = _ffn(*args)
    h, v = _norm_ref(x, weight, 1e-5, res, 0.0)
    _check16(y, v)
    a = P.rms_norm(x, weight, 1e-5, residual=res, residual_out=torch.empty_like(res), fp8=True)
    _check8(a.q, a.scale, v)
    yg, yu = P.gemm_fp8(a.q, a.scale, [gate[0], up[0]], [gate[1], up[1]])
    _check_product(yg, a.q, a.scale, *gate)
    _check_product(yu, a.q, a.scale, *up)
    b = P.gated_act(yg, yu, fp8=True)
    _check8(b.q, b.scale, _act_ref(yg, yu, "silu"))
    _check_product(out, b.q, b.scale, *down)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = _ffn(*args, stream=s)
    s.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(other, (y, r, out)))
    with torch.cuda.stream(s):
        _ffn(*args)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        captured = _ffn(*args)
    for k in range(3):
        x.copy_(_randn(g, *x.shape))
        want = _ffn(*args)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(captured, want)), k


def test_two_streams_at_once():
    g = _gen(8)
    jobs = [_layer(g, n, 2048, 2816) for n in (16, 500)]
    want = [_ffn(*j) for j in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(10):
        got = [_ffn(*j, stream=s) for j, s in zip(jobs, streams)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_two_graphs_of_the_same_inputs():
    """Calls have no workspace: graphs captured of the same inputs replay side by side."""
    g = _gen(12)
    args = _layer(g, 64, 1024, 1536)
    want = _ffn(*args)
    graphs = []
    for _ in range(2):
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            out = _ffn(*args)
        graphs.append((s, graph, out))
    torch.cuda.synchronize()
    for _ in range(20):
        for s, graph, _ in graphs:
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for _, _, out in graphs:
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_weights_made_right_before_the_product():
    """The product fetches weights before the kernel in front has ended, if that kernel allows it: one that writes weights does not."""
    g = _gen(13)
    x, xs = _matrix8(g, 3, 4096, 1)
    a, b = (_randn(g, 2048, 4096).to(BF) for _ in range(2))
    qa, qb = P.quant_weight(a), P.quant_weight(b)
    want = [P.gemm_fp8(x, xs, *qa), P.gemm_fp8(x, xs, *qb)]
    for i in range(20):
        w, s = P.quant_weight((a, b)[i % 2])
        assert torch.equal(P.gemm_fp8(x, xs, w, s), want[i % 2])
        w.view(torch.uint8).copy_((qb, qa)[i % 2][0].view(torch.uint8))
        s.copy_((qb, qa)[i % 2][1])
        assert torch.equal(P.gemm_fp8(x, xs, w, s), want[1 - i % 2])


def test_block_example():
    """A decoder block on all the calls (examples/serve_layer.py) against the same block in 64 bits from its 16-bit weights.  8-bit
    values are off by 0.026 in the mean square, so each of a block's four products in a row by 0.037 of its spread and all of them by
    0.074; the worst of some 10^5 outputs and the largest of them lie about as many spreads out."""
    import importlib.util
    from pathlib import Path
    path = Path(__file__).resolve().parent.parent / "examples" / "serve_layer.py"
    spec = importlib.util.spec_from_file_location("serve_layer", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    assert example.main(steps=2, block=True) <= 0.12
