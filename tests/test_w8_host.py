"""The 8-bit calls without a GPU: layouts of the argument structures, and refusals before anything is launched."""
import ctypes

import pytest
import torch

import paper_2608_05483_b200 as P
from paper_2608_05483_b200 import binding


def _flat(s):
    out = []
    for name, _ in s._fields_:
        v = getattr(s, name)
        out += list(v) if isinstance(v, ctypes.Array) else [v]
    return out


@pytest.mark.parametrize("pack,struct", [(binding._NORM_PACK, P.RmsNormArgs), (binding._ACT_PACK, P.GatedActArgs),
                                         (binding._GEMM_PACK, P.GemmFp8Args)])
def test_packed_arguments_have_the_structures_layout(pack, struct):
    assert pack.size == ctypes.sizeof(struct)
    values = list(range(1, 1 + len(_flat(struct()))))
    assert _flat(struct.from_buffer_copy(pack.pack(*values))) == values


AT = 4096        # an address that is never followed: every call below is refused first, or has nothing to do


def _norm(**kw):
    a = P.RmsNormArgs(P.INPUT_FP32, P.INPUT_BF16, P.INPUT_BF16, P.INPUT_BF16, 2, 64, 0, 0, 0, 0, 0, AT, AT, AT, AT, AT, AT, AT, 1e-5, 0.0)
    for k, v in kw.items():
        setattr(a, k, v)
    return P.plora_rms_norm(a)


def _act(**kw):
    a = P.GatedActArgs(P.INPUT_FP32, P.INPUT_BF16, P.ACT_SILU, 2, 64, 0, 0, 0, 0, AT, AT, AT, AT, AT)
    for k, v in kw.items():
        setattr(a, k, v)
    return P.plora_gated_act(a)


def _gemm(**kw):
    a = P.GemmFp8Args(P.INPUT_FP32, 2, 64, 2)
    a.x = a.x_scale = AT
    for i in range(2):
        a.n[i], a.w[i], a.w_scale[i], a.out[i] = 64, AT, AT, AT
    for k, v in kw.items():
        if isinstance(v, tuple):
            getattr(a, k)[v[0]] = v[1]
        else:
            setattr(a, k, v)
    return P.plora_gemm_fp8(a)


def test_nothing_to_do():
    assert _norm(n=0) == _act(n=0) == _gemm(m=0) == P.OK
    assert P.plora_quant_weight(AT, P.INPUT_BF16, 0, 64, 0, AT, 0, AT) == P.OK


@pytest.mark.parametrize("kw", [
    dict(n=-1), dict(d=0), dict(type=P.INPUT_FP32), dict(type=7), dict(in_type=P.INPUT_FP16), dict(weight_type=P.INPUT_FP16),
    dict(residual_type=P.INPUT_FP16), dict(eps=-1.0), dict(eps=float("nan")), dict(offset=float("inf")), dict(x=None), dict(residual=None),
    dict(residual_out=None), dict(q=None), dict(scale=None), dict(y=None, q=None, scale=None, residual=None, residual_out=None),
    dict(x_stride=63), dict(residual_stride=8), dict(residual_out_stride=-64), dict(y_stride=1), dict(q_stride=72), dict(q_stride=48),
    dict(q=AT + 8), dict(x=AT + 2), dict(y=AT + 1), dict(scale=AT + 2)])
def test_norm_refuses(kw):
    assert _norm(**kw) == P.ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [
    dict(n=-1), dict(d=0), dict(type=P.INPUT_FP32), dict(in_type=P.INPUT_FP16), dict(act=3), dict(act=-1), dict(gate=None), dict(q=None),
    dict(scale=None), dict(y=None, q=None, scale=None), dict(gate_stride=63), dict(up_stride=63), dict(y_stride=63), dict(q_stride=72),
    dict(q=AT + 1), dict(up=AT + 2), dict(y=AT + 1)])
def test_act_refuses(kw):
    assert _act(**kw) == P.ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [
    dict(m=-1), dict(k=0), dict(n_weights=0), dict(n_weights=5), dict(n_weights=3), dict(out_type=3), dict(n=(1, 0)), dict(x=None),
    dict(x_scale=None), dict(w=(0, None)), dict(w_scale=(1, None)), dict(out=(1, None)), dict(x=AT + 8), dict(w=(1, AT + 4)),
    dict(out=(0, AT + 2)), dict(x_stride=72), dict(x_stride=48), dict(w_stride=(1, 72)), dict(out_stride=(0, 63)), dict(status=AT + 2)])
def test_gemm_refuses(kw):
    assert _gemm(**kw) == P.ERR_INVALID_ARG


def test_more_refusals():
    lib = binding.load()
    assert lib.plora_rms_norm(None, 0) == lib.plora_gated_act(None, 0) == lib.plora_gemm_fp8(None, 0) == P.ERR_INVALID_ARG
    assert _norm(d=32769) == P.ERR_UNSUPPORTED
    assert _act(n=1 << 24, d=1 << 14) == P.ERR_UNSUPPORTED
    assert _gemm(m=(1 << 30) + 1) == _gemm(n=(0, (1 << 30) + 1), out_stride=(0, 1 << 31)) == _gemm(k=(1 << 30) + 1) == P.ERR_UNSUPPORTED
    q = P.plora_quant_weight
    for bad in ((None, 0, 4, 64, 0, AT, 0, AT), (AT, 3, 4, 64, 0, AT, 0, AT), (AT, 0, -1, 64, 0, AT, 0, AT), (AT, 0, 4, 0, 0, AT, 0, AT),
                (AT, 0, 4, 64, 32, AT, 0, AT), (AT, 0, 4, 64, 0, AT + 8, 0, AT), (AT, 0, 4, 64, 0, AT, 72, AT), (AT, 0, 4, 64, 0, AT, 0, None),
                (AT + 1, 0, 4, 64, 0, AT, 0, AT)):
        assert q(*bad) == P.ERR_INVALID_ARG
    assert q(AT, 0, 65536 * 128, 64, 0, AT, 0, AT) == P.ERR_UNSUPPORTED


class _OnGpu:
    """Stands for a CUDA tensor of this shape and stride where only its layout is looked at."""

    def __init__(self, shape, stride, dtype=torch.float32, device=0):
        self.shape, self._stride, self.dtype, self.is_cuda, self.device = shape, stride, dtype, device >= 0, device

    def stride(self):
        return self._stride

    def get_device(self):
        return self.device

    def is_contiguous(self):
        return self._stride == (self.shape[1], 1)

    def data_ptr(self):
        return AT


def test_layouts_that_the_binding_refuses():
    rows, q_rows, scales = binding._rows, binding._q_rows, binding._scales
    assert rows("x", _OnGpu((4, 64), (200, 1)), 4, 64, 0) == 200
    assert rows("x", _OnGpu((1, 64), (0, 1)), 1, 64, 0) == 64 and rows("x", _OnGpu((0, 64), (64, 1)), 0, 64, 0) == 64
    assert rows("x", _OnGpu((4, 1), (8, 5)), 4, 1, 0) == 8
    f8 = torch.float8_e4m3fn
    assert q_rows("q", _OnGpu((4, 50), (64, 1), f8), 4, 50, 0) == 64 and q_rows("q", _OnGpu((1, 50), (50, 1), f8), 1, 50, 0) == 64
    assert scales("s", _OnGpu((4, 2), (2, 1)), 4, 2, 0) == AT
    for bad in (lambda: rows("x", _OnGpu((4, 64), (0, 1)), 4, 64, 0),               # expanded along its rows
                lambda: rows("x", _OnGpu((4, 64), (32, 1)), 4, 64, 0),              # rows that overlap
                lambda: rows("x", _OnGpu((4, 64), (1, 4)), 4, 64, 0),               # transposed
                lambda: rows("x", _OnGpu((4, 64), (64, 1)), 4, 65, 0),
                lambda: rows("x", _OnGpu((4, 64), (64, 1), device=1), 4, 64, 0),    # another device
                lambda: rows("x", _OnGpu((4, 64), (64, 1), device=-1), 4, 64, 0),   # not on a GPU
                lambda: q_rows("q", _OnGpu((4, 50), (50, 1), f8), 4, 50, 0),
                lambda: q_rows("q", _OnGpu((4, 64), (64, 1)), 4, 64, 0),
                lambda: q_rows("q", _OnGpu((4, 64), (64, 1), torch.float8_e5m2), 4, 64, 0),
                lambda: scales("s", _OnGpu((4, 2), (4, 1)), 4, 2, 0),
                lambda: scales("s", _OnGpu((2, 4), (4, 1)), 4, 2, 0),
                lambda: scales("s", _OnGpu((4, 2), (2, 1), torch.bfloat16), 4, 2, 0),
                lambda: scales("s", _OnGpu((4, 2), (2, 1), device=1), 4, 2, 0)):
        with pytest.raises(ValueError):
            bad()


def test_tensors_that_are_not_on_the_gpu_are_refused():
    x, f8 = torch.zeros(4, 64), torch.float8_e4m3fn
    with pytest.raises(ValueError):
        P.rms_norm(x, y=torch.zeros(4, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        P.rms_norm(x)                       # nothing to write
    with pytest.raises(ValueError):
        P.gated_act(x, act="tanh", fp8=True)
    with pytest.raises(ValueError):
        P.gated_act(x, x.bfloat16(), fp8=True)
    with pytest.raises(ValueError):
        P.gated_act(x, x)
    with pytest.raises(ValueError):
        P.gemm_fp8(x.to(f8), torch.ones(4, 1), x.to(f8), torch.ones(1, 1))
    with pytest.raises(ValueError):
        P.gemm_fp8(x.to(f8), torch.ones(4, 1), [], [])
