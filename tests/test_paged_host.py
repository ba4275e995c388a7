"""The paged cache's calls without a GPU: layouts of the argument structures, sizes, and refusals before anything is launched."""
import ctypes
import subprocess
import sys
from pathlib import Path

import pytest
import torch

import paper_2608_05483_b200 as P
from paper_2608_05483_b200 import binding


def test_packed_arguments_have_the_structures_layout():
    assert binding._ROPE_PACK.size == ctypes.sizeof(P.RopeCacheArgs)
    assert binding._PAGED_PACK.size == ctypes.sizeof(P.PagedAttn)
    for pack, struct in ((binding._ROPE_PACK, P.RopeCacheArgs), (binding._PAGED_PACK, P.PagedAttn)):
        values = list(range(1, 1 + len(struct._fields_)))
        s = struct.from_buffer_copy(pack.pack(*values))
        assert [getattr(s, name) for name, _ in struct._fields_] == values


def test_workspace_sizes():
    size = P.plora_attn_paged_workspace_bytes
    base = size(64, 64, 32, 8, 128, 16, 256)
    assert base > 256 and base % 256 == 0
    # more tokens, more requests or longer tables never need less
    assert size(128, 64, 32, 8, 128, 16, 256) >= base and size(64, 64, 32, 8, 128, 16, 512) >= base
    assert size(64, 128, 32, 8, 128, 16, 256) >= base
    for bad in ((0, 1, 8, 8, 128, 16, 4), (1, 0, 8, 8, 128, 16, 4), (1, 1, 8, 0, 128, 16, 4), (1, 1, 8, 8, 128, 16, 0),
                (1, 1, 8, 8, 96, 16, 4), (1, 1, 8, 8, 128, 24, 4), (1, 1, 8, 3, 128, 16, 4), (1, 1, 256, 1, 128, 16, 4)):
        assert size(*bad) == 0


def test_refusals_before_the_device_is_touched():
    a = P.PagedAttn()
    assert P.plora_attn_paged(a) == P.OK                      # no tokens: nothing to do
    assert binding.load().plora_attn_paged(None, 0) == P.ERR_INVALID_ARG
    a.n_tok = 1
    assert P.plora_attn_paged(a) == P.ERR_INVALID_ARG
    a.n_tok = -1
    assert P.plora_attn_paged(a) == P.ERR_INVALID_ARG
    r = P.RopeCacheArgs()
    assert binding.load().plora_rope_cache(None, 0) == P.ERR_INVALID_ARG
    assert P.plora_rope_cache(r) == P.ERR_INVALID_ARG         # neither q nor k and v
    r.n_q_heads, r.head_dim, r.in_type = 2, 64, P.INPUT_FP32
    assert P.plora_rope_cache(r) == P.OK                      # no tokens
    r.n_tok = 3
    assert P.plora_rope_cache(r) == P.ERR_INVALID_ARG         # null pointers
    r.head_dim = 63
    assert P.plora_rope_cache(r) == P.ERR_UNSUPPORTED
    r.head_dim, r.in_type, r.out_type = 64, P.INPUT_FP16, P.INPUT_BF16
    assert P.plora_rope_cache(r) == P.ERR_INVALID_ARG
    assert P.plora_rope_table(P.RopeDesc(64, 0, 10000.0, 1.0, 0.0, 0.0, 0.0, 1.0), 8, None) == P.ERR_INVALID_ARG
    assert P.plora_kv_plan(None, None, 1, 16, None, 0, None, None, 4, 4, None, None, None, None, None, None) == P.ERR_INVALID_ARG


def test_tensors_that_are_not_on_the_gpu_are_refused():
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    q, c = torch.zeros(2, 2, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        P.kv_plan(i(2), i(2), 16, i(4), i(2, 3), 8)
    with pytest.raises(ValueError):
        P.rope_cache(q, q, q, i(2), i(2), None, c, c.clone())
    with pytest.raises(ValueError):
        P.attn_paged(q, c, c.clone(), i(2, 3), i(2), 1.0)
    with pytest.raises(ValueError):
        P.rope_table(64, 8, scaling="no such scaling")

@pytest.mark.parametrize("n_tok,hq,hk,d,page,blocks", [(16384, 64, 8, 128, 128, 35157), (40000, 8, 8, 64, 16, 400000)])
def test_workspace_holds_the_partial_results_of_the_longest_caches(n_tok, hq, hk, d, page, blocks):
    """A piece of a split has at most 2^22 keys: every token of a prompt behind a longer cache leaves a partial result per piece."""
    pieces = -(-blocks * page // (1 << 22))
    assert pieces > 1
    assert P.plora_attn_paged_workspace_bytes(n_tok, 1, hq, hk, d, page, blocks) >= n_tok * pieces * hq * (d + 2) * 4


class _OnGpu:
    """Stands for a CUDA tensor of this shape and stride where only its layout is looked at."""

    def __init__(self, shape, stride, dtype=torch.bfloat16):
        self.shape, self._stride, self.dtype, self.is_cuda = shape, stride, dtype, True

    def stride(self):
        return self._stride


def test_expanded_tensors_are_refused():
    """A stride of 0 means packed in the C structures: a tensor expanded along its tokens would be read as n packed rows."""
    row = lambda stride, n=4: _OnGpu((n, 2, 64), (stride, 64, 1))
    assert torch.zeros(1, 2, 64).expand(4, 2, 64).stride() == row(0).stride()
    with pytest.raises(ValueError):
        binding._token_stride("q", row(0))
    assert binding._token_stride("q", row(320)) == 320
    assert binding._token_stride("q", row(0, 1)) == 128 and binding._token_stride("q", row(128, 0)) == 128
    cache = lambda stride, n=4: _OnGpu((n, 2, 16, 64), (stride, 1024, 64, 1))
    with pytest.raises(ValueError):
        binding._page_stride(cache(0), cache(0))
    assert binding._page_stride(cache(4096), cache(4096)) == 4096
    assert binding._page_stride(cache(0, 1), cache(0, 1)) == 2048


def test_the_c_abi_is_used_without_torch():
    code = ("import sys; sys.modules['torch'] = None\n"
            "import paper_2608_05483_b200 as P\n"
            "assert P.load() and P.status_string(P.OK) and P.plora_attn_paged_workspace_bytes(1, 1, 8, 8, 128, 16, 4) > 0\n"
            "assert P.plora_attn_paged(P.PagedAttn()) == P.OK\n")
    run = subprocess.run([sys.executable, "-c", code], cwd=Path(__file__).resolve().parent.parent, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stderr[-2000:]
