"""ctypes binding of the C ABI in include/plora.h.

Argument marshalling only: every step of the path runs in the CUDA library.
The module-level `plora_*` functions mirror the C entry points one to one
(pointers as ints, status codes returned); `Context` wraps them for torch
tensors and raises `PloraError` on a non-zero status.  There is no CPU
fallback: if the shared library is missing or cannot be loaded, import of the
functions fails loudly.
"""
from __future__ import annotations

import ctypes
import struct
from pathlib import Path
from typing import Any, NamedTuple

import numpy as np

from . import _build


class _Torch:
    """Stands in for the module until the torch layer first needs it: the C ABI is used without torch, too."""

    def __getattr__(self, name):
        global torch
        import torch
        return getattr(torch, name)


torch = _Torch()

OK = 0
ERR_INVALID_ARG = -1
ERR_NOT_REGISTERED = -2
ERR_BAD_ADAPTER_ID = -3
ERR_WORKSPACE = -4
ERR_CUDA = -5
ERR_TIMEOUT = -6
ERR_UNSUPPORTED = -7
ERR_DEBUG_CHECK = -8

PATH_AUTO, PATH_UNFUSED, PATH_FUSED, PATH_SGMV, PATH_SGMV_SPLIT = 0, 1, 2, 3, 4

EXPORTS = (
    "plora_create", "plora_destroy", "plora_pool_slab_bytes", "plora_register_pool", "plora_pool_max_rank",
    "plora_bucket", "plora_bucket_view", "plora_lora_delta", "plora_lora_delta_group", "plora_shrink", "plora_expand",
    "plora_shrink_m16", "plora_expand_m16", "plora_set_input_type",
    "plora_lora_delta_host", "plora_lora_delta_host_async", "plora_host_sync", "plora_lora_delta_noalloc", "plora_set_path", "plora_device_status", "plora_launch_count", "plora_status_string",
    "plora_cost_model", "plora_attn_workspace_bytes", "plora_attn_decode", "plora_attn_status", "plora_attn_set_debug",
    "plora_set_wait_limit", "plora_set_test_hook", "plora_set_inputs_resident", "plora_stream_read",
    "plora_kv_plan", "plora_rope_table", "plora_rope_cache", "plora_attn_paged_workspace_bytes", "plora_attn_paged",
    "plora_rms_norm", "plora_gated_act", "plora_quant_weight", "plora_gemm_fp8",
    "plora_gemm_fp8_status",
)

INPUT_BF16, INPUT_FP16, INPUT_FP32 = 0, 1, 2
ROPE_HALF, ROPE_INTERLEAVED = 0, 1
ROPE_NONE, ROPE_LINEAR, ROPE_NTK, ROPE_BANDS, ROPE_RAMP = 0, 1, 2, 3, 4
ACT_NONE, ACT_SILU, ACT_GELU = 0, 1, 2

HOOK_NONE, HOOK_WITHHOLD_RELEASE, HOOK_MAX_CYCLES = 0, 1, 1 << 24


class PoolDesc(ctypes.Structure):
    _fields_ = [
        ("layer", ctypes.c_int32), ("proj", ctypes.c_int32),
        ("d_in", ctypes.c_int32), ("d_out", ctypes.c_int32),
        ("n_adapters", ctypes.c_int32), ("ab_on_device", ctypes.c_int32),
        ("ranks", ctypes.c_void_p), ("scales", ctypes.c_void_p),
        ("A", ctypes.c_void_p), ("B", ctypes.c_void_p),
    ]


class CostHw(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("c_gpu", "w_gpu", "c_dev", "w_dram", "n_dev", "l_link", "w_link")]


class CostTerms(ctypes.Structure):
    _fields_ = [("t_gpu", ctypes.c_double * 4), ("t_dev_cpt", ctypes.c_double * 4), ("t_dev_trs", ctypes.c_double * 4),
                ("t_lora_gpu", ctypes.c_double), ("t_lora_dev", ctypes.c_double), ("t_lora", ctypes.c_double)]


class RopeDesc(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_int32), ("scaling", ctypes.c_int32)] + [
        (n, ctypes.c_double) for n in ("base", "factor", "orig_len", "low", "high", "magnitude")]


class RopeCacheArgs(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("in_type", "out_type", "layout", "n_tok", "n_q_heads", "n_kv_heads", "head_dim",
                                               "rot_dim", "max_pos", "page_size", "n_pages")]
                + [(n, ctypes.c_int64) for n in ("q_stride", "k_stride", "v_stride", "page_stride")]
                + [(n, ctypes.c_void_p) for n in ("q", "k", "v", "positions", "slots", "table", "q_out", "k_cache", "v_cache",
                                                  "status")])


class PagedAttn(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("type", "n_tok", "n_req", "n_groups", "n_q_heads", "n_kv_heads", "head_dim",
                                               "page_size", "n_pages", "max_blocks")]
                + [(n, ctypes.c_int64) for n in ("q_stride", "page_stride")]
                + [(n, ctypes.c_void_p) for n in ("q", "k_cache", "v_cache", "block_table", "kv_len", "tok_start", "group_start",
                                                  "prefix_len", "key_lo", "key_hi", "slopes")]
                + [("scale", ctypes.c_float), ("softcap", ctypes.c_float), ("out", ctypes.c_void_p),
                   ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)])


class RmsNormArgs(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("in_type", "type", "weight_type", "residual_type", "n", "d")]
                + [(n, ctypes.c_int64) for n in ("x_stride", "residual_stride", "residual_out_stride", "y_stride", "q_stride")]
                + [(n, ctypes.c_void_p) for n in ("x", "weight", "residual", "residual_out", "y", "q", "scale")]
                + [("eps", ctypes.c_float), ("offset", ctypes.c_float)])


class GatedActArgs(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("in_type", "type", "act", "n", "d")]
                + [(n, ctypes.c_int64) for n in ("gate_stride", "up_stride", "y_stride", "q_stride")]
                + [(n, ctypes.c_void_p) for n in ("gate", "up", "y", "q", "scale")])


class GemmFp8Args(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("out_type", "m", "k", "n_weights")]
                + [("n", ctypes.c_int32 * 4), ("x_stride", ctypes.c_int64), ("w_stride", ctypes.c_int64 * 4),
                   ("out_stride", ctypes.c_int64 * 4), ("x", ctypes.c_void_p), ("x_scale", ctypes.c_void_p), ("w", ctypes.c_void_p * 4),
                   ("w_scale", ctypes.c_void_p * 4), ("out", ctypes.c_void_p * 4), ("status", ctypes.c_void_p), ("wait_cycles", ctypes.c_int64),
                   ("weights_ready", ctypes.c_int32), ("test_hook", ctypes.c_int32)])


class PloraError(RuntimeError):
    def __init__(self, status: int, where: str = ""):
        self.status = int(status)
        super().__init__(f"{where}: {status_string(status)} ({status})" if where else f"{status_string(status)} ({status})")


_lib = None


def _debug_build() -> bool:
    """PLORA_DEBUG_BUILD=1 in the environment selects the checked build of the library (same sources compiled with
    -DPLORA_DEBUG: the delta kernels and the paged attention check every address against its buffer and report
    PLORA_ERR_DEBUG_CHECK)."""
    import os
    return os.environ.get("PLORA_DEBUG_BUILD", "") == "1"


def library_path() -> Path:
    return _build.LIB_DEBUG if _debug_build() else _build.LIB


def load(build_if_missing: bool = True):
    """Load libplora_b200.so (building it with nvcc first if it is not there)."""
    global _lib
    if _lib is not None:
        return _lib
    path = library_path()
    if not path.exists():
        if not build_if_missing:
            raise RuntimeError(f"{path} is missing: run __graft_entry__.build() (nvcc, sm_100a); there is no fallback path")
        _build.build(debug=_debug_build())
    lib = ctypes.CDLL(str(path))
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    sig = {
        "plora_create": (i32, [ctypes.POINTER(vp), ctypes.c_int, i32, i32]),
        "plora_destroy": (i32, [vp]),
        "plora_pool_slab_bytes": (ctypes.c_size_t, [ctypes.POINTER(PoolDesc)]),
        "plora_register_pool": (i32, [vp, ctypes.POINTER(PoolDesc), vp, ctypes.c_size_t, vp]),
        "plora_pool_max_rank": (i32, [vp, i32, i32]),
        "plora_bucket": (i32, [vp, vp, i32, i32, vp]),
        "plora_bucket_view": (i32, [vp] + [ctypes.POINTER(vp)] * 5),
        "plora_lora_delta": (i32, [vp, vp, vp, i32, i32, i32, vp, vp]),
        "plora_lora_delta_group": (i32, [vp, i32, vp, vp, i32, vp, vp, vp, vp]),
        "plora_shrink": (i32, [vp, vp, vp, i32, i32, i32, vp, i32, vp]),
        "plora_expand": (i32, [vp, vp, i32, vp, i32, i32, i32, vp, vp]),
        "plora_shrink_m16": (i32, [vp, vp, vp, i32, i32, i32, vp, i32, vp]),
        "plora_expand_m16": (i32, [vp, vp, i32, vp, i32, i32, i32, vp, vp]),
        "plora_lora_delta_host": (i32, [vp, vp, vp, i32, i32, i32, vp, vp]),
        "plora_lora_delta_noalloc": (i32, [vp, vp, vp, i32, i32, i32, vp, vp]),
        "plora_lora_delta_host_async": (i32, [vp, i32, vp, vp, i32, vp, vp, vp, vp]),
        "plora_host_sync": (i32, [vp]),
        "plora_set_path": (i32, [vp, i32, i32]),
        "plora_set_input_type": (i32, [vp, i32]),
        "plora_device_status": (i32, [vp, vp, ctypes.POINTER(i32)]),
        "plora_launch_count": (i64, [vp]),
        "plora_status_string": (ctypes.c_char_p, [i32]),
        "plora_attn_workspace_bytes": (ctypes.c_size_t, [i32, i32, i32, i32]),
        "plora_attn_decode": (i32, [vp, vp, vp, vp, i32, i32, i32, i32, i32, ctypes.c_float, vp, vp, ctypes.c_size_t, vp]),
        "plora_attn_status": (i32, [vp, vp, ctypes.POINTER(i32)]),
        "plora_attn_set_debug": (i32, [vp, i64, i32, vp]),
        "plora_set_wait_limit": (i32, [vp, i64]),
        "plora_set_test_hook": (i32, [vp, i32]),
        "plora_set_inputs_resident": (i32, [vp, i32]),
        "plora_stream_read": (i32, [vp, ctypes.c_size_t, vp, ctypes.c_size_t, vp]),
        "plora_cost_model": (i32, [ctypes.POINTER(CostHw), i32, vp, vp, ctypes.c_double, ctypes.c_double, ctypes.c_double,
                                   ctypes.POINTER(CostTerms)]),
        "plora_kv_plan": (i32, [vp, vp, i32, i32, vp, i32, vp, vp, i32, i32, vp, vp, vp, vp, vp, vp, vp]),
        "plora_rope_table": (i32, [ctypes.POINTER(RopeDesc), i32, vp, vp]),
        "plora_rope_cache": (i32, [vp, vp]),
        "plora_attn_paged_workspace_bytes": (ctypes.c_size_t, [i32] * 7),
        "plora_attn_paged": (i32, [vp, vp]),
        "plora_rms_norm": (i32, [vp, vp]),
        "plora_gated_act": (i32, [vp, vp]),
        "plora_quant_weight": (i32, [vp, i32, i32, i32, i64, vp, i64, vp, vp]),
        "plora_gemm_fp8": (i32, [vp, vp]),
        "plora_gemm_fp8_status": (i32, [vp, ctypes.POINTER(i32)]),
    }
    for name in EXPORTS:
        fn = getattr(lib, name)  # AttributeError here = the library does not export what the header declares
        fn.restype, fn.argtypes = sig[name]
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load().plora_status_string(int(status)).decode()


# ---- one-to-one wrappers (ints for pointers) ------------------------------------------
def plora_create(device: int, max_tokens: int, max_adapters: int):
    h = ctypes.c_void_p()
    rc = load().plora_create(ctypes.byref(h), int(device), int(max_tokens), int(max_adapters))
    return rc, h.value


def plora_destroy(ctx):
    return load().plora_destroy(ctx)


def plora_cost_model(hw: dict, ranks, batch, d: float, value_bytes: float, t_base: float):
    """(status, terms): the cost terms of the paper's four strategies (Section VI-B) as a dict of lists / floats.
    hw: c_gpu, w_gpu, c_dev, w_dram, n_dev, l_link, w_link.  batch: [n_adapters][4] request counts."""
    import numpy as np
    r = np.ascontiguousarray(ranks, np.int32)
    b = np.ascontiguousarray(batch, np.float64).reshape(len(r), 4)
    chw = CostHw(**{k: float(v) for k, v in hw.items()})
    out = CostTerms()
    rc = load().plora_cost_model(ctypes.byref(chw), len(r), r.ctypes.data, b.ctypes.data, float(d), float(value_bytes),
                                 float(t_base), ctypes.byref(out))
    terms = dict(t_gpu=list(out.t_gpu), t_dev_cpt=list(out.t_dev_cpt), t_dev_trs=list(out.t_dev_trs),
                 t_lora_gpu=out.t_lora_gpu, t_lora_dev=out.t_lora_dev, t_lora=out.t_lora)
    return rc, terms


def plora_attn_workspace_bytes(n_req: int, max_kv_len: int, n_kv_heads: int, q_per_kv: int) -> int:
    return int(load().plora_attn_workspace_bytes(n_req, max_kv_len, n_kv_heads, q_per_kv))


def plora_attn_decode(q_ptr, k_ptr, v_ptr, kv_len_ptr, n_req, max_kv_len, n_kv_heads, q_per_kv, head_dim, scale, out_ptr,
                      ws_ptr, ws_bytes, stream=0):
    return load().plora_attn_decode(q_ptr, k_ptr, v_ptr, kv_len_ptr, n_req, max_kv_len, n_kv_heads, q_per_kv, head_dim,
                                    float(scale), out_ptr, ws_ptr, ws_bytes, stream)


def plora_attn_status(ws_ptr, stream=0):
    v = ctypes.c_int32(0)
    rc = load().plora_attn_status(ws_ptr, stream, ctypes.byref(v))
    return rc, int(v.value)


def plora_attn_set_debug(ws_ptr, cycles: int, hook: int, stream=0):
    return load().plora_attn_set_debug(ws_ptr, int(cycles), int(hook), stream)


def plora_set_wait_limit(ctx, cycles: int):
    return load().plora_set_wait_limit(ctx, int(cycles))


def plora_set_test_hook(ctx, hook: int):
    return load().plora_set_test_hook(ctx, int(hook))


def plora_set_inputs_resident(ctx, resident: bool):
    return load().plora_set_inputs_resident(ctx, 1 if resident else 0)


def plora_stream_read(buf_ptr, nbytes: int, sink_ptr, sink_bytes: int, stream=0):
    return load().plora_stream_read(buf_ptr, int(nbytes), sink_ptr, int(sink_bytes), stream)


def _new_on(stream, make, *size, **kw):
    """A tensor made on the stream that the call runs on: zeroed before the kernels read it, and its memory handed on only
    behind them."""
    if stream is None:
        return make(*size, **kw)
    with torch.cuda.stream(stream):
        return make(*size, **kw)


def attn_decode(q, k_cache, v_cache, kv_len, scale, out=None, workspace=None, stream=None):
    """Torch convenience: q bf16 [B, Hq, 128], k_cache / v_cache bf16 [B, Hkv, Lmax, 128], kv_len int32 [B] (all CUDA);
    returns (out fp32 [B, Hq, 128], workspace).  Pass the returned workspace back in to reuse it."""
    import torch
    B, Hq, d = q.shape
    Hkv, Lmax = int(k_cache.shape[1]), int(k_cache.shape[2])
    need = plora_attn_workspace_bytes(B, Lmax, Hkv, Hq // Hkv)
    if workspace is None:
        workspace = _new_on(stream, torch.zeros, need, dtype=torch.uint8, device=q.device)
    if out is None:
        out = _new_on(stream, torch.empty, (B, Hq, d), dtype=torch.float32, device=q.device)
    _check(plora_attn_decode(q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), kv_len.data_ptr(), B, Lmax, Hkv, Hq // Hkv,
                             d, scale, out.data_ptr(), workspace.data_ptr(), int(workspace.numel()), _stream_handle(stream)),
           "plora_attn_decode")
    return out, workspace


# ---- serving over a paged KV cache ------------------------------------------------------
def plora_kv_plan(kv_len_ptr, new_len_ptr, n_req, page_size, free_ptr, n_free, cursor_in_ptr, table_ptr, max_blocks, max_tokens,
                  tok_start_ptr, positions_ptr, tok_req_ptr, slots_ptr, kv_len_out_ptr, cursor_out_ptr, stream=0):
    return load().plora_kv_plan(kv_len_ptr, new_len_ptr, n_req, page_size, free_ptr, n_free, cursor_in_ptr, table_ptr, max_blocks,
                                max_tokens, tok_start_ptr, positions_ptr, tok_req_ptr, slots_ptr, kv_len_out_ptr, cursor_out_ptr,
                                stream)


def plora_rope_table(desc: RopeDesc, max_pos: int, table_ptr: int, stream=0):
    return load().plora_rope_table(ctypes.byref(desc), max_pos, table_ptr, stream)


def plora_rope_cache(args: RopeCacheArgs, stream=0):
    return load().plora_rope_cache(ctypes.byref(args), stream)


def plora_attn_paged_workspace_bytes(n_tok, n_req, n_q_heads, n_kv_heads, head_dim, page_size, max_blocks) -> int:
    return int(load().plora_attn_paged_workspace_bytes(n_tok, n_req, n_q_heads, n_kv_heads, head_dim, page_size, max_blocks))


def plora_attn_paged(args: PagedAttn, stream=0):
    return load().plora_attn_paged(ctypes.byref(args), stream)


class KvPlan(NamedTuple):
    """What kv_plan writes (int32 device tensors): tok_start [n_req + 1], positions / tok_req / slots [max_tokens],
    kv_len [n_req] and cursor [1] after the step."""
    tok_start: Any
    positions: Any
    tok_req: Any
    slots: Any
    kv_len: Any
    cursor: Any


# These calls are made once per layer or step, at a few microseconds of GPU work each, so the checks are written for
# speed: plain comparisons, the argument structures packed in one go (laid out as RopeCacheArgs and PagedAttn).
_ROPE_PACK = struct.Struct("@11i4q10P")
_PAGED_PACK = struct.Struct("@10i2q11P2f2PN")


def _bad(what: str):
    raise ValueError(what)


def _ints(name, t, shape) -> int:
    """Address of an int32 CUDA tensor, packed, of this shape."""
    if t.dtype is not torch.int32 or t.shape != shape or not t.is_cuda or not t.is_contiguous():
        _bad(f"{name}: packed int32 CUDA tensor {list(shape)} expected, got {t.dtype} {list(t.shape)} on {t.device}")
    return t.data_ptr()


def _opt_ints(name, t, shape) -> int:
    return 0 if t is None else _ints(name, t, shape)


def _type16(t) -> int:
    if t.dtype is torch.bfloat16:
        return INPUT_BF16
    if t.dtype is torch.float16:
        return INPUT_FP16
    _bad(f"bfloat16 or float16 expected, got {t.dtype}")


def _token_stride(name, t) -> int:
    """Elements between the tokens of a CUDA tensor [n_tok, heads, head_dim] whose heads are packed."""
    n, h, d = t.shape
    st, sh, sd = t.stride()
    if not t.is_cuda or (sd != 1 and d > 1) or (sh != d and h > 1):
        _bad(f"{name}: CUDA tensor [n_tok, heads, head_dim] with packed heads expected")
    if n < 2:
        return h * d
    if st == 0:      # (the C structures read 0 as packed)
        _bad(f"{name}: a tensor that is expanded along its tokens is not supported")
    return st


def _page_stride(k_cache, v_cache) -> int:
    """Elements between the pages of a cache pair [n_pages, n_kv_heads, page_size, head_dim] whose pages are packed."""
    n, h, s, d = k_cache.shape
    st = k_cache.stride()
    if (v_cache.shape != k_cache.shape or v_cache.dtype is not k_cache.dtype or v_cache.stride() != st or not k_cache.is_cuda
            or not v_cache.is_cuda or st[3] != 1 or st[2] != d or (st[1] != s * d and h > 1)):
        _bad("k_cache, v_cache: alike CUDA tensors [n_pages, n_kv_heads, page_size, head_dim] with packed pages expected")
    if n < 2:
        return h * s * d
    if st[0] == 0:   # (the C structures read 0 as packed)
        _bad("k_cache, v_cache: a cache that is expanded along its pages is not supported")
    return st[0]


def _raw_stream(stream, t) -> int:
    return torch._C._cuda_getCurrentRawStream(t.get_device()) if stream is None else stream.cuda_stream


def kv_plan(kv_len, new_len, page_size: int, free_pages, block_table, max_tokens: int, cursor=None, out=None, stream=None) -> KvPlan:
    """Pages, slots and positions of a step (plora_kv_plan): kv_len, new_len int32 [n_req], free_pages int32 [n_free],
    block_table int32 [n_req, max_blocks] (updated in place), cursor int32 [1] or None (the free list's first unused
    entry; the result's cursor is the next step's).  out: a KvPlan of an earlier step, to be overwritten."""
    n, = kv_len.shape
    one, toks = (n,), (max_tokens,)
    if out is None:
        size = 2 * n + 2 + 3 * max_tokens
        buf = (torch.empty(size, dtype=torch.int32, device=kv_len.device) if stream is None
               else _new_on(stream, torch.empty, size, dtype=torch.int32, device=kv_len.device))
        out = KvPlan(*buf.split_with_sizes((n + 1, max_tokens, max_tokens, max_tokens, n, 1)))
        at = buf.data_ptr()
        ptrs = (at, at + 4 * (n + 1), at + 4 * (n + 1 + max_tokens), at + 4 * (n + 1 + 2 * max_tokens),
                at + 4 * (n + 1 + 3 * max_tokens), at + 4 * (2 * n + 1 + 3 * max_tokens))
    else:
        ptrs = (_ints("tok_start", out.tok_start, (n + 1,)), _ints("positions", out.positions, toks),
                _ints("tok_req", out.tok_req, toks), _ints("slots", out.slots, toks), _ints("kv_len", out.kv_len, one),
                _ints("cursor", out.cursor, (1,)))
    n_free, = free_pages.shape
    width = block_table.shape[-1]
    rc = load().plora_kv_plan(_ints("kv_len", kv_len, one), _ints("new_len", new_len, one), n, page_size,
                              _ints("free_pages", free_pages, (n_free,)), n_free, _opt_ints("cursor", cursor, (1,)),
                              _ints("block_table", block_table, (n, width)), width, max_tokens, *ptrs, _raw_stream(stream, kv_len))
    if rc != OK:
        raise PloraError(rc, "plora_kv_plan")
    return out


_SCALINGS = {"none": ROPE_NONE, "linear": ROPE_LINEAR, "ntk": ROPE_NTK, "bands": ROPE_BANDS, "ramp": ROPE_RAMP}


def rope_table(rot_dim: int, max_pos: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
               orig_len: float = 0.0, low: float | None = None, high: float | None = None, magnitude: float = 1.0, device="cuda",
               stream=None):
    """The fp32 table [max_pos, rot_dim // 2, 2] of cosines and sines (plora_rope_table).  low and high, the turns over orig_len
    between which "bands" and "ramp" change over: 1 and 4 for bands, 1 and 32 for a ramp unless given."""
    if scaling not in _SCALINGS:
        _bad(f"scaling: one of {sorted(_SCALINGS)} expected, got {scaling!r}")
    table = _new_on(stream, torch.empty, (max(0, int(max_pos)), int(rot_dim) // 2, 2), dtype=torch.float32, device=device)
    low = 1.0 if low is None else low
    high = (32.0 if scaling == "ramp" else 4.0) if high is None else high
    d = RopeDesc(int(rot_dim), _SCALINGS[scaling], base, factor, orig_len, low, high, magnitude)
    _check(plora_rope_table(d, int(max_pos), table.data_ptr(), _raw_stream(stream, table)), "plora_rope_table")
    return table


def rope_cache(q, k, v, positions, slots, table, k_cache, v_cache, q_out=None, interleaved: bool = False, status=None, stream=None):
    """Rotates q and k, writes k and v to their cache slots and returns the rotated q (plora_rope_cache).  q, k, v:
    [n_tok, heads, head_dim], fp32 or the cache's type, rows of any stride; table: rope_table's (None: nothing turns)."""
    n, hq, d = q.shape
    hk = k.shape[1]
    out_type = _type16(k_cache)
    page_stride = _page_stride(k_cache, v_cache)
    n_pages, ch, page, cd = k_cache.shape
    if q.dtype is torch.float32:
        in_type = INPUT_FP32
    elif q.dtype is k_cache.dtype:
        in_type = out_type
    else:
        _bad("q, k, v: float32 or the cache's type expected")
    if k.dtype is not q.dtype or v.dtype is not q.dtype:
        _bad("q, k, v: one type expected")
    if k.shape != (n, hk, d) or v.shape != (n, hk, d) or ch != hk or cd != d:
        _bad("q, k, v and the caches: shapes do not agree")
    if q_out is None:
        q_out = (torch.empty((n, hq, d), dtype=k_cache.dtype, device=q.device) if stream is None
                 else _new_on(stream, torch.empty, (n, hq, d), dtype=k_cache.dtype, device=q.device))
    elif q_out.dtype is not k_cache.dtype or q_out.shape != (n, hq, d) or not q_out.is_cuda or not q_out.is_contiguous():
        _bad("q_out: packed, of the cache's type and q's shape, expected")
    rot = max_pos = at = 0
    if table is not None:
        max_pos, half, two = table.shape
        if two != 2 or table.dtype is not torch.float32 or not table.is_cuda or not table.is_contiguous():
            _bad("table: float32 [max_pos, rot_dim // 2, 2] expected")
        rot, at = 2 * half, table.data_ptr()
    a = _ROPE_PACK.pack(in_type, out_type, ROPE_INTERLEAVED if interleaved else ROPE_HALF, n, hq, hk, d, rot, max_pos, page, n_pages,
                        _token_stride("q", q), _token_stride("k", k), _token_stride("v", v), page_stride, q.data_ptr(), k.data_ptr(),
                        v.data_ptr(), _ints("positions", positions, (n,)), _ints("slots", slots, (n,)), at, q_out.data_ptr(),
                        k_cache.data_ptr(), v_cache.data_ptr(), _opt_ints("status", status, (1,)))
    rc = load().plora_rope_cache(a, _raw_stream(stream, q))
    if rc != OK:
        raise PloraError(rc, "plora_rope_cache")
    return q_out


def attn_paged_workspace(q, k_cache, n_req: int, max_blocks=None):
    """A workspace for attn_paged on batches of q's size over this cache (max_blocks: the block table's width, None: any),
    zeroed on the current stream."""
    n_pages, hk, page, d = k_cache.shape
    need = plora_attn_paged_workspace_bytes(max(1, q.shape[0]), max(1, int(n_req)), q.shape[1], hk, d, page,
                                            n_pages if max_blocks is None else min(n_pages, int(max_blocks)))
    if need == 0:
        raise PloraError(ERR_UNSUPPORTED, "plora_attn_paged_workspace_bytes")
    return torch.zeros(need, dtype=torch.uint8, device=q.device)


def attn_paged(q, k_cache, v_cache, block_table, kv_len, scale: float, tok_start=None, group_start=None, prefix_len=None,
               softcap: float = 0.0, slopes=None, key_lo=None, key_hi=None, out=None, workspace=None, stream=None):
    """Attention of the new tokens q [n_tok, n_q_heads, head_dim] over the paged cache (plora_attn_paged); returns
    (out, workspace).  tok_start None: one token per request.  Pass the returned workspace back in to reuse it."""
    n, hq, d = q.shape
    n_pages, hk, page, cd = k_cache.shape
    n_req, = kv_len.shape
    width = block_table.shape[-1]
    page_stride = _page_stride(k_cache, v_cache)
    if q.dtype is not k_cache.dtype or cd != d or hk == 0 or hq % hk != 0:
        _bad("q and the caches do not agree")
    if out is None:
        out = (torch.empty((n, hq, d), dtype=q.dtype, device=q.device) if stream is None
               else _new_on(stream, torch.empty, (n, hq, d), dtype=q.dtype, device=q.device))
    elif out.dtype is not q.dtype or out.shape != (n, hq, d) or not out.is_cuda or not out.is_contiguous():
        _bad("out: packed, of q's shape and type, expected")
    if workspace is None:
        workspace = _new_on(stream, attn_paged_workspace, q, k_cache, n_req, width)
    elif workspace.dtype is not torch.uint8 or not workspace.is_cuda or not workspace.is_contiguous():
        _bad("workspace: packed uint8 CUDA tensor expected")
    if (group_start is None) != (prefix_len is None):
        _bad("group_start and prefix_len go together")
    n_groups = 0 if prefix_len is None else prefix_len.shape[0]
    if slopes is not None and (slopes.dtype is not torch.float32 or not slopes.is_cuda or slopes.shape != (hq,)
                               or not slopes.is_contiguous()):
        _bad("slopes: packed float32 CUDA tensor [n_q_heads] expected")
    a = _PAGED_PACK.pack(_type16(q), n, n_req, n_groups, hq, hk, d, page, n_pages, width, _token_stride("q", q), page_stride,
                         q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), _ints("block_table", block_table, (n_req, width)),
                         _ints("kv_len", kv_len, (n_req,)), _opt_ints("tok_start", tok_start, (n_req + 1,)),
                         _opt_ints("group_start", group_start, (n_groups + 1,)), _opt_ints("prefix_len", prefix_len, (n_groups,)),
                         _opt_ints("key_lo", key_lo, (n,)), _opt_ints("key_hi", key_hi, (n,)),
                         0 if slopes is None else slopes.data_ptr(), scale, softcap, out.data_ptr(), workspace.data_ptr(),
                         workspace.numel())
    rc = load().plora_attn_paged(a, _raw_stream(stream, q))
    if rc != OK:
        raise PloraError(rc, "plora_attn_paged")
    return out, workspace


# ---- a layer's base projections in 8 bits -------------------------------------------------
def plora_rms_norm(args: RmsNormArgs, stream=0):
    return load().plora_rms_norm(ctypes.byref(args), stream)


def plora_gated_act(args: GatedActArgs, stream=0):
    return load().plora_gated_act(ctypes.byref(args), stream)


def plora_quant_weight(w_ptr, type_, n, k, w_stride, q_ptr, q_stride, scale_ptr, stream=0):
    return load().plora_quant_weight(w_ptr, type_, n, k, w_stride, q_ptr, q_stride, scale_ptr, stream)


def plora_gemm_fp8(args: GemmFp8Args, stream=0):
    return load().plora_gemm_fp8(ctypes.byref(args), stream)


def plora_gemm_fp8_status(stream=0):
    v = ctypes.c_int32(0)
    rc = load().plora_gemm_fp8_status(stream, ctypes.byref(v))
    return rc, int(v.value)


class Act8(NamedTuple):
    """What rms_norm and gated_act write: y [n, d] in 16 bits, q [n, d] e4m3 with scale [n, ceil(d / 128)], the residual sum (each
    None where it was not asked for)."""
    y: Any
    q: Any
    scale: Any
    residual: Any = None


# (packed as RmsNormArgs, GatedActArgs and GemmFp8Args are laid out)
_NORM_PACK = struct.Struct("@6i5q7P2f")
_ACT_PACK = struct.Struct("@5i4x4q5P")
_GEMM_PACK = struct.Struct("@8i9q15Pq2i")


_kinds = {}       # type codes by torch type, filled when the torch layer is first used


def _type_of(name, t) -> int:
    kind = _kinds.get(t.dtype)
    if kind is None:
        if not _kinds:
            _kinds.update({torch.bfloat16: INPUT_BF16, torch.float16: INPUT_FP16, torch.float32: INPUT_FP32})
            return _type_of(name, t)
        _bad(f"{name}: float32, bfloat16 or float16 expected, got {t.dtype}")
    return kind


# (The calls look at the usual layout in place, one line per tensor, and leave what is not usual to these helpers, which refuse what has
# to be refused: a helper call per tensor cost 0.6 us of the 8 that a small norm takes.)
def _rows(name, t, n: int, d: int, dev: int) -> int:
    """Elements between the rows of a CUDA tensor [n, d] whose rows are packed (dev: the inputs' device, at least 0)."""
    if t.shape != (n, d) or t.get_device() != dev:
        _bad(f"{name}: CUDA tensor [{n}, {d}] on the inputs' device expected, got {list(t.shape)} on {t.device}")
    st, one = t.stride()
    if one != 1 and d > 1:
        _bad(f"{name}: packed rows expected")
    if st < d:       # (the C structures read 0 as packed; rows that overlap are not rows)
        if n > 1:
            _bad(f"{name}: a tensor that is expanded along its rows is not supported")
        return d
    return st


def _q_rows(name, q, n: int, d: int, dev: int) -> int:
    """Bytes between the rows of an e4m3 CUDA tensor [n, d]."""
    if q.dtype is not torch.float8_e4m3fn:
        _bad(f"{name}: float8_e4m3fn expected, got {q.dtype}")
    st = _rows(name, q, n, d, dev)
    if st % 16:
        if n > 1:
            _bad(f"{name}: rows have to lie a multiple of 16 bytes apart")
        return -(-d // 16) * 16
    return st


def _scales(name, t, rows: int, cols: int, dev: int) -> int:
    if t.dtype is not torch.float32 or t.shape != (rows, cols) or not t.is_contiguous() or t.get_device() != dev:
        _bad(f"{name}: packed float32 CUDA tensor {[rows, cols]} on the inputs' device expected, got {t.dtype} {list(t.shape)} on {t.device}")
    return t.data_ptr()


def _device_of(name, t) -> int:
    dev = t.get_device()
    if dev < 0:
        _bad(f"{name}: CUDA tensor expected, got one on {t.device}")
    return dev


def _q_empty(stream, n: int, d: int, device):
    """An 8-bit matrix's buffers: rows a multiple of 16 bytes apart."""
    width = -(-d // 16) * 16
    q = _new_on(stream, torch.empty, (n, width), dtype=torch.float8_e4m3fn, device=device)
    scale = _new_on(stream, torch.empty, (n, -(-d // 128)), dtype=torch.float32, device=device)
    return (q if width == d else q[:, :d]), scale


def _call_on(name: str, dev: int, args, stream):
    """Makes the call with the inputs' device as the current one."""
    fn = getattr(_lib or load(), name)
    if dev == torch._C._cuda_getDevice():
        rc = fn(args, torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream)
    else:
        with torch.cuda.device(dev):
            rc = fn(args, torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream)
    if rc != OK:
        raise PloraError(rc, name)


def _output_type(name, kind) -> int:
    if kind == INPUT_FP32:
        _bad(f"{name}: bfloat16 or float16 expected")
    return kind


def rms_norm(x, weight=None, eps: float = 1e-5, residual=None, residual_out=None, offset: float = 0.0, out_type=None, fp8: bool = False,
             y=None, q=None, scale=None, stream=None) -> Act8:
    """Root-mean-square norm of the rows of x [n, d] (plora_rms_norm), x + residual first if there is a residual: the sum goes to
    residual_out (None: to residual itself).  x is fp32, or of the 16-bit type; weight [d] of either.
    Outputs: y in 16 bits (out_type=torch.bfloat16 / float16, or a buffer) and an 8-bit matrix (fp8=True, or buffers q and scale)."""
    shape = x.shape
    n, d = shape
    dev = _device_of("x", x)
    in_type = kind = _type_of("x", x)
    if y is None and out_type is not None:
        y = _new_on(stream, torch.empty, (n, d), dtype=out_type, device=x.device)
    if fp8 and q is None and scale is None:
        q, scale = _q_empty(stream, n, d, x.device)
    xs, one = x.stride()
    if one != 1 or xs < d:
        xs = _rows("x", x, n, d, dev)
    wt = rt = -1
    w_at = rs = ros = r_at = ro_at = ys = y_at = qs = q_at = s_at = 0
    if y is not None:
        kind = _output_type("y", _type_of("y", y))
        ys, one = y.stride()
        if y.shape != shape or one != 1 or ys < d or y.get_device() != dev:
            ys = _rows("y", y, n, d, dev)
        y_at = y.data_ptr()
    if weight is not None:
        wt = _type_of("weight", weight)
        if weight.shape != (d,) or not weight.is_contiguous() or weight.get_device() != dev:
            _bad(f"weight: packed CUDA tensor [{d}] on x's device expected")
        w_at = weight.data_ptr()
    if residual is not None:
        rt = _type_of("residual", residual)
        rs, one = residual.stride()
        if residual.shape != shape or one != 1 or rs < d or residual.get_device() != dev:
            rs = _rows("residual", residual, n, d, dev)
        r_at = residual.data_ptr()
        if residual_out is None:
            residual_out, ros, ro_at = residual, rs, r_at
        else:
            if residual_out.dtype is not residual.dtype:
                _bad("residual_out: residual's type expected")
            ros, one = residual_out.stride()
            if residual_out.shape != shape or one != 1 or ros < d or residual_out.get_device() != dev:
                ros = _rows("residual_out", residual_out, n, d, dev)
            ro_at = residual_out.data_ptr()
    elif residual_out is not None:
        _bad("residual_out without a residual")
    if q is not None and scale is not None:
        qs, one = q.stride()
        if q.shape != shape or one != 1 or qs < d or qs % 16 or q.dtype is not torch.float8_e4m3fn or q.get_device() != dev:
            qs = _q_rows("q", q, n, d, dev)
        q_at, s_at = q.data_ptr(), _scales("scale", scale, n, (d + 127) // 128, dev)
    elif q is not None or scale is not None:
        _bad("q and scale go together")
    elif y is None and residual is None:
        _bad("nothing to write: neither y, q nor a residual")
    # one 16-bit type: y's, or that of whichever of the others is not fp32 (bf16 where all are)
    for t in (in_type, wt, rt):
        if t >= 0 and t != INPUT_FP32 and t != kind:
            if kind != INPUT_FP32:
                _bad("x, weight, residual, y: float32 or one 16-bit type expected")
            kind = t
    if kind == INPUT_FP32:
        kind = INPUT_BF16
    _call_on("plora_rms_norm", dev, _NORM_PACK.pack(in_type, kind, kind if wt < 0 else wt, kind if rt < 0 else rt, n, d, xs, rs, ros, ys, qs,
                                                    x.data_ptr(), w_at, r_at, ro_at, y_at, q_at, s_at, eps, offset), stream)
    return Act8(y, q, scale, residual_out)


_ACTS = {"none": ACT_NONE, "silu": ACT_SILU, "gelu": ACT_GELU}


def gated_act(gate, up=None, act: str = "silu", out_type=None, fp8: bool = False, y=None, q=None, scale=None, stream=None) -> Act8:
    """act(gate) * up, or act(gate), for gate and up [n, d] (plora_gated_act); outputs as of rms_norm.  act: "silu", "gelu" (tanh form) or
    "none": with up=None the 8-bit form of a matrix."""
    code = _ACTS.get(act)
    if code is None:
        _bad(f"act: one of {sorted(_ACTS)} expected, got {act!r}")
    shape = gate.shape
    n, d = shape
    dev = _device_of("gate", gate)
    in_type = kind = _type_of("gate", gate)
    if y is None and out_type is not None:
        y = _new_on(stream, torch.empty, (n, d), dtype=out_type, device=gate.device)
    if fp8 and q is None and scale is None:
        q, scale = _q_empty(stream, n, d, gate.device)
    gs, one = gate.stride()
    if one != 1 or gs < d:
        gs = _rows("gate", gate, n, d, dev)
    us = u_at = ys = y_at = qs = q_at = s_at = 0
    if up is not None:
        if up.dtype is not gate.dtype:
            _bad("gate and up: one type expected")
        us, one = up.stride()
        if up.shape != shape or one != 1 or us < d or up.get_device() != dev:
            us = _rows("up", up, n, d, dev)
        u_at = up.data_ptr()
    if y is not None:
        kind = _output_type("y", _type_of("y", y))
        if in_type != INPUT_FP32 and in_type != kind:
            _bad("gate, up, y: float32 or one 16-bit type expected")
        ys, one = y.stride()
        if y.shape != shape or one != 1 or ys < d or y.get_device() != dev:
            ys = _rows("y", y, n, d, dev)
        y_at = y.data_ptr()
    if q is not None and scale is not None:
        qs, one = q.stride()
        if q.shape != shape or one != 1 or qs < d or qs % 16 or q.dtype is not torch.float8_e4m3fn or q.get_device() != dev:
            qs = _q_rows("q", q, n, d, dev)
        q_at, s_at = q.data_ptr(), _scales("scale", scale, n, (d + 127) // 128, dev)
    elif q is not None or scale is not None:
        _bad("q and scale go together")
    elif y is None:
        _bad("nothing to write: neither y nor q")
    if kind == INPUT_FP32:
        kind = INPUT_BF16
    _call_on("plora_gated_act", dev, _ACT_PACK.pack(in_type, kind, code, n, d, gs, us, ys, qs, gate.data_ptr(),
                                                    u_at, y_at, q_at, s_at), stream)
    return Act8(y, q, scale)


def quant_weight(w, stream=None):
    """A weight [n, k] (n: outputs, k: inputs) as an 8-bit matrix (q [n, k] e4m3, scale [ceil(n / 128), ceil(k / 128)]): a set-up call
    (plora_quant_weight)."""
    n, k = w.shape
    dev = _device_of("w", w)
    kind, st = _type_of("w", w), _rows("w", w, n, k, dev)
    width = -(-k // 16) * 16
    q = _new_on(stream, torch.empty, (n, width), dtype=torch.float8_e4m3fn, device=w.device)[:, :k]
    scale = _new_on(stream, torch.empty, (-(-n // 128), -(-k // 128)), dtype=torch.float32, device=w.device)
    with torch.cuda.device(dev):
        _check(plora_quant_weight(w.data_ptr(), kind, n, k, st, q.data_ptr(), width, scale.data_ptr(), _raw_stream(stream, w)),
               "plora_quant_weight")
    return q, scale


def gemm_fp8(x, x_scale, w, w_scale, out_type=None, out=None, status=None, stream=None, weights_ready: bool = False,
             wait_cycles: int = 0):
    """x w^T for an 8-bit matrix x [m, k] with x_scale and an 8-bit weight w [n, k] with w_scale, or up to four of them (lists) that
    share x, in one launch (plora_gemm_fp8).  Returns [m, n] (a list of them for lists): fp32, or out_type, or the buffers `out`.
    weights_ready: the caller's word that the weights were complete before the kernel in front of this call on the stream began (laid out
    once, and waited for since); their first copies then start while that kernel drains.
    wait_cycles: limit of the kernel's waits in SM clock cycles, 0: about two seconds.  A wait that ran out leaves ERR_TIMEOUT in status
    (int32 [1]), or without one in the word that gemm_fp8_status reads."""
    many = isinstance(w, (list, tuple))
    ws, scales = (w, w_scale) if many else ((w,), (w_scale,))
    count = len(ws)
    if count < 1 or count > 4 or len(scales) != count:
        _bad("w, w_scale: one to four weights, each with its scales, expected")
    m, k = x.shape
    dev = _device_of("x", x)
    blocks = (k + 127) // 128
    if out is None:
        kind = out_type or torch.float32
        outs = [_new_on(stream, torch.empty, (m, t.shape[0]), dtype=kind, device=x.device) for t in ws]
    else:
        outs = out if many else (out,)
        if len(outs) != count:
            _bad("out: a buffer for each weight expected")
    ns, strides, out_strides, at, s_at, o_at = [0] * 4, [0] * 4, [0] * 4, [0] * 4, [0] * 4, [0] * 4
    kind, f8 = outs[0].dtype, torch.float8_e4m3fn
    for i, (t, s, o) in enumerate(zip(ws, scales, outs)):
        n, tk = t.shape
        if o.dtype is not kind:
            _bad("out: one type expected")
        st, one = t.stride()
        if tk != k or one != 1 or st < k or st % 16 or t.dtype is not f8 or t.get_device() != dev:
            st = _q_rows("w", t, n, k, dev)
        ost, one = o.stride()
        if o.shape != (m, n) or one != 1 or ost < n or o.get_device() != dev:
            ost = _rows("out", o, m, n, dev)
        ns[i], strides[i], out_strides[i] = n, st, ost
        at[i], s_at[i], o_at[i] = t.data_ptr(), _scales("w_scale", s, (n + 127) // 128, blocks, dev), o.data_ptr()
    xs, one = x.stride()
    if one != 1 or xs < k or xs % 16 or x.dtype is not f8:
        xs = _q_rows("x", x, m, k, dev)
    status_at = 0
    if status is not None:
        status_at = _ints("status", status, (1,))
        if status.get_device() != dev:
            _bad("status: on the inputs' device expected")
    _call_on("plora_gemm_fp8", dev, _GEMM_PACK.pack(_type_of("out", outs[0]), m, k, count, *ns, xs, *strides, *out_strides, x.data_ptr(),
                                                    _scales("x_scale", x_scale, m, blocks, dev), *at, *s_at, *o_at, status_at, wait_cycles,
                                                      1 if weights_ready else 0, HOOK_NONE), stream)
    return list(outs) if many else outs[0]


def gemm_fp8_status(device=None, stream=None) -> int:
    """The sticky status of the gemm_fp8 calls that were given no status word, on `device` (None: the current one); waits for the stream
    and clears the word (plora_gemm_fp8_status)."""
    with torch.cuda.device(device):
        rc, status = plora_gemm_fp8_status(torch.cuda.current_stream().cuda_stream if stream is None else stream.cuda_stream)
    _check(rc, "plora_gemm_fp8_status")
    return status


def plora_pool_slab_bytes(desc: PoolDesc) -> int:
    return int(load().plora_pool_slab_bytes(ctypes.byref(desc)))


def plora_register_pool(ctx, desc: PoolDesc, slab_ptr: int, slab_bytes: int, stream: int = 0):
    return load().plora_register_pool(ctx, ctypes.byref(desc), slab_ptr, slab_bytes, stream)


def plora_pool_max_rank(ctx, layer: int, proj: int) -> int:
    return load().plora_pool_max_rank(ctx, layer, proj)


def plora_bucket(ctx, ids_ptr: int, n_tok: int, n_adapters: int, stream: int = 0):
    return load().plora_bucket(ctx, ids_ptr, n_tok, n_adapters, stream)


def plora_bucket_view(ctx):
    ptrs = [ctypes.c_void_p() for _ in range(5)]
    rc = load().plora_bucket_view(ctx, *[ctypes.byref(p) for p in ptrs])
    return rc, tuple(p.value for p in ptrs)


def plora_lora_delta(ctx, x_ptr: int, ids_ptr: int, n_tok: int, layer: int, proj: int, y_ptr: int, stream: int = 0):
    return load().plora_lora_delta(ctx, x_ptr, ids_ptr, n_tok, layer, proj, y_ptr, stream)


def plora_lora_delta_group(ctx, x_ptrs, ids_ptr, n_tok, layers, projs, y_ptrs, stream=0):
    """x_ptrs / y_ptrs: sequences of device pointers; layers / projs: sequences of ints (all of length n)."""
    n = len(x_ptrs)
    xs = (ctypes.c_void_p * n)(*x_ptrs)
    ys = (ctypes.c_void_p * n)(*y_ptrs)
    ls = (ctypes.c_int32 * n)(*layers)
    ps = (ctypes.c_int32 * n)(*projs)
    return load().plora_lora_delta_group(ctx, n, ctypes.cast(xs, ctypes.c_void_p), ids_ptr, n_tok,
                                         ctypes.cast(ls, ctypes.c_void_p), ctypes.cast(ps, ctypes.c_void_p),
                                         ctypes.cast(ys, ctypes.c_void_p), stream)


def plora_shrink(ctx, x_ptr, ids_ptr, n_tok, layer, proj, m_ptr, ldm, stream=0):
    return load().plora_shrink(ctx, x_ptr, ids_ptr, n_tok, layer, proj, m_ptr, ldm, stream)


def plora_expand(ctx, m_ptr, ldm, ids_ptr, n_tok, layer, proj, y_ptr, stream=0):
    return load().plora_expand(ctx, m_ptr, ldm, ids_ptr, n_tok, layer, proj, y_ptr, stream)


def plora_shrink_m16(ctx, x_ptr, ids_ptr, n_tok, layer, proj, m_ptr, ldm, stream=0):
    return load().plora_shrink_m16(ctx, x_ptr, ids_ptr, n_tok, layer, proj, m_ptr, ldm, stream)


def plora_expand_m16(ctx, m_ptr, ldm, ids_ptr, n_tok, layer, proj, y_ptr, stream=0):
    return load().plora_expand_m16(ctx, m_ptr, ldm, ids_ptr, n_tok, layer, proj, y_ptr, stream)


def plora_lora_delta_host(ctx, x_host_ptr, ids_host_ptr, n_tok, layer, proj, y_host_ptr, stream=0):
    return load().plora_lora_delta_host(ctx, x_host_ptr, ids_host_ptr, n_tok, layer, proj, y_host_ptr, stream)


def plora_lora_delta_host_async(ctx, x_host_ptr, ids_host_ptr, n_tok, layers, projs, y_host_ptrs, stream=0):
    n = len(layers)
    la = (ctypes.c_int32 * n)(*layers)
    pa = (ctypes.c_int32 * n)(*projs)
    ya = (ctypes.c_void_p * n)(*y_host_ptrs)
    return load().plora_lora_delta_host_async(ctx, n, x_host_ptr, ids_host_ptr, n_tok, la, pa, ya, stream)


def plora_host_sync(ctx):
    return load().plora_host_sync(ctx)


def plora_lora_delta_noalloc(ctx, x_ptr, ids_ptr, n_tok, layer, proj, y_ptr, stream=0):
    return load().plora_lora_delta_noalloc(ctx, x_ptr, ids_ptr, n_tok, layer, proj, y_ptr, stream)


def plora_set_path(ctx, path: int, sgmv_min_rows: int = 0):
    return load().plora_set_path(ctx, path, sgmv_min_rows)


def plora_device_status(ctx, stream: int = 0):
    v = ctypes.c_int32(0)
    rc = load().plora_device_status(ctx, stream, ctypes.byref(v))
    return rc, int(v.value)


def plora_launch_count(ctx) -> int:
    return int(load().plora_launch_count(ctx))


# ---- torch-facing convenience layer -------------------------------------------------------
class _DevArray:
    """Exposes a raw device pointer to torch through the CUDA array interface."""

    def __init__(self, ptr: int, n: int, typestr: str = "<i4"):
        self.__cuda_array_interface__ = {"shape": (n,), "typestr": typestr, "data": (ptr, False), "version": 2}


def _stream_handle(stream) -> int:
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream)


def _check(rc: int, where: str):
    if rc != OK:
        raise PloraError(rc, where)


def _data_ptr(t) -> int:
    if isinstance(t, np.ndarray):
        return int(t.ctypes.data)
    return int(t.data_ptr())


class Context:
    """One library context (one device, one stream at a time)."""

    def __init__(self, max_tokens: int, max_adapters: int, device: int = 0):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("no CUDA device: this library has no CPU path")
        rc, h = plora_create(device, max_tokens, max_adapters)
        _check(rc, "plora_create")
        self._h = h
        self.device = device
        self.max_tokens, self.max_adapters = max_tokens, max_adapters
        self._slabs = {}
        self._n_tok = 0
        self._n_adapters = 0

    def close(self):
        if getattr(self, "_h", None):
            plora_destroy(self._h)
            self._h = None
            self._slabs.clear()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def handle(self):
        return self._h

    def register_pool(self, layer, proj, d_in, d_out, ranks, scales, A, B, stream=None):
        """A, B: per-adapter lists of bf16 matrices [d_in, r_a] / [r_a, d_out]: torch tensors
        (all on the device, or all on the host) or numpy uint16 bit patterns.  Returns the slab tensor."""
        import torch
        n = len(A)
        ranks = np.ascontiguousarray(ranks, dtype=np.int32)
        scales = np.ascontiguousarray(scales, dtype=np.float32)
        assert len(B) == n and ranks.shape == (n,) and scales.shape == (n,)
        on_dev = bool(n) and (not isinstance(A[0], np.ndarray)) and A[0].is_cuda
        keep = []
        pa = (ctypes.c_void_p * n)()
        pb = (ctypes.c_void_p * n)()
        for a in range(n):
            ma, mb = A[a], B[a]
            if isinstance(ma, np.ndarray):
                ma = np.ascontiguousarray(ma, dtype=np.uint16)
                mb = np.ascontiguousarray(mb, dtype=np.uint16)
            else:
                assert ma.is_cuda == on_dev and mb.is_cuda == on_dev and ma.dtype in (torch.bfloat16, torch.float16)
                ma, mb = ma.contiguous(), mb.contiguous()
            assert tuple(ma.shape) == (d_in, int(ranks[a])), (a, tuple(ma.shape))
            assert tuple(mb.shape) == (int(ranks[a]), d_out), (a, tuple(mb.shape))
            keep += [ma, mb]
            pa[a], pb[a] = _data_ptr(ma), _data_ptr(mb)
        desc = PoolDesc(layer, proj, d_in, d_out, n, 1 if on_dev else 0, ranks.ctypes.data, scales.ctypes.data,
                        ctypes.cast(pa, ctypes.c_void_p).value, ctypes.cast(pb, ctypes.c_void_p).value)
        nbytes = plora_pool_slab_bytes(desc)
        if nbytes == 0:
            raise PloraError(ERR_UNSUPPORTED, "plora_pool_slab_bytes")
        slab = torch.empty(nbytes, dtype=torch.uint8, device=f"cuda:{self.device}")
        assert slab.data_ptr() % 256 == 0
        _check(plora_register_pool(self._h, desc, slab.data_ptr(), nbytes, _stream_handle(stream)), "plora_register_pool")
        del keep
        self._slabs[(layer, proj)] = slab
        return slab

    def pool_max_rank(self, layer, proj) -> int:
        r = plora_pool_max_rank(self._h, layer, proj)
        if r < 0:
            raise PloraError(r, "plora_pool_max_rank")
        return r

    def bucket(self, ids, n_adapters: int, stream=None):
        self._n_tok, self._n_adapters = int(ids.numel()), int(n_adapters)
        _check(plora_bucket(self._h, ids.data_ptr(), self._n_tok, n_adapters, _stream_handle(stream)), "plora_bucket")

    def bucket_view(self):
        """Host copies of the current bucket: dict(perm, seg_adapter, seg_start, n_seg, n_active)."""
        import torch
        rc, (perm, seg_adapter, seg_start, n_seg, n_active) = plora_bucket_view(self._h)
        _check(rc, "plora_bucket_view")
        torch.cuda.synchronize()
        cap = min(self._n_tok, self._n_adapters)
        dev = f"cuda:{self.device}"

        def grab(ptr, n):
            if n == 0:
                return np.zeros(0, np.int32)
            return torch.as_tensor(_DevArray(ptr, n), device=dev).cpu().numpy().copy()

        return dict(perm=grab(perm, self._n_tok), seg_adapter=grab(seg_adapter, cap), seg_start=grab(seg_start, cap + 1),
                    n_seg=int(grab(n_seg, 1)[0]), n_active=int(grab(n_active, 1)[0]))

    def lora_delta(self, x, ids, layer, proj, y, stream=None):
        _check(plora_lora_delta(self._h, x.data_ptr(), ids.data_ptr(), int(ids.numel()), layer, proj, y.data_ptr(),
                                _stream_handle(stream)), "plora_lora_delta")

    def lora_delta_group(self, xs, ids, layers, projs, ys, stream=None):
        """Independent projections (q/k/v of a layer, up/gate) in one call; same-shape pools share a launch."""
        _check(plora_lora_delta_group(self._h, [t.data_ptr() for t in xs], ids.data_ptr(), int(ids.numel()),
                                      list(layers), list(projs), [t.data_ptr() for t in ys], _stream_handle(stream)),
               "plora_lora_delta_group")

    def shrink(self, x, ids, layer, proj, m, stream=None):
        _check(plora_shrink(self._h, x.data_ptr(), ids.data_ptr(), int(ids.numel()), layer, proj, m.data_ptr(),
                            int(m.shape[1]), _stream_handle(stream)), "plora_shrink")

    def expand(self, m, ids, layer, proj, y, stream=None):
        _check(plora_expand(self._h, m.data_ptr(), int(m.shape[1]), ids.data_ptr(), int(ids.numel()), layer, proj,
                            y.data_ptr(), _stream_handle(stream)), "plora_expand")

    def shrink_m16(self, x, ids, layer, proj, m_bf16, stream=None):
        _check(plora_shrink_m16(self._h, x.data_ptr(), ids.data_ptr(), int(ids.numel()), layer, proj, m_bf16.data_ptr(),
                                int(m_bf16.shape[1]), _stream_handle(stream)), "plora_shrink_m16")

    def expand_m16(self, m_bf16, ids, layer, proj, y, stream=None):
        _check(plora_expand_m16(self._h, m_bf16.data_ptr(), int(m_bf16.shape[1]), ids.data_ptr(), int(ids.numel()), layer,
                                proj, y.data_ptr(), _stream_handle(stream)), "plora_expand_m16")

    def lora_delta_host(self, x_host, ids_host, layer, proj, y_host, stream=None):
        """x_host / ids_host / y_host: CPU torch tensors (pinned or not) or numpy arrays; y_host is updated in place."""
        n_tok = int(ids_host.shape[0])
        _check(plora_lora_delta_host(self._h, _data_ptr(x_host), _data_ptr(ids_host), n_tok, layer, proj,
                                     _data_ptr(y_host), _stream_handle(stream)), "plora_lora_delta_host")

    def lora_delta_host_async(self, x_host, ids_host, layers, projs, ys_host, stream=None):
        """Queues y_host[g] += delta of pool (layers[g], projs[g]) for projections that share x_host;
        the results are in host memory after host_sync().  The host tensors must stay alive and
        untouched until then."""
        n_tok = int(ids_host.shape[0])
        _check(plora_lora_delta_host_async(self._h, _data_ptr(x_host), _data_ptr(ids_host), n_tok, list(layers), list(projs),
                                           [_data_ptr(y) for y in ys_host], _stream_handle(stream)),
               "plora_lora_delta_host_async")

    def host_sync(self):
        _check(plora_host_sync(self._h), "plora_host_sync")

    def lora_delta_noalloc(self, x, ids, layer, proj, y, stream=None):
        """The delta for callers that must not allocate: same result as lora_delta, with the
        intermediate m in the library's fixed scratch array (see plora_lora_delta_noalloc)."""
        _check(plora_lora_delta_noalloc(self._h, x.data_ptr(), ids.data_ptr(), int(ids.numel()), layer, proj,
                                        y.data_ptr(), _stream_handle(stream)), "plora_lora_delta_noalloc")

    def set_path(self, path: int, sgmv_min_rows: int = 0):
        _check(plora_set_path(self._h, path, sgmv_min_rows), "plora_set_path")

    def set_wait_limit(self, cycles: int):
        _check(plora_set_wait_limit(self._h, cycles), "plora_set_wait_limit")

    def set_test_hook(self, hook: int):
        _check(plora_set_test_hook(self._h, hook), "plora_set_test_hook")

    def set_inputs_resident(self, resident: bool):
        _check(plora_set_inputs_resident(self._h, resident), "plora_set_inputs_resident")

    def set_input_type(self, fp16: bool):
        _check(load().plora_set_input_type(self._h, 1 if fp16 else 0), "plora_set_input_type")

    def device_status(self, stream=None) -> int:
        rc, v = plora_device_status(self._h, _stream_handle(stream))
        _check(rc, "plora_device_status")
        return v

    def launch_count(self) -> int:
        return plora_launch_count(self._h)
