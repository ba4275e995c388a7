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
)

INPUT_BF16, INPUT_FP16, INPUT_FP32 = 0, 1, 2
ROPE_HALF, ROPE_INTERLEAVED = 0, 1
ROPE_NONE, ROPE_LINEAR, ROPE_NTK, ROPE_BANDS, ROPE_RAMP = 0, 1, 2, 3, 4

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
    import torch
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
