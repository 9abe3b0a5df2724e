"""Thin ctypes binding over libhill's C ABI (include/hill.h).

Every function here only marshals arguments: tensors become device pointers,
a descriptor is filled from tensor shapes and strides, and a non-OK status
raises :class:`HillError`.  All arithmetic runs in the CUDA kernels of
libhill.so; there is no other implementation behind these names, and loading
fails loudly if the library has not been built.

Names follow the C ABI: :func:`hill_score`, :func:`hill_topk_select`,
:func:`hill_gather_sparse_attn`, :func:`hill_evict_step`, :func:`hill_topk_select_bkp`,
:func:`hill_evict_step_bkp`, :func:`hill_quantize_k`, :func:`hill_score_f8`, :func:`hill_evict_step_f8`,
:func:`hill_evict_step_kvh`, :func:`hill_evict_step_begin`, :func:`hill_evict_step_begin_f8`,
:func:`hill_evict_step_end`, :func:`hill_workspace_bytes`, :func:`hill_sync_status`; for a cache of bounded
size :func:`hill_window_attn`, :func:`hill_window_attn_q4`, :func:`hill_cache_insert`, :func:`hill_cache_insert_q4`,
:func:`hill_cache_read_q4`, :func:`hill_window_workspace_bytes`; for prompts :func:`hill_prompt_attn`,
:func:`hill_prompt_importance`; for a cache in pages :func:`hill_paged_attn`, :func:`hill_paged_write`,
:func:`hill_paged_read`.
"""
from __future__ import annotations

import ctypes
import os
import struct

import torch

from . import build as _build

HILL_OK = 0
HILL_ERR_INVALID_ARG = 1
HILL_ERR_UNSUPPORTED = 2
HILL_ERR_WORKSPACE = 3
HILL_ERR_CUDA = 4
HILL_ERR_TIMEOUT = 5
HILL_ERR_DEVICE = 6

HILL_F16, HILL_BF16 = 0, 1
HILL_SCORE_ATTN, HILL_SCORE_RAW = 0, 1

LIB_PATH = _build.LIB


class HillError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


class hill_desc(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
        ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
        ("capacity", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("q_sb", ctypes.c_int64), ("q_sh", ctypes.c_int64),
        ("k_sb", ctypes.c_int64), ("k_sh", ctypes.c_int64), ("k_sn", ctypes.c_int64),
        ("v_sb", ctypes.c_int64), ("v_sh", ctypes.c_int64), ("v_sn", ctypes.c_int64),
    ]


class hill_new_rows(ctypes.Structure):
    _fields_ = [
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
        ("k_sb", ctypes.c_int64), ("k_sh", ctypes.c_int64), ("k_sn", ctypes.c_int64),
        ("v_sb", ctypes.c_int64), ("v_sh", ctypes.c_int64), ("v_sn", ctypes.c_int64),
        ("max_new", ctypes.c_int32), ("count", ctypes.c_void_p), ("weight", ctypes.c_void_p),
    ]


# the same in one call (a fifth of the time that filling the fields takes)
_pack_rows = struct.Struct("@PPqqqqqqiPP").pack
assert struct.calcsize("@PPqqqqqqiPP") == ctypes.sizeof(hill_new_rows)

class hill_packed(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "num_q_heads", "num_kv_heads", "head_dim", "dtype", "q_rows", "k_rows")] + [
        (n, ctypes.c_int64) for n in ("q_st", "q_sh", "k_st", "k_sh", "v_st", "v_sh")]


class hill_pages(ctypes.Structure):
    _fields_ = [
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("table", ctypes.c_void_p),
        ("pages", ctypes.c_int32), ("page", ctypes.c_int32), ("cols", ctypes.c_int32),
    ]


class hill_rows(ctypes.Structure):
    _fields_ = [
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
        ("k_st", ctypes.c_int64), ("k_sh", ctypes.c_int64), ("v_st", ctypes.c_int64), ("v_sh", ctypes.c_int64),
        ("rows", ctypes.c_int32),
    ]


_pack_packed_rows = struct.Struct("@PPqqqqi4x").pack
assert struct.calcsize("@PPqqqqi4x") == ctypes.sizeof(hill_rows)

_lib = None


def load(path: str | None = None) -> ctypes.CDLL:
    """Load libhill.so (raises OSError if it is missing: build it first)."""
    global _lib
    if _lib is not None:
        return _lib
    path = path or LIB_PATH
    if not os.path.exists(path):
        raise OSError(f"libhill.so not built ({path}); run python -m paper_2602_18750_gb300.build")
    lib = ctypes.CDLL(path)
    P, I32, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    D = ctypes.POINTER(hill_desc)
    lib.hill_workspace_bytes.argtypes = [D, I32, I32]
    lib.hill_workspace_bytes.restype = SZ
    lib.hill_score.argtypes = [D, P, P, P, I32, P, P, P, SZ, P]
    lib.hill_topk_select.argtypes = [D, P, P, P, I32, P, P, P, SZ, P]
    lib.hill_gather_sparse_attn.argtypes = [D, P, P, P, P, P, I32, P, P, SZ, P]
    lib.hill_evict_step.argtypes = [D, P, P, P, P, P, I32, I32, P, P, P, P, P, P, SZ, P]
    lib.hill_topk_select_bkp.argtypes = [D, P, P, P, I32, I32, P, P, P, P, SZ, P]
    lib.hill_evict_step_bkp.argtypes = [D, P, P, P, P, P, I32, I32, I32, P, P, P, P, P, P, P, SZ, P]
    lib.hill_quantize_k.argtypes = [D, P, P, P, I32, P, P, P]
    lib.hill_evict_step_kvh.argtypes = [D, P, P, P, P, P, I32, I32, P, P, P, P, P, P, SZ, P]
    lib.hill_evict_step_begin.argtypes = [D, P, P, P, I32, I32, P, P, P, SZ, P]
    lib.hill_evict_step_begin_f8.argtypes = [D, P, P, P, P, I32, I32, P, P, P, SZ, P]
    lib.hill_evict_step_end.argtypes = [D, P, P, I32, I32, I32, P, P, P, P, P, P, SZ, P]
    lib.hill_selftest_wait.argtypes = [ctypes.c_uint32, P]
    lib.hill_score_f8.argtypes = [D, P, P, P, P, I32, P, P, P, SZ, P]
    lib.hill_evict_step_f8.argtypes = [D, P, P, P, P, P, P, P, I32, I32, P, P, P, P, P, P, SZ, P]
    lib.hill_score_noalloc.argtypes = [D, P, P, P, I32, P, P, P]
    lib.hill_score_noalloc.restype = I32
    lib.hill_window_workspace_bytes.argtypes = [D, I32]
    lib.hill_window_workspace_bytes.restype = SZ
    lib.hill_window_attn.argtypes = [D, P, P, P, P, I32, I32, I32, P, P, P, SZ, P]
    lib.hill_window_attn_q4.argtypes = [D, P, P, P, P, P, I32, I32, I32, P, P, P, SZ, P]
    # (the second: a hill_new_rows, by reference or packed)
    lib.hill_cache_insert.argtypes = [D, P, P, P, P, P, P, I32, I32, I32, P, P]
    lib.hill_cache_insert_q4.argtypes = [D, P, P, P, P, P, P, P, I32, I32, I32, P, P]
    lib.hill_cache_read_q4.argtypes = [D, P, P, P, P, P, I32, P, P, P]
    K, G = ctypes.POINTER(hill_packed), ctypes.POINTER(hill_pages)
    lib.hill_prompt_workspace_bytes.argtypes = [K]
    lib.hill_prompt_workspace_bytes.restype = SZ
    lib.hill_prompt_attn.argtypes = [K, P, P, P, P, P, I32, I32, P, P, P]
    lib.hill_prompt_importance.argtypes = [K, P, P, P, P, P, I32, I32, I32, I32, P, I32, P, SZ, P]
    lib.hill_paged_attn.argtypes = [D, P, G, P, I32, I32, I32, P, P, P, SZ, P]
    lib.hill_paged_write.argtypes = [D, G, P, P, P, P]   # (the third: a hill_rows, by reference or packed)
    lib.hill_paged_read.argtypes = [D, G, P, P, I32, P, P, P]
    lib.hill_sync_status.argtypes = [P]
    lib.hill_status_string.argtypes = [I32]
    lib.hill_status_string.restype = ctypes.c_char_p
    lib.hill_abi_version.restype = I32
    lib.hill_kernel_launches.restype = ctypes.c_uint64
    for name in ("hill_score", "hill_topk_select", "hill_gather_sparse_attn", "hill_evict_step",
                 "hill_topk_select_bkp", "hill_evict_step_bkp", "hill_quantize_k", "hill_score_f8",
                 "hill_evict_step_f8", "hill_evict_step_kvh", "hill_evict_step_begin", "hill_evict_step_begin_f8",
                 "hill_evict_step_end", "hill_selftest_wait", "hill_sync_status", "hill_window_attn",
                 "hill_window_attn_q4", "hill_cache_insert", "hill_cache_insert_q4", "hill_cache_read_q4",
                 "hill_prompt_attn", "hill_prompt_importance", "hill_paged_attn", "hill_paged_write", "hill_paged_read"):
        getattr(lib, name).restype = I32
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load().hill_status_string(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != HILL_OK:
        raise HillError(status, where)


def _ptr(t) -> int | None:
    return t if t is None or isinstance(t, int) else t.data_ptr()


_I32, _F32 = torch.int32, torch.float32


def _typed(t, dtype, what: str) -> int | None:
    """The pointer of a tensor that the kernels read or write as dense elements of dtype."""
    if t is None or isinstance(t, int):
        return t
    if t.dtype is not dtype or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous, of {dtype}; got {t.dtype}, strides {t.stride()}")
    return t.data_ptr()


# the handle of the current stream without a Stream object around it (2.5 us of a call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int | None:
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def make_desc(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor | None = None) -> hill_desc:
    """Descriptor from q [B][H][d] and K/V [B][Hkv][cap][d] (any element strides, d contiguous)."""
    B, H, d = q.shape
    Bk, Hkv, cap, dk = k_cache.shape
    if Bk != B or dk != d:
        raise ValueError(f"shape mismatch q {tuple(q.shape)} vs K {tuple(k_cache.shape)}")
    if q.stride(-1) != 1 or k_cache.stride(-1) != 1:
        raise ValueError("head dimension must be contiguous")
    if q.dtype != k_cache.dtype:
        raise ValueError("q and K must share a dtype")
    dt = {torch.float16: HILL_F16, torch.bfloat16: HILL_BF16}.get(q.dtype)
    if dt is None:
        raise ValueError(f"unsupported dtype {q.dtype}")
    v = v_cache if v_cache is not None else k_cache
    if tuple(v.shape) != tuple(k_cache.shape) or v.stride(-1) != 1 or v.dtype != q.dtype:
        raise ValueError("V must match K in shape and dtype")
    desc = hill_desc(B, H, Hkv, d, cap, dt,
                     q.stride(0), q.stride(1),
                     k_cache.stride(0), k_cache.stride(1), k_cache.stride(2),
                     v.stride(0), v.stride(1), v.stride(2))
    desc.caches = k_cache.dtype, k_cache.shape, k_cache.stride(), v.stride()
    return desc


def hill_workspace_bytes(desc: hill_desc, mode: int, max_k: int) -> int:
    return int(load().hill_workspace_bytes(ctypes.byref(desc), int(mode), int(max_k)))


def alloc_workspace(desc: hill_desc, mode: int, max_k: int, device="cuda") -> torch.Tensor:
    n = hill_workspace_bytes(desc, mode, max_k)
    if n == 0:
        raise HillError(HILL_ERR_INVALID_ARG, "hill_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def _ws(ws):
    if ws is None:
        return None, 0
    return ws.data_ptr(), ws.numel() * ws.element_size()


def hill_score(desc, q, k_cache, lens, mode, scores, accum=None, ws=None, stream=None) -> None:
    wp, wn = _ws(ws)
    _check(load().hill_score(ctypes.byref(desc), _ptr(q), _ptr(k_cache), _ptr(lens), int(mode),
                             _ptr(scores), _ptr(accum), wp, wn, _stream(stream)), "hill_score")


def hill_score_noalloc(desc, q, k_cache, lens, mode, scores, accum=None, stream=None) -> None:
    """hill_score without a workspace: scratch lives in a fixed array inside
    the library (for callers that cannot allocate device memory)."""
    _check(load().hill_score_noalloc(ctypes.byref(desc), _ptr(q), _ptr(k_cache), _ptr(lens), int(mode),
                                     _ptr(scores), _ptr(accum), _stream(stream)), "hill_score_noalloc")


def hill_topk_select(desc, scores, lens, k, max_k, idx, count, ws=None, stream=None) -> None:
    wp, wn = _ws(ws)
    _check(load().hill_topk_select(ctypes.byref(desc), _ptr(scores), _ptr(lens), _ptr(k), int(max_k),
                                   _ptr(idx), _ptr(count), wp, wn, _stream(stream)), "hill_topk_select")


def hill_gather_sparse_attn(desc, q, k_cache, v_cache, idx, count, max_k, out, ws=None, stream=None) -> None:
    wp, wn = _ws(ws)
    _check(load().hill_gather_sparse_attn(ctypes.byref(desc), _ptr(q), _ptr(k_cache), _ptr(v_cache),
                                          _ptr(idx), _ptr(count), int(max_k), _ptr(out), wp, wn,
                                          _stream(stream)), "hill_gather_sparse_attn")


def hill_evict_step(desc, q, k_cache, v_cache, lens, k, max_k, mode, accum, scores, idx, count, out,
                    ws, stream=None) -> None:
    wp, wn = _ws(ws)
    _check(load().hill_evict_step(ctypes.byref(desc), _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(lens),
                                  _ptr(k), int(max_k), int(mode), _ptr(accum), _ptr(scores), _ptr(idx),
                                  _ptr(count), _ptr(out), wp, wn, _stream(stream)), "hill_evict_step")


def hill_topk_select_bkp(desc, scores, lens, k, recent, max_k, idx, count, hits=None, ws=None,
                         stream=None) -> None:
    """BKP selection (Sec. 4.2): the `recent` newest tokens pinned, the top-k of
    the older ones, and hits[b][j] += 1 (saturating uint16) for kept tokens."""
    wp, wn = _ws(ws)
    _check(load().hill_topk_select_bkp(ctypes.byref(desc), _ptr(scores), _ptr(lens), _ptr(k), int(recent),
                                       int(max_k), _ptr(idx), _ptr(count), _ptr(hits), wp, wn,
                                       _stream(stream)), "hill_topk_select_bkp")


def hill_evict_step_bkp(desc, q, k_cache, v_cache, lens, k, recent, max_k, mode, accum, scores, idx, count,
                        hits, out, ws, stream=None) -> None:
    wp, wn = _ws(ws)
    _check(load().hill_evict_step_bkp(ctypes.byref(desc), _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(lens),
                                      _ptr(k), int(recent), int(max_k), int(mode), _ptr(accum), _ptr(scores),
                                      _ptr(idx), _ptr(count), _ptr(hits), _ptr(out), wp, wn,
                                      _stream(stream)), "hill_evict_step_bkp")


def hill_evict_step_begin(desc, q, k_cache, lens, max_k, mode, accum, scores, ws, stream=None) -> None:
    """First half of the split step: the scoring kernel (K stream)."""
    wp, wn = _ws(ws)
    _check(load().hill_evict_step_begin(ctypes.byref(desc), _ptr(q), _ptr(k_cache), _ptr(lens), int(max_k),
                                        int(mode), _ptr(accum), _ptr(scores), wp, wn, _stream(stream)),
           "hill_evict_step_begin")


def hill_evict_step_begin_f8(desc, q, k8, kscale, lens, max_k, mode, accum, scores, ws, stream=None) -> None:
    """First half of the split step from the E4M3 key shadow."""
    wp, wn = _ws(ws)
    _check(load().hill_evict_step_begin_f8(ctypes.byref(desc), _ptr(q), _ptr(k8), _ptr(kscale), _ptr(lens),
                                           int(max_k), int(mode), _ptr(accum), _ptr(scores), wp, wn,
                                           _stream(stream)), "hill_evict_step_begin_f8")


def hill_evict_step_end(desc, lens, k, max_k, mode, accum, scores, idx, count, ws, recent=0, hits=None,
                        stream=None) -> None:
    """Second half of the split step: normalisation (ATTN) and selection."""
    wp, wn = _ws(ws)
    _check(load().hill_evict_step_end(ctypes.byref(desc), _ptr(lens), _ptr(k), int(recent), int(max_k), int(mode),
                                      _ptr(accum), _ptr(scores), _ptr(idx), _ptr(count), _ptr(hits), wp, wn,
                                      _stream(stream)), "hill_evict_step_end")


def hill_evict_step_kvh(desc, q, k_cache, v_cache, lens, k, max_k, mode, accum, scores, idx, count, out, ws,
                        stream=None) -> None:
    """Per-KV-head selection: scores [B][Hkv][cap], idx [B][Hkv][max_k], count [B][Hkv]."""
    wp, wn = _ws(ws)
    _check(load().hill_evict_step_kvh(ctypes.byref(desc), _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(lens),
                                      _ptr(k), int(max_k), int(mode), _ptr(accum), _ptr(scores), _ptr(idx),
                                      _ptr(count), _ptr(out), wp, wn, _stream(stream)), "hill_evict_step_kvh")


def shadow_shape(desc):
    """Shapes of the E4M3 key shadow: (codes [B][Hkv][cap][128], scales [B][Hkv][cap32])."""
    cap32 = (desc.capacity + 31) // 32 * 32
    return ((desc.batch, desc.num_kv_heads, desc.capacity, desc.head_dim),
            (desc.batch, desc.num_kv_heads, cap32))


def alloc_shadow(desc, device="cuda"):
    cs, ss = shadow_shape(desc)
    return torch.zeros(cs, dtype=torch.uint8, device=device), torch.zeros(ss, dtype=torch.float32, device=device)


def hill_quantize_k(desc, k_cache, row_begin, row_end, max_rows, k8, kscale, stream=None) -> None:
    _check(load().hill_quantize_k(ctypes.byref(desc), _ptr(k_cache), _ptr(row_begin), _ptr(row_end),
                                  int(max_rows), _ptr(k8), _ptr(kscale), _stream(stream)), "hill_quantize_k")


def hill_score_f8(desc, q, k8, kscale, lens, mode, scores, accum=None, ws=None, stream=None) -> None:
    wp, wn = _ws(ws)
    _check(load().hill_score_f8(ctypes.byref(desc), _ptr(q), _ptr(k8), _ptr(kscale), _ptr(lens), int(mode),
                                _ptr(scores), _ptr(accum), wp, wn, _stream(stream)), "hill_score_f8")


def hill_evict_step_f8(desc, q, k8, kscale, k_cache, v_cache, lens, k, max_k, mode, accum, scores, idx, count,
                       out, ws, stream=None) -> None:
    wp, wn = _ws(ws)
    _check(load().hill_evict_step_f8(ctypes.byref(desc), _ptr(q), _ptr(k8), _ptr(kscale), _ptr(k_cache),
                                     _ptr(v_cache), _ptr(lens), _ptr(k), int(max_k), int(mode), _ptr(accum),
                                     _ptr(scores), _ptr(idx), _ptr(count), _ptr(out), wp, wn, _stream(stream)),
           "hill_evict_step_f8")


def make_desc_q4(q: torch.Tensor, k4: torch.Tensor) -> hill_desc:
    """Descriptor from q [B][H][d] and the codes of a 4-bit cache [B][Hkv][cap][d / 2]."""
    B, H, d = q.shape
    Bk, Hkv, cap, half = k4.shape
    if Bk != B or 2 * half != d:
        raise ValueError(f"shape mismatch q {tuple(q.shape)} vs codes {tuple(k4.shape)}")
    if k4.element_size() != 1 or not k4.is_contiguous():
        raise ValueError("codes must be bytes, contiguous")
    if q.stride(-1) != 1:
        raise ValueError("head dimension must be contiguous")
    dt = {torch.float16: HILL_F16, torch.bfloat16: HILL_BF16}.get(q.dtype)
    if dt is None:
        raise ValueError(f"unsupported dtype {q.dtype}")
    return hill_desc(B, H, Hkv, d, cap, dt, q.stride(0), q.stride(1), Hkv * cap * d, cap * d, d, Hkv * cap * d, cap * d, d)


def q4_shape(B: int, Hkv: int, cap: int, d: int = 128):
    """Shapes of a 4-bit cache: codes (of K, and of V) [B][Hkv][cap][d / 2], params [B][Hkv][cap32][4]."""
    return (B, Hkv, cap, d // 2), (B, Hkv, (cap + 31) // 32 * 32, 4)


def alloc_q4(B: int, Hkv: int, cap: int, dtype=torch.float16, device="cuda"):
    """(k4, v4, params) of an empty 4-bit cache."""
    cs, ps = q4_shape(B, Hkv, cap)
    return (torch.zeros(cs, dtype=torch.uint8, device=device), torch.zeros(cs, dtype=torch.uint8, device=device),
            torch.zeros(ps, dtype=dtype, device=device))


def hill_window_workspace_bytes(desc: hill_desc, with_accum: bool) -> int:
    return int(load().hill_window_workspace_bytes(ctypes.byref(desc), int(bool(with_accum))))


def alloc_window_workspace(desc: hill_desc, with_accum: bool, device="cuda") -> torch.Tensor:
    n = hill_window_workspace_bytes(desc, with_accum)
    if n == 0:
        raise HillError(HILL_ERR_INVALID_ARG, "hill_window_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def hill_window_attn(desc, q, k_cache, v_cache, lens, sinks, window, out, accum=None, kvh=False, ws=None,
                     stream=None) -> None:
    """Attention over the first `sinks` and the newest `window` tokens; accum += the weights."""
    wp, wn = _ws(ws)
    _check(load().hill_window_attn(ctypes.byref(desc), _ptr(q), _ptr(k_cache), _ptr(v_cache),
                                   _typed(lens, _I32, "lens"), int(sinks), int(window), int(bool(kvh)),
                                   _typed(accum, _F32, "accum"), _typed(out, _F32, "out"), wp, wn,
                                   _stream(stream)), "hill_window_attn")


def hill_window_attn_q4(desc, q, k4, v4, params, lens, sinks, window, out, accum=None, kvh=False, ws=None,
                        stream=None) -> None:
    """hill_window_attn over a cache held in 4 bits."""
    wp, wn = _ws(ws)
    _check(load().hill_window_attn_q4(ctypes.byref(desc), _ptr(q), _ptr(k4), _ptr(v4), _ptr(params),
                                      _typed(lens, _I32, "lens"), int(sinks), int(window), int(bool(kvh)),
                                      _typed(accum, _F32, "accum"), _typed(out, _F32, "out"), wp, wn,
                                      _stream(stream)), "hill_window_attn_q4")


def _new_rows(desc, k_new, v_new, n_new, w_new, kvh) -> bytes:
    """The hill_new_rows of new tokens, packed."""
    shape, dtype = k_new.shape, torch.bfloat16 if desc.dtype else torch.float16
    if len(shape) != 4 or shape != v_new.shape or k_new.dtype != dtype or v_new.dtype != dtype:
        raise ValueError("new rows must be [B][Hkv][T][d], K and V alike, in the cache's type")
    (kb, kh, kn, k1), (vb, vh, vn, v1) = k_new.stride(), v_new.stride()
    B, Hkv, T, d = shape
    if B != desc.batch or Hkv != desc.num_kv_heads or d != desc.head_dim or k1 != 1 or v1 != 1:
        raise ValueError(f"new rows must be [{desc.batch}][{desc.num_kv_heads}][T][{desc.head_dim}], the last dimension "
                         f"contiguous; got {tuple(shape)}")
    n = w = 0
    if n_new is not None:
        n = _typed(n_new, _I32, "n_new")
        if n_new is not n and n_new.numel() < B:
            raise ValueError(f"n_new must be [{B}], got {tuple(n_new.shape)}")
    if w_new is not None:
        w = _typed(w_new, _F32, "w_new")
        if w_new is not w and w_new.numel() != B * (Hkv if kvh else 1) * T:
            raise ValueError(f"w_new must be [{B}]{[Hkv] if kvh else ''}[{T}], got {tuple(w_new.shape)}")
    return _pack_rows(k_new.data_ptr(), v_new.data_ptr(), kb, kh, kn, vb, vh, vn, T, n, w)


def _state(seen, pos, accum, slots):
    """Their pointers; the usual case without a call for each (1 us of an insert's host time)."""
    try:
        if (seen.dtype is _I32 and pos.dtype is _I32 and slots.dtype is _I32 and accum.dtype is _F32
                and seen.is_contiguous() and pos.is_contiguous() and slots.is_contiguous() and accum.is_contiguous()):
            return seen.data_ptr(), pos.data_ptr(), accum.data_ptr(), slots.data_ptr()
    except AttributeError:   # pointers among them
        pass
    return _typed(seen, _I32, "seen"), _typed(pos, _I32, "pos"), _typed(accum, _F32, "accum"), _typed(slots, _I32, "slots")


def hill_cache_insert(desc, k_new, v_new, k_cache, v_cache, seen, pos, accum, sinks, recent, slots, n_new=None,
                      w_new=None, kvh=False, stream=None) -> None:
    """New tokens [B][Hkv][T][d] into a cache of fixed size, in place; a full one evicts by accumulated weight."""
    rows = _new_rows(desc, k_new, v_new, n_new, w_new, kvh)
    seen, pos, accum, slots = _state(seen, pos, accum, slots)
    _check(load().hill_cache_insert(ctypes.byref(desc), rows, _ptr(k_cache), _ptr(v_cache), seen, pos, accum,
                                    int(sinks), int(recent), 1 if kvh else 0, slots, _stream(stream)),
           "hill_cache_insert")


def hill_cache_insert_q4(desc, k_new, v_new, k4, v4, params, seen, pos, accum, sinks, recent, slots, n_new=None,
                         w_new=None, kvh=False, stream=None) -> None:
    """hill_cache_insert into a 4-bit cache."""
    rows = _new_rows(desc, k_new, v_new, n_new, w_new, kvh)
    seen, pos, accum, slots = _state(seen, pos, accum, slots)
    _check(load().hill_cache_insert_q4(ctypes.byref(desc), rows, _ptr(k4), _ptr(v4), _ptr(params), seen, pos, accum,
                                       int(sinks), int(recent), 1 if kvh else 0, slots, _stream(stream)),
           "hill_cache_insert_q4")


def hill_cache_read_q4(desc, k4, v4, params, row_begin, row_end, max_rows, k_cache, v_cache, stream=None) -> None:
    """What slots [row_begin, row_end) of a 4-bit cache stand for, into 16-bit caches."""
    _check(load().hill_cache_read_q4(ctypes.byref(desc), _ptr(k4), _ptr(v4), _ptr(params),
                                     _typed(row_begin, _I32, "row_begin"),
                                     _typed(row_end, _I32, "row_end"), int(max_rows), _ptr(k_cache),
                                     _ptr(v_cache), _stream(stream)), "hill_cache_read_q4")


_DTYPES = {torch.float16: HILL_F16, torch.bfloat16: HILL_BF16}


def _dtype_of(desc):
    return torch.bfloat16 if desc.dtype else torch.float16


def make_packed(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, batch: int) -> hill_packed:
    """Descriptor of packed prompts: q [q_rows][H][d], k and v [k_rows][Hkv][d] (any strides of rows and heads)."""
    if q.dim() != 3 or k.dim() != 3 or v.shape != k.shape or k.shape[2] != q.shape[2]:
        raise ValueError(f"packed rows must be [rows][heads][d], K and V alike; got q {tuple(q.shape)}, K {tuple(k.shape)}, "
                         f"V {tuple(v.shape)}")
    if q.dtype not in _DTYPES or k.dtype != q.dtype or v.dtype != q.dtype:
        raise ValueError(f"q, K and V must share fp16 or bf16; got {q.dtype}, {k.dtype}, {v.dtype}")
    if q.stride(2) != 1 or k.stride(2) != 1 or v.stride(2) != 1:
        raise ValueError("head dimension must be contiguous")
    desc = hill_packed(int(batch), q.shape[1], k.shape[1], q.shape[2], _DTYPES[q.dtype], q.shape[0], k.shape[0],
                       q.stride(0), q.stride(1), k.stride(0), k.stride(1), v.stride(0), v.stride(1))
    # what a call's tensors are held against (told apart field by field they would take as long as the launch)
    desc.made_for = tuple((t.dtype, t.shape, t.stride()) for t in (q, k, v)), torch.Size((q.shape[0], q.shape[1])), torch.Size((int(batch) + 1,))
    return desc


def hill_prompt_workspace_bytes(desc: hill_packed) -> int:
    return int(load().hill_prompt_workspace_bytes(ctypes.byref(desc)))


def alloc_prompt_workspace(desc: hill_packed, device="cuda") -> torch.Tensor:
    n = hill_prompt_workspace_bytes(desc)
    if n == 0:
        raise HillError(HILL_ERR_INVALID_ARG, "hill_prompt_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def _packed_rows(t, like, what: str):
    """The pointer of packed rows that a descriptor was made for."""
    if t is None or isinstance(t, int):
        return t
    if t.dtype is not like[0] or t.shape != like[1] or t.stride() != like[2]:
        raise ValueError(f"{what} must be {list(like[1])} of {like[0]}, strides {like[2]}, as the descriptor was made for; "
                         f"got {list(t.shape)} of {t.dtype}, strides {t.stride()}")
    return t.data_ptr()


def _dense(t, dtype, shape, what: str):
    """The pointer of a contiguous tensor of this type and shape."""
    if t is None or isinstance(t, int):
        return t
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what} must be {list(shape)} of {dtype}, contiguous; got {list(t.shape)} of {t.dtype}, strides "
                         f"{t.stride()}")
    return t.data_ptr()


def hill_prompt_attn(desc, q, k, v, q_start, k_start, sinks, window, out, lse=None, stream=None) -> None:
    """Causal attention over packed prompts into out (desc's type); lse: the log of every query's sum of exponentials."""
    (lq, lk, lv), heads, offsets = desc.made_for
    _check(load().hill_prompt_attn(desc, _packed_rows(q, lq, "q"), _packed_rows(k, lk, "K"), _packed_rows(v, lv, "V"),
                                   _dense(q_start, _I32, offsets, "q_start"), _dense(k_start, _I32, offsets, "k_start"),
                                   int(sinks), int(window), _dense(out, lq[0], lq[1], "out"),
                                   _dense(lse, _F32, heads, "lse"), _stream(stream)), "hill_prompt_attn")


def hill_prompt_importance(desc, q, k, lse, q_start, k_start, sinks, window, newest, accum, kvh=False, ws=None,
                           stream=None) -> None:
    """accum [B][cap] (kvh: [B][Hkv][cap]) += the weights that the prompts' tokens receive from the newest queries."""
    wp, wn = _ws(ws)
    (lq, lk, _), heads, offsets = desc.made_for
    rows = (desc.batch, desc.num_kv_heads) if kvh else (desc.batch,)
    if accum.shape[:-1] != rows:
        raise ValueError(f"accum must be {list(rows)}[cap], got {tuple(accum.shape)}")
    _check(load().hill_prompt_importance(desc, _packed_rows(q, lq, "q"), _packed_rows(k, lk, "K"),
                                         _dense(lse, _F32, heads, "lse"), _dense(q_start, _I32, offsets, "q_start"),
                                         _dense(k_start, _I32, offsets, "k_start"), int(sinks), int(window), int(newest),
                                         1 if kvh else 0, _typed(accum, _F32, "accum"), accum.shape[-1], wp, wn,
                                         _stream(stream)), "hill_prompt_importance")


def make_pages(k_pool: torch.Tensor, v_pool: torch.Tensor, table: torch.Tensor, scales: torch.Tensor | None = None) -> hill_pages:
    """A cache in pages: pools [pages][Hkv][page][d] in 16 bits, or E4M3 codes with scales [pages][Hkv][page][2], and
    the page table [B][cols].  The handle keeps the tensors alive; their contents may change under it."""
    if k_pool.dim() != 4 or v_pool.shape != k_pool.shape or k_pool.shape[3] != 128 or v_pool.dtype != k_pool.dtype:
        raise ValueError(f"pools must be [pages][Hkv][page][128], K and V alike; got {tuple(k_pool.shape)} of {k_pool.dtype}, "
                         f"{tuple(v_pool.shape)} of {v_pool.dtype}")
    if not k_pool.is_contiguous() or not v_pool.is_contiguous():
        raise ValueError("pools must be contiguous")
    if scales is None:
        if k_pool.dtype not in _DTYPES:
            raise ValueError(f"pools without scales must be fp16 or bf16, got {k_pool.dtype}")
    else:
        if k_pool.dtype not in (torch.float8_e4m3fn, torch.uint8):
            raise ValueError(f"pools with scales must hold E4M3 codes, got {k_pool.dtype}")
        if scales.shape != (*k_pool.shape[:3], 2):
            raise ValueError(f"scales must be {[*k_pool.shape[:3], 2]}, got {tuple(scales.shape)}")
    if table.dim() != 2:
        raise ValueError(f"the table must be [B][cols], got {tuple(table.shape)}")
    p = hill_pages(k_pool.data_ptr(), v_pool.data_ptr(), _typed(scales, _F32, "scales"), _typed(table, _I32, "the table"),
                   k_pool.shape[0], k_pool.shape[2], table.shape[1])
    p.tensors = (k_pool, v_pool, table, scales)
    p.kv_heads, p.batch, p.dtype = k_pool.shape[1], table.shape[0], None if scales is not None else k_pool.dtype
    p.offsets, p.rows = torch.Size((p.batch + 1,)), torch.Size((p.batch,))
    cap = p.cols * p.page
    # the shapes of lens and accum: of sequences, and of KV heads
    p.held = (p.rows, torch.Size((p.batch, cap))), (torch.Size((p.batch, p.kv_heads)), torch.Size((p.batch, p.kv_heads, cap)))
    return p


def _fits(desc, pages) -> None:
    if desc.num_kv_heads != pages.kv_heads or desc.batch != pages.batch or (pages.dtype and pages.dtype is not _dtype_of(desc)):
        raise ValueError(f"pages of {pages.batch} sequences, {pages.kv_heads} KV heads{f', {pages.dtype}' if pages.dtype else ''} "
                         f"do not fit a descriptor of {desc.batch}, {desc.num_kv_heads}, {_dtype_of(desc)}")


def make_desc_paged(q: torch.Tensor, pages: hill_pages) -> hill_desc:
    """Descriptor from q [B][H][d] and a cache in pages; its capacity is what the table covers."""
    B, H, d = q.shape
    if q.stride(-1) != 1 or d != 128:
        raise ValueError("head dimension must be 128, contiguous")
    if q.dtype not in _DTYPES:
        raise ValueError(f"unsupported dtype {q.dtype}")
    desc = hill_desc(B, H, pages.kv_heads, d, pages.cols * pages.page, _DTYPES[q.dtype], q.stride(0), q.stride(1))
    _fits(desc, pages)
    desc.made_for = q.dtype, q.shape, q.stride()
    return desc


def hill_paged_attn(desc, q, pages, lens, sinks, window, out, accum=None, kvh=False, ws=None, stream=None) -> None:
    """hill_window_attn over a cache in pages; desc is make_desc_paged's."""
    _fits(desc, pages)
    wp, wn = _ws(ws)
    rows, held = pages.held[1 if kvh else 0]
    _check(load().hill_paged_attn(desc, _packed_rows(q, desc.made_for, "q"), pages, _dense(lens, _I32, rows, "lens"), int(sinks), int(window), 1 if kvh else 0,
                                  _dense(accum, _F32, held, "accum"), _dense(out, _F32, desc.made_for[1], "out"), wp, wn,
                                  _stream(stream)), "hill_paged_attn")


def hill_paged_write(desc, pages, k_new, v_new, starts, begin, stream=None) -> None:
    """New rows [rows][Hkv][d] of several sequences into their pages; E4M3 caches quantise them."""
    _fits(desc, pages)
    shape, dt = k_new.shape, _dtype_of(desc)
    if len(shape) != 3 or v_new.shape != shape or shape[1] != pages.kv_heads or shape[2] != 128 or k_new.dtype is not dt or v_new.dtype is not dt:
        raise ValueError(f"new rows must be [rows][{pages.kv_heads}][128] of {dt}, K and V alike; got {tuple(shape)} of "
                         f"{k_new.dtype}, {tuple(v_new.shape)} of {v_new.dtype}")
    (kt, kh, k1), (vt, vh, v1) = k_new.stride(), v_new.stride()
    if k1 != 1 or v1 != 1:
        raise ValueError("head dimension must be contiguous")
    rows = _pack_packed_rows(k_new.data_ptr(), v_new.data_ptr(), kt, kh, vt, vh, shape[0])
    _check(load().hill_paged_write(desc, pages, rows, _dense(starts, _I32, pages.offsets, "starts"),
                                   _dense(begin, _I32, pages.rows, "begin"), _stream(stream)), "hill_paged_write")


def _cache(t, dtype, shape, strides, what: str):
    """The pointer of a 16-bit cache that lies as the descriptor has it."""
    if t is None or isinstance(t, int):
        return t
    if t.dtype is not dtype or t.shape != shape or (t.stride() != strides and any(
            n > 1 and x != y for n, x, y in zip(shape, t.stride(), strides))):
        raise ValueError(f"{what} must be {list(shape)} of {dtype}, strides {strides}, as the descriptor was made for; "
                         f"got {list(t.shape)} of {t.dtype}, strides {t.stride()}")
    return t.data_ptr()


def hill_paged_read(desc, pages, row_begin, row_end, max_rows, k_cache, v_cache, stream=None) -> None:
    """What positions [row_begin, row_end) of a cache in pages stand for, into 16-bit caches [B][Hkv][capacity][128].

    desc is make_desc's of those caches, or make_desc_paged's: then the caches say how their rows lie."""
    _fits(desc, pages)
    caches = getattr(desc, "caches", None)
    if caches is None:
        if hasattr(desc, "made_for"):
            desc = hill_desc.from_buffer_copy(desc)
            desc.k_sb, desc.k_sh, desc.k_sn = k_cache.stride()[:3]
            desc.v_sb, desc.v_sh, desc.v_sn = v_cache.stride()[:3]
        caches = (_dtype_of(desc), torch.Size((desc.batch, desc.num_kv_heads, desc.capacity, 128)),
                  (desc.k_sb, desc.k_sh, desc.k_sn, 1), (desc.v_sb, desc.v_sh, desc.v_sn, 1))
    dtype, shape, ks, vs = caches
    kp, vp = _cache(k_cache, dtype, shape, ks, "k_cache"), _cache(v_cache, dtype, shape, vs, "v_cache")
    _check(load().hill_paged_read(desc, pages, _dense(row_begin, _I32, pages.rows, "row_begin"),
                                  _dense(row_end, _I32, pages.rows, "row_end"), int(max_rows), kp, vp, _stream(stream)),
           "hill_paged_read")


def hill_selftest_wait(limit_us: int, stream=None) -> None:
    """Run the bounded-wait self test (its expiry shows up in hill_sync_status)."""
    _check(load().hill_selftest_wait(int(limit_us), _stream(stream)), "hill_selftest_wait")


def hill_kernel_launches() -> int:
    return int(load().hill_kernel_launches())


def hill_sync_status(stream=None) -> None:
    _check(load().hill_sync_status(_stream(stream)), "hill_sync_status")


class Evictor:
    """Holds the workspace and output buffers for repeated steps of one shape.

    ``step()`` issues exactly one hill_evict_step call; buffers are allocated
    once with torch (device memory plumbing only).
    """

    def __init__(self, q, k_cache, v_cache, max_k: int, mode: int = HILL_SCORE_ATTN,
                 with_scores: bool = True, with_attn: bool = True):
        self.desc = make_desc(q, k_cache, v_cache)
        self.mode = int(mode)
        self.max_k = int(max_k)
        dev = q.device
        B, H, d = q.shape
        cap = k_cache.shape[2]
        self.ws = alloc_workspace(self.desc, self.mode, self.max_k, dev)
        self.scores = torch.empty(B, cap, dtype=torch.float32, device=dev) if with_scores else None
        self.idx = torch.empty(B, max(self.max_k, 1), dtype=torch.int32, device=dev)
        self.count = torch.empty(B, dtype=torch.int32, device=dev)
        self.out = torch.empty(B, H, d, dtype=torch.float32, device=dev) if with_attn else None

    def step(self, q, k_cache, v_cache, lens, k, accum=None, stream=None):
        hill_evict_step(self.desc, q, k_cache, v_cache, lens, k, self.max_k, self.mode, accum,
                        self.scores, self.idx, self.count, self.out, self.ws, stream)
        return self


class BoundedCache:
    """The cache of one layer with a fixed number of slots: its buffers and state, allocated once.

    ``insert`` puts new tokens in (a full cache evicts by accumulated weight), ``attend`` runs the attention over
    what is held and adds the weights; ``step`` does both.  ``bits`` is 16 or 4.  With ``kvh`` every KV head keeps
    tokens of its own.  ``sinks`` + max(``recent``, ``max_new``) slots are needed.  With ``recent`` = ``capacity`` -
    ``sinks`` the oldest tokens after the sinks go first, whatever their weights: a sliding window (whose attention
    needs no weights: ``hill_window_attn`` on the same buffers without an accum leaves them out).
    """

    def __init__(self, batch: int, heads: int, kv_heads: int, capacity: int, dtype=torch.float16, bits: int = 16,
                 sinks: int = 4, recent: int = 0, kvh: bool = False, max_new: int = 1, device="cuda"):
        if bits not in (4, 16):
            raise ValueError("bits must be 16 or 4")
        if min(sinks, recent, max_new) < 0 or sinks + max(recent, max_new) > capacity:
            raise ValueError(f"{capacity} slots do not hold {sinks} sinks and {max(recent, max_new)} tokens that stay")
        self.bits, self.sinks, self.recent, self.kvh, self.max_new = bits, int(sinks), int(recent), bool(kvh), int(max_new)
        self.dtype = dtype
        rows = (batch, kv_heads) if kvh else (batch,)
        q = torch.empty(batch, heads, 128, dtype=dtype, device=device)
        if bits == 4:
            self.k4, self.v4, self.params = alloc_q4(batch, kv_heads, capacity, dtype, device)
            self.desc = make_desc_q4(q, self.k4)
        else:
            self.K, self.V = (torch.zeros(batch, kv_heads, capacity, 128, dtype=dtype, device=device) for _ in range(2))
            self.desc = make_desc(q, self.K, self.V)
        self.seen = torch.zeros(rows, dtype=torch.int32, device=device)
        self.pos = torch.zeros(*rows, capacity, dtype=torch.int32, device=device)
        self.accum = torch.zeros(*rows, capacity, dtype=torch.float32, device=device)
        self.slots = torch.full((*rows, self.max_new), -1, dtype=torch.int32, device=device)
        self.out = torch.empty(batch, heads, 128, dtype=torch.float32, device=device)
        self.ws = alloc_window_workspace(self.desc, True, device)

    def insert(self, k_new, v_new, n_new=None, w_new=None, stream=None):
        """New tokens [B][Hkv][T][d], T <= max_new; slots[..., :T] says where they went."""
        T = k_new.shape[2]
        if T > self.max_new:
            raise ValueError(f"{T} new tokens, at most {self.max_new}")
        slots = self.slots if T == self.max_new else self.slots.flatten()[:self.seen.numel() * T].view(*self.seen.shape, T)
        if self.bits == 4:
            hill_cache_insert_q4(self.desc, k_new, v_new, self.k4, self.v4, self.params, self.seen, self.pos, self.accum,
                                 self.sinks, self.recent, slots, n_new, w_new, self.kvh, stream)
        else:
            hill_cache_insert(self.desc, k_new, v_new, self.K, self.V, self.seen, self.pos, self.accum, self.sinks,
                              self.recent, slots, n_new, w_new, self.kvh, stream)
        return slots

    def attend(self, q, stream=None):
        """Attention of q [B][H][d] over the held tokens; their weights are added to accum."""
        if q.shape != self.out.shape or q.stride(-1) != 1 or q.dtype is not self.dtype:
            raise ValueError(f"q must be {tuple(self.out.shape)} of {self.dtype}, the last dimension contiguous")
        self.desc.q_sb, self.desc.q_sh = q.stride(0), q.stride(1)
        everything = self.desc.capacity
        if self.bits == 4:
            hill_window_attn_q4(self.desc, q, self.k4, self.v4, self.params, self.seen, 0, everything, self.out,
                                self.accum, self.kvh, self.ws, stream)
        else:
            hill_window_attn(self.desc, q, self.K, self.V, self.seen, 0, everything, self.out, self.accum, self.kvh,
                             self.ws, stream)
        return self.out

    def step(self, q, k_new, v_new, stream=None):
        """One decode step: the new token in, then its attention."""
        self.insert(k_new, v_new, stream=stream)
        return self.attend(q, stream)
