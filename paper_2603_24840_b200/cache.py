"""ctypes binding of the paged 8-bit cache: appending keys and values with their rotary positions, and attention of one token per rollout (marshalling only)."""
from __future__ import annotations

import ctypes as C
from typing import Optional

import torch

from . import attention as A
from . import binding as B
from . import rotary

_ready = False


class _Cache(C.Structure):
    _fields_ = [("k_cache", C.c_void_p), ("v_cache", C.c_void_p), ("k_page_stride", C.c_int64), ("v_page_stride", C.c_int64), ("k_scale", C.c_void_p),
                ("v_scale", C.c_void_p), ("k_scale_stride", C.c_int64), ("v_scale_stride", C.c_int64), ("pages", C.c_int32), ("page", C.c_int32),
                ("Hkv", C.c_int32), ("D", C.c_int32)]


class _Append(C.Structure):
    _fields_ = [("cache", _Cache), ("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("q_stride", C.c_int64), ("k_stride", C.c_int64),
                ("v_stride", C.c_int64), ("q_out", C.c_void_p), ("k_out", C.c_void_p), ("q_out_stride", C.c_int64), ("k_out_stride", C.c_int64),
                ("page_table", C.c_void_p), ("table_stride", C.c_int64), ("lengths", C.c_void_p), ("cu_new", C.c_void_p), ("keep", C.c_void_p),
                ("prompt_lengths", C.c_void_p), ("frequencies", C.c_void_p), ("rows", C.c_int64), ("table_pages", C.c_int32), ("N", C.c_int32),
                ("P", C.c_int32), ("G", C.c_int32), ("Hq", C.c_int32), ("R", C.c_int32), ("interleaved", C.c_int32), ("factor", C.c_float)]


class _Attend(C.Structure):
    _fields_ = [("cache", _Cache), ("q", C.c_void_p), ("q_stride", C.c_int64), ("page_table", C.c_void_p), ("table_stride", C.c_int64),
                ("lengths", C.c_void_p), ("keep", C.c_void_p), ("prompt_table", C.c_void_p), ("prompt_table_stride", C.c_int64),
                ("prompt_lengths", C.c_void_p), ("table_pages", C.c_int32), ("prompt_table_pages", C.c_int32), ("N", C.c_int32), ("P", C.c_int32),
                ("G", C.c_int32), ("Hq", C.c_int32), ("scale", C.c_float), ("reserved", C.c_int32), ("o", C.c_void_p), ("o_stride", C.c_int64),
                ("lse", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


def _lib():
    global _ready
    lib = B.load_library()
    if not _ready:
        for fn, res, args in (("arrol_cache_append", C.c_int, [C.c_void_p, C.POINTER(_Append), C.c_void_p]),
                              ("arrol_cache_attention_workspace", C.c_size_t, [C.c_void_p] + [C.c_int32] * 6),
                              ("arrol_cache_attention", C.c_int, [C.c_void_p, C.POINTER(_Attend), C.c_void_p])):
            getattr(lib, fn).restype = res
            getattr(lib, fn).argtypes = args
        _ready = True
    return lib


_CODES = (torch.float8_e4m3fn, torch.uint8)


def _pool(k_cache, v_cache, k_scale, v_scale) -> _Cache:
    # shapes and strides are asked for once a tensor: small calls are bound by the host
    shape, ks, vs, kss, vss = k_cache.shape, k_cache.stride(), v_cache.stride(), k_scale.stride(), v_scale.stride()
    if len(shape) != 4 or v_cache.shape != shape or k_scale.shape != shape[:2] or v_scale.shape != shape[:2]:
        raise ValueError("k_cache and v_cache are [pages, Hkv, page, D], their scales [pages, Hkv]")
    if k_cache.dtype not in _CODES or v_cache.dtype not in _CODES:
        raise TypeError("caches are float8_e4m3fn, or uint8 of the same bits")
    if k_scale.dtype is not torch.float32 or v_scale.dtype is not torch.float32:
        raise TypeError("scales are float32")
    pages, Hkv, page, D = shape
    inner = (page * D, D, 1)
    if ks[1:] != inner or vs[1:] != inner:      # heads, tokens of which there is one, and empty pools may have any
        for s in (ks, vs):
            if pages * Hkv * page * D and (s[3] != 1 or s[2] != D and page > 1 or s[1] != page * D and Hkv > 1):
                raise ValueError("a page's heads, tokens and dimensions lie side by side")
    if (kss[1] != 1 or vss[1] != 1) and Hkv > 1 and pages:
        raise ValueError("a page's scales lie side by side")
    if pages == 1:
        ks = vs = (Hkv * page * D,)
        kss = vss = (Hkv,)
    return _Cache(k_cache.data_ptr(), v_cache.data_ptr(), ks[0], vs[0], k_scale.data_ptr(), v_scale.data_ptr(), kss[0], vss[0], pages, page, Hkv, D)


def _table(name: str, t: Optional[torch.Tensor], rows: int):
    """(pointer, stride, entries a row)"""
    if t is None:
        return None, 0, 0
    shape, stride = t.shape, t.stride()
    if t.dtype is not torch.int32 or len(shape) != 2 or shape[0] != rows or shape[1] > 1 and stride[1] != 1:
        raise ValueError("%s is an int32 tensor [%d, pages]" % (name, rows))
    return t.data_ptr(), stride[0] if rows > 1 else shape[1], shape[1]


def arrol_cache_append(ctx: B.Context, k, v, k_cache, v_cache, k_scale, v_scale, page_table, lengths, cu_new=None, keep=None, q=None, q_out=None, k_out=None,
                       frequencies=None, factor: float = 1.0, interleaved: bool = False, prompt_lengths=None, G: int = 1, stream=None):
    """k, v [rows, Hkv, D], q, q_out [rows, Hq, D], k_out as k, bfloat16 (rows may be strided; outputs may be the inputs): one row per sequence, or rows cu_new[i] ..
    cu_new[i + 1] - 1 of sequence i; lengths int32 [N] with the new tokens; page_table int32 [N, pages]."""
    cache = _pool(k_cache, v_cache, k_scale, v_scale)
    rows, N, Hkv, D = k.shape[0], lengths.numel(), cache.Hkv, cache.D
    Hq = 0 if q is None else q.shape[1]
    if (q is None) != (q_out is None):
        raise ValueError("q_out receives q")
    if cu_new is None and rows != N:
        raise ValueError("one row per sequence, or cu_new")
    k_at, k_stride = A._rows(k, rows, Hkv, D)
    v_at, v_stride = A._rows(v, rows, Hkv, D)
    q_at, q_stride = A._rows(q, rows, Hq, D)
    qo_at, qo_stride = A._rows(q_out, rows, Hq, D)
    ko_at, ko_stride = A._rows(k_out, rows, Hkv, D)
    table, table_stride, table_pages = _table("page_table", page_table, N)
    f, R = rotary.frequencies_of(frequencies)
    P = 0 if prompt_lengths is None else prompt_lengths.numel()
    a = _Append(cache, q_at, k_at, v_at, q_stride, k_stride, v_stride, qo_at, ko_at, qo_stride, ko_stride, table, table_stride,
                A._ints("lengths", lengths, torch.int32, N), A._ints("cu_new", cu_new, torch.int64, N + 1), A._ints("keep", keep, torch.uint8, N),
                A._ints("prompt_lengths", prompt_lengths, torch.int32), f, rows, table_pages, N, P, G, Hq, R, 1 if interleaved else 0, factor)
    B._check(_lib().arrol_cache_append(ctx.handle, C.byref(a), B._stream(stream)), "arrol_cache_append")


def arrol_cache_attention_workspace(ctx: B.Context, N: int, P: int, G: int, Hq: int, Hkv: int, D: int) -> int:
    return int(_lib().arrol_cache_attention_workspace(ctx.handle, int(N), int(P), int(G), int(Hq), int(Hkv), int(D)))


def arrol_cache_attention(ctx: B.Context, q, k_cache, v_cache, k_scale, v_scale, page_table, lengths, o, lse, workspace, keep=None,
                          scale: Optional[float] = None, prompt_table=None, prompt_lengths=None, G: int = 1, stream=None):
    """One token per rollout: q, o [N, Hq, D] bfloat16, lse float32 [N, Hq] or None; page_table int32 [N, pages], prompt_table int32 [P, pages]; scale defaults to
    1 / sqrt(D)."""
    cache = _pool(k_cache, v_cache, k_scale, v_scale)
    N, Hq, D = q.shape
    if D != cache.D:
        raise ValueError("q has the cache's head dimension")
    q_at, q_stride = A._rows(q, N, Hq, D)
    o_at, o_stride = A._rows(o, N, Hq, D)
    table, table_stride, table_pages = _table("page_table", page_table, N)
    P = 0
    if (prompt_table is None) != (prompt_lengths is None):
        raise ValueError("prompts are given by prompt_table and prompt_lengths")
    if prompt_table is not None:
        P = prompt_table.shape[0]
    p_table, p_stride, p_pages = _table("prompt_table", prompt_table, P)
    a = _Attend(cache, q_at, q_stride, table, table_stride, A._ints("lengths", lengths, torch.int32, N), A._ints("keep", keep, torch.uint8, N), p_table, p_stride,
                A._ints("prompt_lengths", prompt_lengths, torch.int32, P), table_pages, p_pages, N, P, G, Hq, D ** -0.5 if scale is None else scale, 0, o_at, o_stride,
                A._lse(lse, N, Hq), B._ptr(workspace), A._bytes(workspace))
    B._check(_lib().arrol_cache_attention(ctx.handle, C.byref(a), B._stream(stream)), "arrol_cache_attention")
