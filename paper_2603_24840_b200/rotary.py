"""ctypes binding of the rotary positions of packed queries and keys, and of their gradients (marshalling only)."""
from __future__ import annotations

import ctypes as C
from typing import Optional, Tuple

import torch

from . import attention as A
from . import binding as B

PLAIN, LINEAR, BANDS, RAMP = 0, 1, 2, 3

_ready = False


class _Rotary(C.Structure):
    _fields_ = [("q", C.c_void_p), ("k", C.c_void_p), ("q_stride", C.c_int64), ("k_stride", C.c_int64), ("q_out", C.c_void_p), ("k_out", C.c_void_p),
                ("q_out_stride", C.c_int64), ("k_out_stride", C.c_int64), ("frequencies", C.c_void_p), ("positions", C.c_void_p),
                ("cu_seqlens", C.c_void_p), ("d_num", C.c_void_p), ("cu_prompts", C.c_void_p), ("survivor_idx", C.c_void_p), ("T_max", C.c_int64),
                ("S_max", C.c_int32), ("P", C.c_int32), ("G", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32), ("D", C.c_int32), ("R", C.c_int32),
                ("interleaved", C.c_int32), ("factor", C.c_float), ("reserved", C.c_int32)]


def _lib():
    global _ready
    lib = B.load_library()
    if not _ready:
        for fn, args in (("arrol_rotary_frequencies", [C.c_int32, C.c_double, C.c_int32] + [C.c_double] * 4 + [C.c_void_p, C.POINTER(C.c_double)]),
                         ("arrol_rotary", [C.c_void_p, C.POINTER(_Rotary), C.c_void_p]), ("arrol_rotary_backward", [C.c_void_p, C.POINTER(_Rotary), C.c_void_p])):
            getattr(lib, fn).restype = C.c_int
            getattr(lib, fn).argtypes = args
        _ready = True
    return lib


def frequencies_of(t: Optional[torch.Tensor]):
    """(pointer, R) of the frequencies, a dense float64 tensor [R / 2]."""
    if t is None:
        return None, 0
    if t.dtype is not torch.float64 or t.dim() != 1 or not t.is_contiguous() or t.numel() == 0:
        raise ValueError("frequencies is a dense float64 tensor [R / 2]")
    if not t.is_cuda:              # arrol_rotary_frequencies leaves them in host memory
        raise ValueError("frequencies are in device memory")
    return t.data_ptr(), 2 * t.numel()


def arrol_rotary_frequencies(R: int, base: float = 10000.0, kind: int = PLAIN, stretch: float = 1.0, low: float = 1.0, high: float = 4.0,
                             original: float = 8192.0) -> Tuple[torch.Tensor, float]:
    """Radians per position of each pair, float64 [R / 2] in host memory, and the factor on cosine and sine."""
    f, factor = torch.empty(max(int(R) // 2, 0), dtype=torch.float64), C.c_double()
    B._check(_lib().arrol_rotary_frequencies(int(R), float(base), int(kind), float(stretch), float(low), float(high), float(original), f.data_ptr() or None,
                                             C.byref(factor)), "arrol_rotary_frequencies")
    return f, factor.value


def _args(q, k, frequencies, q_out, k_out, positions, cu_seqlens, d_num, cu_prompts, survivor_idx, G, factor, interleaved) -> _Rotary:
    one = k if q is None else q
    if one is None:
        raise ValueError("there are queries or keys")
    T, D = one.shape[0], one.shape[2]
    Hq, Hkv = 0 if q is None else q.shape[1], 0 if k is None else k.shape[1]
    if (q is None) != (q_out is None) or (k is None) != (k_out is None):
        raise ValueError("q_out receives q, k_out receives k")
    q_at, q_stride = A._rows(q, T, Hq, D)
    k_at, k_stride = A._rows(k, T, Hkv, D)
    qo_at, qo_stride = A._rows(q_out, T, Hq, D)
    ko_at, ko_stride = A._rows(k_out, T, Hkv, D)
    f, R = frequencies_of(frequencies)
    S = P = 0
    if positions is None:
        if cu_seqlens is None or d_num is None:
            raise ValueError("tokens are placed by positions, or by cu_seqlens and d_num")
        S = cu_seqlens.numel() - 1
        if survivor_idx is not None:
            S = min(S, survivor_idx.numel())
        if cu_prompts is not None:
            P = cu_prompts.numel() - 1
    elif cu_seqlens is not None or cu_prompts is not None or survivor_idx is not None:
        raise ValueError("tokens are placed by positions, or by cu_seqlens and d_num")
    return _Rotary(q_at, k_at, q_stride, k_stride, qo_at, ko_at, qo_stride, ko_stride, f, A._ints("positions", positions, torch.int32, T),
                   A._ints("cu_seqlens", cu_seqlens, torch.int64, 1), A._ints("d_num", d_num, torch.int64, 2), A._ints("cu_prompts", cu_prompts, torch.int64, 1),
                   A._ints("survivor_idx", survivor_idx, torch.int32), T, S, P, G, Hq, Hkv, D, R, 1 if interleaved else 0, factor, 0)


def arrol_rotary(ctx: B.Context, q, k, frequencies, q_out, k_out, positions=None, cu_seqlens=None, d_num=None, cu_prompts=None, survivor_idx=None,
                 G: int = 1, factor: float = 1.0, interleaved: bool = False, stream=None):
    """q, q_out [T_max, Hq, D], k, k_out [T_max, Hkv, D] bfloat16 (rows may be strided; outputs may be the inputs; q or k may be None); placed by positions
    (int32 [T_max]) or by what arrol_compact leaves, with the prompts' lengths from cu_prompts."""
    a = _args(q, k, frequencies, q_out, k_out, positions, cu_seqlens, d_num, cu_prompts, survivor_idx, G, factor, interleaved)
    B._check(_lib().arrol_rotary(ctx.handle, C.byref(a), B._stream(stream)), "arrol_rotary")


def arrol_rotary_backward(ctx: B.Context, dq_out, dk_out, frequencies, dq, dk, positions=None, cu_seqlens=None, d_num=None, cu_prompts=None,
                          survivor_idx=None, G: int = 1, factor: float = 1.0, interleaved: bool = False, stream=None):
    """Gradients of arrol_rotary's inputs, dq and dk, from those of its outputs."""
    a = _args(dq_out, dk_out, frequencies, dq, dk, positions, cu_seqlens, d_num, cu_prompts, survivor_idx, G, factor, interleaved)
    B._check(_lib().arrol_rotary_backward(ctx.handle, C.byref(a), B._stream(stream)), "arrol_rotary_backward")
