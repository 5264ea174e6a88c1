"""ctypes binding of the attention calls: packed survivors over their prompts and own tokens, its backward, and one generated token per
rollout (marshalling only)."""
from __future__ import annotations

import ctypes as C
import math
from typing import Optional

import torch

from . import binding as B

_ready = False


class _Attention(C.Structure):
    _fields_ = [("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("q_stride", C.c_int64), ("k_stride", C.c_int64),
                ("v_stride", C.c_int64), ("cu_seqlens", C.c_void_p), ("d_num", C.c_void_p), ("prompt_k", C.c_void_p),
                ("prompt_v", C.c_void_p), ("prompt_k_stride", C.c_int64), ("prompt_v_stride", C.c_int64), ("cu_prompts", C.c_void_p),
                ("survivor_idx", C.c_void_p), ("T_max", C.c_int64), ("prompt_rows", C.c_int64), ("S_max", C.c_int32), ("P", C.c_int32),
                ("G", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32), ("D", C.c_int32), ("scale", C.c_float), ("reserved", C.c_int32),
                ("o", C.c_void_p), ("o_stride", C.c_int64), ("lse", C.c_void_p), ("d_o", C.c_void_p), ("d_o_stride", C.c_int64),
                ("dq", C.c_void_p), ("dk", C.c_void_p), ("dv", C.c_void_p), ("dq_stride", C.c_int64), ("dk_stride", C.c_int64),
                ("dv_stride", C.c_int64), ("dprompt_k", C.c_void_p), ("dprompt_v", C.c_void_p), ("dprompt_k_stride", C.c_int64),
                ("dprompt_v_stride", C.c_int64), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


class _Decode(C.Structure):
    _fields_ = [("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("q_stride", C.c_int64), ("k_stride", C.c_int64),
                ("v_stride", C.c_int64), ("src_tok_off", C.c_void_p), ("lengths", C.c_void_p), ("keep", C.c_void_p),
                ("prompt_k", C.c_void_p), ("prompt_v", C.c_void_p), ("prompt_k_stride", C.c_int64), ("prompt_v_stride", C.c_int64),
                ("cu_prompts", C.c_void_p), ("cache_rows", C.c_int64), ("prompt_rows", C.c_int64), ("N", C.c_int32), ("P", C.c_int32),
                ("G", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32), ("D", C.c_int32), ("scale", C.c_float), ("reserved", C.c_int32),
                ("o", C.c_void_p), ("o_stride", C.c_int64), ("lse", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


def _lib():
    global _ready
    lib = B.load_library()
    if not _ready:
        for fn, res, args in (
                ("arrol_attention_workspace", C.c_size_t, [C.c_void_p, C.c_int32, C.c_int64, C.c_int64] + [C.c_int32] * 4),
                ("arrol_attention", C.c_int, [C.c_void_p, C.POINTER(_Attention), C.c_void_p]),
                ("arrol_attention_backward", C.c_int, [C.c_void_p, C.POINTER(_Attention), C.c_void_p]),
                ("arrol_attention_decode_workspace", C.c_size_t, [C.c_void_p] + [C.c_int32] * 5),
                ("arrol_attention_decode", C.c_int, [C.c_void_p, C.POINTER(_Decode), C.c_void_p])):
            getattr(lib, fn).restype = res
            getattr(lib, fn).argtypes = args
        _ready = True
    return lib


def _rows(t: Optional[torch.Tensor], heads: int, D: int):
    """(pointer, row stride) of a [rows, heads, D] tensor whose heads lie side by side."""
    if t is None:
        return None, 0
    if t.dtype != torch.bfloat16:
        raise TypeError("attention tensors are bfloat16")
    if t.dim() != 3 or t.shape[1] != heads or t.shape[2] != D or t.numel() and (
            (D > 1 and t.stride(2) != 1) or (heads > 1 and t.stride(1) != D)):
        raise ValueError("attention tensors are [rows, heads, D] with the heads of a row side by side")
    return t.data_ptr(), max(t.stride(0), heads * D) if t.shape[0] < 2 else t.stride(0)


def _same_rows(name: str, t: torch.Tensor, rows: int):
    if t.shape[0] < rows:
        raise ValueError("%s has fewer rows than its counterpart" % name)


def _lse(t: Optional[torch.Tensor], rows: int, heads: int):
    if t is None:
        return None
    if t.dtype != torch.float32 or not t.is_contiguous() or t.numel() < rows * heads:
        raise ValueError("lse is a dense float32 tensor [rows, heads]")
    return t.data_ptr()


def _ints(name: str, t: Optional[torch.Tensor], dtype, count: int = 0):
    if t is None:
        return None
    if t.dtype != dtype or not t.is_contiguous() or t.numel() < count:
        raise ValueError("%s is a dense %s tensor of at least %d entries" % (name, dtype, count))
    return t.data_ptr()


def arrol_attention_workspace(ctx: B.Context, S_max: int, T_max: int, prompt_rows: int, Hq: int, Hkv: int, D: int,
                              backward: bool = False) -> int:
    return int(_lib().arrol_attention_workspace(ctx.handle, int(S_max), int(T_max), int(prompt_rows), int(Hq), int(Hkv), int(D),
                                                1 if backward else 0))


def _packed(q, k, v, cu_seqlens, d_num, o, lse, workspace, scale, prompt_k, prompt_v, cu_prompts, survivor_idx, G) -> _Attention:
    (T, Hq, D), Hkv = q.shape, k.shape[1]
    a = _Attention()
    a.q, a.q_stride = _rows(q, Hq, D)
    a.k, a.k_stride = _rows(k, Hkv, D)
    a.v, a.v_stride = _rows(v, Hkv, D)
    a.o, a.o_stride = _rows(o, Hq, D)
    for name, t in (("k", k), ("v", v), ("o", o)):
        _same_rows(name, t, T)
    a.lse = _lse(lse, T, Hq)
    S = cu_seqlens.numel() - 1
    a.cu_seqlens = _ints("cu_seqlens", cu_seqlens, torch.int64, 1)
    a.d_num = _ints("d_num", d_num, torch.int64, 2)
    if prompt_k is not None:
        a.prompt_k, a.prompt_k_stride = _rows(prompt_k, Hkv, D)
        a.prompt_v, a.prompt_v_stride = _rows(prompt_v, Hkv, D)
        _same_rows("prompt_v", prompt_v, prompt_k.shape[0])
        a.cu_prompts = _ints("cu_prompts", cu_prompts, torch.int64, 1)
        a.prompt_rows, a.P = prompt_k.shape[0], cu_prompts.numel() - 1
    if survivor_idx is not None:
        S = min(S, survivor_idx.numel())
        a.survivor_idx = _ints("survivor_idx", survivor_idx, torch.int32)
    a.T_max, a.S_max, a.G, a.Hq, a.Hkv, a.D = T, S, int(G), Hq, Hkv, D
    a.scale = 1.0 / math.sqrt(D) if scale is None else float(scale)
    a.workspace = B._ptr(workspace)
    a.workspace_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    return a


def arrol_attention(ctx: B.Context, q, k, v, cu_seqlens, d_num, o, lse, workspace, scale: Optional[float] = None, prompt_k=None,
                    prompt_v=None, cu_prompts=None, survivor_idx=None, G: int = 1, stream=None):
    """q, o [T_max, Hq, D], k, v [T_max, Hkv, D] bfloat16 (rows may be strided), lse float32 [T_max, Hq]; cu_seqlens, d_num, survivor_idx
    as arrol_compact leaves them; scale defaults to 1 / sqrt(D)."""
    a = _packed(q, k, v, cu_seqlens, d_num, o, lse, workspace, scale, prompt_k, prompt_v, cu_prompts, survivor_idx, G)
    B._check(_lib().arrol_attention(ctx.handle, C.byref(a), B._stream(stream)), "arrol_attention")


def arrol_attention_backward(ctx: B.Context, q, k, v, cu_seqlens, d_num, o, lse, d_o, dq, dk, dv, workspace,
                             scale: Optional[float] = None, prompt_k=None, prompt_v=None, dprompt_k=None, dprompt_v=None, cu_prompts=None,
                             survivor_idx=None, G: int = 1, stream=None):
    """Gradients (overwritten) of arrol_attention's o; o and lse are what that call wrote."""
    a = _packed(q, k, v, cu_seqlens, d_num, o, lse, workspace, scale, prompt_k, prompt_v, cu_prompts, survivor_idx, G)
    a.d_o, a.d_o_stride = _rows(d_o, a.Hq, a.D)
    a.dq, a.dq_stride = _rows(dq, a.Hq, a.D)
    a.dk, a.dk_stride = _rows(dk, a.Hkv, a.D)
    a.dv, a.dv_stride = _rows(dv, a.Hkv, a.D)
    for name, t in (("d_o", d_o), ("dq", dq), ("dk", dk), ("dv", dv)):
        _same_rows(name, t, a.T_max)
    if prompt_k is not None:
        a.dprompt_k, a.dprompt_k_stride = _rows(dprompt_k, a.Hkv, a.D)
        a.dprompt_v, a.dprompt_v_stride = _rows(dprompt_v, a.Hkv, a.D)
        for name, t in (("dprompt_k", dprompt_k), ("dprompt_v", dprompt_v)):
            _same_rows(name, t, a.prompt_rows)
    B._check(_lib().arrol_attention_backward(ctx.handle, C.byref(a), B._stream(stream)), "arrol_attention_backward")


def arrol_attention_decode_workspace(ctx: B.Context, N: int, P: int, Hq: int, Hkv: int, D: int) -> int:
    return int(_lib().arrol_attention_decode_workspace(ctx.handle, int(N), int(P), int(Hq), int(Hkv), int(D)))


def arrol_attention_decode(ctx: B.Context, q, k, v, src_tok_off, lengths, o, lse, workspace, keep=None, scale: Optional[float] = None,
                           prompt_k=None, prompt_v=None, cu_prompts=None, G: int = 1, stream=None):
    """One token per rollout: q, o [N, Hq, D], caches k, v [cache_rows, Hkv, D] bfloat16, lse float32 [N, Hq] or None."""
    (N, Hq, D), Hkv = q.shape, k.shape[1]
    a = _Decode()
    a.q, a.q_stride = _rows(q, Hq, D)
    a.k, a.k_stride = _rows(k, Hkv, D)
    a.v, a.v_stride = _rows(v, Hkv, D)
    a.o, a.o_stride = _rows(o, Hq, D)
    _same_rows("o", o, N)
    _same_rows("v", v, k.shape[0])
    a.lse = _lse(lse, N, Hq)
    a.src_tok_off = _ints("src_tok_off", src_tok_off, torch.int64, N)
    a.lengths = _ints("lengths", lengths, torch.int32, N)
    a.keep = _ints("keep", keep, torch.uint8, N)
    if prompt_k is not None:
        a.prompt_k, a.prompt_k_stride = _rows(prompt_k, Hkv, D)
        a.prompt_v, a.prompt_v_stride = _rows(prompt_v, Hkv, D)
        _same_rows("prompt_v", prompt_v, prompt_k.shape[0])
        a.cu_prompts = _ints("cu_prompts", cu_prompts, torch.int64, 1)
        a.prompt_rows, a.P = prompt_k.shape[0], cu_prompts.numel() - 1
    a.cache_rows, a.N, a.G, a.Hq, a.Hkv, a.D = k.shape[0], N, int(G), Hq, Hkv, D
    a.scale = 1.0 / math.sqrt(D) if scale is None else float(scale)
    a.workspace = B._ptr(workspace)
    a.workspace_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    B._check(_lib().arrol_attention_decode(ctx.handle, C.byref(a), B._stream(stream)), "arrol_attention_decode")
