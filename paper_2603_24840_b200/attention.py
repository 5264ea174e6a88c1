"""ctypes binding of the attention calls: packed survivors over their prompts and own tokens, its backward, and one generated token per
rollout (marshalling only)."""
from __future__ import annotations

import ctypes as C
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


# Small calls are bound by the host: shapes and strides are asked for once a tensor, structures filled in one constructor call.
def _rows(t: Optional[torch.Tensor], rows: int, heads: int, D: int):
    """(pointer, row stride) of a [rows or more, heads, D] tensor whose heads lie side by side."""
    if t is None:
        return None, 0
    if t.dtype is not torch.bfloat16:
        raise TypeError("attention tensors are bfloat16")
    shape, stride = t.shape, t.stride()
    if len(shape) != 3 or shape[1] != heads or shape[2] != D or shape[0] < rows or (stride[1] != D and heads > 1 or stride[2] != 1 and D > 1) and t.numel():
        raise ValueError("attention tensors are [rows, heads, D] with the heads of a row side by side, %d rows at least here" % rows)
    return t.data_ptr(), stride[0] if shape[0] > 1 else max(stride[0], heads * D)


def _lse(t: Optional[torch.Tensor], rows: int, heads: int):
    if t is None:
        return None
    if t.dtype is not torch.float32 or not t.is_contiguous() or t.numel() < rows * heads:
        raise ValueError("lse is a dense float32 tensor [rows, heads]")
    return t.data_ptr()


def _ints(name: str, t: Optional[torch.Tensor], dtype, count: int = 0):
    if t is None:
        return None
    if t.dtype is not dtype or not t.is_contiguous() or t.numel() < count:
        raise ValueError("%s is a dense %s tensor of at least %d entries" % (name, dtype, count))
    return t.data_ptr()


def _prompts(prompt_k, prompt_v, cu_prompts, Hkv: int, D: int):
    """(rows, prompts, k, v, k stride, v stride, cu)"""
    if prompt_k is None and prompt_v is None and cu_prompts is None:
        return 0, 0, None, None, 0, 0, None
    if prompt_k is None or prompt_v is None or cu_prompts is None:
        raise ValueError("prompts are given by prompt_k, prompt_v and cu_prompts")
    rows = prompt_k.shape[0]
    k, k_stride = _rows(prompt_k, rows, Hkv, D)
    v, v_stride = _rows(prompt_v, rows, Hkv, D)
    return rows, cu_prompts.numel() - 1, k, v, k_stride, v_stride, _ints("cu_prompts", cu_prompts, torch.int64, 1)


def _bytes(workspace: Optional[torch.Tensor]) -> int:
    return 0 if workspace is None else workspace.numel() * workspace.element_size()


def arrol_attention_workspace(ctx: B.Context, S_max: int, T_max: int, prompt_rows: int, Hq: int, Hkv: int, D: int,
                              backward: bool = False) -> int:
    return int(_lib().arrol_attention_workspace(ctx.handle, int(S_max), int(T_max), int(prompt_rows), int(Hq), int(Hkv), int(D),
                                                1 if backward else 0))


def _packed(q, k, v, cu_seqlens, d_num, o, lse, workspace, scale, prompt_k, prompt_v, cu_prompts, survivor_idx, G, grads=(None, 0) * 6) -> _Attention:
    (T, Hq, D), Hkv = q.shape, k.shape[1]
    q_at, q_stride = _rows(q, T, Hq, D)
    k_at, k_stride = _rows(k, T, Hkv, D)
    v_at, v_stride = _rows(v, T, Hkv, D)
    o_at, o_stride = _rows(o, T, Hq, D)
    S = cu_seqlens.numel() - 1
    if survivor_idx is not None:
        S = min(S, survivor_idx.numel())
    rows, P, pk, pv, pk_stride, pv_stride, cu_p = _prompts(prompt_k, prompt_v, cu_prompts, Hkv, D)
    d_o, d_o_stride, dq, dq_stride, dk, dk_stride, dv, dv_stride, dpk, dpk_stride, dpv, dpv_stride = grads
    return _Attention(q_at, k_at, v_at, q_stride, k_stride, v_stride, _ints("cu_seqlens", cu_seqlens, torch.int64, 1),
                      _ints("d_num", d_num, torch.int64, 2), pk, pv, pk_stride, pv_stride, cu_p,
                      _ints("survivor_idx", survivor_idx, torch.int32), T, rows, S, P, G, Hq, Hkv, D, D ** -0.5 if scale is None else scale, 0,
                      o_at, o_stride, _lse(lse, T, Hq), d_o, d_o_stride, dq, dk, dv, dq_stride, dk_stride, dv_stride, dpk, dpv, dpk_stride,
                      dpv_stride, B._ptr(workspace), _bytes(workspace))


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
    (T, Hq, D), Hkv, rows = q.shape, k.shape[1], 0 if prompt_k is None else prompt_k.shape[0]
    grads = _rows(d_o, T, Hq, D) + _rows(dq, T, Hq, D) + _rows(dk, T, Hkv, D) + _rows(dv, T, Hkv, D)
    if prompt_k is None and (dprompt_k is not None or dprompt_v is not None):
        raise ValueError("dprompt_k and dprompt_v are the gradients of prompt_k and prompt_v")
    grads += _rows(dprompt_k, rows, Hkv, D) + _rows(dprompt_v, rows, Hkv, D)
    a = _packed(q, k, v, cu_seqlens, d_num, o, lse, workspace, scale, prompt_k, prompt_v, cu_prompts, survivor_idx, G, grads)
    B._check(_lib().arrol_attention_backward(ctx.handle, C.byref(a), B._stream(stream)), "arrol_attention_backward")


def arrol_attention_decode_workspace(ctx: B.Context, N: int, P: int, Hq: int, Hkv: int, D: int) -> int:
    return int(_lib().arrol_attention_decode_workspace(ctx.handle, int(N), int(P), int(Hq), int(Hkv), int(D)))


def arrol_attention_decode(ctx: B.Context, q, k, v, src_tok_off, lengths, o, lse, workspace, keep=None, scale: Optional[float] = None,
                           prompt_k=None, prompt_v=None, cu_prompts=None, G: int = 1, stream=None):
    """One token per rollout: q, o [N, Hq, D], caches k, v [cache_rows, Hkv, D] bfloat16, lse float32 [N, Hq] or None."""
    (N, Hq, D), Hkv, cache_rows = q.shape, k.shape[1], k.shape[0]
    q_at, q_stride = _rows(q, N, Hq, D)
    k_at, k_stride = _rows(k, cache_rows, Hkv, D)
    v_at, v_stride = _rows(v, cache_rows, Hkv, D)
    o_at, o_stride = _rows(o, N, Hq, D)
    rows, P, pk, pv, pk_stride, pv_stride, cu_p = _prompts(prompt_k, prompt_v, cu_prompts, Hkv, D)
    a = _Decode(q_at, k_at, v_at, q_stride, k_stride, v_stride, _ints("src_tok_off", src_tok_off, torch.int64, N),
                _ints("lengths", lengths, torch.int32, N), _ints("keep", keep, torch.uint8, N), pk, pv, pk_stride, pv_stride, cu_p, cache_rows,
                rows, N, P, G, Hq, Hkv, D, D ** -0.5 if scale is None else scale, 0, o_at, o_stride, _lse(lse, N, Hq), B._ptr(workspace),
                _bytes(workspace))
    B._check(_lib().arrol_attention_decode(ctx.handle, C.byref(a), B._stream(stream)), "arrol_attention_decode")
