"""CPU-only checks around the attention calls: the 64-bit reference that the GPU tests use, and the calls' refusals, which come before anything
touches a device."""
import ctypes as C
import math

import pytest
import torch

import attention_reference as R
from paper_2603_24840_b200 import attention as A
from paper_2603_24840_b200 import build as libbuild


@pytest.fixture(scope="module")
def lib():
    libbuild.build()
    return A._lib()


def _problem(seed, D=5, Hq=4, Hkv=2):
    g = torch.Generator().manual_seed(seed)
    mk = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    cu, idx, G, cup = [0, 3, 3, 7, 8], [0, 1, 5, 7], 4, [0, 4, 6]
    seqs = R.sequences(cu, idx, G, cup)
    assert seqs == [(0, 3, 0, 4), (3, 0, 0, 4), (3, 4, 4, 2), (7, 1, 4, 2)]
    return mk(8, Hq, D), mk(8, Hkv, D), mk(8, Hkv, D), mk(6, Hkv, D), mk(6, Hkv, D), seqs, mk(8, Hq, D)


def test_reference_agrees_with_a_softmax_over_the_whole_batch():
    q, k, v, pk, pv, seqs, _ = _problem(0)
    res, _ = R.packed(q, k, v, pk, pv, seqs, 0.3)
    key, val = torch.cat([pk, k]).repeat_interleave(2, 1), torch.cat([pv, v]).repeat_interleave(2, 1)
    see = torch.zeros(8, 14, dtype=torch.bool)
    for row, n, a, shared in seqs:
        for t in range(n):
            see[row + t, a:a + shared] = True
            see[row + t, 6 + row:6 + row + t + 1] = True
    z = torch.einsum("thd,jhd->htj", q, key) * 0.3
    z = z.masked_fill(~see, -math.inf)
    o = torch.einsum("htj,jhd->thd", torch.softmax(z, -1), val)
    assert torch.allclose(res["o"], o, atol=1e-12) and torch.allclose(res["lse"], torch.logsumexp(z, -1).T, atol=1e-12)


@pytest.mark.parametrize("name", ["q", "k", "v", "pk", "pv"])
def test_reference_gradients_agree_with_differences(name):
    q, k, v, pk, pv, seqs, d_o = _problem(1)
    args = {"q": q, "k": k, "v": v, "pk": pk, "pv": pv}
    grad = R.packed(**args, seqs=seqs, scale=0.4, d_o=d_o)[0]["d" + name]
    x, h = args[name], 1e-5
    for at in torch.randperm(x.numel(), generator=torch.Generator().manual_seed(2))[:12].tolist():
        f = []
        for step in (h, -h):
            y = x.clone()
            y.view(-1)[at] += step
            f.append((R.packed(**{**args, name: y}, seqs=seqs, scale=0.4)[0]["o"] * d_o).sum().item())
        assert abs((f[0] - f[1]) / (2 * h) - grad.view(-1)[at].item()) < 1e-7


def test_decode_reference_is_the_last_row_of_the_packed_one():
    q, k, v, pk, pv, seqs, _ = _problem(3)
    res, _ = R.packed(q, k, v, pk, pv, seqs, 0.5)
    last = [2, 6, 7]
    off, lengths, which = [0, 3, 7], [3, 4, 1], [0, 1, 1]
    for i in range(3):
        o, _, lse = R.decode(q[last[i]:last[i] + 1], k, v, [off[i]], [lengths[i]], None, pk, pv, [[0, 4], [4, 6]][which[i]], 1, 0.5)
        assert torch.allclose(o[0], res["o"][last[i]], atol=1e-12) and torch.allclose(lse[0], res["lse"][last[i]], atol=1e-12)
    o, _, lse = R.decode(q[:1], k, v, [0], [0], None, pk, pv, [0, 0], 1, 0.5)
    assert not o.any() and (lse == -math.inf).all()


# ---- refusals: the context is never looked at, so a block of zeros stands for it ---------------------------------------------------

ADDR = 1 << 20        # an aligned address that nothing follows


def _ctx():
    return C.create_string_buffer(1 << 16)


def _packed_args(**over):
    a = A._Attention()
    for n in ("q", "k", "v", "cu_seqlens", "d_num", "prompt_k", "prompt_v", "cu_prompts", "o", "lse", "d_o", "dq", "dk", "dv", "dprompt_k", "dprompt_v", "workspace"):
        setattr(a, n, ADDR)
    for n in ("q", "k", "v", "prompt_k", "prompt_v", "o", "d_o", "dq", "dk", "dv", "dprompt_k", "dprompt_v"):
        setattr(a, n + "_stride", 8 * 64)
    a.T_max, a.prompt_rows, a.S_max, a.P, a.G, a.Hq, a.Hkv, a.D, a.scale = 100, 10, 4, 2, 4, 8, 4, 64, 0.125
    for n, x in over.items():
        setattr(a, n, x)
    return a


PACKED_REFUSALS = [
    (dict(q=None), -1), (dict(k=ADDR + 8), -1), (dict(v_stride=4 * 64 - 8), -1), (dict(q_stride=8 * 64 + 4), -1), (dict(o=None), -1), (dict(lse=None), -1),
    (dict(cu_seqlens=None), -1), (dict(d_num=None), -1), (dict(prompt_k=None), -1), (dict(cu_prompts=None), -1), (dict(prompt_v_stride=0), -1),
    (dict(P=0), -1), (dict(T_max=-1), -1), (dict(S_max=-1), -1), (dict(prompt_rows=-1), -1), (dict(G=0), -1), (dict(Hq=6), -1), (dict(Hkv=0), -1),
    (dict(scale=0.0), -1), (dict(scale=-1.0), -1), (dict(scale=math.nan), -1), (dict(scale=math.inf), -1),
    (dict(D=136, Hq=4), -2), (dict(D=60), -2), (dict(D=4), -2), (dict(Hq=65, Hkv=1), -2), (dict(T_max=(1 << 31) - 512), -2), (dict(prompt_rows=1 << 32), -2),
    (dict(workspace=None), -3), (dict(workspace=ADDR + 16), -3), (dict(workspace_bytes=255), -3),
]


@pytest.mark.parametrize("over,code", PACKED_REFUSALS)
@pytest.mark.parametrize("call", ["arrol_attention", "arrol_attention_backward"])
def test_packed_calls_refuse(lib, call, over, code):
    assert getattr(lib, call)(_ctx(), C.byref(_packed_args(**over)), None) == code


@pytest.mark.parametrize("name", ["d_o", "dq", "dk", "dv", "dprompt_k", "dprompt_v"])
def test_backward_refuses_missing_and_misaligned_gradients(lib, name):
    for over in ({name: None}, {name: ADDR + 8}, {name + "_stride": 8}, {name + "_stride": 8 * 64 + 1}):
        assert lib.arrol_attention_backward(_ctx(), C.byref(_packed_args(**over)), None) == -1


def test_null_contexts_and_empty_calls(lib):
    null = C.c_void_p()
    assert lib.arrol_attention(null, C.byref(_packed_args()), None) == -1
    assert lib.arrol_attention(_ctx(), None, None) == -1
    assert lib.arrol_attention_backward(null, None, None) == -1
    assert lib.arrol_attention_decode(null, None, None) == -1
    assert lib.arrol_attention_workspace(null, 1, 1, 0, 8, 4, 64, 0) == 0
    assert lib.arrol_attention_decode_workspace(null, 1, 0, 8, 4, 64) == 0
    empty = A._Attention(S_max=0, G=1, Hq=8, Hkv=4, D=64, scale=1.0)
    assert lib.arrol_attention(_ctx(), C.byref(empty), None) == 0 and lib.arrol_attention_backward(_ctx(), C.byref(empty), None) == 0
    assert lib.arrol_attention_decode(_ctx(), C.byref(A._Decode(G=1, Hq=8, Hkv=4, D=64, scale=1.0)), None) == 0


def _decode_args(**over):
    a = A._Decode()
    for n in ("q", "k", "v", "src_tok_off", "lengths", "keep", "prompt_k", "prompt_v", "cu_prompts", "o", "lse", "workspace"):
        setattr(a, n, ADDR)
    for n in ("q", "k", "v", "prompt_k", "prompt_v", "o"):
        setattr(a, n + "_stride", 8 * 64)
    a.cache_rows, a.prompt_rows, a.N, a.P, a.G, a.Hq, a.Hkv, a.D, a.scale = 100, 10, 8, 2, 4, 8, 4, 64, 0.125
    for n, x in over.items():
        setattr(a, n, x)
    return a


@pytest.mark.parametrize("over,code", [
    (dict(q=None), -1), (dict(k=None), -1), (dict(v=ADDR + 2), -1), (dict(o_stride=8), -1), (dict(src_tok_off=None), -1), (dict(lengths=None), -1),
    (dict(prompt_k=None), -1), (dict(cu_prompts=None), -1), (dict(N=9), -1), (dict(G=0), -1), (dict(P=0), -1), (dict(N=-1), -1), (dict(cache_rows=-1), -1),
    (dict(scale=0.0), -1), (dict(Hq=7), -1), (dict(D=132, Hq=4), -2), (dict(G=1025, N=2050), -2), (dict(cache_rows=1 << 31), -2), (dict(Hq=65, Hkv=1), -2),
    (dict(workspace=None), -3), (dict(workspace=ADDR + 128), -3), (dict(workspace_bytes=0), -3)])
def test_decode_refuses(lib, over, code):
    assert lib.arrol_attention_decode(_ctx(), C.byref(_decode_args(**over)), None) == code


def test_binding_refuses_other_layouts():
    q = torch.zeros(4, 8, 64, dtype=torch.bfloat16)
    assert A._rows(q[:, :4], 4, 4, 64) == (q.data_ptr(), 8 * 64)            # heads of a wider row
    assert A._rows(q[:1, :4], 1, 4, 64)[1] >= 4 * 64
    assert A._rows(q[:, :1], 4, 1, 64) == (q.data_ptr(), 8 * 64)
    assert A._rows(None, 4, 8, 64) == (None, 0)
    for bad in (q.transpose(0, 1), q[:, ::2], q[..., ::2], q.view(4, -1)):
        with pytest.raises(ValueError):
            A._rows(bad, bad.shape[0], bad.shape[1], bad.shape[-1])
    with pytest.raises(ValueError):
        A._rows(q, 5, 8, 64)                                                # fewer rows than its counterpart
    with pytest.raises(ValueError):
        A._rows(q, 4, 4, 64)
    with pytest.raises(TypeError):
        A._rows(q.float(), 4, 8, 64)
    with pytest.raises(ValueError):
        A._lse(torch.zeros(3, 8), 4, 8)
    with pytest.raises(ValueError):
        A._ints("lengths", torch.zeros(3, dtype=torch.int32), torch.int32, 4)
    with pytest.raises(ValueError):
        A._ints("lengths", torch.zeros(4, dtype=torch.int64), torch.int32, 4)


def test_binding_refuses_prompts_in_part():
    class Ctx:
        handle = 0

    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    q, k, lse = bf(4, 4, 64), bf(4, 2, 64), torch.zeros(4, 4)
    cu, num, ws = torch.tensor([0, 4]), torch.tensor([1, 4]), torch.zeros(1 << 12, dtype=torch.uint8)
    pk, cup = bf(6, 2, 64), torch.tensor([0, 6])
    for prompts in (dict(prompt_k=pk, prompt_v=pk), dict(prompt_k=pk, cu_prompts=cup), dict(prompt_v=pk, cu_prompts=cup), dict(prompt_v=pk)):
        with pytest.raises(ValueError):
            A.arrol_attention(Ctx, q, k, k, cu, num, q, lse, ws, **prompts)
        with pytest.raises(ValueError):
            A.arrol_attention_decode(Ctx, q, k, k, torch.zeros(4, dtype=torch.int64), torch.zeros(4, dtype=torch.int32), q, lse, ws, G=4, **prompts)


def test_binding_refuses_what_belongs_to_prompts_without_them():
    class Ctx:
        handle = 0

    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    q, k, lse = bf(4, 4, 64), bf(4, 2, 64), torch.zeros(4, 4)
    cu, num, ws = torch.tensor([0, 4]), torch.tensor([1, 4]), torch.zeros(1 << 12, dtype=torch.uint8)
    pk, cup = bf(6, 2, 64), torch.tensor([0, 6])
    with pytest.raises(ValueError):
        A.arrol_attention(Ctx, q, k, k, cu, num, q, lse, ws, cu_prompts=cup)
    with pytest.raises(ValueError):
        A.arrol_attention_decode(Ctx, q, k, k, torch.zeros(4, dtype=torch.int64), torch.zeros(4, dtype=torch.int32), q, lse, ws, G=4, cu_prompts=cup)
    for prompts in (dict(cu_prompts=cup), dict(dprompt_k=pk), dict(dprompt_v=pk), dict(dprompt_k=pk, dprompt_v=pk)):
        with pytest.raises(ValueError):
            A.arrol_attention_backward(Ctx, q, k, k, cu, num, q, lse, q, q, k, k, ws, **prompts)
