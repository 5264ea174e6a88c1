"""Attention with results that are slices of wider rows, rows whose offsets pass 2^32 elements, and index lists that name a rollout more than once."""
import math

import pytest
import torch

from paper_2603_24840_b200 import attention as A
from paper_2603_24840_b200 import binding as B
from test_gpu_attention import Problem
from test_gpu_attention_decode import Problem as Decode

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("D,Hq,Hkv", [(64, 8, 2), (128, 4, 4), (40, 6, 1)])
def test_results_are_slices_of_wider_rows(ctx, D, Hq, Hkv):
    """What lies between the slices, and behind the live rows, stays as it was."""
    for lens, prompts in (([100, 3, 190], [65, 40]), ([20, 30], [3000, 700])):         # whole keys; split keys
        p = Problem(lens, prompts, list(range(len(lens))), 2, Hq, Hkv, D, seed=60, spare=9)
        want = p.run(ctx)
        rows, shared = p.q.shape[0], p.pk.shape[0]
        wide, wide_o, wide_p = [torch.full((n, w, D), -7.0, dtype=BF, device="cuda") for n, w in
                                ((rows, Hq + 2 * Hkv + 3), (rows, Hq + 2), (shared, 2 * Hkv + 1))]
        out = {"o": wide_o[:, 1:1 + Hq], "lse": want["lse"].clone().fill_(-7.0), "dq": wide[:, :Hq], "dk": wide[:, Hq + 1:Hq + 1 + Hkv], "dv": wide[:, Hq + 3 + Hkv:],
               "dprompt_k": wide_p[:, :Hkv], "dprompt_v": wide_p[:, Hkv + 1:]}
        ws = p.workspace(ctx)
        p.forward(ctx, out, ws)
        p.backward(ctx, out, ws)
        torch.cuda.synchronize()
        assert B.arrol_poll_status(ctx) == 0
        for name in want:
            assert torch.equal(out[name], want[name]), name
        gaps = [wide_o[:, :1], wide_o[:, 1 + Hq:], wide[:, Hq:Hq + 1], wide[:, Hq + 1 + Hkv:Hq + 3 + Hkv], wide_p[:, Hkv:Hkv + 1]]
        assert all((g.float() == -7).all() for g in gaps)


def _far(stride, rows, *parts):
    """Slices [rows, heads, D] of one buffer whose rows lie `stride` elements apart."""
    buffer = torch.empty(stride * rows, dtype=BF, device="cuda").view(rows, stride)
    out, at = [], 0
    for heads, D in parts:
        out.append(buffer[:, at:at + heads * D].unflatten(1, (heads, D)))
        at += heads * D
    return out


@pytest.mark.parametrize("D", [64, 128])
def test_offsets_beyond_32_bits(ctx, D):
    """Rows 2^22 elements apart: the 1,100 of them reach past 2^32 elements and 2^33 bytes, for every input and result, and for a generation step's cache."""
    Hq, Hkv, spare = 4, 2, 5
    near = Problem([700, 395], [900, 100], [0, 1], 1, Hq, Hkv, D, seed=61, spare=spare)
    want = near.run(ctx)
    far, rows, shared = Problem([700, 395], [900, 100], [0, 1], 1, Hq, Hkv, D, seed=61, spare=spare), near.q.shape[0], near.pk.shape[0]
    x = _far(1 << 22, rows, (Hq, D), (Hkv, D), (Hkv, D), (Hq, D), (Hq, D), (Hq, D), (Hkv, D), (Hkv, D), (Hkv, D), (Hkv, D), (Hkv, D), (Hkv, D))
    far.q, far.k, far.v, far.d_o = x[:4]
    far.pk, far.pv = x[8][:shared], x[9][:shared]
    for n in ("q", "k", "v", "d_o", "pk", "pv"):
        getattr(far, n).copy_(getattr(near, n))
    out = {"o": x[4], "lse": want["lse"].clone().fill_(-7.0), "dq": x[5], "dk": x[6], "dv": x[7], "dprompt_k": x[10][:shared], "dprompt_v": x[11][:shared]}
    for n, t in out.items():
        t.fill_(-7.0)
    ws = far.workspace(ctx)
    far.forward(ctx, out, ws)
    far.backward(ctx, out, ws)
    torch.cuda.synchronize()
    assert B.arrol_poll_status(ctx) == 0
    for n in want:
        assert torch.equal(out[n], want[n]), n

    d = Decode([500, 3, 590], [300, 0, 700], 1, Hq, Hkv, D, seed=62, gap=0)
    o, lse = d.run(ctx)
    q, k, v, pk, pv, o2 = _far(1 << 22, 1100, (Hq, D), (Hkv, D), (Hkv, D), (Hkv, D), (Hkv, D), (Hq, D))
    k, v, pk, pv = k[:1093], v[:1093], pk[:1000], pv[:1000]
    for a, b in ((k, d.k), (v, d.v), (pk, d.pk), (pv, d.pv)):
        a.copy_(b)
    q, o2 = q[::500], o2[::500]                 # three rows, 2^31 elements apart
    q.copy_(d.q)
    lse2 = torch.full_like(lse, -7.0)
    A.arrol_attention_decode(ctx, q, k, v, d.d_off, d.d_len, o2, lse2, d.workspace(ctx), scale=d.scale, G=1, prompt_k=pk, prompt_v=pv, cu_prompts=d.d_cup)
    torch.cuda.synchronize()
    assert B.arrol_poll_status(ctx) == 0
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("D", [64, 128])
def test_a_rollout_that_is_named_more_than_once(ctx, D):
    """survivor_idx must not decrease; equal entries are survivors of one prompt like others."""
    p = Problem([60, 0, 150, 60, 33], [70, 90, 20], [1, 1, 2, 2, 5], 2, 4, 2, D, seed=63)
    out = p.run(ctx)
    p.check(out)
    assert (out["dprompt_k"][160:].float().abs().sum() > 0) and math.isfinite(out["lse"].sum().item())
