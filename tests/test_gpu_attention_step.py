"""The attention calls where they are used: generation up to the prune step, the re-batched survivors' forward and backward around the lm_head."""
import math

import pytest
import torch

import attention_reference as R
from paper_2603_24840_b200 import attention as A
from paper_2603_24840_b200 import binding as B
from paper_2603_24840_b200 import update as U

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def test_prune_attend_score_and_back():
    """keep from arrol_select, the survivors packed by arrol_compact, attention over its outputs as they lie on the device, log-probs of the result,
    policy loss, lm_head backward, attention backward.  Then the same rollouts' generation step at the cut, with the same mask."""
    ctx = B.Context(0)
    P, G, K, Hq, Hkv, D, V = 3, 4, 2, 4, 2, 64, 512
    N, d, scale = P * G, Hq * D, 1 / math.sqrt(D)
    g = torch.Generator("cuda").manual_seed(0)
    mk = lambda *s, by=1.0: (torch.randn(*s, generator=g, device="cuda") * by).to(BF)  # noqa: E731
    ints = lambda v, t: torch.tensor(v, dtype=t, device="cuda")  # noqa: E731
    lengths = [40, 70, 33, 129, 90, 64, 65, 200, 31, 77, 150, 101]
    off, cap = [0], 0
    for n in lengths:
        off.append(off[-1] + n)
    cap = sum(sorted(lengths, reverse=True)[:P * K])
    prompts = [50, 0, 130]
    cup = [0, 50, 50, 180]
    # per source token: queries, keys and values side by side, one row of arrol_compact's row plane
    width = (Hq + 2 * Hkv) * D
    src = mk(off[-1], width)
    src_tokens = torch.randint(0, V, (off[-1],), generator=g, device="cuda", dtype=torch.int32)
    pk, pv, W = mk(180, Hkv, D), mk(180, Hkv, D), mk(V, d, by=0.05)
    q_score, rewards = torch.rand(N, generator=g, device="cuda"), ints([1, 0] * 6, torch.float32)
    d_len, d_off, d_cup = ints(lengths, torch.int32), ints(off[:-1], torch.int64), ints(cup, torch.int64)
    keep = torch.empty(N, dtype=torch.uint8, device="cuda")
    B.arrol_select(ctx, q_score, P, G, K, 0.5, keep)
    cu = torch.full((N + 1,), -1, dtype=torch.int64, device="cuda")
    idx = torch.full((N,), -1, dtype=torch.int32, device="cuda")
    adv, num = torch.empty(N, device="cuda"), torch.empty(2, dtype=torch.int64, device="cuda")
    rows = torch.full((cap, width), math.nan, dtype=BF, device="cuda")
    toks = torch.empty(cap, dtype=torch.int32, device="cuda")
    tok_adv, tok_seq = torch.empty(cap, device="cuda"), torch.empty(cap, dtype=torch.int32, device="cuda")
    B.arrol_compact(ctx, keep, d_len, d_off, N, G, rewards, cap, cu, idx, adv, num, src_tokens=src_tokens, dst_tokens=toks, src_rows=src, dst_rows=rows,
                    row_bytes=width * 2, tok_adv=tok_adv, tok_seq=tok_seq)
    qkv = rows.view(cap, Hq + 2 * Hkv, D)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    o, lse = torch.zeros(cap, Hq, D, dtype=BF, device="cuda"), torch.zeros(cap, Hq, device="cuda")
    ws = torch.empty(A.arrol_attention_workspace(ctx, N, cap, 180, Hq, Hkv, D, backward=True), dtype=torch.uint8, device="cuda")
    shared = dict(prompt_k=pk, prompt_v=pv, cu_prompts=d_cup, survivor_idx=idx, G=G, scale=scale)
    A.arrol_attention(ctx, q, k, v, cu, num, o, lse, ws, **shared)
    # log-probs, loss and lm_head backward of the attention's output, T on the device
    d_T = num[1:]
    logp, lse_v = torch.zeros(cap, device="cuda"), torch.zeros(cap, device="cuda")
    ws2 = torch.empty(B.arrol_token_logprob_workspace(ctx, cap, d, V), dtype=torch.uint8, device="cuda")
    B.arrol_token_logprob(ctx, o.view(cap, d), W, toks, cap, d, V, logp, ws2, lse=lse_v, d_T=d_T)
    grad, loss = torch.zeros(cap, device="cuda"), torch.zeros(1, dtype=torch.float64, device="cuda")
    U.arrol_policy_loss(ctx, logp, logp - 0.01, tok_adv, tok_seq, cu, num, cap, grad, loss)
    dH, dW = torch.zeros(cap, d, device="cuda"), torch.empty(V, d, device="cuda")
    ws3 = torch.empty(U.arrol_lm_head_backward_workspace(ctx, cap, d, V), dtype=torch.uint8, device="cuda")
    U.arrol_lm_head_backward(ctx, o.view(cap, d), W, toks, grad, lse_v, cap, d, V, dH, dW, ws3, d_T=d_T)
    d_o = dH.to(BF).view(cap, Hq, D)
    grads = {"dq": torch.zeros_like(o), "dk": torch.zeros(cap, Hkv, D, dtype=BF, device="cuda"), "dv": torch.zeros(cap, Hkv, D, dtype=BF, device="cuda"),
             "dprompt_k": torch.empty_like(pk), "dprompt_v": torch.empty_like(pv)}
    A.arrol_attention_backward(ctx, q, k, v, cu, num, o, lse, d_o, workspace=ws, **shared, **grads)
    torch.cuda.synchronize()
    assert B.arrol_poll_status(ctx) == 0

    S, T = num.tolist()
    assert S == P * K and keep.view(P, G).sum(1).tolist() == [K] * P and T < cap
    seqs = R.sequences(cu[:S + 1].tolist(), idx[:S].tolist(), G, cup)
    res, tol = R.packed(q[:T], k[:T], v[:T], pk, pv, seqs, scale, d_o[:T])
    for name, ref, x in (("o", "o", o), ("dq", "dq", grads["dq"]), ("dk", "dk", grads["dk"]), ("dv", "dv", grads["dv"])):
        assert ((x[:T].double() - res[ref]).abs() <= tol[ref]).all(), name
        assert (x[T:] == 0).all(), name
    for name, ref in (("dprompt_k", "dpk"), ("dprompt_v", "dpv")):
        assert ((grads[name].double() - res[ref]).abs() <= tol[ref]).all(), name
    z = o[:T].view(T, d).double() @ W.double().T
    want = torch.log_softmax(z, -1).gather(1, toks[:T, None].long())[:, 0]
    assert (logp[:T].double() - want).abs().max() <= 2e-3

    # generation at the cut: every live rollout's token at the cut attends to its prompt and to its own tokens so far
    cut = 30
    at = d_off + cut - 1
    all_qkv = src.view(-1, Hq + 2 * Hkv, D)
    q1 = all_qkv[at, :Hq].contiguous()
    o1, lse1 = torch.zeros(N, Hq, D, dtype=BF, device="cuda"), torch.zeros(N, Hq, device="cuda")
    ws4 = torch.empty(A.arrol_attention_decode_workspace(ctx, N, P, Hq, Hkv, D), dtype=torch.uint8, device="cuda")
    A.arrol_attention_decode(ctx, q1, all_qkv[:, Hq:Hq + Hkv], all_qkv[:, Hq + Hkv:], d_off, torch.full_like(d_len, cut), o1, lse1, ws4, keep=keep, scale=scale,
                             prompt_k=pk, prompt_v=pv, cu_prompts=d_cup, G=G)
    torch.cuda.synchronize()
    assert B.arrol_poll_status(ctx) == 0
    assert (o1[keep == 0] == 0).all()
    for s in range(S):          # the packed forward's row of the same token: both within their bounds of the same value
        i, r = idx[s].item(), cu[s].item() + cut - 1
        assert ((o1[i].double() - o[r].double()).abs() <= 2 * tol["o"][r]).all()
        assert (lse1[i] - lse[r]).abs().max() <= 1e-4
    ctx.close()
