"""Attention of packed sequences over shared prompts in 64 bits, from the definition: one sequence, one key head at a time.  Returns results and,
beside each, how far a kernel may be from it that computes in fp32 and rounds to bf16 what the interface says it rounds."""
import math

import torch

BF16 = 2.0 ** -8       # half a step of bf16, relative
F32 = 2.0 ** -13       # products' sums over D and over keys, exponentials and logarithms in fp32: far above a few hundred half steps of 2^-24


def sequences(cu_seqlens, survivor_idx, G, cu_prompts):
    """[(first row, rows, prompt's first row, prompt's rows)]"""
    out = []
    for s in range(len(cu_seqlens) - 1):
        p = (survivor_idx[s] if survivor_idx is not None else s) // G
        a, b = (cu_prompts[p], cu_prompts[p + 1]) if cu_prompts is not None else (0, 0)
        out.append((cu_seqlens[s], cu_seqlens[s + 1] - cu_seqlens[s], a, b - a))
    return out


def _one(q, key, val, scale, allowed):
    """q [r, m, D], key, val [n, D] -> probabilities, o, lse and o's bound."""
    z = scale * (q @ key.T)
    z = torch.where(allowed, z, -math.inf)
    m = z.max(-1, keepdim=True).values
    m = torch.where(m == -math.inf, 0.0, m)
    e = torch.exp(z - m)
    total = e.sum(-1, keepdim=True)
    p = torch.where(total > 0, e / total, 0.0)
    o, spread = p @ val, p @ val.abs()
    # o is rounded; so is every probability before the product with v
    return p, o, (m + total.log()).squeeze(-1), BF16 * o.abs() + (BF16 + F32) * spread


def packed(q, k, v, pk, pv, seqs, scale, d_o=None):
    """Rows of bf16 tensors in 64 bits.  {"o", "lse"[, "dq", "dk", "dv", "dpk", "dpv"]}, and the same names with bounds."""
    f64 = lambda t: None if t is None else t.double()  # noqa: E731
    q, k, v, pk, pv, d_o = map(f64, (q, k, v, pk, pv, d_o))
    (T, Hq, D), Hkv = q.shape, k.shape[1]
    r = Hq // Hkv
    zeros = lambda t: torch.zeros_like(t)  # noqa: E731
    res = {"o": zeros(q), "lse": torch.zeros(T, Hq, dtype=torch.float64, device=q.device)}
    if d_o is not None:
        res |= {"dq": zeros(q), "dk": zeros(k), "dv": zeros(v)}
        if pk is not None:
            res |= {"dpk": zeros(pk), "dpv": zeros(pv)}
    tol = {n: zeros(t) for n, t in res.items()}
    for row, n, a, shared in seqs:
        if n == 0:
            continue
        own = slice(row, row + n)
        allowed = torch.ones(n, shared + n, dtype=torch.bool, device=q.device).tril(shared)
        for g in range(Hkv):
            hs = slice(g * r, (g + 1) * r)
            key, val = k[own, g], v[own, g]
            if shared:
                key, val = torch.cat([pk[a:a + shared, g], key]), torch.cat([pv[a:a + shared, g], val])
            qq = q[own, hs].transpose(0, 1)
            p, o, lse, o_tol = _one(qq, key, val, scale, allowed)
            res["o"][own, hs], tol["o"][own, hs] = o.transpose(0, 1), o_tol.transpose(0, 1)
            res["lse"][own, hs] = lse.T
            tol["lse"][own, hs] = (2e-5 * (1 + lse.abs())).T
            if d_o is None:
                continue
            go = d_o[own, hs].transpose(0, 1)
            dp = go @ val.T
            ds = p * (dp - (go * o).sum(-1, keepdim=True))
            # ds is rounded; d_o . o is that of the o that was written; the rest is fp32
            delta_tol = (go.abs() * o_tol).sum(-1, keepdim=True)
            ds_tol = BF16 * ds.abs() + (1 + BF16) * p * (delta_tol + F32 * (go.abs() @ val.abs().T + (go * o).abs().sum(-1, keepdim=True)))
            dq = scale * (ds @ key)
            res["dq"][own, hs] = dq.transpose(0, 1)
            tol["dq"][own, hs] = (BF16 * dq.abs() + scale * (ds_tol @ key.abs()) + 1e-30).transpose(0, 1)
            flat = lambda t: t.reshape(-1, t.shape[-1])  # noqa: E731
            dk, dk_tol = scale * (flat(ds).T @ flat(qq)), scale * (flat(ds_tol).T @ flat(qq).abs())
            dv, dv_tol = flat(p).T @ flat(go), (BF16 + F32) * (flat(p).T @ flat(go).abs())
            for name, x, t in (("k", dk, dk_tol), ("v", dv, dv_tol)):
                res["d" + name][own, g] = x[shared:]
                tol["d" + name][own, g] = t[shared:]
                if shared:
                    res["dp" + name][a:a + shared, g] += x[:shared]
                    tol["dp" + name][a:a + shared, g] += t[:shared]
    for name in ("dk", "dv", "dpk", "dpv"):
        if name in res:
            tol[name] += BF16 * res[name].abs() + 1e-30
    return res, tol


def decode(q, k, v, off, lengths, keep, pk, pv, cu_prompts, G, scale):
    """One row per rollout; rows that are not kept: zeros."""
    q, k, v = q.double(), k.double(), v.double()
    (N, Hq, D), Hkv = q.shape, k.shape[1]
    r = Hq // Hkv
    o, lse = torch.zeros_like(q), torch.zeros(N, Hq, dtype=torch.float64, device=q.device)
    o_tol = torch.zeros_like(q)
    for i in range(N):
        if keep is not None and not keep[i]:
            continue
        for g in range(Hkv):
            key, val = k[off[i]:off[i] + lengths[i], g], v[off[i]:off[i] + lengths[i], g]
            if cu_prompts is not None:
                a, b = cu_prompts[i // G], cu_prompts[i // G + 1]
                key, val = torch.cat([pk[a:b, g].double(), key]), torch.cat([pv[a:b, g].double(), val])
            hs = slice(g * r, (g + 1) * r)
            if key.shape[0] == 0:
                lse[i, hs] = -math.inf
                continue
            allowed = torch.ones(1, key.shape[0], dtype=torch.bool, device=q.device)
            _, oo, ll, tt = _one(q[i, hs].unsqueeze(1), key, val, scale, allowed)
            o[i, hs], o_tol[i, hs], lse[i, hs] = oo[:, 0], tt[:, 0], ll[:, 0]
    return o, o_tol, lse
