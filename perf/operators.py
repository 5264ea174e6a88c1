"""Performance cases of the attention operators: what a training loop and a generation loop around the prune step ask of them.

Three kinds of pass, each over the range of sizes that its callers have:

  attend   attention of the packed survivors over their prompts and their own tokens (forward; old- or reference-policy scoring)
  train    the same with its gradients with respect to queries, keys, values and the shared prompts' keys and values
  decode   one generated token per rollout over the key/value cache, prompts shared by their group's rollouts

The head layouts are generic ones of grouped-query models; lengths, prompts and group sizes are those of the package's workloads.
"""
from __future__ import annotations

import functools
import math
import random

import torch

own = False

MAX_PAIRS_ATTEND = 2.2e9     # query-head x padded row x padded key products of one pass: bounds time and the plain form's memory
MAX_PAIRS_TRAIN = 1.1e9
MAX_CACHE_BYTES = 2.4e9      # keys and values that one generation step reads


def listed():
    return [
        # A debugging-size step: 4 prompts x 4 survivors of a hundred tokens or two, no grouping. Launches count.
        _packed("attend", "attend-tiny", P=4, G=8, K=4, lo=96, hi=256, plo=17, phi=90, Hq=8, Hkv=8, D=64),
        # A micro-batch of survivors with the smaller head size: 4 prompts x 4 survivors of 512 to 2,048 tokens.
        _packed("attend", "attend-d64", P=4, G=8, K=4, lo=512, hi=2048, plo=120, phi=700, Hq=32, Hkv=8, D=64),
        # Many short answers to long prompts: almost all of the work is on the shared part.
        _packed("attend", "attend-long-prompts", P=6, G=16, K=8, lo=40, hi=333, plo=1500, phi=4000, Hq=28, Hkv=4, D=128),
        # One long document without a prompt: evaluation, or the prompts' own pass.
        _packed("attend", "attend-8k", P=1, G=1, K=1, lo=8192, hi=8192, plo=0, phi=0, Hq=32, Hkv=8, D=128),
        # Training, debugging size.
        _packed("train", "train-tiny", P=2, G=8, K=4, lo=33, hi=190, plo=20, phi=70, Hq=4, Hkv=2, D=64),
        # Training micro-batch of the group size 16, keep 8 workloads: two prompts, 16 query heads on 8.
        _packed("train", "train-d128", P=2, G=16, K=8, lo=300, hi=1900, plo=100, phi=500, Hq=16, Hkv=8, D=128),
        # Two long rollouts of one prompt, groups of four heads.
        _packed("train", "train-4k", P=1, G=8, K=2, lo=3900, hi=4096, plo=211, phi=211, Hq=32, Hkv=8, D=128),
        # Training with the smaller head size and a head ratio that divides no power of two.
        _packed("train", "train-d64-r3", P=3, G=8, K=4, lo=200, hi=1500, plo=64, phi=400, Hq=24, Hkv=8, D=64),
        # Generation, a few rollouts at the start of their answers: latency.
        _decode("decode-tiny", P=2, G=8, lo=1, hi=60, plo=40, phi=200, Hq=8, Hkv=2, D=64, kept=1.0),
        # One prompt of 16 rollouts that have long answers: too few rows to fill the GPU without splitting the cache.
        _decode("decode-one-group", P=1, G=16, lo=5000, hi=8192, plo=2000, phi=2000, Hq=32, Hkv=8, D=128, kept=0.5),
        # Generation of a whole batch after the prune step: half of the rollouts live, ragged answers.
        _decode("decode-batch", P=32, G=16, lo=300, hi=4096, plo=100, phi=1000, Hq=16, Hkv=8, D=128, kept=0.5),
        # Short answers to long shared prompts, before anything is pruned.
        _decode("decode-long-prompts", P=24, G=16, lo=20, hi=300, plo=3000, phi=8192, Hq=32, Hkv=8, D=64, kept=1.0),
    ]


def _packed(kind, name, **sizes):
    return {"kind": kind, "name": name, "layout": 1, **sizes}


def _decode(name, **sizes):
    return {"kind": "decode", "name": name, "layout": 1, **sizes}


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["attend", "train", "decode"])
        Hkv, D = rng.choice([1, 2, 4, 8]), rng.choice([64, 64, 96, 128, 128])
        case = {"kind": kind, "layout": rng.randrange(1 << 20), "P": _log_uniform(rng, 1, 24), "G": rng.choice([4, 8, 16]), "Hq": Hkv * rng.randint(1, 8), "Hkv": Hkv, "D": D}
        hi, phi = _log_uniform(rng, 16, 8192), _log_uniform(rng, 1, 6000)
        case |= {"lo": rng.randint(1, hi), "hi": hi, "plo": rng.randint(0, phi), "phi": phi}
        if kind == "decode":
            case["kept"] = rng.choice([0.25, 0.5, 1.0])
            if work(case)["bytes"] <= MAX_CACHE_BYTES and case["P"] * case["G"] * (hi + phi) * Hkv * D <= MAX_CACHE_BYTES:
                return case
        else:
            case["K"] = rng.randint(1, case["G"])
            lens, prompts, _ = _layout(case)
            padded = len(lens) * case["Hq"] * max(lens) * (max(lens) + max(prompts))
            if padded <= (MAX_PAIRS_ATTEND if kind == "attend" else MAX_PAIRS_TRAIN) and sum(lens) * case["Hq"] * D <= 3e8:
                return case


def _layout(case):
    """Lengths, prompt lengths and the survivors' numbers (of all rollouts, for `decode`): of the case alone, so that work() knows them."""
    rng = random.Random("%(layout)d %(P)d %(G)d %(lo)d %(hi)d" % case)
    prompts = [rng.randint(case["plo"], case["phi"]) for _ in range(case["P"])]
    if case["kind"] == "decode":
        N = case["P"] * case["G"]
        live = sorted(rng.sample(range(N), max(1, int(round(N * case["kept"])))))
        return [rng.randint(case["lo"], case["hi"]) for _ in range(N)], prompts, live
    index = [p * case["G"] + i for p in range(case["P"]) for i in sorted(rng.sample(range(case["G"]), case["K"]))]
    return [rng.randint(case["lo"], case["hi"]) for _ in index], prompts, index


def _starts(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return at


def prepare(case, seed):
    dev = "cuda"
    lens, prompts, index = _layout(case)
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    gen = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=gen, device=dev) * scale).to(torch.bfloat16)

    def ints(values, dtype):
        return torch.tensor(values, dtype=dtype, device=dev)

    s = {"kind": case["kind"], "G": case["G"], "P": case["P"], "scale": 1.0 / math.sqrt(D), "lens": lens, "prompts": prompts}
    s["cu_prompts"] = ints(_starts(prompts), torch.int64)
    if sum(prompts):
        s["prompt_k"], s["prompt_v"] = normal(sum(prompts), Hkv, D), normal(sum(prompts), Hkv, D)
    else:
        s["prompt_k"] = s["prompt_v"] = None
    # scores spread by about 1.5, as between normalised queries and keys with learned gains
    if case["kind"] == "decode":
        N = len(lens)
        room = [(n + 64) // 64 * 64 for n in lens]                     # a rollout's cache grows in steps of 64 tokens
        s["q"] = normal(N, Hq, D, scale=1.5)
        s["k"], s["v"] = normal(sum(room), Hkv, D), normal(sum(room), Hkv, D)
        s["src_tok_off"] = ints(_starts(room)[:-1], torch.int64)
        s["lengths"] = ints(lens, torch.int32)
        keep = torch.zeros(N, dtype=torch.uint8)
        keep[index] = 1
        s["keep"] = keep.to(dev)
        s["o"] = torch.zeros(N, Hq, D, dtype=torch.bfloat16, device=dev)
        s["lse"] = torch.zeros(N, Hq, device=dev)
        return s
    T = sum(lens)
    s["q"], s["k"], s["v"] = normal(T, Hq, D, scale=1.5), normal(T, Hkv, D), normal(T, Hkv, D)
    s["cu_seqlens"] = ints(_starts(lens), torch.int64)
    s["survivor_idx"] = ints(index, torch.int32)
    s["num"] = ints([len(lens), T], torch.int64)
    if case["kind"] == "train":
        s["do"] = normal(T, Hq, D)
    return s


def run(state):
    return {"attend": _run_attend, "train": _run_train, "decode": _run_decode}[state["kind"]](state)


# ---- the framework's calls ----------------------------------------------------------------------------------------------

@functools.lru_cache(maxsize=None)
def _context():
    from paper_2603_24840_b200 import binding
    return binding.Context(0)


def _own_attend(s):
    from paper_2603_24840_b200 import attention as A
    ctx, q, k = _context(), s["q"], s["k"]
    (T, Hq, D), Hkv, S = q.shape, k.shape[1], len(s["lens"])
    o, lse = torch.empty_like(q), torch.empty(T, Hq, device=q.device)
    rows = 0 if s["prompt_k"] is None else s["prompt_k"].shape[0]
    ws = torch.empty(A.arrol_attention_workspace(ctx, S, T, rows, Hq, Hkv, D, backward=s["kind"] == "train"), dtype=torch.uint8, device=q.device)
    shared = {} if rows == 0 else {"prompt_k": s["prompt_k"], "prompt_v": s["prompt_v"], "cu_prompts": s["cu_prompts"], "survivor_idx": s["survivor_idx"], "G": s["G"]}
    A.arrol_attention(ctx, q, k, s["v"], s["cu_seqlens"], s["num"], o, lse, ws, scale=s["scale"], **shared)
    return o, lse, ws, shared


def _own_train(s):
    from paper_2603_24840_b200 import attention as A
    o, lse, ws, shared = _own_attend(s)
    grads = {"dq": torch.empty_like(s["q"]), "dk": torch.empty_like(s["k"]), "dv": torch.empty_like(s["v"])}
    if shared:
        grads |= {"dprompt_k": torch.empty_like(s["prompt_k"]), "dprompt_v": torch.empty_like(s["prompt_v"])}
    A.arrol_attention_backward(_context(), s["q"], s["k"], s["v"], s["cu_seqlens"], s["num"], o, lse, s["do"], workspace=ws, scale=s["scale"], **shared, **grads)
    return {"o": o, "lse": lse, **grads}


def _own_decode(s):
    from paper_2603_24840_b200 import attention as A
    ctx, (N, Hq, D), Hkv = _context(), s["q"].shape, s["k"].shape[1]
    ws = torch.empty(A.arrol_attention_decode_workspace(ctx, N, s["P"], Hq, Hkv, D), dtype=torch.uint8, device=s["q"].device)
    shared = {} if s["prompt_k"] is None else {"prompt_k": s["prompt_k"], "prompt_v": s["prompt_v"], "cu_prompts": s["cu_prompts"], "G": s["G"]}
    A.arrol_attention_decode(ctx, s["q"], s["k"], s["v"], s["src_tok_off"], s["lengths"], s["o"], s["lse"], ws, keep=s["keep"], scale=s["scale"], **shared)
    return {"o": s["o"], "lse": s["lse"]}


# ---- the plain forms: a padded batch, in 32 bits ------------------------------------------------------------------------

def _padded(rows, starts, lengths, most):
    """[B, most, ...] in 32 bits: `lengths[b]` rows from starts[b] on, zeros behind them."""
    j = torch.arange(most, device=rows.device)
    valid = j[None, :] < lengths[:, None]
    at = torch.where(valid, starts[:, None] + j[None, :], 0)
    return torch.where(valid[..., None, None], rows[at].float(), 0.0), valid


def _keys(s, starts, lengths, prompt_of):
    """Keys and values [B, Hkv, prompt part + own part, D] of each sequence, and which of them there are."""
    most = max(max(s["lens"]), 1)
    k, valid = _padded(s["k"], starts, lengths, most)
    v, _ = _padded(s["v"], starts, lengths, most)
    shared = 0
    if s["prompt_k"] is not None:
        cu = s["cu_prompts"]
        shared = max(s["prompts"])
        pk, pvalid = _padded(s["prompt_k"], cu[:-1], cu[1:] - cu[:-1], shared)
        pv, _ = _padded(s["prompt_v"], cu[:-1], cu[1:] - cu[:-1], shared)
        k, v = torch.cat([pk[prompt_of], k], 1), torch.cat([pv[prompt_of], v], 1)
        valid = torch.cat([pvalid[prompt_of], valid], 1)
    return k.transpose(1, 2), v.transpose(1, 2), valid, shared


def _softmax(z, allowed):
    """Probabilities and the logarithm of the sum; a row with nothing allowed: zeros and minus infinity."""
    z = z.masked_fill(~allowed, -math.inf)
    m = z.amax(-1, keepdim=True)
    m0 = torch.where(m == -math.inf, 0.0, m)
    p = (z - m0).exp_()
    total = p.sum(-1, keepdim=True)
    return p / torch.where(total == 0, 1.0, total), (m0 + total.log()).squeeze(-1)


def _plain_packed(s):
    q, cu, dev = s["q"], s["cu_seqlens"], s["q"].device
    Hq, Hkv, D = q.shape[1], s["k"].shape[1], q.shape[2]
    r, B, L = Hq // Hkv, len(s["lens"]), max(s["lens"])
    lengths = cu[1:] - cu[:-1]
    prompt_of = s["survivor_idx"].long() // s["G"]
    k, v, valid, shared = _keys(s, cu[:-1], lengths, prompt_of)
    grouped = lambda x: _padded(x, cu[:-1], lengths, L)[0].reshape(B, L, Hkv, r, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, r * L, D)  # noqa: E731
    qp = grouped(q)
    z = (qp @ k.transpose(2, 3)) * s["scale"]
    i, j = torch.arange(L, device=dev), torch.arange(k.shape[2], device=dev) - shared
    allowed = valid[:, None, :] & (j[None, None, :] <= i[None, :, None])
    p, lse = _softmax(z.view(B, Hkv, r, L, -1), allowed[:, None, None])
    p, z = p.view(B, Hkv, r * L, -1), None
    live = i[None, :] < lengths[:, None]
    packed = lambda x: x.view(B, Hkv, r, L, D).permute(0, 3, 1, 2, 4).reshape(B, L, Hq, D)[live]  # noqa: E731
    o = p @ v
    out = {"o": packed(o).to(torch.bfloat16), "lse": lse.permute(0, 3, 1, 2).reshape(B, L, Hq)[live]}
    return out, (qp, k, v, p, o, grouped, packed, live, shared)


def _run_attend(s):
    if own:
        o, lse, _, _ = _own_attend(s)
        return {"o": o, "lse": lse}
    return _plain_packed(s)[0]


def _run_train(s):
    if own:
        return _own_train(s)
    out, (qp, k, v, p, o, grouped, packed, live, shared) = _plain_packed(s)
    do = grouped(s["do"])
    dv = p.transpose(2, 3) @ do
    ds = do @ v.transpose(2, 3)
    ds -= (do * o).sum(-1, keepdim=True)
    ds *= p
    ds *= s["scale"]
    dq, dk = ds @ k, ds.transpose(2, 3) @ qp
    out["dq"] = packed(dq).to(torch.bfloat16)
    for name, g in (("k", dk), ("v", dv)):
        g = g.transpose(1, 2)
        out["d" + name] = g[:, shared:][live].to(torch.bfloat16)
        if shared:  # the survivors of a prompt, as many for each, add up
            cu = s["cu_prompts"]
            total = g[:, :shared].unflatten(0, (s["P"], -1)).sum(1)
            there = torch.arange(shared, device=g.device)[None, :] < (cu[1:] - cu[:-1])[:, None]
            out["dprompt_" + name] = total[there].to(torch.bfloat16)
    return out


def _run_decode(s):
    if own:
        return _own_decode(s)
    q = s["q"]
    N, Hq, D = q.shape
    Hkv = s["k"].shape[1]
    prompt_of = torch.arange(N, device=q.device) // s["G"]
    k, v, valid, _ = _keys(s, s["src_tok_off"], s["lengths"].long(), prompt_of)
    z = (q.float().view(N, Hkv, Hq // Hkv, D) @ k.transpose(2, 3)) * s["scale"]
    p, lse = _softmax(z, valid[:, None, None])
    keep = s["keep"].bool()
    o = torch.where(keep[:, None, None], (p @ v).view(N, Hq, D), 0.0)
    return {"o": o.to(torch.bfloat16), "lse": torch.where(keep[:, None], lse.reshape(N, Hq), 0.0)}


# ---- what the paths cannot do without -------------------------------------------------------------------------------------

def work(case):
    lens, prompts, index = _layout(case)
    Hq, Hkv, D, G = case["Hq"], case["Hkv"], case["D"], case["G"]
    if case["kind"] == "decode":
        read = sum(lens[i] for i in index) + sum(prompts[p] for p in {i // G for i in index})
        keys = sum(lens[i] + prompts[i // G] for i in index)
        return {"bytes": 4 * read * Hkv * D + len(index) * Hq * (4 * D + 4), "flops": 4 * D * Hq * keys}
    T, pairs = sum(lens), sum(n * (n + 1) // 2 + n * prompts[i // G] for n, i in zip(lens, index))
    kv = 2 * 2 * (T + sum(prompts)) * Hkv * D
    row = 2 * T * Hq * D
    if case["kind"] == "attend":
        return {"bytes": 2 * row + kv + 4 * T * Hq, "flops": 4 * D * Hq * pairs}
    return {"bytes": 4 * row + 2 * kv + 4 * T * Hq, "flops": 14 * D * Hq * pairs}


# ---- the definition in 64 bits, sequence by sequence ------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    lens, prompts, index = _layout(case)
    Hq, Hkv, D, G = case["Hq"], case["Hkv"], case["D"], case["G"]
    r, decode, train = Hq // Hkv, case["kind"] == "decode", case["kind"] == "train"
    f64 = dict(dtype=torch.float64, device=s["q"].device)
    out = {"o": torch.zeros(s["q"].shape, **f64), "lse": torch.zeros(s["q"].shape[:2], **f64)}
    if train:
        out |= {n: torch.zeros(s[n[1:]].shape, **f64) for n in ("dq", "dk", "dv")}
        if s["prompt_k"] is not None:
            out |= {n: torch.zeros(s[n[1:]].shape, **f64) for n in ("dprompt_k", "dprompt_v")}
    at_prompt = _starts(prompts)
    at = s["src_tok_off"].tolist() if decode else _starts(lens)
    for n, i in enumerate(index):
        p, b, length = i // G, at[i if decode else n], lens[i if decode else n]
        a, shared = at_prompt[p], prompts[p]
        rows = slice(i, i + 1) if decode else slice(b, b + length)
        m = rows.stop - rows.start
        # key c of row j: the prompt's keys, then the own ones up to the row itself (all that are there, for `decode`)
        mask = None
        if not decode:
            mask = torch.ones(m, shared + length, dtype=torch.bool, device=s["q"].device).tril(shared)
        for g in range(Hkv):
            heads = slice(g * r, (g + 1) * r)
            key, val = s["k"][b:b + length, g], s["v"][b:b + length, g]
            if shared:
                key, val = torch.cat([s["prompt_k"][a:a + shared, g], key]), torch.cat([s["prompt_v"][a:a + shared, g], val])
            key, val = key.double(), val.double()
            q = s["q"][rows, heads].double().transpose(0, 1)                 # [r, m, D]
            if key.shape[0] == 0:
                out["lse"][rows, heads] = -math.inf
                continue
            z = torch.matmul(q, key.T) * s["scale"]
            if mask is not None:
                z = torch.where(mask, z, -math.inf)
            lse = torch.logsumexp(z, -1)
            w = torch.exp(z - lse[..., None])
            o = torch.matmul(w, val)
            out["o"][rows, heads], out["lse"][rows, heads] = o.transpose(0, 1), lse.transpose(0, 1)
            if train:
                do = s["do"][rows, heads].double().transpose(0, 1)
                dv = torch.einsum("rmk,rmd->kd", w, do)
                dz = w * (torch.matmul(do, val.T) - (do * o).sum(-1, keepdim=True)) * s["scale"]
                dk = torch.einsum("rmk,rmd->kd", dz, q)
                out["dq"][rows, heads] = torch.matmul(dz, key).transpose(0, 1)
                for name, grad in (("k", dk), ("v", dv)):
                    out["d" + name][b:b + length, g] = grad[shared:]
                    if shared:
                        out["dprompt_" + name][a:a + shared, g] += grad[:shared]
    return out
