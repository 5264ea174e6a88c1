"""Performance cases of positions and the 8-bit cache: what training and generation around the attention calls ask of them.

Five kinds of pass, each over the range of sizes that its callers have:

  rotate   rotary positions of the packed survivors' queries and keys; `back`: the gradients' way
  one      one generated token per live rollout: rotate its query and key, append key and value to the rollout's pages
  rows     prompts, or pieces of them: rotate and append runs of tokens, queries and keys also as bf16 for the attention of the piece itself
  attend   attention of one token per live rollout over its group's prompt and its own tokens, both in 8-bit pages

A cache holds numbers of the type e4m3 and, for each page and key head, a scale (a power of two); the passes that write return both as they stand.
Head layouts are generic ones of grouped-query models; lengths, prompts and group sizes are those of the package's workloads.
"""
from __future__ import annotations

import functools
import math
import random

import torch

own = False

F8, BF = torch.float8_e4m3fn, torch.bfloat16
TOP, LOWEST = 448.0, -100               # the largest e4m3 number; the exponent of the least scale
MAX_ROTATE_BYTES = 1.7e9
MAX_APPEND_BYTES = 1.0e9
MAX_CACHE_BYTES = 1.25e9                # of one generation step, and of the plain form's padded copies of it (an eighth each)
MAX_PADDED = 1.4e9


def listed():
    return [
        # A debugging-size step: 4 prompts x 4 survivors of a hundred tokens or two, whole heads, halves as pairs.
        _rotate("rotate-tiny", P=4, G=8, K=4, lo=96, hi=256, plo=17, phi=90, Hq=8, Hkv=8, D=64, R=64),
        # The policy's forward over a whole step's survivors: 16 prompts x 8, slices of a fused projection, frequencies in bands for long contexts.
        _rotate("rotate-step", P=16, G=16, K=8, lo=300, hi=1900, plo=100, phi=500, Hq=16, Hkv=8, D=128, R=128, fused=True, scaling="bands"),
        # The gradients of a micro-batch, half of the head rotated, neighbours as pairs, positions given token by token.
        _rotate("rotate-back", P=5, G=16, K=8, lo=211, hi=1013, plo=0, phi=300, Hq=28, Hkv=4, D=128, R=64, interleaved=True, back=True, given=True),
        # Two long rollouts, heads of 80, a context stretched by parts of the frequencies.
        _rotate("rotate-d80", P=1, G=8, K=2, lo=7001, hi=8192, plo=333, phi=333, Hq=20, Hkv=4, D=80, R=80, scaling="ramp"),
        # Generation, a few rollouts at the start of their answers: latency.
        _append("one-tiny", "one", P=2, G=8, lo=1, hi=60, plo=40, phi=200, Hq=8, Hkv=2, D=64, R=64, page=16, kept=1.0),
        # Generation of a whole batch after the prune step: half of 1,024 rollouts live, early in their answers.
        _append("one-batch", "one", P=64, G=16, lo=30, hi=300, plo=100, phi=1000, Hq=32, Hkv=8, D=128, R=128, page=64, kept=0.5, scaling="bands"),
        # The batch's prompts, all of their tokens at once.
        _append("rows-prompts", "rows", P=48, G=1, lo=100, hi=1500, new=1.0, Hq=16, Hkv=8, D=128, R=128, page=64, kept=1.0, fused=True),
        # Pieces of long prompts that begin and end inside pages; part of the head, neighbours as pairs.
        _append("rows-pieces", "rows", P=7, G=1, lo=900, hi=5000, new=0.15, Hq=14, Hkv=2, D=64, R=32, page=32, kept=0.8, interleaved=True),
        # Generation, a few rollouts: latency.
        _attend("attend-tiny", P=2, G=8, lo=1, hi=60, plo=40, phi=200, Hq=8, Hkv=2, D=64, page=16, kept=1.0),
        # One prompt of 16 rollouts that have long answers, half of them live: few rows, long pages' lists.
        _attend("attend-one-group", P=1, G=16, lo=5000, hi=8192, plo=2000, phi=2000, Hq=32, Hkv=8, D=128, page=64, kept=0.5),
        # Generation of a whole batch after the prune step.
        _attend("attend-batch", P=32, G=16, lo=300, hi=4096, plo=100, phi=1000, Hq=16, Hkv=8, D=128, page=64, kept=0.5),
        # Short answers to long shared prompts, before anything is pruned.
        _attend("attend-long-prompts", P=24, G=16, lo=20, hi=300, plo=1500, phi=8192, Hq=32, Hkv=8, D=64, page=32, kept=1.0),
    ]


def _rotate(name, **sizes):
    return {"kind": "rotate", "name": name, "layout": 1, "fused": False, "interleaved": False, "scaling": "plain", "back": False, "given": False, **sizes}


def _append(name, kind, **sizes):
    return {"kind": kind, "name": name, "layout": 1, "plo": 0, "phi": 0, "new": 0.0, "fused": False, "interleaved": False, "scaling": "plain", **sizes}


def _attend(name, **sizes):
    return {"kind": "attend", "name": name, "layout": 1, **sizes}


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["rotate", "rotate", "one", "rows", "attend", "attend"])
        Hkv, D = rng.choice([1, 2, 4, 8]), rng.choice([64, 64, 80, 96, 128, 128])
        case = {"kind": kind, "layout": rng.randrange(1 << 20), "P": _log_uniform(rng, 1, 32), "G": rng.choice([4, 8, 16]), "Hq": Hkv * rng.randint(1, 8), "Hkv": Hkv, "D": D}
        hi, phi = _log_uniform(rng, 16, 8192), _log_uniform(rng, 1, 6000)
        case |= {"lo": rng.randint(1, hi), "hi": hi, "plo": rng.randint(0, phi), "phi": phi}
        if kind != "attend":
            case |= {"R": rng.choice([D, D, D, D // 2, D // 4 * 2]), "interleaved": rng.random() < 0.4, "fused": rng.random() < 0.5,
                     "scaling": rng.choice(["plain", "linear", "bands", "ramp"])}
        if kind == "rotate":
            case |= {"K": rng.randint(1, case["G"]), "back": rng.random() < 0.5, "given": rng.random() < 0.3}
            if work(case)["bytes"] <= MAX_ROTATE_BYTES:
                return case
            continue
        case |= {"page": rng.choice([16, 32, 64, 128]), "kept": rng.choice([0.25, 0.5, 1.0])}
        lens, prompts, live, new = _layout(case | {"new": 0.0})
        if kind == "attend":
            padded = len(live) * (max(lens) + max(prompts)) * Hkv * D
            if work(case)["bytes"] <= MAX_CACHE_BYTES and padded <= MAX_PADDED and sum(lens) * Hkv * D <= MAX_CACHE_BYTES:
                return case
            continue
        case |= {"new": 0.0 if kind == "one" else rng.choice([0.02, 0.2, 1.0])}
        if kind == "rows":
            case |= {"G": 1, "plo": 0, "phi": 0}
        if work(case)["bytes"] <= MAX_APPEND_BYTES and sum(_layout(case)[0]) * Hkv * D <= MAX_CACHE_BYTES / 4:
            return case


def _layout(case):
    """Of the case alone, so that work() knows it.  rotate: the survivors' lengths, the prompts', the survivors' numbers.  Else the tokens that each
    rollout (or prompt, for `rows`) has after the pass, the prompts' lengths, the live ones, and how many tokens are new."""
    rng = random.Random("%(layout)d %(P)d %(G)d %(lo)d %(hi)d" % case)
    prompts = [rng.randint(case["plo"], case["phi"]) for _ in range(case["P"])]
    if case["kind"] == "rotate":
        index = [p * case["G"] + i for p in range(case["P"]) for i in sorted(rng.sample(range(case["G"]), case["K"]))]
        return [rng.randint(case["lo"], case["hi"]) for _ in index], prompts, index
    N = case["P"] * case["G"]
    live = sorted(rng.sample(range(N), max(1, int(round(N * case["kept"])))))
    lens = [rng.randint(case["lo"], case["hi"]) for _ in range(N)]
    new = [1] * N if not case["new"] else [n if case["new"] == 1.0 else rng.randint(1, max(1, int(n * case["new"]))) for n in lens]
    return lens, prompts, live, new


def _starts(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return at


# ---- inputs -------------------------------------------------------------------------------------------------------------

def _frequencies(R, scaling):
    """Angle per position of each pair, and the factor on cosine and sine: base 500,000 where contexts are stretched, else 10,000."""
    base = 10000.0 if scaling in ("plain", "linear") else 500000.0
    f = [base ** (-2.0 * i / R) for i in range(R // 2)]
    if scaling == "linear":
        return [x / 4.0 for x in f], 1.0
    if scaling == "bands":        # long waves are slowed down 32 times, short ones not, those between in part; trained on 8,192 positions
        out = []
        for x in f:
            turns = 8192 * x / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - 1.0) / (4.0 - 1.0)))
            out.append((1 - keep) * x / 32.0 + keep * x)
        return out, 1.0
    if scaling == "ramp":         # by the pairs' numbers: from the one that turns 32 times in 4,096 positions to the one that turns once
        at = lambda turns: R * math.log(4096 / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), R - 1)
        slow = [min(1.0, max(0.0, (i - lo) / max(hi - lo, 1e-3))) for i in range(R // 2)]
        return [x * (1 - s) + x / 4.0 * s for x, s in zip(f, slow)], 0.1 * math.log(4.0) + 1.0
    return f, 1.0


def _needed(amax):
    """The least power of two that brings amax to 448 or less."""
    m, x = torch.frexp(amax)
    e = torch.where(amax > 0, x - 9 + (m > 0.875).to(x.dtype), LOWEST).clamp(min=LOWEST)
    return torch.ldexp(torch.ones_like(amax), e)


def _pages(gen, pages, Hkv, page, D):
    """Random pages as the append leaves them: values whose size differs from page to page and head to head."""
    cache, scale = torch.empty(pages, Hkv, page, D, dtype=F8, device="cuda"), torch.empty(pages, Hkv, device="cuda")
    for a in range(0, pages, 4096):
        n = min(4096, pages - a)
        x = torch.randn(n, Hkv, page, D, generator=gen, device="cuda") * torch.exp(0.5 * torch.randn(n, Hkv, 1, 1, generator=gen, device="cuda"))
        scale[a:a + n] = _needed(x.abs().amax((2, 3)))
        cache[a:a + n] = (x / scale[a:a + n, :, None, None]).to(F8)
    return cache, scale


def prepare(case, seed):
    dev = "cuda"
    gen = torch.Generator(device=dev).manual_seed(seed)
    Hq, Hkv, D, kind = case["Hq"], case["Hkv"], case["D"], case["kind"]

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=gen, device=dev) * scale).to(BF)

    def ints(values, dtype=torch.int32):
        return torch.tensor(values, dtype=dtype, device=dev)

    def rows(T):
        if case["fused"]:
            qkv = normal(T, Hq + 2 * Hkv, D)
            return qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        return normal(T, Hq, D), normal(T, Hkv, D), normal(T, Hkv, D)

    s = {"kind": kind, "G": case["G"]}
    if kind != "attend":
        f, s["factor"] = _frequencies(case["R"], case["scaling"])
        s["frequencies"], s["interleaved"] = ints(f, torch.float64), case["interleaved"]
    if kind == "rotate":
        lens, prompts, index = _layout(case)
        T = sum(lens)
        s["q"], s["k"], _ = rows(T)
        s["back"] = case["back"]
        s["cu_seqlens"], s["num"] = ints(_starts(lens), torch.int64), ints([len(lens), T], torch.int64)
        s["cu_prompts"], s["survivor_idx"] = ints(_starts(prompts), torch.int64), ints(index)
        s["positions"] = None
        if case["given"]:
            s["positions"] = ints([prompts[i // case["G"]] + t for i, n in zip(index, lens) for t in range(n)])
        return s
    lens, prompts, live, new = _layout(case | ({"new": 0.0} if kind == "attend" else {}))
    N, page = len(lens), case["page"]
    held = [-(-n // page) for n in lens]
    in_prompts = [-(-n // page) if kind == "attend" else 0 for n in prompts]
    pool = sum(held) + sum(in_prompts)
    s["k_cache"], s["k_scale"] = _pages(gen, pool, Hkv, page, D)
    s["v_cache"], s["v_scale"] = _pages(gen, pool, Hkv, page, D)
    order = torch.randperm(pool, generator=gen, device=dev).to(torch.int32)     # pages come from wherever some were free

    def table(counts, start):
        at = torch.tensor(_starts(counts)[:-1], device=dev)[:, None] + start + torch.arange(max(max(counts), 1), device=dev)
        return torch.where(torch.arange(max(max(counts), 1), device=dev) < ints(counts)[:, None], order[at.clamp(max=pool - 1)], -1).contiguous()

    s["table"] = table(held, 0)
    s["lengths"], s["prompt_lengths"] = ints(lens), ints(prompts)
    keep = torch.zeros(N, dtype=torch.uint8)
    keep[live] = 1
    s["keep"] = keep.to(dev)
    if kind == "attend":
        # scores spread by about 1.5, as between normalised queries and keys with learned gains
        s["q"], s["live"], s["scale"] = normal(N, Hq, D, scale=1.5), ints(live, torch.int64), 1.0 / math.sqrt(D)
        s["longest"], s["longest_prompt"] = max(lens), max(prompts)
        s["prompt_table"] = table(in_prompts, sum(held)) if max(prompts) else None
        s["o"], s["lse"] = torch.zeros(N, Hq, D, dtype=BF, device=dev), torch.zeros(N, Hq, device=dev)
        return s
    T = sum(new)
    s["q"], s["k"], s["v"] = rows(T)
    s["cu_new"] = ints(_starts(new), torch.int64) if kind == "rows" else None
    s["q_out"] = torch.zeros(T, Hq, D, dtype=BF, device=dev)
    s["k_out"] = torch.zeros(T, Hkv, D, dtype=BF, device=dev) if kind == "rows" else None
    return s


def run(state):
    return {"rotate": _run_rotate, "one": _run_append, "rows": _run_append, "attend": _run_attend}[state["kind"]](state)


# ---- the framework's calls ----------------------------------------------------------------------------------------------

@functools.lru_cache(maxsize=None)
def _context():
    from paper_2603_24840_b200 import binding
    return binding.Context(0)


def _own_rotate(s):
    from paper_2603_24840_b200 import rotary
    q, k = s["q"], s["k"]
    out = torch.empty(q.shape, dtype=BF, device=q.device), torch.empty(k.shape, dtype=BF, device=k.device)
    where = {"positions": s["positions"], "d_num": s["num"]} if s["positions"] is not None else {
        "cu_seqlens": s["cu_seqlens"], "d_num": s["num"], "cu_prompts": s["cu_prompts"], "survivor_idx": s["survivor_idx"], "G": s["G"]}
    call = rotary.arrol_rotary_backward if s["back"] else rotary.arrol_rotary
    call(_context(), q, k, s["frequencies"], *out, factor=s["factor"], interleaved=s["interleaved"], **where)
    return out


def _own_append(s):
    from paper_2603_24840_b200 import cache
    more = {"cu_new": s["cu_new"], "k_out": s["k_out"]} if s["kind"] == "rows" else {"prompt_lengths": s["prompt_lengths"], "G": s["G"]}
    cache.arrol_cache_append(_context(), s["k"], s["v"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["table"], s["lengths"], keep=s["keep"],
                             q=s["q"], q_out=s["q_out"], frequencies=s["frequencies"], factor=s["factor"], interleaved=s["interleaved"], **more)


def _own_attend(s):
    from paper_2603_24840_b200 import cache
    ctx, q = _context(), s["q"]
    N, Hq, D = q.shape
    P = 0 if s["prompt_table"] is None else s["prompt_table"].shape[0]
    ws = torch.empty(cache.arrol_cache_attention_workspace(ctx, N, P, s["G"], Hq, s["k_cache"].shape[1], D), dtype=torch.uint8, device=q.device)
    shared = {"prompt_table": s["prompt_table"], "prompt_lengths": s["prompt_lengths"], "G": s["G"]} if P else {}
    cache.arrol_cache_attention(ctx, q, s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["table"], s["lengths"], s["o"], s["lse"], ws, keep=s["keep"],
                                scale=s["scale"], **shared)


# ---- the plain forms: whole arrays, in 32 bits (angles in 64) -------------------------------------------------------------

def _turn(x, positions, s, sign=1.0):
    """[T, H, D] in 32 bits, the first dimensions of each head turned by the positions' angles."""
    f = s["frequencies"]
    n = f.numel()
    a = positions.double()[:, None] * f
    cos, sin = (a.cos() * s["factor"]).float()[:, None], (a.sin() * (s["factor"] * sign)).float()[:, None]
    x = x.float()
    if s["interleaved"]:
        x1, x2 = x[..., 0:2 * n:2], x[..., 1:2 * n:2]
        turned = torch.stack([x1 * cos - x2 * sin, x2 * cos + x1 * sin], -1).flatten(-2)
    else:
        x1, x2 = x[..., :n], x[..., n:2 * n]
        turned = torch.cat([x1 * cos - x2 * sin, x2 * cos + x1 * sin], -1)
    return torch.cat([turned, x[..., 2 * n:]], -1)


def _run_rotate(s):
    if own:
        q, k = _own_rotate(s)
        return {"q": q, "k": k}
    positions = s["positions"]
    if positions is None:
        cu, T = s["cu_seqlens"], s["q"].shape[0]
        seq = torch.repeat_interleave(torch.arange(cu.numel() - 1, device=cu.device), cu[1:] - cu[:-1], output_size=T)
        p = s["survivor_idx"].long()[seq] // s["G"]
        positions = torch.arange(T, device=cu.device) - cu[seq] + s["cu_prompts"][p + 1] - s["cu_prompts"][p]
    sign = -1.0 if s["back"] else 1.0
    return {"q": _turn(s["q"], positions, s, sign).to(BF), "k": _turn(s["k"], positions, s, sign).to(BF)}


def _put(cache, scale, x, pages, slots, row_live, first_pages, first_slots):
    """Rows x [T, Hkv, D] at (pages, slots); rows that are not live come with page 0 and are left out.  A page that had tokens (first_slots of first_pages) keeps its
    scale or gets a larger one, and its numbers with it."""
    page = cache.shape[2]
    raw = cache.view(torch.uint8)
    most = torch.zeros_like(scale).scatter_reduce_(0, pages[:, None].expand(-1, scale.shape[1]), torch.where(row_live[:, None], x.abs().amax(-1), 0.0), "amax")
    touched = torch.zeros(cache.shape[0], dtype=torch.bool, device=x.device).index_fill_(0, pages[row_live], True)
    need = _needed(most)
    old = scale[first_pages]
    larger = torch.where(first_slots[:, None] > 0, torch.maximum(old, need[first_pages]), need[first_pages])
    held = (torch.arange(page, device=x.device) < first_slots[:, None])[:, None, :, None]
    was = raw[first_pages]
    now = (was.view(F8).float() * (old / larger)[..., None, None]).to(F8).view(torch.uint8)
    raw[first_pages] = torch.where(held, now, was)
    need[first_pages] = larger
    scale.copy_(torch.where(touched[:, None], need, scale))
    code = (x / scale[pages][..., None]).to(F8).view(torch.uint8)
    raw[pages[row_live], :, slots[row_live]] = code[row_live]


def _run_append(s):
    if own:
        _own_append(s)
    else:
        lengths, table, keep, dev = s["lengths"].long(), s["table"].long(), s["keep"].bool(), s["k"].device
        N, T, page = lengths.numel(), s["k"].shape[0], s["k_cache"].shape[2]
        seqs = torch.arange(N, device=dev)
        if s["cu_new"] is None:
            seq, at, first = seqs, lengths - 1, lengths - 1
            positions = at + s["prompt_lengths"].long().repeat_interleave(s["G"])
        else:
            cu = s["cu_new"]
            first = lengths - (cu[1:] - cu[:-1])
            seq = torch.repeat_interleave(seqs, cu[1:] - cu[:-1], output_size=T)
            at = positions = torch.arange(T, device=dev) - cu[seq] + first[seq]
        live, q, k = keep[seq], _turn(s["q"], positions, s), _turn(s["k"], positions, s)
        s["q_out"].copy_(torch.where(live[:, None, None], q, 0.0).to(BF))
        if s["k_out"] is not None:
            s["k_out"].copy_(torch.where(live[:, None, None], k, 0.0).to(BF))
        pages = torch.where(live, table[seq, at // page], 0)
        first = first[keep]
        first_pages = table[keep].gather(1, (first // page)[:, None])[:, 0]
        _put(s["k_cache"], s["k_scale"], k, pages, at % page, live, first_pages, first % page)
        _put(s["v_cache"], s["v_scale"], s["v"].float(), pages, at % page, live, first_pages, first % page)
    return {n: s[n] for n in ("q_out", "k_out", "k_cache", "v_cache", "k_scale", "v_scale") if s[n] is not None}


def _from_pages(cache, scale, table, lengths, most):
    """[B, Hkv, most, D] in 32 bits, zeros behind each length."""
    page = cache.shape[2]
    j = torch.arange(most, device=cache.device)
    valid = j[None, :] < lengths[:, None]
    pages = torch.where(valid, table[:, j // page], 0).long()
    x = cache.view(torch.uint8)[pages, :, (j % page)[None, :]].view(F8).float() * scale[pages][..., None]
    return torch.where(valid[..., None, None], x, 0.0).transpose(1, 2), valid


def _run_attend(s):
    if own:
        _own_attend(s)
        return {"o": s["o"], "lse": s["lse"]}
    live, (N, Hq, D), Hkv = s["live"], s["q"].shape, s["k_cache"].shape[1]
    k, valid = _from_pages(s["k_cache"], s["k_scale"], s["table"][live], s["lengths"][live], s["longest"])
    v, _ = _from_pages(s["v_cache"], s["v_scale"], s["table"][live], s["lengths"][live], s["longest"])
    if s["prompt_table"] is not None:
        p = live // s["G"]
        pk, pvalid = _from_pages(s["k_cache"], s["k_scale"], s["prompt_table"], s["prompt_lengths"], s["longest_prompt"])
        pv, _ = _from_pages(s["v_cache"], s["v_scale"], s["prompt_table"], s["prompt_lengths"], s["longest_prompt"])
        k, v, valid = torch.cat([pk[p], k], 2), torch.cat([pv[p], v], 2), torch.cat([pvalid[p], valid], 1)
    z = (s["q"][live].float().view(-1, Hkv, Hq // Hkv, D) @ k.transpose(2, 3)) * s["scale"]
    z = z.masked_fill_(~valid[:, None, None], -math.inf)
    m = z.amax(-1, keepdim=True)
    e = (z - m).exp_()
    total = e.sum(-1, keepdim=True)
    o = (e @ v) / total
    s["o"][live] = o.reshape(-1, Hq, D).to(BF)
    s["lse"][live] = (m + total.log()).reshape(-1, Hq)
    return {"o": s["o"], "lse": s["lse"]}


# ---- what the paths cannot do without -------------------------------------------------------------------------------------

def work(case):
    Hq, Hkv, D, G = case["Hq"], case["Hkv"], case["D"], case["G"]
    if case["kind"] == "rotate":
        T = sum(_layout(case)[0])
        return {"bytes": 4 * T * (Hq + Hkv) * D, "flops": 3 * T * (Hq + Hkv) * case["R"]}
    lens, prompts, live, new = _layout(case | ({"new": 0.0} if case["kind"] == "attend" else {}))
    if case["kind"] == "attend":
        read = sum(lens[i] for i in live) + sum(prompts[p] for p in {i // G for i in live})
        keys = sum(lens[i] + prompts[i // G] for i in live)
        return {"bytes": 2 * read * Hkv * D + len(live) * Hq * (4 * D + 4), "flops": 4 * D * Hq * keys}
    T = sum(new[i] for i in live)
    return {"bytes": T * D * (4 * Hq + (4 + 2 + (2 if case["kind"] == "rows" else 0)) * Hkv), "flops": T * (3 * (Hq + Hkv) * case["R"] + 4 * Hkv * D)}


# ---- the definition in 64 bits ----------------------------------------------------------------------------------------------

def _turned(x, positions, case):
    """Pairs as complex numbers, turned by multiplication."""
    f, factor = _frequencies(case["R"], case["scaling"])
    sign = -1.0 if case.get("back") else 1.0
    at = torch.tensor(positions, dtype=torch.float64, device=x.device)[:, None] * torch.tensor(f, dtype=torch.float64, device=x.device)
    by = torch.polar(torch.full_like(at, factor), sign * at)[:, None]
    x = x.double()
    R = case["R"]
    if case["interleaved"]:
        z = torch.complex(x[..., 0:R:2].contiguous(), x[..., 1:R:2].contiguous()) * by
        x[..., 0:R:2], x[..., 1:R:2] = z.real, z.imag
    else:
        z = torch.complex(x[..., :R // 2].contiguous(), x[..., R // 2:R].contiguous()) * by
        x[..., :R // 2], x[..., R // 2:R] = z.real, z.imag
    return x


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rotate":
        lens, prompts, index = _layout(case)
        positions = [prompts[i // case["G"]] + t for i, n in zip(index, lens) for t in range(n)]
        return {"q": _turned(s["q"], positions, case), "k": _turned(s["k"], positions, case)}
    lens, prompts, live, new = _layout(case | ({"new": 0.0} if case["kind"] == "attend" else {}))
    return _exact_attend(case, s, lens, prompts, live) if case["kind"] == "attend" else _exact_append(case, s, lens, prompts, live, new)


def _exact_append(case, s, lens, prompts, live, new):
    """Sequence by sequence, page by page: the numbers before they are rounded to 8 bits."""
    page, G, table, cu = case["page"], case["G"], s["table"].tolist(), _starts(new)
    out = {n: s[n].double() for n in ("q_out", "k_out", "k_cache", "v_cache", "k_scale", "v_scale") if s[n] is not None}
    rows = [r for i in live for r in range(cu[i], cu[i + 1])]
    positions = [prompts[i // G] + lens[i] - new[i] + t for i in live for t in range(new[i])]
    at = torch.tensor(rows, device=s["k"].device)
    q, k, v = _turned(s["q"][at], positions, case), _turned(s["k"][at], positions, case), s["v"][at].double()
    out["q_out"][at] = q
    if "k_out" in out:
        out["k_out"][at] = k
    from_row, pieces = 0, []                                  # (page, slots, rows) of every page that gets some
    for i in live:
        token, end = lens[i] - new[i], lens[i]
        while token < end:
            n = min(page - token % page, end - token)
            pieces.append((table[i][token // page], token % page, n, from_row))
            token, from_row = token + n, from_row + n
    for name, x in (("k", k), ("v", v)):
        cache, scale = out[name + "_cache"], out[name + "_scale"]
        sizes = x.abs().amax(-1)
        for p, slot, n, r in pieces:
            need = torch.exp2(torch.ceil(torch.log2(sizes[r:r + n].amax(0).clamp(min=2.0 ** -90) / TOP)))
            if slot:
                new_scale = torch.maximum(scale[p], need)
                cache[p, :, :slot] *= (scale[p] / new_scale)[:, None, None]
                need = new_scale
            scale[p] = need
            cache[p, :, slot:slot + n] = (x[r:r + n] / need[None, :, None]).transpose(0, 1)
    return out


def _exact_attend(case, s, lens, prompts, live):
    Hq, Hkv, D, G, page = case["Hq"], case["Hkv"], case["D"], case["G"], case["page"]
    out = {"o": s["o"].double(), "lse": s["lse"].double()}
    table, shared = s["table"].tolist(), None if s["prompt_table"] is None else s["prompt_table"].tolist()

    def tokens(cache, scale, pages, n):
        at = torch.tensor(pages[:-(-n // page)], dtype=torch.int64, device=s["q"].device)
        x = cache.view(torch.uint8)[at].view(F8).double() * scale[at].double()[..., None, None]
        return x.transpose(1, 2).reshape(-1, Hkv, D)[:n]

    for i in live:
        parts = [(shared[i // G], prompts[i // G])] if shared else []
        parts = [x for x in parts + [(table[i], lens[i])] if x[1]]
        key, val = (torch.cat([tokens(s[n + "_cache"], s[n + "_scale"], *x) for x in parts]) for n in "kv")
        q = s["q"][i].double().view(Hkv, Hq // Hkv, D)
        z = torch.einsum("grd,jgd->grj", q, key) * s["scale"]
        lse = torch.logsumexp(z, -1)
        out["o"][i] = torch.einsum("grj,jgd->grd", torch.exp(z - lse[..., None]), val).reshape(Hq, D)
        out["lse"][i] = lse.reshape(-1)
    return out
