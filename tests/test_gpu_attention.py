"""GPU parity of the packed attention calls against the 64-bit reference: every result within the bound that the roundings of the interface give."""
import math

import pytest
import torch

import attention_reference as R
from paper_2603_24840_b200 import attention as A
from paper_2603_24840_b200 import binding as B

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    c.close()


def _starts(n):
    out = [0]
    for x in n:
        out.append(out[-1] + x)
    return out


class Problem:
    """A packed batch with `spare` rows behind the live ones; `prompts` = None: no prompts.  `wide`: rows of one fused projection."""

    def __init__(self, lens, prompts=None, index=None, G=1, Hq=4, Hkv=2, D=64, seed=0, spare=0, wide=False, fill=0.0, q_scale=1.5, scale=None, extra_S=0):
        dev, g = "cuda", torch.Generator("cuda").manual_seed(seed)
        mk = lambda *s, by=1.0: (torch.randn(*s, generator=g, device=dev) * by).to(BF)  # noqa: E731
        self.T, self.G, self.Hq, self.Hkv, self.D = sum(lens), G, Hq, Hkv, D
        self.cu, self.index = _starts(lens), index
        self.cu_prompts = None if prompts is None else _starts(prompts)
        self.scale = 1 / math.sqrt(D) if scale is None else scale
        rows = self.T + spare
        if wide:
            w = mk(rows, Hq + 2 * Hkv, D)
            w[:, :Hq] *= q_scale
            self.q, self.k, self.v = w[:, :Hq], w[:, Hq:Hq + Hkv], w[:, Hq + Hkv:]
        else:
            self.q, self.k, self.v = mk(rows, Hq, D, by=q_scale), mk(rows, Hkv, D), mk(rows, Hkv, D)
        self.d_o = mk(rows, Hq, D)
        self.pk = self.pv = None
        if prompts is not None:
            self.pk, self.pv = mk(sum(prompts) + spare, Hkv, D), mk(sum(prompts) + spare, Hkv, D)
        if spare:
            for t in (self.q, self.k, self.v, self.d_o):
                t[self.T:] = fill
            if self.pk is not None:
                self.pk[sum(prompts):] = fill
                self.pv[sum(prompts):] = fill
        junk = [7 << 40] * extra_S
        self.d_cu = torch.tensor(self.cu + junk, dtype=torch.int64, device=dev)
        self.d_num = torch.tensor([len(lens), self.T], dtype=torch.int64, device=dev)
        self.d_cup = None if prompts is None else torch.tensor(self.cu_prompts, dtype=torch.int64, device=dev)
        self.d_idx = None if index is None else torch.tensor(index + [-5] * extra_S, dtype=torch.int32, device=dev)
        self.seqs = R.sequences(self.cu, index, G, self.cu_prompts)

    def shared(self):
        return {} if self.pk is None else dict(prompt_k=self.pk, prompt_v=self.pv, cu_prompts=self.d_cup, survivor_idx=self.d_idx, G=self.G)

    def outputs(self, fill=-7.0):
        rows, full = self.q.shape[0], lambda *s: torch.full(s, fill, dtype=BF, device="cuda")  # noqa: E731
        out = {"o": full(rows, self.Hq, self.D), "lse": torch.full((rows, self.Hq), fill, device="cuda"), "dq": full(rows, self.Hq, self.D),
               "dk": full(rows, self.Hkv, self.D), "dv": full(rows, self.Hkv, self.D)}
        if self.pk is not None:
            out |= {"dprompt_k": full(*self.pk.shape), "dprompt_v": full(*self.pv.shape)}
        return out

    def workspace(self, ctx, backward=True):
        n = A.arrol_attention_workspace(ctx, len(self.cu) - 1, self.q.shape[0], 0 if self.pk is None else self.pk.shape[0], self.Hq, self.Hkv, self.D, backward)
        assert n > 0
        return torch.full((n,), 0xAB, dtype=torch.uint8, device="cuda")

    def forward(self, ctx, out, ws, **kw):
        A.arrol_attention(ctx, self.q, self.k, self.v, self.d_cu, self.d_num, out["o"], out["lse"], ws, scale=self.scale, **self.shared(), **kw)

    def backward(self, ctx, out, ws, **kw):
        grads = {n: t for n, t in out.items() if n.startswith("d")}
        A.arrol_attention_backward(ctx, self.q, self.k, self.v, self.d_cu, self.d_num, out["o"], out["lse"], self.d_o, workspace=ws, scale=self.scale,
                                   **self.shared(), **grads, **kw)

    def run(self, ctx, backward=True):
        out, ws = self.outputs(), self.workspace(ctx, backward)
        self.forward(ctx, out, ws)
        if backward:
            self.backward(ctx, out, ws)
        torch.cuda.synchronize()
        assert B.arrol_poll_status(ctx) == 0
        return out

    def reference(self, backward=True):
        return R.packed(self.q, self.k, self.v, self.pk, self.pv, self.seqs, self.scale, self.d_o if backward else None)

    def check(self, out, backward=True, skip=None):
        res, tol = self.reference(backward)
        names = {"o": "o", "lse": "lse"} | ({"dq": "dq", "dk": "dk", "dv": "dv", "dprompt_k": "dpk", "dprompt_v": "dpv"} if backward else {})
        for name, ref in names.items():
            if name not in out:
                continue
            live = self.T if not name.startswith("dp") else self.cu_prompts[-1]
            x, y, t = out[name][:live].double(), res[ref][:live], tol[ref][:live]
            ok = (x - y).abs() <= t
            if skip is not None and not name.startswith("dp"):
                ok |= skip[:live].view(-1, *[1] * (ok.dim() - 1))
            assert ok.all(), "%s: %g of %g at %s" % (name, ((x - y).abs() / t)[~ok].max(), 1.0, (~ok).nonzero()[0].tolist())
            assert (out[name][live:].double() == -7.0).all(), name + ": rows behind the live ones"


SHAPES = [
    # lens, prompts, index, G, Hq, Hkv, D
    ([1], None, None, 1, 1, 1, 64),
    ([0, 1, 2, 0, 3, 0], None, None, 1, 2, 1, 64),
    ([1, 1, 1, 1, 1], [1, 0, 2, 1, 1], None, 1, 4, 4, 128),
    ([127, 128, 129, 1, 64, 63], None, None, 1, 4, 2, 128),
    ([300, 5, 260], [200, 70, 3], [0, 2, 9], 4, 8, 2, 64),
    ([513, 31], [129, 0], [1, 2], 2, 6, 2, 64),
    ([90, 700], [0, 640], [0, 7], 4, 7, 1, 128),
    ([200, 45, 45, 2, 333], [17, 128, 256], [0, 1, 3, 4, 9], 4, 5, 1, 96),
    ([150, 260], [40], [2, 3], 4, 16, 1, 128),
    ([33, 70], [130], [0, 1], 2, 64, 1, 64),
    ([50, 129], [64], [0, 1], 2, 33, 1, 128),
    ([64, 200], [64], [0, 3], 4, 3, 3, 8),
    ([64, 200], [64], [0, 3], 4, 6, 3, 72),
    ([1500], [700], [0], 1, 4, 1, 128),
    ([1100, 900], None, None, 1, 2, 2, 64),
    ([7] * 90, [300, 0, 1, 65], [i for i in range(90)], 23, 4, 2, 64),
]


@pytest.mark.parametrize("lens,prompts,index,G,Hq,Hkv,D", SHAPES)
def test_forward_and_backward_match_the_definition(ctx, lens, prompts, index, G, Hq, Hkv, D):
    p = Problem(lens, prompts, index, G, Hq, Hkv, D, seed=len(lens) + D)
    p.check(p.run(ctx))


def test_strided_rows_spare_rows_and_counts_on_the_device(ctx):
    """Slices of one fused projection, rows behind the last sequence full of NaN and left as they were, arrays longer than the count."""
    for fill in (math.nan, math.inf):
        p = Problem([100, 3, 190], [65, 40], [0, 1, 5], 4, 6, 2, 128, seed=3, spare=37, wide=True, fill=fill, extra_S=2)
        p.check(p.run(ctx))
        p = Problem([100, 3, 190], None, None, 1, 8, 8, 64, seed=4, spare=200, fill=fill, extra_S=3)
        p.check(p.run(ctx))


def test_no_live_tokens_writes_nothing_but_the_prompts_zeros(ctx):
    p = Problem([0, 0], [10, 60], [0, 1], 1, 4, 2, 64, spare=130)
    out = p.run(ctx)
    for name in ("o", "lse", "dq", "dk", "dv"):
        assert (out[name].float() == -7).all()
    for name in ("dprompt_k", "dprompt_v"):
        assert (out[name][:70] == 0).all() and (out[name][70:].float() == -7).all()


def test_a_prompt_without_survivors_has_zero_gradients(ctx):
    p = Problem([40, 50], [100, 77, 30], [0, 8], 4, 4, 2, 64)
    out = p.run(ctx)
    p.check(out)
    assert (out["dprompt_k"][100:177] == 0).all() and (out["dprompt_v"][100:177] == 0).all()


def test_large_scores_and_small_scale(ctx):
    """Scores of hundreds: one key takes nearly all of the weight, maxima change from block to block."""
    for q_scale, scale in ((60.0, None), (1.5, 1e-6), (8.0, 1.0)):
        p = Problem([400, 150], [300], [0, 1], 2, 4, 2, 64, seed=5, q_scale=q_scale, scale=scale)
        out = p.run(ctx, backward=False)
        res, tol = p.reference(False)
        # the exponent's error grows with the scores: their products are summed in fp32, |z| 2^-20 covers 64 terms
        zmax = (p.q.float().norm(dim=-1).max() * max(p.k.float().norm(dim=-1).max(), p.pk.float().norm(dim=-1).max()) * p.scale).item()
        extra = zmax * 2.0 ** -20
        spread = p.v.abs().max().double()
        assert ((out["o"].double() - res["o"]).abs() <= tol["o"] + 2 * extra * spread).all()
        assert ((out["lse"].double() - res["lse"]).abs() <= tol["lse"] + extra).all()


@pytest.mark.parametrize("where", ["q", "k", "v", "d_o", "pk", "pv"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_not_a_number_reaches_only_what_attends_to_it(ctx, where, value):
    """One row of one tensor is not finite: rows of other sequences, earlier rows of the same one (keys, values) and other prompts are as before."""
    make = lambda: Problem([70, 90, 200, 40], [33, 50], [0, 1, 5, 6], 4, 4, 2, 64, seed=6)  # noqa: E731
    clean = make()
    good = clean.run(ctx)
    p = make()
    getattr(p, where)[{"pk": 40, "pv": 40}.get(where, 70 + 60), 1, 3] = value
    out = p.run(ctx)
    seq, prompt = slice(70, 160), slice(0, 33)
    rows = torch.zeros(400, dtype=torch.bool, device="cuda")            # rows of dq / o that may differ
    keys = rows.clone()                                                  # rows of dk, dv that may differ
    prompts = torch.zeros(83, dtype=torch.bool, device="cuda")
    if where in ("pk", "pv"):
        rows[160:], keys[160:], prompts[33:] = True, True, True         # the second prompt and its two sequences
    elif where in ("k", "v"):
        rows[130:160], keys[seq], prompts[prompt] = True, True, True    # rows from 130 on attend to it, and their gradients reach all of their keys
    else:
        rows[130], keys[70:131], prompts[prompt] = True, True, True
    for name, may in (("o", rows), ("lse", rows), ("dq", rows), ("dk", keys), ("dv", keys), ("dprompt_k", prompts), ("dprompt_v", prompts)):
        if where == "d_o" and name in ("o", "lse"):
            may = torch.zeros_like(may)
        assert torch.equal(out[name][~may], good[name][~may]), name
    heads = slice(2, 4) if where not in ("q", "d_o") else slice(1, 2)
    if where in ("v", "pv"):
        first = 130 if where == "v" else 160
        last = 160 if where == "v" else 400
        bad = out["o"][first:last, heads]
        assert not torch.isfinite(bad[:, :, 3]).any()
    if where == "d_o":
        assert not torch.isfinite(out["dq"][130, 1]).all()


@pytest.mark.parametrize("D,Hq,Hkv", [(64, 4, 2), (128, 4, 2), (128, 6, 1), (96, 3, 3)])
@pytest.mark.parametrize("at", [0, 5, 127, 128, 300, 511, 699])
def test_not_a_number_in_a_long_sequence(ctx, D, Hq, Hkv, at):
    """Blocks that some rows see whole and others in part, or not at all: NaN in one value (key, query row) of a sequence between two others."""
    make = lambda: Problem([200, 700, 333], [150, 260], [0, 1, 4], 4, Hq, Hkv, D, seed=18)  # noqa: E731
    good = make().run(ctx)
    for where in ("v", "k", "q", "d_o"):
        p = make()
        getattr(p, where)[200 + at, 0, D // 2] = math.nan
        out = p.run(ctx)
        rows = torch.zeros(1233, dtype=torch.bool, device="cuda")
        keys, prompts = rows.clone(), torch.zeros(410, dtype=torch.bool, device="cuda")
        prompts[:150] = True
        if where in ("k", "v"):
            rows[200 + at:900], keys[200:900] = True, True
        else:
            rows[200 + at], keys[200:201 + at] = True, True
        for name, may in (("o", rows), ("dq", rows), ("dk", keys), ("dv", keys), ("dprompt_k", prompts), ("dprompt_v", prompts)):
            if where == "d_o" and name == "o":
                may = torch.zeros_like(may)
            assert torch.equal(out[name][~may], good[name][~may]), (where, name)
        r = Hq // Hkv
        if where != "d_o":
            heads = slice(0, r) if where in ("k", "v") else slice(0, 1)
            last = 900 if where in ("k", "v") else 201 + at
            shown = out["o"][200 + at:last, heads]
            assert not torch.isfinite(shown[..., D // 2]).any(), where
        assert not torch.isfinite(out["dk"][200:201 + at, 0]).all(-1).any(), where


def test_same_bits_every_time_and_on_another_stream(ctx):
    p = Problem([300, 500, 20, 260], [200, 130], [0, 1, 5, 6], 4, 8, 2, 128, seed=7)
    first = p.run(ctx)
    for _ in range(3):
        again = p.run(ctx)
        assert all(torch.equal(first[n], again[n]) for n in first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out, ws = p.outputs(), p.workspace(ctx)
    torch.cuda.synchronize()
    p.forward(ctx, out, ws, stream=side)
    p.backward(ctx, out, ws, stream=side)
    side.synchronize()
    assert all(torch.equal(first[n], out[n]) for n in first)


def test_two_streams_at_once_with_workspaces_of_their_own(ctx):
    probs = [Problem([900, 300, 77], [300], [0, 1, 2], 4, 8, 2, 64, seed=8), Problem([130] * 9, None, None, 1, 4, 4, 128, seed=9)]
    want = [p.run(ctx) for p in probs]
    streams = [torch.cuda.Stream() for _ in probs]
    outs, wss = [p.outputs() for p in probs], [p.workspace(ctx) for p in probs]
    torch.cuda.synchronize()
    for _ in range(5):
        for p, s, out, ws in zip(probs, streams, outs, wss):
            p.forward(ctx, out, ws, stream=s)
            p.backward(ctx, out, ws, stream=s)
    torch.cuda.synchronize()
    for w, out in zip(want, outs):
        assert all(torch.equal(w[n], out[n]) for n in w)


def test_captured_and_replayed_with_other_lengths(ctx):
    """A graph of forward and backward follows the counts and the packing of the moment, as long as the capacities hold."""
    p = Problem([200, 100, 60], [50, 90], [0, 1, 5], 4, 4, 2, 64, seed=10, spare=40)
    q = Problem([10, 250, 99], [120, 20], [2, 4, 7], 4, 4, 2, 64, seed=11, spare=41)
    out, ws = p.outputs(), p.workspace(ctx)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.forward(ctx, out, ws)
        p.backward(ctx, out, ws)
    graph.replay()
    torch.cuda.synchronize()
    p.check(out)
    for n in ("q", "k", "v", "d_o", "pk", "pv", "d_cu", "d_num", "d_cup", "d_idx"):
        getattr(p, n).copy_(getattr(q, n)[:getattr(p, n).shape[0]])
    p.T, p.cu, p.index, p.cu_prompts, p.seqs = q.T, q.cu, q.index, q.cu_prompts, q.seqs
    for t in out.values():
        t.fill_(-7.0)
    graph.replay()
    torch.cuda.synchronize()
    p.check(out)


def test_bad_row_numbers_are_reported_and_not_followed(ctx):
    def broken(change):
        p = Problem([60, 80], [30, 40], [0, 5], 4, 4, 2, 64)
        change(p)
        out, ws = p.outputs(), p.workspace(ctx)
        p.forward(ctx, out, ws)
        p.backward(ctx, out, ws)
        torch.cuda.synchronize()
        assert B.arrol_poll_status(ctx, raise_on_error=False) == 16
        assert B.arrol_poll_status(ctx) == 0

    def put(name, at, value):
        def change(p):
            getattr(p, name)[at] = value
        return change

    for change in (put("d_cu", 1, -4), put("d_cu", 1, 1 << 50), put("d_cu", 2, 100), put("d_cu", 0, 9), put("d_cup", 1, 1 << 40), put("d_cup", 2, 71),
                   put("d_cup", 1, -1), put("d_idx", 1, 8), put("d_idx", slice(0, 2), torch.tensor([5, 0], dtype=torch.int32)), put("d_idx", 0, -1), put("d_num", 0, 0)):
        broken(change)


def test_counts_beyond_the_capacities_are_clamped(ctx):
    p = Problem([60, 80], [30, 40], [0, 5], 4, 4, 2, 64, seed=12)
    want = p.run(ctx)
    p.d_num.copy_(torch.tensor([1 << 40, 1 << 40]))
    got = p.run(ctx)
    assert all(torch.equal(want[n], got[n]) for n in want)


def test_refuses_a_workspace_that_is_too_small(ctx):
    p = Problem([60], None, None, 1, 4, 2, 64)
    out = p.outputs()
    for call, backward in ((p.forward, False), (p.backward, True)):
        ws = p.workspace(ctx, backward)
        with pytest.raises(B.ArrolError) as e:
            call(ctx, out, ws[:-256])
        assert e.value.code == -3
    assert (out["o"].float() == -7).all()


def test_empty_prompts_and_sequences_without_an_index(ctx):
    """Prompts that are all empty; every rollout present (no survivor_idx); a single prompt row."""
    p = Problem([30, 200], [0, 0], [0, 5], 4, 4, 2, 64, seed=13)
    p.check(p.run(ctx))
    p = Problem([30, 0, 70, 129], [5, 66], None, 2, 4, 2, 64, seed=14)
    p.check(p.run(ctx))
    p = Problem([300], [1], [3], 4, 8, 1, 128, seed=15)
    p.check(p.run(ctx))


def test_no_tokens_at_all(ctx):
    p = Problem([], [40, 3], [], 4, 4, 2, 64)
    out = p.run(ctx)
    assert (out["dprompt_k"] == 0).all() and (out["dprompt_v"] == 0).all()
    p = Problem([], None, None, 1, 4, 2, 64)
    p.run(ctx)


def test_a_prompt_whose_tokens_are_split_into_parts(ctx):
    """Few tiles and many tokens that pass by them: the prompt's gradients come from parts of the tokens that are added up, in one order."""
    p = Problem([700, 650, 720, 30], [200], [0, 1, 2, 3], 4, 8, 2, 64, seed=16)
    out = p.run(ctx)
    p.check(out)
    again = p.run(ctx)
    assert torch.equal(out["dprompt_k"], again["dprompt_k"]) and torch.equal(out["dprompt_v"], again["dprompt_v"])


# Few query rows and many keys: the keys are split over blocks and joined.  Parts without a key (their number comes from the arrays' sizes, the lengths
# from the device), parts of the prompt alone and of own keys alone, and parts that only one of a pair of tiles needs.
SPLIT = [
    # lens, prompts, index, G, Hq, Hkv, D
    ([64], [6000], [0], 1, 4, 1, 128),
    ([1], [5000], [0], 1, 2, 1, 64),
    ([30, 25, 31, 28], [3000, 2900], [0, 1, 2, 3], 2, 8, 2, 64),
    ([100, 3], [4500, 1], [0, 1], 1, 4, 2, 128),
    ([3, 100], [1, 4500], [0, 1], 1, 4, 2, 64),
    ([2, 200], [0, 5000], [0, 1], 1, 7, 1, 96),
    ([3000], None, None, 1, 1, 1, 128),
    ([3001], None, None, 1, 2, 1, 64),
    ([2500, 900], [1500, 10], [0, 1], 1, 2, 1, 72),
    ([40] * 6, [700] * 6, [0, 1, 2, 3, 4, 5], 1, 4, 4, 8),
]


@pytest.mark.parametrize("lens,prompts,index,G,Hq,Hkv,D", SPLIT)
def test_few_rows_whose_keys_are_split(ctx, lens, prompts, index, G, Hq, Hkv, D):
    p = Problem(lens, prompts, index, G, Hq, Hkv, D, seed=len(lens) + D, spare=5, fill=math.nan)
    out = p.run(ctx)
    p.check(out)
    again = p.run(ctx)
    assert all(torch.equal(out[n][:1], again[n][:1]) for n in out) and torch.equal(out["o"][:p.T], again["o"][:p.T])


@pytest.mark.parametrize("D,Hq,Hkv", [(64, 4, 1), (128, 4, 2), (128, 7, 1)])
@pytest.mark.parametrize("at", [0, 127, 128, 1500, 2559])
def test_not_a_number_where_the_keys_are_split(ctx, D, Hq, Hkv, at):
    """One key or value of a shared prompt: every row of its sequences has it, and no row of the others."""
    make = lambda: Problem([60, 70, 50], [2560, 900], [0, 1, 3], 2, Hq, Hkv, D, seed=21)  # noqa: E731
    good = make().run(ctx, backward=False)
    for where, value in (("pv", math.nan), ("pv", math.inf), ("pk", math.nan)):
        p = make()
        getattr(p, where)[at, 0, D // 2] = value
        out = p.run(ctx, backward=False)
        assert torch.equal(out["o"][130:], good["o"][130:]) and torch.equal(out["lse"][130:], good["lse"][130:])
        assert not torch.isfinite(out["o"][:130, :Hq // Hkv, D // 2]).any(), where


@pytest.mark.parametrize("D", [64, 128])
def test_split_keys_captured_and_replayed_with_other_lengths(ctx, D):
    """The number of parts is the launch's; a replay with short prompts leaves most of them without a key, one with none and no rows all of them."""
    p = Problem([64, 40], [3500, 2000], [0, 1], 1, 4, 2, D, seed=22, spare=20)
    others = [Problem([1, 70], [3, 130], [0, 1], 1, 4, 2, D, seed=23, spare=5420), Problem([0, 0], [0, 0], [0, 1], 1, 4, 2, D, seed=24, spare=6000),
              Problem([100, 2], [100, 5000], [0, 1], 1, 4, 2, D, seed=25, spare=450)]
    out, ws = p.outputs(), p.workspace(ctx, False)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.forward(ctx, out, ws)
    for q in [None] + others:
        if q is not None:
            for n in ("q", "k", "v", "pk", "pv", "d_cu", "d_num", "d_cup", "d_idx"):
                getattr(p, n).copy_(getattr(q, n)[:getattr(p, n).shape[0]])
            p.T, p.cu, p.index, p.cu_prompts, p.seqs = q.T, q.cu, q.index, q.cu_prompts, q.seqs
        for t in out.values():
            t.fill_(-7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert B.arrol_poll_status(ctx) == 0
        if p.T:
            p.check({"o": out["o"], "lse": out["lse"]}, backward=False)
        else:
            assert (out["o"].float() == -7).all() and (out["lse"] == -7).all()


def test_large_scores_where_the_keys_are_split(ctx):
    """Parts whose maxima lie hundreds apart."""
    p = Problem([50], [4000], [0], 1, 4, 1, 64, seed=26, q_scale=60.0)
    p.pk *= torch.linspace(0, 1, 4000, device="cuda").view(-1, 1, 1).to(BF)
    out = p.run(ctx, backward=False)
    res, tol = p.reference(False)
    # as above: sums of 64 products in fp32, |z| 2^-20
    extra = (p.q.float().norm(dim=-1).max() * max(p.k.float().norm(dim=-1).max(), p.pk.float().norm(dim=-1).max()) * p.scale).item() * 2.0 ** -20
    spread = max(p.v.abs().max(), p.pv.abs().max()).double()
    assert ((out["o"].double() - res["o"]).abs() <= tol["o"] + 2 * extra * spread).all()
    assert ((out["lse"].double() - res["lse"]).abs() <= tol["lse"] + extra).all()


def test_a_workspace_for_the_largest_call_serves_the_smaller_ones(ctx):
    """Fewer tokens may mean more parts, but never more bytes."""
    for Hq, Hkv, D in ((4, 1, 128), (8, 2, 64), (32, 8, 128), (7, 1, 96), (200, 100, 8)):
        for backward in (False, True):
            ask = lambda T, rows: A.arrol_attention_workspace(ctx, 4, T, rows, Hq, Hkv, D, backward)  # noqa: E731
            tokens, prompts = (1, 64, 65, 300, 1000, 2500, 8192, 40000, 300000), (0, 1, 500, 2600, 6000, 30000, 200000)
            for rows in prompts:
                sizes = [ask(T, rows) for T in tokens]
                assert sizes == sorted(sizes), (Hq, Hkv, D, backward, rows, sizes)
            for T in tokens:
                sizes = [ask(T, rows) for rows in prompts]
                assert sizes == sorted(sizes), (Hq, Hkv, D, backward, T, sizes)
    p = Problem([64], [6000], [0], 1, 4, 1, 128, seed=27)
    ws, out = torch.full((A.arrol_attention_workspace(ctx, 1, 8192, 6000, 4, 1, 128, True),), 0xAB, dtype=torch.uint8, device="cuda"), p.outputs()
    p.forward(ctx, out, ws)
    p.backward(ctx, out, ws)
    torch.cuda.synchronize()
    p.check(out)


def test_gradients_agree_with_differences(ctx):
    """The loss changes by gradient times step: coarse, as q, k, v are bf16, but of the kernel's own forward."""
    p = Problem([90, 60], [40], [0, 1], 2, 4, 2, 64, seed=17)
    out = p.run(ctx)
    g = torch.Generator("cuda").manual_seed(1)
    for name, grad in (("q", "dq"), ("k", "dk"), ("v", "dv"), ("pk", "dprompt_k"), ("pv", "dprompt_v")):
        x = getattr(p, name)
        old = x.clone()
        step = (torch.randn(x.shape, generator=g, device="cuda") * 0.05).to(BF)
        losses = []
        for sign in (1, -1):
            x.copy_((old.float() + sign * step.float()).to(BF))
            moved = (x.double() - old.double())
            o = p.run(ctx, backward=False)["o"]
            losses.append(((o.double() * p.d_o.double()).sum().item(), (moved * out[grad].double()).sum().item()))
        x.copy_(old)
        found, expected = losses[0][0] - losses[1][0], losses[0][1] - losses[1][1]
        # what the roundings of o (2^-8 of each, of either sign) and of the gradient leave of a difference of two sums
        noise = 2 * 2.0 ** -8 * ((out["o"].double() * p.d_o.double()) ** 2).sum().sqrt().item() * 2
        assert abs(found - expected) <= noise + 0.02 * abs(expected), (name, found, expected, noise)


@pytest.mark.parametrize("D,Hq,Hkv,first,rows", [(64, 32, 8, 8, 75), (64, 32, 8, 8, 80), (64, 32, 8, 8, 64), (64, 32, 8, 16, 33), (40, 28, 4, 6, 90), (128, 32, 8, 8, 40)])
def test_many_values_that_are_not_finite_beside_another_prompt(ctx, D, Hq, Hkv, first, rows):
    """The first tile of an item holds short sequences whose prompts, several blocks in all, are full of NaN; the second tile's prompt begins behind them,
    inside a block, and so keeps its values from a stage that those blocks had before it.  Its rows are those of a clean call, bit for bit."""
    tile = 128 // (Hq // Hkv)
    lens, prompts, clean = [], [], []
    for _ in range(3):                          # three items
        each = [tile // first] * first
        each[-1] += tile - sum(each)
        lens += each + [tile]
        prompts += [rows] * first + [100]
        clean += [False] * first + [True]
    make = lambda: Problem(lens, prompts, list(range(len(lens))), 1, Hq, Hkv, D, seed=31)  # noqa: E731
    good, p = make().run(ctx), make()
    for i, c in enumerate(clean):
        if not c:
            p.pv[p.cu_prompts[i]:p.cu_prompts[i + 1], :, ::3] = math.nan
    keep = torch.tensor([c for c, n in zip(clean, lens) for _ in range(n)], device="cuda")
    kept_prompts = torch.tensor([c for c, n in zip(clean, prompts) for _ in range(n)], device="cuda")
    for _ in range(20):
        out = p.run(ctx)
        for name in ("o", "lse", "dq", "dk", "dv"):
            assert torch.equal(out[name][keep], good[name][keep]), name
        for name in ("dprompt_k", "dprompt_v"):
            assert torch.equal(out[name][kept_prompts], good[name][kept_prompts]), name
        assert not torch.isfinite(out["o"][~keep][..., 0]).any()


@pytest.mark.parametrize("n", [32, 64, 128])
@pytest.mark.parametrize("D,Hq,Hkv", [(64, 4, 4), (128, 4, 2), (16, 1, 1), (128, 32, 1), (64, 64, 1)])
def test_prompts_and_sequences_as_long_as_a_block(ctx, D, Hq, Hkv, n):
    """Ranges of keys as long as a block of them, but not at its beginning: the first token's prompt begins the blocks, a prompt and a sequence of exactly n
    rows follow at odd places, so that every row of a warp has n keys of which some are in the block."""
    p = Problem([37, 150, n, n + 1, 200, n], [29, n, n, 1, n], [0, 1, 1, 2, 3, 4], 1, Hq, Hkv, D, seed=32)
    p.check(p.run(ctx))
