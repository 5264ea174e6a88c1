"""GPU parity of the single-token attention call against the 64-bit reference."""
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


class Problem:
    """lengths[i] rows of rollout i's cache, `gap` rows between the caches (and `fill` in them); prompts = None: none."""

    def __init__(self, lengths, prompts=None, G=1, Hq=4, Hkv=2, D=64, keep=None, seed=0, gap=3, fill=0.0, wide=False, q_scale=1.5):
        dev, g = "cuda", torch.Generator("cuda").manual_seed(seed)
        mk = lambda *s, by=1.0: (torch.randn(*s, generator=g, device=dev) * by).to(BF)  # noqa: E731
        N, rows, self.off = len(lengths), 0, []
        for n in lengths:
            rows += gap
            self.off.append(rows)
            rows += n
        rows += gap
        self.N, self.G, self.Hq, self.Hkv, self.D, self.scale = N, G, Hq, Hkv, D, 1 / math.sqrt(D)
        self.lengths, self.keep = lengths, keep
        self.q = mk(N, Hq, D, by=q_scale)
        if wide:
            kv = mk(rows, 2 * Hkv, D)
            self.k, self.v = kv[:, :Hkv], kv[:, Hkv:]
        else:
            self.k, self.v = mk(rows, Hkv, D), mk(rows, Hkv, D)
        live = torch.zeros(rows, dtype=torch.bool, device=dev)
        for a, n in zip(self.off, lengths):
            live[a:a + n] = True
        self.k[~live] = fill
        self.v[~live] = fill
        self.pk = self.pv = self.cup = self.d_cup = None
        if prompts is not None:
            self.cup = [0]
            for n in prompts:
                self.cup.append(self.cup[-1] + n)
            self.pk, self.pv = mk(self.cup[-1] + gap, Hkv, D), mk(self.cup[-1] + gap, Hkv, D)
            self.pk[self.cup[-1]:] = fill
            self.pv[self.cup[-1]:] = fill
            self.d_cup = torch.tensor(self.cup, dtype=torch.int64, device=dev)
        self.d_off = torch.tensor(self.off, dtype=torch.int64, device=dev)
        self.d_len = torch.tensor(lengths, dtype=torch.int32, device=dev)
        self.d_keep = None if keep is None else torch.tensor(keep, dtype=torch.uint8, device=dev)

    def workspace(self, ctx):
        n = A.arrol_attention_decode_workspace(ctx, self.N, 0 if self.cup is None else len(self.cup) - 1, self.Hq, self.Hkv, self.D)
        assert n > 0
        return torch.full((n,), 0xAB, dtype=torch.uint8, device="cuda")

    def outputs(self):
        return torch.full((self.N, self.Hq, self.D), -7.0, dtype=BF, device="cuda"), torch.full((self.N, self.Hq), -7.0, device="cuda")

    def call(self, ctx, o, lse, ws, **kw):
        shared = {} if self.pk is None else dict(prompt_k=self.pk, prompt_v=self.pv, cu_prompts=self.d_cup)
        A.arrol_attention_decode(ctx, self.q, self.k, self.v, self.d_off, self.d_len, o, lse, ws, keep=self.d_keep, scale=self.scale, G=self.G, **shared, **kw)

    def run(self, ctx, status=0):
        o, lse = self.outputs()
        self.call(ctx, o, lse, self.workspace(ctx))
        torch.cuda.synchronize()
        assert B.arrol_poll_status(ctx, raise_on_error=False) == status
        return o, lse

    def check(self, o, lse):
        ro, tol, rl = R.decode(self.q, self.k, self.v, self.off, self.lengths, self.keep, self.pk, self.pv, self.cup, self.G, self.scale)
        kept = torch.ones(self.N, dtype=torch.bool) if self.keep is None else torch.tensor(self.keep).bool()
        kept = kept.cuda()
        d = (o.double() - ro).abs()
        assert (d <= tol)[kept].all(), (d / tol.clamp(min=1e-30))[kept].max()
        none = rl == -math.inf
        assert (lse[none & kept[:, None]] == -math.inf).all()
        some = ~none & kept[:, None]
        assert ((lse.double() - rl).abs()[some] <= (2e-5 * (1 + rl.abs()))[some]).all()
        assert (o[~kept].float() == -7).all() and (lse[~kept] == -7).all()


CASES = [
    # lengths, prompts, G, Hq, Hkv, D, keep
    ([1], None, 1, 1, 1, 64, None),
    ([0], None, 1, 4, 2, 64, None),
    ([0, 5, 0, 1], [0, 3], 2, 4, 2, 128, None),
    ([0, 0, 9, 0], [40, 0], 2, 4, 1, 64, [1, 0, 1, 1]),
    ([127, 128, 129, 1000], None, 1, 8, 2, 128, None),
    ([17, 300, 64, 65, 2, 0, 511, 90], [129, 700], 4, 8, 2, 64, [1, 1, 0, 1, 0, 0, 1, 1]),
    ([20] * 16, [900], 16, 32, 8, 128, [1, 0] * 8),
    ([40] * 33, [333], 33, 8, 1, 64, None),                     # 264 query rows of one key head
    ([70] * 6, [50, 64], 3, 64, 1, 128, None),                  # 192
    ([30, 2, 100], [10], 3, 21, 3, 96, None),
    ([30, 2, 100], [10], 3, 5, 1, 8, None),
    ([4000, 1], [2500, 0], 1, 7, 1, 128, None),
    ([9000], None, 1, 2, 1, 64, None),
    ([60, 200] * 40, [100] * 20, 4, 4, 2, 72, [1, 1, 0, 0] * 20),
    ([500] * 4, [77], 4, 16, 16, 128, [0, 0, 0, 1]),
]


@pytest.mark.parametrize("lengths,prompts,G,Hq,Hkv,D,keep", CASES)
def test_decode_matches_the_definition(ctx, lengths, prompts, G, Hq, Hkv, D, keep):
    p = Problem(lengths, prompts, G, Hq, Hkv, D, keep, seed=len(lengths) + Hq)
    p.check(*p.run(ctx))


@pytest.mark.parametrize("fill", [math.nan, math.inf])
def test_rows_between_the_caches_may_hold_anything(ctx, fill):
    p = Problem([100, 3, 0, 190], [65, 40], 2, 6, 2, 128, [1, 1, 1, 0], seed=3, gap=70, fill=fill, wide=True)
    p.check(*p.run(ctx))
    p = Problem([1, 33, 64, 900], None, 1, 8, 8, 64, seed=4, gap=1, fill=fill)
    p.check(*p.run(ctx))


def test_not_a_number_in_a_cache_reaches_its_rollout_alone(ctx):
    for where, value in (("k", math.nan), ("v", math.nan), ("v", math.inf)):
        p = Problem([100, 150, 30, 64], [65, 40], 2, 4, 2, 64, seed=5)
        good = p.run(ctx)
        getattr(p, where)[p.off[1] + 149, 0, 5] = value
        bad = p.run(ctx)
        for x, y in zip(good, bad):
            assert torch.equal(x[[0, 2, 3]], y[[0, 2, 3]])
        assert not torch.isfinite(bad[0][1, :2, 5]).any()


def test_same_bits_every_time_on_streams_and_in_graphs(ctx):
    p = Problem([300, 1200, 20, 0, 777, 64, 65, 3000], [500, 90], 4, 8, 2, 128, [1, 1, 1, 1, 0, 1, 1, 1], seed=6)
    first = p.run(ctx)
    for _ in range(3):
        again = p.run(ctx)
        assert all(torch.equal(x, y) for x, y in zip(first, again))
    other = Problem([5, 700, 60, 2] * 30, None, 1, 4, 4, 64, seed=7)
    want = other.run(ctx)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs, wss = [x.outputs() for x in (p, other)], [x.workspace(ctx) for x in (p, other)]
    torch.cuda.synchronize()
    for _ in range(5):
        for x, s, out, ws in zip((p, other), streams, outs, wss):
            x.call(ctx, *out, ws, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(first + want, outs[0] + outs[1]))
    # a captured step follows the lengths and the mask of the moment
    out, ws = p.outputs(), p.workspace(ctx)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.call(ctx, *out, ws)
    p.lengths, p.keep = [299, 1000, 21 - 4, 0, 700, 60, 65, 100], [1, 0, 1, 1, 1, 1, 0, 1]
    p.d_len.copy_(torch.tensor(p.lengths, dtype=torch.int32))
    p.d_keep.copy_(torch.tensor(p.keep, dtype=torch.uint8))
    for t in out:
        t.fill_(-7.0)
    graph.replay()
    torch.cuda.synchronize()
    p.check(*out)


def test_bad_cache_rows_are_reported_and_not_followed(ctx):
    for name, at, value, other in (("d_off", 1, -1, [0, 2, 3]), ("d_off", 2, 1 << 50, [0, 1, 3]), ("d_len", 3, 1 << 30, [0, 1, 2]), ("d_len", 0, -5, [1, 2, 3]),
                                   ("d_cup", 1, 1 << 40, []), ("d_cup", 0, -3, [2, 3]), ("d_cup", 2, 5, [0, 1])):
        p = Problem([100, 150, 30, 64], [65, 40], 2, 4, 2, 64, seed=8)
        good = p.run(ctx)
        getattr(p, name)[at] = value
        bad = p.run(ctx, status=16)
        for x, y in zip(good, bad):
            assert torch.equal(x[other], y[other])
    # a rollout that is not kept is not looked at
    p = Problem([100, 150, 30, 64], [65, 40], 2, 4, 2, 64, [1, 0, 1, 1], seed=8)
    good = p.run(ctx)
    p.d_off[1], p.d_len[1] = -(1 << 60), -1
    assert all(torch.equal(x, y) for x, y in zip(good, p.run(ctx)))


def test_lse_is_optional(ctx):
    p = Problem([100, 0, 30], None, 1, 4, 2, 64, seed=9)
    o, lse = p.run(ctx)
    o2, _ = p.outputs()
    p.call(ctx, o2, None, p.workspace(ctx))
    torch.cuda.synchronize()
    assert torch.equal(o, o2)


def test_nothing_kept_and_no_rollouts(ctx):
    p = Problem([10, 20], [30], 2, 4, 2, 64, [0, 0])
    o, lse = p.run(ctx)
    assert (o.float() == -7).all() and (lse == -7).all()
    p = Problem([], None, 1, 4, 2, 64)
    p.run(ctx)


def test_empty_caches_and_empty_prompts(ctx):
    """No cache rows at all, prompts alone; prompts that are all empty."""
    p = Problem([0, 0], [70], 2, 4, 2, 64, seed=10, gap=0)
    p.check(*p.run(ctx))
    p = Problem([5, 90, 0], [0], 3, 4, 2, 128, seed=11, gap=0)
    p.check(*p.run(ctx))


def test_caches_may_share_rows(ctx):
    """Rollouts that were forked read the same rows."""
    p = Problem([200, 90, 90], None, 1, 8, 2, 64, seed=12)
    p.off = [p.off[0], p.off[0] + 10, p.off[0] + 10]
    p.d_off.copy_(torch.tensor(p.off))
    o, lse = p.run(ctx)
    p.check(o, lse)


def test_large_scores(ctx):
    """One key takes nearly all of the weight; maxima change from tile to tile."""
    p = Problem([900, 300], [500], 2, 8, 2, 64, seed=13, q_scale=60.0)
    o, lse = p.run(ctx)
    ro, tol, rl = R.decode(p.q, p.k, p.v, p.off, p.lengths, None, p.pk, p.pv, p.cup, p.G, p.scale)
    zmax = (p.q.float().norm(dim=-1).max() * max(p.k.float().norm(dim=-1).max(), p.pk.float().norm(dim=-1).max()) * p.scale).item()
    extra = zmax * 2.0 ** -20          # the exponent's error: 64 products summed in fp32
    assert ((o.double() - ro).abs() <= tol + 2 * extra * p.v.abs().max().double()).all()
    assert ((lse.double() - rl).abs() <= 2e-5 * (1 + rl.abs()) + extra).all()


@pytest.mark.parametrize("D,Hq,Hkv", [(64, 4, 2), (128, 8, 1), (72, 3, 3)])
def test_keys_whose_scores_are_minus_infinity_are_keys(ctx, D, Hq, Hkv):
    """A softmax over scores of minus infinity alone is not a number; no key at all gives zeros.  One key, several chunks of them, a prompt's."""
    make = lambda: Problem([1, 400, 0, 60, 0], [0, 90, 0, 0, 130], 1, Hq, Hkv, D, seed=14)  # noqa: E731
    good, p = make().run(ctx), make()
    p.q[:, :, 0] = 1.0
    for i in (0, 1):
        p.k[p.off[i]:p.off[i] + p.lengths[i], :, 0] = -math.inf
    for i in (1, 4):
        p.pk[p.cup[i]:p.cup[i + 1], :, 0] = -math.inf
    o, lse = p.run(ctx)
    for i in (0, 1, 4):
        assert not torch.isfinite(o[i]).any() and not torch.isfinite(lse[i]).any(), i
    assert (o[2] == 0).all() and (lse[2] == -math.inf).all()
    assert torch.isfinite(o[3]).all() and torch.isfinite(lse[3]).all()
    # beside a key with a score they weigh nothing
    p = make()
    p.q[:, :, 0] = 1.0
    clean = p.run(ctx)
    p.k[p.off[1]:p.off[1] + 300, :, 0] = -math.inf
    p.pk[p.cup[4]:p.cup[5] - 1, :, 0] = -math.inf
    o, lse = p.run(ctx)
    assert torch.isfinite(o).all() and torch.isfinite(lse[[0, 1, 3, 4]]).all()
    assert all(torch.equal(x[[0, 2, 3]], y[[0, 2, 3]]) for x, y in zip(clean, (o, lse)))
    assert torch.equal(o[4], p.pv[p.cup[5] - 1].repeat_interleave(Hq // Hkv, 0))
    assert good[0].shape == o.shape


@pytest.mark.parametrize("where,value", [("pk", math.nan), ("pv", math.nan), ("pv", math.inf), ("pk", math.inf), ("pk", -math.inf), ("k", math.inf), ("k", -math.inf)])
def test_not_a_number_in_a_prompt_or_a_key_reaches_its_rollouts_alone(ctx, where, value):
    p = Problem([100, 150, 30, 64], [65, 40], 2, 4, 2, 64, seed=15)
    p.q[:, :, 5] = 1.0
    good = p.run(ctx)
    at, reached = (70, [2, 3]) if where[0] == "p" else (p.off[1] + 149, [1])
    getattr(p, where)[at, 0, 5] = value
    bad = p.run(ctx)
    others = [i for i in range(4) if i not in reached]
    for x, y in zip(good, bad):
        assert torch.equal(x[others], y[others]) and torch.equal(x[reached, 2:], y[reached, 2:])
    if value != -math.inf:                     # a key of no weight is all that a score of minus infinity makes
        assert not torch.isfinite(bad[0][reached, :2, 5]).any()


@pytest.mark.parametrize("lengths,prompts,G,Hq,Hkv,D", [
    ([0, 226, 0, 834, 156, 705, 550, 757, 0, 547, 1, 0, 1, 24, 595, 0, 1, 0, 0, 96, 0, 1, 1, 0, 0, 1, 0, 170, 205, 0, 0, 0, 1, 565, 1, 0, 219, 140, 281, 193, 462, 188, 24, 177,
      771, 157, 651, 387, 379, 0, 1, 83, 74, 86, 268, 1, 392, 3, 281, 1], [55, 178, 0, 142], 15, 32, 8, 64),
    ([700, 30, 608, 250] * 10, [227, 80, 1, 300], 10, 64, 8, 128),
    ([33, 64, 407, 851] * 14, None, 1, 128, 8, 128),
])
def test_same_bits_over_many_calls(ctx, lengths, prompts, G, Hq, Hkv, D):
    """The stages of the ring change hands between readers and copies thousands of times: calls one behind another, all results compared on the device."""
    p = Problem(lengths, prompts, G, Hq, Hkv, D, seed=16, gap=70, fill=math.nan)
    o, lse = p.run(ctx)
    p.check(o, lse)
    ws, other = p.workspace(ctx), torch.zeros((), dtype=torch.bool, device="cuda")
    for _ in range(1500):
        again = p.outputs()
        p.call(ctx, *again, ws)
        other |= (again[0] != o).any() | (again[1] != lse).any()
    assert B.arrol_poll_status(ctx) == 0 and not other.item()
