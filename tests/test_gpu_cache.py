"""GPU parity of the paged 8-bit cache: appends and attention of one token per rollout against the 64-bit reference, and a generation loop of them."""
import math

import pytest
import torch

import cache_reference as CR
from paper_2603_24840_b200 import binding as B
from paper_2603_24840_b200 import cache as K
from paper_2603_24840_b200 import rotary as R

pytestmark = pytest.mark.gpu

BF, F8 = torch.bfloat16, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    c.close()


class Pool:
    """Pages that no sequence has hold NaN, and so do their scales.  `both`: keys and values of a page in one buffer."""

    def __init__(self, pages, Hkv, page, D, seed=0, both=False):
        self.g = torch.Generator("cuda").manual_seed(seed)
        if both:
            buffer = torch.full((pages, 2, Hkv, page, D), 0x7F, dtype=torch.uint8, device="cuda").view(F8)
            self.k, self.v = buffer[:, 0], buffer[:, 1]
            scales = torch.full((pages, 2, Hkv), math.nan, device="cuda")
            self.ks, self.vs = scales[:, 0], scales[:, 1]
        else:
            self.k, self.v = (torch.full((pages, Hkv, page, D), 0x7F, dtype=torch.uint8, device="cuda").view(F8) for _ in range(2))
            self.ks, self.vs = (torch.full((pages, Hkv), math.nan, device="cuda") for _ in range(2))
        self.order = torch.randperm(pages, generator=self.g, device="cuda").to(torch.int32)
        self.used, self.page, self.Hkv, self.D, self.pages = 0, page, Hkv, D, pages

    def table(self, counts, spare=1):
        """Rows of page numbers for so many tokens each, behind them numbers that are none."""
        most = max([-(-n // self.page) for n in counts] + [0]) + spare
        t = torch.full((len(counts), most), -(1 << 30), dtype=torch.int32, device="cuda")
        for i, n in enumerate(counts):
            m = -(-n // self.page)
            t[i, :m] = self.order[self.used:self.used + m]
            self.used += m
        assert self.used <= self.pages
        return t

    def fill(self, table, counts, spread=1.0):
        """Random numbers in the slots of these tokens, scales from 2^-9 spread-wide powers of two."""
        for i, n in enumerate(counts):
            for x in range(-(-n // self.page)):
                p, m = int(table[i, x]), min(self.page, n - x * self.page)
                for c, s in ((self.k, self.ks), (self.v, self.vs)):
                    # e4m3 numbers of an ordinary size times scales that bring them to about 1
                    power = torch.round(torch.randn(self.Hkv, generator=self.g, device="cuda") * spread) - 7
                    c.view(torch.uint8)[p, :, :m] = (torch.randn(self.Hkv, m, self.D, generator=self.g, device="cuda") * 100).clamp(-448, 448).to(F8).view(torch.uint8)
                    s[p] = torch.exp2(power)

    def args(self):
        return self.k, self.v, self.ks, self.vs


class Attend:
    def __init__(self, lengths, prompts=None, G=1, Hq=4, Hkv=2, D=64, page=32, keep=None, seed=0, both=False, q_scale=1.5, spread=0.5):
        self.N, self.Hq, self.lengths, self.prompts, self.G, self.keep, self.scale = len(lengths), Hq, lengths, prompts, G, keep, 1 / math.sqrt(D)
        need = sum(-(-n // page) for n in lengths) + sum(-(-n // page) for n in prompts or [])
        self.pool = Pool(need + 3, Hkv, page, D, seed, both)
        self.table = self.pool.table(lengths)
        self.pool.fill(self.table, lengths, spread)
        self.p_table = self.d_prompts = None
        if prompts is not None:
            self.p_table = self.pool.table(prompts, spare=2)
            self.pool.fill(self.p_table, prompts, spread)
            self.d_prompts = torch.tensor(prompts, dtype=torch.int32, device="cuda")
        self.q = (torch.randn(self.N, Hq, D, generator=self.pool.g, device="cuda") * q_scale).to(BF)
        self.d_len = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.d_keep = None if keep is None else torch.tensor(keep, dtype=torch.uint8, device="cuda")

    def workspace(self, ctx):
        n = K.arrol_cache_attention_workspace(ctx, self.N, len(self.prompts or []), self.G, self.Hq, self.pool.Hkv, self.pool.D)
        assert n > 0
        return torch.full((n,), 0xAB, dtype=torch.uint8, device="cuda")

    def outputs(self):
        return torch.full(self.q.shape, -7.0, dtype=BF, device="cuda"), torch.full((self.N, self.Hq), -7.0, device="cuda")

    def call(self, ctx, o, lse, ws, **kw):
        shared = {} if self.prompts is None else dict(prompt_table=self.p_table, prompt_lengths=self.d_prompts)
        K.arrol_cache_attention(ctx, self.q, *self.pool.args(), self.table, self.d_len, o, lse, ws, keep=self.d_keep, scale=self.scale, G=self.G, **shared, **kw)

    def run(self, ctx, status=0):
        o, lse = self.outputs()
        self.call(ctx, o, lse, self.workspace(ctx))
        torch.cuda.synchronize()
        assert B.arrol_poll_status(ctx, raise_on_error=False) == status
        return o, lse

    def check(self, o, lse, extra=0.0):
        own = [CR.read_many(c, s, self.table, self.lengths) for c, s in ((self.pool.k, self.pool.ks), (self.pool.v, self.pool.vs))]
        shared = [CR.read_many(c, s, self.p_table, self.prompts) for c, s in ((self.pool.k, self.pool.ks), (self.pool.v, self.pool.vs))] if self.prompts is not None else None
        for i in range(self.N):
            if self.keep is not None and not self.keep[i]:
                assert (o[i].float() == -7).all() and (lse[i] == -7).all()
                continue
            key, val = ((torch.cat([shared[x][i // self.G], own[x][i]]) if shared else own[x][i]) for x in range(2))
            want, tol, ll = CR.attend(self.q[i], key, val, self.scale)
            d = (o[i].double() - want).abs()
            big = val.abs().max() if extra else 0.0
            fine = torch.isfinite(want)                       # where the formula is not finite, the call is not
            assert torch.equal(fine, torch.isfinite(o[i])) and torch.equal(torch.isfinite(ll), torch.isfinite(lse[i])) or not len(key), i
            assert (d <= tol + 2 * extra * big)[fine].all(), (i, (d / tol)[fine].max())
            if len(key):
                assert ((lse[i].double() - ll).abs() <= 2e-5 * (1 + ll.abs()) + extra)[torch.isfinite(ll)].all(), i
            else:
                assert (lse[i] == -math.inf).all() and not o[i].any()


ATTEND = [
    # lengths, prompts, G, Hq, Hkv, D, page, keep
    ([1], None, 1, 1, 1, 64, 16, None),
    ([0], None, 1, 4, 2, 64, 16, None),
    ([0, 5, 0, 1], [0, 3], 2, 4, 2, 128, 32, None),
    ([0, 0, 9, 0], [40, 0], 2, 4, 1, 64, 64, [1, 0, 1, 1]),
    ([15, 16, 17, 31, 32, 33, 127, 128, 129, 1000], None, 1, 8, 2, 128, 16, None),
    ([127, 128, 129, 1000], None, 1, 8, 2, 64, 128, None),
    ([17, 300, 64, 65, 2, 0, 511, 90], [129, 700], 4, 8, 2, 64, 32, [1, 1, 0, 1, 0, 0, 1, 1]),
    ([20] * 16, [900], 16, 32, 8, 128, 64, [1, 0] * 8),
    ([40] * 33, [333], 33, 8, 1, 64, 16, None),                     # 264 query rows of one key head: five units of 8 rollouts
    ([70] * 6, [50, 64], 3, 64, 1, 128, 32, None),                  # 64 query heads a key head: own tokens are shared units too
    ([70, 400, 0], None, 1, 17, 1, 48, 16, None),
    ([30, 200, 100, 4], [10, 500], 2, 40, 2, 112, 64, [1, 1, 0, 1]),      # 20 a key head: three tiles of 16 rows for two rollouts
    ([30, 2, 100], [10], 3, 21, 3, 96, 32, None),
    ([30, 2, 100], [300], 3, 33, 3, 80, 16, None),                  # 33 rows: a fourth warp without any
    ([30, 2, 100], [10], 3, 5, 1, 16, 16, None),
    ([4000, 1], [2500, 0], 1, 7, 1, 128, 64, None),
    ([9000], None, 1, 2, 1, 64, 128, None),
    ([9000], None, 1, 9, 1, 128, 32, None),                         # rows 8 .. 15 of a tile
    ([60, 200] * 40, [100] * 20, 4, 4, 2, 32, 16, [1, 1, 0, 0] * 20),
    ([500] * 4, [77], 4, 16, 16, 128, 64, [0, 0, 0, 1]),
    ([3, 50] * 150, [20, 0, 170] * 50, 2, 4, 4, 64, 16, [1, 0, 1, 1] * 75),       # more entries than threads
]


@pytest.mark.parametrize("lengths,prompts,G,Hq,Hkv,D,page,keep", ATTEND)
def test_attention_matches_the_definition(ctx, lengths, prompts, G, Hq, Hkv, D, page, keep):
    p = Attend(lengths, prompts, G, Hq, Hkv, D, page, keep, seed=len(lengths) + Hq, both=len(lengths) % 2 == 0)
    p.check(*p.run(ctx))


@pytest.mark.parametrize("D,Hq,Hkv", [(64, 4, 2), (128, 8, 1), (128, 20, 1)])
def test_scales_that_differ_from_page_to_page(ctx, D, Hq, Hkv):
    """Values' scales from 2^-40 to 2^26 of their middle: the larger ones come late, early and alone."""
    p = Attend([200, 333, 64], [150], 3, Hq, Hkv, D, 16, seed=1, spread=0.5)
    power = torch.randint(-40, 27, p.pool.vs.shape, generator=p.pool.g, device="cuda").float()
    p.pool.vs.copy_(torch.exp2(power))
    p.check(*p.run(ctx))
    p.pool.ks.mul_(torch.exp2(torch.randint(-6, 2, p.pool.ks.shape, generator=p.pool.g, device="cuda").float()))
    p.check(*p.run(ctx))


WIDE = [
    # lengths, prompts, G, Hq, Hkv, D, page: a few query rows a key head, 9 to 16, 17 to 32, 33 to 64; pages of half a piece, of one, of several
    ([300, 33, 700], None, 1, 4, 2, 64, 16),
    ([300, 33, 700], None, 1, 8, 1, 128, 32),
    ([1500, 20], None, 1, 12, 1, 128, 16),
    ([300, 150], None, 1, 20, 1, 64, 16),
    ([40, 100, 1, 7], [600, 90], 2, 16, 1, 128, 64),
    ([40, 100, 1, 7], [600], 4, 16, 1, 64, 16),
    ([40, 100, 1], [600], 3, 16, 1, 128, 128),
]


def _weigh(p, page, nats):
    """All tokens of this page score so much more than others do, whose keys have 0 in that dimension; queries have sqrt(D) there."""
    codes = p.pool.k.view(torch.uint8)
    codes[page] = 0
    codes[page, :, :, 1] = torch.tensor(nats * 4.0, device="cuda").to(F8).view(torch.uint8)
    p.pool.ks[page] = 0.25


@pytest.mark.parametrize("place", [0.0, 0.5, 1.0])
@pytest.mark.parametrize("lengths,prompts,G,Hq,Hkv,D,page", WIDE)
def test_a_page_with_values_far_larger_than_the_others(ctx, lengths, prompts, G, Hq, Hkv, D, page, place):
    """Large in one dimension and zero in the others, first, in the middle and last: it carries that dimension, or nothing of it, and the other pages the rest.  Its tokens weigh 2^12
    to 2^-58 of the others'."""
    p = Attend(lengths, prompts, G, Hq, Hkv, D, page, seed=30, q_scale=0.25, spread=0.5)
    p.q[..., 1] = math.sqrt(D)
    p.pool.k.view(torch.uint8)[..., 1] = 0
    tables = [(p.table, lengths)] + ([(p.p_table, prompts)] if prompts else [])
    far = [int(t[i, int(place * (-(-n // page) - 1))]) for t, counts in tables for i, n in enumerate(counts) if n > page]
    far = far[:1] if prompts is None else far[-1:]
    codes, scale = p.pool.v.view(torch.uint8), p.pool.vs[far].clone()
    codes[far, :, :, :3] = 0
    codes[far, :, :, 4:] = 0
    for weight in (0, 8, 12, -58):
        for x in far:
            _weigh(p, x, weight * math.log(2))
        for ratio in (4, 5, 8, 12, 16, 20, 26, 34, 60, 100, -4, -5, -9, -60, -90):
            p.pool.vs[far] = scale * 2.0 ** ratio
            p.check(*p.run(ctx))


@pytest.mark.parametrize("most", [3, 8, 30, 90])
@pytest.mark.parametrize("lengths,prompts,G,Hq,Hkv,D,page", WIDE)
def test_pages_of_values_of_all_sizes(ctx, lengths, prompts, G, Hq, Hkv, D, page, most):
    """Every page has a scale of its own, up to 2^most either way, an eighth of the dimensions, and scores 2^-6 to 2^6 of the others'."""
    p = Attend(lengths, prompts, G, Hq, Hkv, D, page, seed=31 + most, q_scale=0.25, spread=0.5)
    p.q[..., 1] = math.sqrt(D)
    g = p.pool.g
    used = torch.cat([t[t >= 0] for t in [p.table] + ([p.p_table] if prompts else [])]).long()
    codes = p.pool.k.view(torch.uint8)
    codes[..., 1] = (torch.randint(-6, 7, (p.pool.pages, 1, 1), generator=g, device="cuda") * (math.log(2) * 2.0 ** 6)).expand(-1, p.pool.Hkv, page).to(F8).view(torch.uint8)
    p.pool.ks[used] = 2.0 ** -6
    p.pool.vs[used] = torch.exp2(torch.randint(-most, most + 1, (len(used), p.pool.Hkv), generator=g, device="cuda").float())
    p.pool.v.view(torch.uint8)[torch.rand(p.pool.pages, p.pool.Hkv, 1, D, generator=g, device="cuda").expand(p.pool.v.shape) > 0.125] = 0
    p.check(*p.run(ctx))
    p.pool.v.view(torch.uint8)[used[::3]] = 0          # zeros and nothing else: the least scale
    p.pool.vs[used[::3]] = 2.0 ** -100
    p.check(*p.run(ctx))


def _far_apart(p, most=40):
    """Scales of values up to 2^most either way, each page with an eighth of the dimensions."""
    g = p.pool.g
    used = torch.isfinite(p.pool.vs)
    p.pool.vs.copy_(torch.where(used, torch.exp2(torch.randint(-most, most + 1, p.pool.vs.shape, generator=g, device="cuda").float()), p.pool.vs))
    values = p.pool.v.view(torch.uint8)
    drop = torch.rand(p.pool.pages, p.pool.Hkv, 1, p.pool.D, generator=g, device="cuda").expand(values.shape) > 0.125
    values[drop & used[:, :, None, None]] = 0
    return p


@pytest.mark.parametrize("lengths,prompts,G,Hq,Hkv,D,page,keep", ATTEND)
def test_scales_far_apart_match_the_definition(ctx, lengths, prompts, G, Hq, Hkv, D, page, keep):
    p = _far_apart(Attend(lengths, prompts, G, Hq, Hkv, D, page, keep, seed=len(lengths) + Hq, both=len(lengths) % 2 == 0, q_scale=0.5))
    p.check(*p.run(ctx))


@pytest.mark.parametrize("lengths,prompts,G,Hq,Hkv,D", [([33, 20] * 20, None, 1, 64, 8, 128), ([7, 40] * 40, [50] * 10, 8, 64, 4, 64)])
def test_scales_far_apart_in_many_rows(ctx, lengths, prompts, G, Hq, Hkv, D):
    """More rows than the merge spreads over its blocks; some of them ordinary."""
    p = Attend(lengths, prompts, G, Hq, Hkv, D, 16, seed=34, q_scale=0.5)
    _far_apart(p, 6)
    p.check(*p.run(ctx))


def test_rows_with_scales_far_apart_beside_ordinary_ones(ctx):
    """One rollout's, or one key head's: the others keep their bits; the same bits every time, with strided rows, without lse and from a graph; NaN and infinities reach their rows alone."""
    p = Attend([400, 150, 900, 64], [165, 40], 2, 12, 3, 128, 16, seed=33)
    plain = p.run(ctx)
    at = int(p.table[2, 7])
    p.pool.vs[at, 1] *= 2.0 ** 30
    p.pool.v.view(torch.uint8)[at, 1, :, 1:] = 0
    o, lse = p.run(ctx)
    p.check(o, lse)
    others = torch.ones(4, 12, dtype=torch.bool, device="cuda")
    others[2, 4:8] = False
    assert torch.equal(o[others], plain[0][others]) and torch.equal(lse[others], plain[1][others]) and not torch.equal(o[~others], plain[0][~others])
    wide, ws = torch.full((4, 20, 128), -7.0, dtype=BF, device="cuda"), p.workspace(ctx)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        p.call(ctx, wide[:, 3:15], None, ws)
    for _ in range(3):
        wide.fill_(-7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, wide[:, 3:15]) and (wide[:, :3] == -7).all() and (wide[:, 15:] == -7).all()
    first = int(p.table[2, 0])
    for name, value in (("k", 0x7F), ("v", 0x7F)):
        codes = getattr(p.pool, name).view(torch.uint8)
        had = int(codes[first, 1, 3, 5])
        codes[first, 1, 3, 5] = value
        bad = p.run(ctx)
        p.check(*bad)
        assert torch.equal(o[others], bad[0][others]) and not torch.isfinite(bad[0][2, 4:8, 5]).any()
        codes[first, 1, 3, 5] = had
    p.q[2, 5, 9], p.q[2, 6, 0] = math.nan, math.inf
    bad = p.run(ctx)
    assert torch.equal(o[others], bad[0][others]) and not torch.isfinite(bad[0][2, 5:7]).any() and torch.equal(o[2, [4, 7]], bad[0][2, [4, 7]])


def test_scales_far_apart_in_pages_beyond_32_bit_offsets_and_bad_pages(ctx):
    p = _far_apart(Attend([70, 33, 1, 200], [40], 4, 4, 2, 64, 32, seed=20))
    want = p.run(ctx)
    p.check(*want)
    p.table[3, 4], p.table[1, 0] = -3, 1 << 30
    for x, y in zip(want, p.run(ctx, status=16)):
        assert torch.equal(x[[0, 2]], y[[0, 2]])
    p = _far_apart(Attend([70, 33, 1, 200], [40], 4, 4, 2, 64, 32, seed=20))
    _spread(p.pool, -(-(1 << 33) // p.pool.pages) // 16 * 16)
    assert all(torch.equal(x, y) for x, y in zip(want, p.run(ctx)))


def test_a_long_tail_behind_one_key_that_takes_most(ctx):
    """Eight thousand keys at 2^-18 of the first's weight carry a thirtieth of the sum: probabilities of four or five bits would lose them."""
    for D, Hq, Hkv in ((64, 4, 1), (128, 32, 1)):
        p = Attend([8200], None, 1, Hq, Hkv, D, 64, seed=2, spread=0.0)
        p.q.zero_()
        p.q[..., 0] = 1.0
        codes = p.pool.k.view(torch.uint8)
        codes[..., 0] = torch.zeros((), device="cuda").to(F8).view(torch.uint8)
        first = int(p.table[0, 0])
        codes[first, :, 0, 0] = torch.tensor(256.0, device="cuda").to(F8).view(torch.uint8)
        p.pool.ks.fill_(1.0)
        p.scale = 18 * math.log(2) / 256
        p.check(*p.run(ctx))


def test_large_scores(ctx):
    p = Attend([900, 300], [500], 2, 8, 2, 64, 32, seed=13, q_scale=60.0)
    o, lse = p.run(ctx)
    key = max(x.norm(dim=-1).max().item() for x in CR.read_many(p.pool.k, p.pool.ks, p.table, p.lengths) + CR.read_many(p.pool.k, p.pool.ks, p.p_table, p.prompts))
    zmax = p.q.float().norm(dim=-1).max().item() * key * p.scale
    p.check(o, lse, extra=zmax * 2.0 ** -20)          # the exponent's error: 64 products summed in fp32


def test_queries_of_any_size(ctx):
    """Rows whose entries lie sixty powers of two apart: what is cut is below 2^-22 of the row's largest."""
    p = Attend([40, 500, 33], None, 1, 12, 3, 128, 16, seed=3)
    p.q.mul_(torch.exp2(torch.randint(-60, 1, p.q.shape, generator=p.pool.g, device="cuda").float()).to(BF))
    p.q[0] *= 2.0 ** -40
    p.q[1, :4] = 0.0
    p.check(*p.run(ctx))


def test_free_slots_and_pages_may_hold_anything(ctx):
    """They hold NaN in all tests; here infinite and negative scales and page numbers far outside behind the last page too."""
    p = Attend([100, 3, 0, 190], [65, 40], 2, 6, 2, 128, 64, [1, 1, 1, 0], seed=4)
    used = set(p.table[p.table >= 0].tolist()) | set(p.p_table[p.p_table >= 0].tolist())
    for x in set(range(p.pool.pages)) - used:
        p.pool.ks[x], p.pool.vs[x] = math.inf, -math.inf
    p.check(*p.run(ctx))


def test_not_a_number_in_a_page_reaches_its_rollouts_alone(ctx):
    for prompt in (False, True):
        for name in ("k", "v"):
            p = Attend([100, 150, 30, 64], [65, 40], 2, 4, 2, 64, 16, seed=5)
            good = p.run(ctx)
            at = int(p.p_table[1, 1]) if prompt else int(p.table[1, 9])
            getattr(p.pool, name).view(torch.uint8)[at, 0, 3, 5] = 0x7F
            bad = p.run(ctx)
            reached = [2, 3] if prompt else [1]
            others = [i for i in range(4) if i not in reached]
            for x, y in zip(good, bad):
                assert torch.equal(x[others], y[others]) and torch.equal(x[reached, 2:], y[reached, 2:])
            assert not torch.isfinite(bad[0][reached, :2, 5]).any()
    p = Attend([100, 150, 30, 64], [65, 40], 2, 4, 2, 64, 16, seed=5)
    good = p.run(ctx)
    p.q[2, 1, 9], p.q[0, 3, 0] = math.nan, math.inf
    bad = p.run(ctx)
    other = torch.ones(4, 4, dtype=torch.bool, device="cuda")
    other[2, 1] = other[0, 3] = False
    assert all(torch.equal(x[other], y[other]) for x, y in zip(good, bad)) and not torch.isfinite(bad[0][~other]).any()


def test_same_bits_every_time_on_streams_and_in_graphs(ctx):
    p = Attend([300, 1200, 20, 0, 777, 64, 65, 3000], [500, 90], 4, 8, 2, 128, 32, [1, 1, 1, 1, 0, 1, 1, 1], seed=6)
    first = p.run(ctx)
    for _ in range(3):
        assert all(torch.equal(x, y) for x, y in zip(first, p.run(ctx)))
    other = Attend([5, 70, 60, 2] * 30, None, 1, 4, 4, 64, 16, seed=7)
    want = other.run(ctx)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs, wss = [x.outputs() for x in (p, other)], [x.workspace(ctx) for x in (p, other)]
    torch.cuda.synchronize()
    for _ in range(5):
        for x, s, out, ws in zip((p, other), streams, outs, wss):
            x.call(ctx, *out, ws, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(first + want, outs[0] + outs[1]))
    # a captured step follows the lengths and the mask of the moment; two graphs share a workspace in turn
    out, ws = p.outputs(), p.workspace(ctx)
    graphs = []
    for x in (p, other):
        graphs.append(torch.cuda.CUDAGraph())
        big = ws if x is p else torch.empty(max(ws.numel(), wss[1].numel()), dtype=torch.uint8, device="cuda")
        with torch.cuda.graph(graphs[-1]):
            x.call(ctx, *(out if x is p else outs[1]), big)
    p.lengths, p.keep = [299, 1000, 17, 0, 700, 60, 65, 100], [1, 0, 1, 1, 1, 1, 0, 1]
    p.d_len.copy_(torch.tensor(p.lengths, dtype=torch.int32))
    p.d_keep.copy_(torch.tensor(p.keep, dtype=torch.uint8))
    for t in out:
        t.fill_(-7.0)
    graphs[1].replay()
    graphs[0].replay()
    graphs[1].replay()
    torch.cuda.synchronize()
    p.check(*out)
    assert all(torch.equal(x, y) for x, y in zip(want, outs[1]))


@pytest.mark.parametrize("lengths,prompts,G,Hq,Hkv,D", [
    ([0, 226, 0, 834, 156, 705, 550, 757, 0, 547, 1, 0, 1, 24, 595, 0, 1, 0, 0, 96, 0, 1, 1, 0, 0, 1, 0, 170, 205, 0], [55, 178], 15, 32, 8, 64),
    ([700, 30, 608, 250] * 10, [227, 80, 1, 300], 10, 64, 8, 128),
    ([33, 64, 407, 851] * 14, None, 1, 24, 8, 128),
])
def test_same_bits_over_many_calls(ctx, lengths, prompts, G, Hq, Hkv, D):
    p = Attend(lengths, prompts, G, Hq, Hkv, D, 16, seed=16)
    o, lse = p.run(ctx)
    p.check(o, lse)
    ws, other = p.workspace(ctx), torch.zeros((), dtype=torch.bool, device="cuda")
    for _ in range(500):
        again = p.outputs()
        p.call(ctx, *again, ws)
        other |= (again[0] != o).any() | (again[1] != lse).any()
    assert B.arrol_poll_status(ctx) == 0 and not other.item()


def test_bad_lengths_and_pages_are_reported_and_not_followed(ctx):
    for name, at, value, other in (("d_len", 3, 1 << 30, [0, 1, 2]), ("d_len", 0, -5, [1, 2, 3]), ("d_prompts", 1, 1 << 30, [0, 1]), ("d_prompts", 0, -1, [2, 3]),
                                   ("table", (1, 2), -1, [0, 2, 3]), ("table", (1, 0), 1 << 30, [0, 2, 3]), ("p_table", (0, 1), -7, [2, 3])):
        p = Attend([100, 150, 30, 64], [65, 40], 2, 4, 2, 64, 32, seed=8)
        good = p.run(ctx)
        getattr(p, name)[at] = value
        bad = p.run(ctx, status=16)
        for x, y in zip(good, bad):
            assert torch.equal(x[other], y[other])
        if name == "d_len":
            p.lengths = [0 if i == at else n for i, n in enumerate(p.lengths)]
            p.check(*bad)
    # a rollout that is not kept is not looked at
    p = Attend([100, 150, 30, 64], [65, 40], 2, 4, 2, 64, 32, [1, 0, 1, 1], seed=8)
    good = p.run(ctx)
    p.table[1], p.d_len[1] = -5, -1
    assert all(torch.equal(x, y) for x, y in zip(good, p.run(ctx)))


def test_lse_is_optional_rows_are_strided_nothing_kept_no_rollouts(ctx):
    p = Attend([100, 0, 30], None, 1, 4, 2, 64, 16, seed=9)
    o, lse = p.run(ctx)
    wide = torch.full((3, 9, 64), -7.0, dtype=BF, device="cuda")
    p.q = torch.cat([p.q, p.q * 0], 1)[:, :4]
    p.call(ctx, wide[:, 2:6], None, p.workspace(ctx))
    torch.cuda.synchronize()
    assert torch.equal(o, wide[:, 2:6]) and (wide[:, :2] == -7).all() and (wide[:, 6:] == -7).all()
    p = Attend([10, 20], [30], 2, 4, 2, 64, 16, [0, 0])
    p.check(*p.run(ctx))
    Attend([], None, 1, 4, 2, 64).run(ctx)
    p = Attend([0, 0], [70], 2, 4, 2, 64, 16, seed=10)               # prompts alone, no page of their own
    p.table = p.table[:, :0]
    p.check(*p.run(ctx))


def test_forked_rollouts_share_pages(ctx):
    p = Attend([200, 90, 90], None, 1, 8, 2, 64, 32, seed=12)
    p.table[1] = p.table[0, :p.table.shape[1]]
    p.table[2] = p.table[1]
    p.check(*p.run(ctx))


def _spread(pool, stride):
    """The pool with its pages this many bytes apart, keys and values in one buffer."""
    shape, size = pool.k.shape, pool.Hkv * pool.page * pool.D
    buffer = torch.full(((pool.pages - 1) * stride + 2 * size,), 0x7F, dtype=torch.uint8, device="cuda")
    for at, name in ((0, "k"), (size, "v")):
        far = buffer[at:].as_strided(shape, (stride,) + pool.k[0].contiguous().stride())
        far.copy_(getattr(pool, name).view(torch.uint8))
        setattr(pool, name, far)


def test_pages_beyond_32_bit_offsets(ctx):
    p = Attend([70, 33, 1], [40], 3, 4, 2, 64, 32, seed=20)
    stride = -(-(1 << 33) // p.pool.pages) // 16 * 16
    want = p.run(ctx)
    _spread(p.pool, stride)
    assert all(torch.equal(x, y) for x, y in zip(want, p.run(ctx)))
    for new in (None, [9, 40, 1]):
        p = Append([70, 41, 17], new, page=32, seed=21)
        p.pool.k, p.pool.v = p.pool.k.view(torch.uint8), p.pool.v.view(torch.uint8)
        _spread(p.pool, stride)
        p.check(p.run(ctx))


@pytest.mark.parametrize("Hq,Hkv,D,pages", [(8, 4, 64, 1 << 24), (24, 2, 128, 1 << 25), (64, 2, 128, 1 << 23)])
def test_tables_for_very_long_sequences(ctx, Hq, Hkv, D, pages):
    """Room for more tokens than the line counts in its finer steps, few of them there."""
    p = Attend([70, 3000, 1, 555, 0, 64, 33, 1200], [40, 900], 4, Hq, Hkv, D, 16, [1, 1, 1, 0, 1, 1, 1, 1], seed=26)
    want = p.run(ctx)
    p.check(*want)
    wide = torch.full((p.N, pages), -5, dtype=torch.int32, device="cuda")
    wide[:, :p.table.shape[1]] = p.table
    p.table = wide
    p.check(*p.run(ctx))


def test_a_workspace_for_more_serves_less(ctx):
    """Of the same heads: with fewer rollouts, prompts or rollouts a prompt; what an earlier call left there does not matter."""
    big = Attend([50, 300] * 20, [100, 9, 0, 400], 10, 8, 2, 64, 16, seed=22)
    ws = big.workspace(ctx)
    for x in (big, Attend([7, 0, 900], None, 1, 8, 2, 64, 16, seed=23), Attend([20] * 6, [500, 3], 3, 8, 2, 64, 16, [1, 1, 0, 1, 0, 0], seed=24), big, Attend([3000], [70], 1, 8, 2, 64, 16, seed=25)):
        out = x.outputs()
        assert x.workspace(ctx).numel() <= ws.numel()
        x.call(ctx, *out, ws)
        torch.cuda.synchronize()
        x.check(*out)


# ---- appends ----------------------------------------------------------------------------------------------------------------------------------

class Append:
    """lengths with the new tokens, new[i] of them.  Old tokens are in the pool already, with scales that fit them."""

    def __init__(self, lengths, new=None, prompts=None, G=1, Hq=4, Hkv=2, D=64, n=64, page=16, keep=None, seed=0, both=False, interleaved=False, by=1.0, fused=False):
        self.N, self.lengths, self.new, self.prompts, self.G, self.keep, self.interleaved = len(lengths), lengths, new, prompts, G, keep, interleaved
        self.pool = pool = Pool(sum(-(-m // page) for m in lengths) + 2, Hkv, page, D, seed, both)
        self.table = pool.table(lengths)
        counts = new or [1] * self.N
        self.olds = [a - b for a, b in zip(lengths, counts)]
        for i, m in enumerate(self.olds):
            for x in range(-(-m // page)):
                at, many = int(self.table[i, x]), min(page, m - x * page)
                for c, s in ((pool.k, pool.ks), (pool.v, pool.vs)):
                    v = torch.randn(Hkv, many, D, generator=pool.g, device="cuda")
                    scale = torch.tensor([CR.scale_of(v[h].abs().max().item()) for h in range(Hkv)], device="cuda")
                    c.view(torch.uint8)[at, :, :many] = (v / scale[:, None, None]).to(F8).view(torch.uint8)
                    s[at] = scale
        T = sum(counts)
        make = lambda h: (torch.randn(T, h, D, generator=pool.g, device="cuda") * by).to(BF)  # noqa: E731
        if fused:
            qkv = make(Hq + 2 * Hkv)
            self.q, self.k, self.v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        else:
            self.q, self.k, self.v = make(Hq), make(Hkv), make(Hkv)
        self.cu = None
        self.starts = [0]
        for m in counts:
            self.starts.append(self.starts[-1] + m)
        if new is not None:
            self.cu = torch.tensor(self.starts, dtype=torch.int64, device="cuda")
        self.f = R.arrol_rotary_frequencies(n)[0].cuda() if n else None
        self.d_len = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.d_keep = None if keep is None else torch.tensor(keep, dtype=torch.uint8, device="cuda")
        self.d_prompts = None if prompts is None else torch.tensor(prompts, dtype=torch.int32, device="cuda")
        self.q_out, self.k_out = torch.full(self.q.shape, -7.0, dtype=BF, device="cuda"), torch.full(self.k.shape, -7.0, dtype=BF, device="cuda")

    def call(self, ctx, **kw):
        K.arrol_cache_append(ctx, self.k, self.v, *self.pool.args(), self.table, self.d_len, **(dict(cu_new=self.cu, keep=self.d_keep, q=self.q, q_out=self.q_out, k_out=self.k_out,
                             frequencies=self.f, factor=1.1 if self.f is not None else 1.0, interleaved=self.interleaved, prompt_lengths=self.d_prompts, G=self.G) | kw))

    def snapshot(self):
        return [x.clone() for x in (self.pool.k.view(torch.uint8), self.pool.v.view(torch.uint8), self.pool.ks, self.pool.vs)]

    def run(self, ctx, status=0, **kw):
        before = self.snapshot()
        self.call(ctx, **kw)
        torch.cuda.synchronize()
        assert B.arrol_poll_status(ctx, raise_on_error=False) == status
        return before

    def check(self, before):
        page, f = self.pool.page, [] if self.f is None else self.f.tolist()
        factor = 1.1 if f else 1.0
        touched = torch.zeros(self.pool.pages, dtype=torch.bool, device="cuda")
        for i in range(self.N):
            rows = slice(self.starts[i], self.starts[i + 1])
            if self.keep is not None and not self.keep[i]:
                assert (self.q_out[rows] == -7).all() and (self.k_out[rows] == -7).all()
                continue
            if rows.start == rows.stop:
                continue
            base = self.prompts[i // self.G] if self.prompts is not None else 0
            at = torch.arange(self.olds[i], self.lengths[i], device="cuda") + base
            for x, y in ((self.q, self.q_out), (self.k, self.k_out)):
                want, tol = CR.turn(x[rows], at, f, self.interleaved, factor)
                assert ((y[rows].double() - want).abs() <= CR.BF16 * (want.abs() + tol) + tol).all()
            for x, cache, scales, old_codes, old_scales in ((self.k, self.pool.k, self.pool.ks, before[0], before[2]), (self.v, self.pool.v, self.pool.vs, before[1], before[3])):
                want, tol = CR.turn(x[rows], at, f, self.interleaved, factor) if x is self.k else (x[rows].double(), torch.zeros_like(x[rows], dtype=torch.float64))
                got = CR.read(cache, scales, self.table[i], self.lengths[i])
                was = CR.read(old_codes, old_scales, self.table[i], self.olds[i])
                for first in range(self.olds[i] // page * page, self.lengths[i], page):
                    p, lo, hi = int(self.table[i, first // page]), max(first, self.olds[i]), min(first + page, self.lengths[i])
                    touched[p] = True
                    fresh = slice(lo - self.olds[i], hi - self.olds[i])
                    for h in range(self.pool.Hkv):
                        w, t = want[fresh, h], tol[fresh, h]
                        least, most = CR.scale_of(max((w.abs() - t).max().item(), 0.0)), CR.scale_of((w.abs() + t).max().item())
                        if lo > first:
                            held = old_scales[p, h].item()
                            least, most = max(least, held), max(most, held)
                        s = scales[p, h].item()
                        assert least <= s <= most, (s, least, most)
                        # half a step of e4m3, or of its subnormals
                        assert ((got[lo:hi, h] - w).abs() <= CR.E4M3 * (w.abs() + t) + t + s * 2.0 ** -10).all()
                        if lo > first:        # numbers that were there: as they were, or with a larger scale rounded among its subnormals
                            a, b = got[first:lo, h], was[first:lo, h]
                            assert torch.equal(a, b) if s == held else ((a - b).abs() <= torch.where(b.abs() < s * 2.0 ** -6, s * 2.0 ** -10, 0.0)).all()
                    end = hi - first      # slots behind the last token are left as they were
                    assert torch.equal(cache.view(torch.uint8)[p, :, end:], old_codes[p, :, end:])
        for now, was in zip((self.pool.k.view(torch.uint8), self.pool.v.view(torch.uint8)), before[:2]):
            assert torch.equal(now[~touched], was[~touched])
        for now, was in zip((self.pool.ks, self.pool.vs), before[2:]):
            assert torch.equal(now[~touched].view(torch.int32), was[~touched].view(torch.int32))


APPEND = [
    # lengths, new, prompts, G, Hq, Hkv, D, n, page, keep, interleaved
    ([1], None, None, 1, 1, 1, 64, 64, 16, None, False),
    ([1, 16, 17, 33, 200], None, None, 1, 8, 2, 128, 128, 16, None, False),
    ([1, 16, 17, 33, 200, 64], None, [50, 7], 3, 6, 2, 64, 64, 64, [1, 0, 1, 1, 1, 0], True),
    ([5, 9], None, None, 1, 7, 1, 80, 40, 128, None, False),
    ([5, 9, 40], None, [1000000], 3, 4, 4, 16, 6, 16, None, True),
    ([5, 9, 40], None, None, 1, 4, 4, 96, 0, 32, None, False),
    ([3] * 70, None, [9] * 35, 2, 4, 2, 32, 32, 16, [1, 0] * 35, False),
    ([1], [1], None, 1, 1, 1, 64, 64, 16, None, False),
    ([100], [100], None, 1, 16, 8, 128, 128, 64, None, False),
    ([100, 33, 64, 5, 300, 17], [100, 1, 30, 0, 299, 2], None, 1, 4, 2, 64, 64, 16, None, True),
    ([100, 33, 64, 5, 300, 17], [10, 33, 64, 5, 150, 16], None, 1, 4, 2, 96, 48, 128, [1, 1, 0, 1, 1, 1], False),
    ([90, 70], [60, 70], None, 1, 3, 3, 128, 40, 128, None, False),               # chunks of 4: two rounds over a page
    ([90, 70], [60, 70], None, 1, 3, 3, 112, 36, 32, None, True),                 # of 2
    ([200, 70], [160, 70], None, 1, 5, 1, 48, 22, 128, None, True),               # of 1
    ([90, 70], [60, 2], None, 1, 3, 3, 128, 0, 64, None, False),
    ([2, 40] * 200, [1, 3] * 200, [11] * 200, 2, 4, 2, 64, 64, 32, [1, 1, 0, 1] * 100, False),      # more sequences than a round of the search asks
    ([1000], [700], [5], 1, 20, 4, 64, 64, 32, None, False),
]


@pytest.mark.parametrize("lengths,new,prompts,G,Hq,Hkv,D,n,page,keep,interleaved", APPEND)
def test_append_matches_the_definition(ctx, lengths, new, prompts, G, Hq, Hkv, D, n, page, keep, interleaved):
    p = Append(lengths, new, prompts, G, Hq, Hkv, D, n, page, keep, seed=len(lengths) + D, both=D % 32 == 0, interleaved=interleaved, fused=len(lengths) % 2 == 1)
    p.check(p.run(ctx))


@pytest.mark.parametrize("Hq,Hkv,D,n,interleaved", [(9, 3, 32, 6, False), (10, 5, 48, 48, False), (16, 2, 16, 10, True), (12, 1, 128, 0, False), (14, 7, 80, 36, False)])
def test_one_token_each_of_many_rollouts(ctx, Hq, Hkv, D, n, interleaved):
    """More heads than there are places for warps: keys, values and queries of a rollout meet in one warp, and some of its places stay empty."""
    N = -(-10000 // (Hq + 2 * Hkv) // 2) * 2
    g = torch.Generator().manual_seed(N)
    lengths = torch.randint(1, 12, (N,), generator=g).tolist()
    keep = (torch.rand(N, generator=g) < 0.7).int().tolist()
    p = Append(lengths, None, [3, 1000], N // 2, Hq, Hkv, D, n, 16, keep, seed=N, interleaved=interleaved, by=3.0)
    p.check(p.run(ctx))


@pytest.mark.parametrize("new", [None, [1, 1, 1], [9, 20, 3]])
@pytest.mark.parametrize("by", [300.0, 1e-3, 1e30, 1e-32, 0.0])
def test_scales_grow_and_do_not_shrink(ctx, by, new):
    """New tokens far larger and far smaller than those of their page; zeros; sizes at the ends of the scales' range."""
    p = Append([10, 37, 64], new, Hkv=2, D=64, n=64, page=16, seed=3, by=by)
    p.check(p.run(ctx))


def test_one_by_one_and_all_at_once_leave_the_same_numbers(ctx):
    """Scales are the same powers of two; numbers differ only where a scale grew under one that it made subnormal."""
    n, page = 75, 32
    a = Append([n, n], [n, n], Hkv=2, D=64, page=page, seed=4)
    a.run(ctx)
    b = Append([n, n], [n, n], Hkv=2, D=64, page=page, seed=4)
    for j in range(n):
        rows = torch.tensor([j, n + j], device="cuda")
        K.arrol_cache_append(ctx, b.k[rows], b.v[rows], *b.pool.args(), b.table, torch.full((2,), j + 1, dtype=torch.int32, device="cuda"), q=b.q[rows],
                             q_out=torch.empty(2, 4, 64, dtype=BF, device="cuda"), frequencies=b.f, factor=1.1)
    torch.cuda.synchronize()
    used = a.table[a.table >= 0].long()
    assert torch.equal(a.pool.ks[used], b.pool.ks[used]) and torch.equal(a.pool.vs[used], b.pool.vs[used])
    for x, y, s in ((a.pool.k, b.pool.k, a.pool.ks), (a.pool.v, b.pool.v, a.pool.vs)):
        for i in range(2):
            u, w = CR.read(x, s, a.table[i], n), CR.read(y, s, a.table[i], n)
            assert ((u - w).abs() <= 2.0 ** -9 * s[used].max().item()).all()
            assert torch.equal(u[u.abs() >= 2.0 ** -5 * s[used].max().item()], w[u.abs() >= 2.0 ** -5 * s[used].max().item()])


def test_again_leaves_the_same(ctx):
    for new in (None, [7, 1, 30]):
        p = Append([20, 33, 64], new, page=16, seed=5, by=3.0)
        p.run(ctx)
        one = p.snapshot() + [p.q_out.clone()]
        p.run(ctx)
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(one, p.snapshot() + [p.q_out]))


def test_in_place_and_without_queries(ctx):
    for new in (None, [7, 1, 30]):
        p = Append([20, 33, 64], new, page=16, seed=6)
        p.run(ctx)
        r = Append([20, 33, 64], new, page=16, seed=6)
        r.run(ctx, q_out=r.q, k_out=r.k)
        assert torch.equal(r.q, p.q_out) and torch.equal(r.k, p.k_out)
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(p.snapshot(), r.snapshot()))
        r = Append([20, 33, 64], new, page=16, seed=6)
        r.run(ctx, q=None, q_out=None, k_out=None)
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(p.snapshot(), r.snapshot()))


def test_infinities_and_nan_are_stored_as_nan(ctx):
    for new in (None, [7, 1, 30]):
        good, bad = (Append([20, 33, 64], new, page=16, seed=7, n=0) for _ in range(2))
        row = bad.starts[1]
        bad.k[row, 0, 5], bad.v[row, 1, 9] = math.inf, math.nan
        good.k[row, 0, 5] = good.v[row, 1, 9] = 0.0
        for p in (good, bad):
            p.run(ctx)
        at, slot = int(bad.table[1, 2]), 0
        for x, y, (h, d) in ((good.pool.k, bad.pool.k, (0, 5)), (good.pool.v, bad.pool.v, (1, 9))):
            assert int(y.view(torch.uint8)[at, h, slot, d]) & 0x7F == 0x7F
            z = y.view(torch.uint8).clone()
            z[at, h, slot, d] = x.view(torch.uint8)[at, h, slot, d]
            assert torch.equal(z, x.view(torch.uint8))
        assert torch.equal(good.pool.ks.nan_to_num(), bad.pool.ks.nan_to_num()) and torch.equal(good.pool.vs.nan_to_num(), bad.pool.vs.nan_to_num())


def test_bad_appends_are_reported_and_not_followed(ctx):
    for new in (None, [7, 1, 30]):
        for name, at, value in (("d_len", 1, 1 << 30), ("d_len", 1, -4), ("d_len", 1, 0), ("table", (1, 2), -1), ("table", (1, 2), 1 << 29)):
            p = Append([20, 33, 64], new, page=16, seed=8)
            getattr(p, name)[at] = value
            before = p.run(ctx, status=16)
            p.keep = [1, 0, 1]
            if name == "table":              # queries may have been turned
                p.q_out[p.starts[1]:p.starts[2]] = p.k_out[p.starts[1]:p.starts[2]] = -7.0
            p.check(before)
    for at, value in ((3, 39), (1, -1), (2, 100), (1, 1 << 40)):
        p = Append([20, 33, 64], [7, 1, 30], page=16, seed=9)
        p.cu[at] = value
        p.run(ctx, status=16)


@pytest.mark.parametrize("N,new", [(3, None), (1500, None), (3, [7, 1, 30])])
def test_rows_of_refused_tokens_are_left_as_they_were(ctx, N, new):
    """Queries too, however many sequences a call has; rows of the sequence's other pages are written."""
    for name, at, value in (("d_len", 1, 1 << 30), ("table", (1, 2), -1), ("table", (1, 2), 1 << 29)):
        good, bad = (Append([20, 33, 64] + [33] * (N - 3), new, page=16, seed=8) for _ in range(2))
        getattr(bad, name)[at] = value
        good.run(ctx)
        bad.run(ctx, status=16)
        left = torch.zeros(good.starts[-1], dtype=torch.bool, device="cuda")
        left[bad.starts[1]:bad.starts[2]] = True              # of 33 tokens the new one is the third page's
        for x, y in ((good.q_out, bad.q_out), (good.k_out, bad.k_out)):
            assert (y[left] == -7).all() and torch.equal(x[~left], y[~left])
    if new is not None:
        p = Append([20, 40, 64], [7, 30, 30], page=16, seed=8)
        p.table[1, 1] = -5                                    # tokens 16 .. 31 of 10 .. 39
        p.run(ctx, status=16)
        for x in (p.q_out, p.k_out):
            rows = x[p.starts[1]:p.starts[2]]
            assert (rows[6:22] == -7).all() and not (rows[:6] == -7).all(-1).any() and not (rows[22:] == -7).all(-1).any()


def test_rows_out_of_order_are_reported_where_nothing_follows_them(ctx):
    """Sequences of which no block is launched, or which are left out: those in front of them are written as ever."""
    for cu, keep in (([0, 7, 10 ** 6, 10 ** 6 + 30], [1, 0, 1]), ([0, 7, 1 << 62, (1 << 62) + 30], [1, 0, 1]), ([0, 7, -(1 << 40), 37], [0, 0, 0]), ([0, 7, 3, 37], [0, 0, 0]),
                     ([0, 7, 37, 39], [1, 0, 0]), ([3, 7, 8, 38], [0, 0, 0]), ([-1, 7, 8, 38], [0, 0, 0])):
        good, bad = (Append([20, 33, 64], [7, 1, 30], page=16, keep=[1 if k and i == 0 else 0 for i, k in enumerate(keep)], seed=9) for _ in range(2))
        bad.cu.copy_(torch.tensor(cu, dtype=torch.int64))
        bad.d_keep.copy_(torch.tensor(keep, dtype=torch.uint8))
        good.run(ctx)
        bad.run(ctx, status=16)
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(good.snapshot() + [good.q_out, good.k_out], bad.snapshot() + [bad.q_out, bad.k_out]))
    many = Append([20] * 600, [2] * 600, page=16, keep=[0] * 600, seed=9)             # more sequences than a block has threads
    many.cu[577] = 1 << 40
    many.run(ctx, status=16)
    p = Append([20, 33, 64], [7, 1, 30], page=16, seed=9)                             # rows behind the last sequence are nobody's
    p.cu = torch.tensor([0, 7, 8, 38], dtype=torch.int64, device="cuda")
    p.k, p.v, p.q = (torch.cat([x, x[:5]]) for x in (p.k, p.v, p.q))
    p.q_out, p.k_out = (torch.cat([x, x[:5]]) for x in (p.q_out, p.k_out))
    p.check(p.run(ctx))
    assert (p.q_out[38:] == -7).all() and (p.k_out[38:] == -7).all()


def test_appends_captured_and_replayed(ctx):
    p = Append([20, 33, 64], None, [3], 3, page=16, seed=10)
    q = Append([20, 33, 64], None, [3], 3, page=16, seed=10)
    p.run(ctx)
    saved = q.snapshot()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        q.call(ctx)
    for t, was in zip((q.pool.k.view(torch.uint8), q.pool.v.view(torch.uint8), q.pool.ks, q.pool.vs), saved):
        t.copy_(was)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(p.snapshot(), q.snapshot())) and torch.equal(p.q_out, q.q_out)


def test_appends_at_once_on_two_streams(ctx):
    """Into different pages of one pool, as two batches that are served side by side."""
    def pair():
        x, y = Append([200] * 30, [70] * 30, page=32, seed=11), Append([64, 33, 17], None, page=32, seed=12)
        both = Pool(x.pool.pages + y.pool.pages, 2, 32, 64)
        n = x.pool.pages
        for part, p in ((slice(0, n), x.pool), (slice(n, None), y.pool)):
            for name in ("k", "v"):
                getattr(both, name).view(torch.uint8)[part] = getattr(p, name).view(torch.uint8)
            both.ks[part], both.vs[part] = p.ks, p.vs
        y.table = torch.where(y.table >= 0, y.table + n, y.table)
        x.pool = y.pool = both
        return x, y
    x, y = pair()
    x.run(ctx)
    y.run(ctx)
    u, w = pair()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for p, s in zip((u, w), streams):
        p.call(ctx, stream=s)
    torch.cuda.synchronize()
    assert B.arrol_poll_status(ctx) == 0
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(x.snapshot(), u.snapshot()))
    assert torch.equal(x.q_out, u.q_out) and torch.equal(y.q_out, w.q_out) and torch.equal(x.k_out, u.k_out) and torch.equal(y.k_out, w.k_out)


# ---- all of it ------------------------------------------------------------------------------------------------------------------------------------

def test_a_generation_with_pruning(ctx):
    """Prompts appended at once, tokens one by one, rollouts pruned on the way, attention after every append; what is turned is what the packed call turns, bit for bit."""
    P, G, Hq, Hkv, D, page, steps = 2, 4, 8, 2, 64, 16, 40
    N, prompts = P * G, [37, 70]
    g = torch.Generator("cuda").manual_seed(0)
    make = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF)  # noqa: E731
    pool = Pool(sum(-(-n // page) for n in prompts) + N * -(-steps // page), Hkv, page, D, 1, both=True)
    p_table, table = pool.table(prompts), pool.table([steps] * N)
    f, factor = R.arrol_rotary_frequencies(D, 500000.0, R.BANDS, stretch=32.0)
    f = f.cuda()
    d_prompts = torch.tensor(prompts, dtype=torch.int32, device="cuda")
    pk, pv = make(sum(prompts), Hkv, D), make(sum(prompts), Hkv, D)
    pk_out = torch.empty_like(pk)
    cup = torch.tensor([0, 37, 107], dtype=torch.int64, device="cuda")
    K.arrol_cache_append(ctx, pk, pv, *pool.args(), p_table, d_prompts, cu_new=cup, k_out=pk_out, frequencies=f, factor=factor)
    turned = torch.empty_like(pk)
    R.arrol_rotary(ctx, None, pk, f, None, turned, cu_seqlens=cup, d_num=torch.tensor([2, 107], device="cuda"), factor=factor)
    torch.cuda.synchronize()
    assert torch.equal(pk_out, turned)
    keep = torch.ones(N, dtype=torch.uint8, device="cuda")
    lengths = torch.zeros(N, dtype=torch.int32, device="cuda")
    ws = torch.empty(K.arrol_cache_attention_workspace(ctx, N, P, G, Hq, Hkv, D), dtype=torch.uint8, device="cuda")
    qs, ks, qo = make(steps, N, Hq, D), make(steps, N, Hkv, D), torch.zeros(steps, N, Hq, D, dtype=BF, device="cuda")
    k_turned = torch.zeros_like(ks)
    vs = make(steps, N, Hkv, D)
    o, lse = torch.zeros(N, Hq, D, dtype=BF, device="cuda"), torch.zeros(N, Hq, device="cuda")
    live = [1] * N
    for t in range(steps):
        if t == 17:
            live = [1, 0, 0, 1, 0, 1, 1, 0]
            keep.copy_(torch.tensor(live, dtype=torch.uint8))
        lengths += keep.int()
        K.arrol_cache_append(ctx, ks[t], vs[t], *pool.args(), table, lengths, keep=keep, q=qs[t], q_out=qo[t], k_out=k_turned[t], frequencies=f, factor=factor,
                             prompt_lengths=d_prompts, G=G)
        K.arrol_cache_attention(ctx, qo[t], *pool.args(), table, lengths, o, lse, ws, keep=keep, prompt_table=p_table, prompt_lengths=d_prompts, G=G)
        if t % 13 in (0, 4) or t == steps - 1:
            n = lengths.tolist()
            shared = [CR.read_many(c, s, p_table, prompts) for c, s in ((pool.k, pool.ks), (pool.v, pool.vs))]
            own = [CR.read_many(c, s, table, n) for c, s in ((pool.k, pool.ks), (pool.v, pool.vs))]
            for i in range(N):
                if live[i]:
                    want, tol, ll = CR.attend(qo[t, i], torch.cat([shared[0][i // G], own[0][i]]), torch.cat([shared[1][i // G], own[1][i]]), D ** -0.5)
                    assert ((o[i].double() - want).abs() <= tol).all() and ((lse[i].double() - ll).abs() <= 2e-5 * (1 + ll.abs())).all()
    assert B.arrol_poll_status(ctx) == 0
    # the packed batch of the survivors, turned by the training call
    index = [i for i in range(N) if live[i]]
    S = len(index)
    q = torch.cat([qs[:, i] for i in index])
    k = torch.cat([ks[:, i] for i in index])
    cu = torch.arange(S + 1, device="cuda", dtype=torch.int64) * steps
    q2, k2 = torch.empty_like(q), torch.empty_like(k)
    R.arrol_rotary(ctx, q, k, f, q2, k2, cu_seqlens=cu, d_num=torch.tensor([S, S * steps], device="cuda"), cu_prompts=cup,
                   survivor_idx=torch.tensor(index, dtype=torch.int32, device="cuda"), G=G, factor=factor)
    torch.cuda.synchronize()
    assert torch.equal(q2, torch.cat([qo[:, i] for i in index])) and torch.equal(k2, torch.cat([k_turned[:, i] for i in index]))
    # what the cache holds of them
    for s, i in enumerate(index):
        got = CR.read(pool.k, pool.ks, table[i], steps)
        want, tol = CR.turn(ks[:, i], torch.arange(steps, device="cuda") + prompts[i // G], f.tolist(), factor=factor)
        scale = pool.ks[table[i, :-(-steps // page)].long()].max().item()
        assert ((got - want).abs() <= CR.E4M3 * (want.abs() + tol) + tol + scale * 2.0 ** -9).all()
