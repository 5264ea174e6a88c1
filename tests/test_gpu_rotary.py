"""GPU parity of the rotary calls against the 64-bit reference."""
import math

import pytest
import torch

import cache_reference as CR
from paper_2603_24840_b200 import binding as B
from paper_2603_24840_b200 import rotary as R

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    c.close()


def _normal(g, *s, by=1.0):
    return (torch.randn(*s, generator=g, device="cuda") * by).to(BF)


def _check(y, x, positions, f, **kw):
    want, tol = CR.turn(x, positions, f.tolist(), **kw)
    off = (y.double() - want).abs()
    bound = CR.BF16 * (want.abs() + tol) + tol
    assert (off <= bound).all(), (off / bound.clamp(min=1e-30)).max()
    n = 2 * f.numel()
    assert torch.equal(y[..., n:], x[..., n:])


CASES = [
    # T, Hq, Hkv, D, R, interleaved
    (1, 1, 1, 64, 64, False),
    (1, 1, 1, 64, 64, True),
    (300, 8, 2, 128, 128, False),
    (77, 28, 4, 128, 64, True),
    (5, 3, 3, 80, 80, False),
    (33, 5, 1, 96, 48, False),           # chunks of 8
    (33, 5, 1, 96, 40, True),            # of 4
    (19, 2, 2, 64, 36, False),           # of 2
    (19, 2, 2, 64, 36, True),
    (21, 4, 1, 40, 22, False),           # of 1
    (21, 4, 1, 40, 22, True),
    (9, 2, 1, 8, 2, False),
    (9, 2, 1, 8, 2, True),
    (9, 2, 1, 8, 6, True),
    (513, 64, 1, 64, 64, False),
    (130, 2, 8, 256, 256, False),
    (130, 1, 1, 256, 2, True),
    (2500, 0, 3, 64, 32, False),
    (2500, 7, 0, 64, 64, True),
]


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("T,Hq,Hkv,D,n,interleaved", CASES)
def test_matches_the_definition(ctx, T, Hq, Hkv, D, n, interleaved, backward):
    g = torch.Generator("cuda").manual_seed(T + D + n)
    q, k = _normal(g, T, Hq, D) if Hq else None, _normal(g, T, Hkv, D) if Hkv else None
    f, _ = R.arrol_rotary_frequencies(n)
    f = f.cuda()
    at = torch.randint(-50, 9000, (T,), generator=g, device="cuda", dtype=torch.int32)
    qo, ko = (None if x is None else torch.full_like(x, -7.0) for x in (q, k))
    (R.arrol_rotary_backward if backward else R.arrol_rotary)(ctx, q, k, f, qo, ko, positions=at, factor=1.25, interleaved=interleaved)
    assert B.arrol_poll_status(ctx) == 0
    for x, y in ((q, qo), (k, ko)):
        if x is not None:
            _check(y, x, at, f, interleaved=interleaved, factor=1.25, backward=backward)


def test_far_positions_keep_their_angles(ctx):
    """In fp32 the angle of position 2^31 - 1 would be off by a hundred turns."""
    g = torch.Generator("cuda").manual_seed(1)
    at = torch.tensor([0, 1, -1, 131071, 1 << 20, (1 << 31) - 1, -(1 << 31)], dtype=torch.int32, device="cuda")
    q = _normal(g, 7, 2, 64)
    f = R.arrol_rotary_frequencies(64, 500000.0)[0].cuda()
    y = torch.empty_like(q)
    R.arrol_rotary(ctx, q, None, f, y, None, positions=at)
    # the angle in 64 bits is itself off by 2^31 x 2^-52 here, 5e-7: twice, in kernel and reference
    want, tol = CR.turn(q, at, f.tolist())
    off, size = (y.double() - want).abs(), q.double().abs().amax(-1, keepdim=True)
    assert (off <= CR.BF16 * want.abs() + tol * 1.01 + 2e-6 * size).all()
    assert torch.equal(y[0], q[0])


class Packed:
    def __init__(self, lens, prompts, index, G, Hq=4, Hkv=2, D=64, n=64, seed=0, spare=5):
        g = torch.Generator("cuda").manual_seed(seed)
        self.T, cu, at = sum(lens), [0], []
        cup = [0]
        for m in prompts or []:
            cup.append(cup[-1] + m)
        for s, m in enumerate(lens):
            cu.append(cu[-1] + m)
            p = (index[s] if index is not None else s) // G
            at += [t + (prompts[p] if prompts is not None else 0) for t in range(m)]
        self.at = torch.tensor(at, dtype=torch.int32, device="cuda")
        self.cu = torch.tensor(cu + [cu[-1] + 1000] * 3, dtype=torch.int64, device="cuda")         # room for more survivors than there are
        self.num = torch.tensor([len(lens), self.T], dtype=torch.int64, device="cuda")
        self.cup = torch.tensor(cup, dtype=torch.int64, device="cuda") if prompts is not None else None
        self.index = torch.tensor(list(index) + [1 << 20] * 3, dtype=torch.int32, device="cuda") if index is not None else None
        self.G, rows = G, self.T + spare
        qkv = _normal(g, rows, Hq + 2 * Hkv, D)
        self.q, self.k = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv]
        self.f = R.arrol_rotary_frequencies(n)[0].cuda()

    def run(self, ctx, status=0, stream=None, out=None):
        qo, ko = out or (torch.full(self.q.shape, -7.0, dtype=BF, device="cuda"), torch.full(self.k.shape, -7.0, dtype=BF, device="cuda"))
        R.arrol_rotary(ctx, self.q, self.k, self.f, qo, ko, cu_seqlens=self.cu, d_num=self.num, cu_prompts=self.cup, survivor_idx=self.index, G=self.G, stream=stream)
        if stream is None and not torch.cuda.is_current_stream_capturing():
            assert B.arrol_poll_status(ctx, raise_on_error=False) == status
        return qo, ko

    def check(self, qo, ko):
        for x, y in ((self.q, qo), (self.k, ko)):
            _check(y[:self.T], x[:self.T], self.at, self.f)
            assert (y[self.T:] == -7).all()


PACKED = [
    ([3, 0, 4, 1], [4, 2], [0, 1, 5, 7], 4),
    ([100, 250, 1], None, None, 1),
    ([0, 0, 7, 0, 0, 90, 0], [11, 0, 5], [0, 1, 2, 9, 10, 16, 20], 8),
    ([1] * 700, [13] * 100, None, 7),                            # more sequences than a round of the search asks
    ([2, 1] * 900, [3, 0, 5] * 200, list(range(0, 5400, 3)), 9),
    ([5000], [0], [3], 4),
    ([], [5], [], 2),
]


@pytest.mark.parametrize("lens,prompts,index,G", PACKED)
def test_positions_of_packed_survivors(ctx, lens, prompts, index, G):
    p = Packed(lens, prompts, index, G)
    p.check(*p.run(ctx))


def test_in_place_gives_the_same_bits(ctx):
    for n, interleaved in ((64, False), (64, True), (36, False), (22, True)):
        g = torch.Generator("cuda").manual_seed(n)
        x = _normal(g, 50, 6, 64)
        f, at = R.arrol_rotary_frequencies(n)[0].cuda(), torch.arange(50, dtype=torch.int32, device="cuda")
        out = torch.empty(50, 6, 64, dtype=BF, device="cuda")
        R.arrol_rotary(ctx, x[:, :4], x[:, 4:], f, out[:, :4], out[:, 4:], positions=at, interleaved=interleaved)
        R.arrol_rotary(ctx, x[:, :4], x[:, 4:], f, x[:, :4], x[:, 4:], positions=at, interleaved=interleaved)
        torch.cuda.synchronize()
        assert torch.equal(x, out)


def test_gradient_is_the_transpose(ctx):
    """<R x, dy> = <x, R' dy>: forward and gradient from the same call's own values, and differences of a sum of products."""
    g = torch.Generator("cuda").manual_seed(3)
    x, dy = _normal(g, 200, 4, 96), _normal(g, 200, 4, 96)
    f, at = R.arrol_rotary_frequencies(64, kind=R.RAMP, stretch=4.0, high=32.0, original=4096)[0].cuda(), torch.arange(200, dtype=torch.int32, device="cuda") * 37
    y, dx = torch.empty_like(x), torch.empty_like(x)
    R.arrol_rotary(ctx, x, None, f, y, None, positions=at, factor=1.5)
    R.arrol_rotary_backward(ctx, dy, None, f, dx, None, positions=at, factor=1.5)
    a, b = (y.double() * dy.double()).sum(-1), (x.double() * dx.double()).sum(-1)
    bound = CR.BF16 * ((y.double() * dy.double()).abs().sum(-1) + (x.double() * dx.double()).abs().sum(-1)) * 1.01
    assert ((a - b).abs() <= bound).all()
    # the call is linear, so a difference along any direction is the call on that direction: steps that bf16 holds exactly
    step = torch.zeros_like(x)
    step[:, :, 5] = 1.0
    e = torch.empty_like(x)
    R.arrol_rotary(ctx, step, None, f, e, None, positions=at, factor=1.5)
    got = (e.double() * dy.double()).sum(-1)
    assert ((got - dx[:, :, 5].double()).abs() <= CR.BF16 * ((e.double() * dy.double()).abs().sum(-1) + dx[:, :, 5].double().abs()) * 1.01).all()


def test_infinities_and_nan_stay_in_their_pair(ctx):
    g = torch.Generator("cuda").manual_seed(4)
    x = _normal(g, 20, 2, 64)
    f, at = R.arrol_rotary_frequencies(64)[0].cuda(), torch.arange(20, dtype=torch.int32, device="cuda")
    good, bad = torch.empty_like(x), torch.empty_like(x)
    R.arrol_rotary(ctx, x, None, f, good, None, positions=at)
    x[3, 1, 7], x[9, 0, 40] = math.nan, math.inf
    R.arrol_rotary(ctx, x, None, f, bad, None, positions=at)
    other = torch.ones_like(x, dtype=torch.bool)
    other[3, 1, [7, 39]] = other[9, 0, [8, 40]] = False
    assert torch.equal(good[other], bad[other]) and not torch.isfinite(bad[~other]).any()


def test_streams_graphs_and_counts_of_the_moment(ctx):
    p = Packed([30, 100, 7], [20, 6], [0, 3, 5], 4, seed=5)
    first = p.run(ctx)
    out = tuple(torch.full_like(x, -7.0) for x in first)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.run(ctx, out=out)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, out))
    # fewer survivors than at capture
    p.num.copy_(torch.tensor([2, 130]))
    for t in out:
        t.fill_(-7.0)
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(first, out):
        assert torch.equal(a[:130], b[:130]) and (b[130:] == -7).all()
    other = torch.cuda.Stream()
    p.num.copy_(torch.tensor([3, 137]))
    torch.cuda.synchronize()
    again = p.run(ctx, stream=other)
    torch.cuda.synchronize()
    assert all(torch.equal(a[:137], b[:137]) for a, b in zip(first, again))


def test_bad_rows_are_reported_and_not_followed(ctx):
    for name, at, value in (("cu", 3, 50), ("cu", 0, 4), ("index", 1, -1), ("index", 2, 1 << 30), ("num", 1, 137 + 3)):
        p = Packed([30, 100, 7], [20, 6], [0, 3, 5], 4, seed=6)
        getattr(p, name)[at] = value
        if name == "cu" and at == 3:
            p.cu[3:] = value
        p.run(ctx, status=16)


def test_rows_beyond_32_bit_offsets(ctx):
    """Rows so far apart that their offsets pass 2^32 elements."""
    stride = (1 << 31) // 8 * 8 + 64
    base = torch.zeros(2 * stride + 64, dtype=BF, device="cuda")
    x = base.as_strided((3, 1, 64), (stride, 64, 1))
    g = torch.Generator("cuda").manual_seed(7)
    x.copy_(_normal(g, 3, 1, 64))
    f, at = R.arrol_rotary_frequencies(64)[0].cuda(), torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda")
    y = torch.empty(3, 1, 64, dtype=BF, device="cuda")
    R.arrol_rotary(ctx, x, None, f, y, None, positions=at)
    _check(y, x, at, f)
    R.arrol_rotary(ctx, x, None, f, x, None, positions=at)
    torch.cuda.synchronize()
    assert torch.equal(x, y)
