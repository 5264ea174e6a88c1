"""CPU-only checks around the rotary and cache calls: frequencies, the 64-bit reference that the GPU tests use, and the calls' refusals, which come before anything touches
a device."""
import ctypes as C
import math

import pytest
import torch

import cache_reference as CR
from paper_2603_24840_b200 import binding as B
from paper_2603_24840_b200 import build as libbuild
from paper_2603_24840_b200 import cache as K
from paper_2603_24840_b200 import rotary as R


@pytest.fixture(scope="module")
def lib():
    libbuild.build()
    R._lib()
    return K._lib()


# ---- frequencies ----------------------------------------------------------------------------------------------------------------------------

def test_plain_and_linear_frequencies(lib):
    for n, base in ((64, 10000.0), (128, 500000.0), (2, 7.0), (10, 1e6)):
        f, factor = R.arrol_rotary_frequencies(n, base)
        assert factor == 1.0 and f.dtype is torch.float64
        want = [base ** (-2 * i / n) for i in range(n // 2)]
        assert all(abs(a - b) <= 2e-15 * b for a, b in zip(f.tolist(), want))
        g, _ = R.arrol_rotary_frequencies(n, base, R.LINEAR, stretch=4.0)
        assert torch.allclose(g * 4, f, rtol=1e-15, atol=0)


def test_bands_leave_short_waves_and_slow_long_ones(lib):
    f, _ = R.arrol_rotary_frequencies(128, 500000.0)
    g, factor = R.arrol_rotary_frequencies(128, 500000.0, R.BANDS, stretch=32.0, low=1.0, high=4.0, original=8192)
    turns = 8192 * f / (2 * math.pi)
    assert factor == 1.0
    assert torch.equal(g[turns >= 4], f[turns >= 4])
    assert torch.allclose(g[turns <= 1], f[turns <= 1] / 32, rtol=1e-15, atol=0)
    between = (turns > 1) & (turns < 4)
    assert between.any()
    s = (turns[between] - 1) / 3
    assert torch.allclose(g[between], (1 - s) * f[between] / 32 + s * f[between], rtol=1e-12, atol=0)


def test_ramp_by_pair_numbers(lib):
    n, base, stretch = 64, 10000.0, 8.0
    f, _ = R.arrol_rotary_frequencies(n, base)
    g, factor = R.arrol_rotary_frequencies(n, base, R.RAMP, stretch=stretch, low=1.0, high=32.0, original=4096)
    assert abs(factor - (0.1 * math.log(8.0) + 1)) < 1e-15
    pair = lambda turns: n * math.log(4096 / (2 * math.pi * turns)) / (2 * math.log(base))  # noqa: E731
    lo, hi = math.floor(pair(32.0)), math.ceil(pair(1.0))
    assert 0 < lo < hi < n // 2
    for i in range(n // 2):
        s = min(1.0, max(0.0, (i - lo) / (hi - lo)))
        assert abs(g[i].item() - ((1 - s) * f[i].item() + s * f[i].item() / stretch)) <= 1e-13 * f[i].item()
    assert R.arrol_rotary_frequencies(n, base, R.RAMP, stretch=0.5, high=32.0)[1] == 1.0


@pytest.mark.parametrize("kw", [dict(R=3), dict(R=0), dict(R=-2), dict(base=1.0), dict(base=math.nan), dict(base=math.inf), dict(kind=4), dict(kind=-1),
                                dict(kind=1, stretch=0.0), dict(kind=2, stretch=math.nan), dict(kind=2, low=0.0), dict(kind=2, low=4.0), dict(kind=3, original=0.0),
                                dict(kind=3, high=math.inf)])
def test_frequencies_refuse(lib, kw):
    args = dict(R=64, base=10000.0, kind=0, stretch=2.0, low=1.0, high=4.0, original=8192.0) | kw
    with pytest.raises(B.ArrolError) as e:
        R.arrol_rotary_frequencies(**args)
    assert e.value.code == -1
    out = (C.c_double * 64)()
    assert lib.arrol_rotary_frequencies(64, 10000.0, 0, 1.0, 1.0, 4.0, 8192.0, None, None) == -1
    assert lib.arrol_rotary_frequencies(64, 10000.0, 0, 1.0, 1.0, 4.0, 8192.0, out, None) == 0


# ---- the reference --------------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("interleaved", [False, True])
def test_reference_turns_depend_on_differences_of_positions_alone(interleaved):
    g = torch.Generator().manual_seed(0)
    q, k = torch.randn(1, 3, 12, generator=g, dtype=torch.float64), torch.randn(1, 3, 12, generator=g, dtype=torch.float64)
    f = [1.0, 0.3, 0.01, 0.002]
    dots = []
    for p in (0, 7, 1000):
        a, _ = CR.turn(q, torch.tensor([p + 5]), f, interleaved, 1.5)
        b, _ = CR.turn(k, torch.tensor([p]), f, interleaved, 1.5)
        assert torch.equal(a[..., 8:], q[..., 8:])
        dots.append((a[..., :8] * b[..., :8]).sum(-1))
    assert torch.allclose(dots[0], dots[1], atol=1e-12) and torch.allclose(dots[0], dots[2], atol=1e-11)
    assert not torch.allclose(dots[0], 2.25 * (q[..., :8] * k[..., :8]).sum(-1), atol=1e-2)
    back, _ = CR.turn(CR.turn(q, torch.tensor([9]), f, interleaved)[0], torch.tensor([9]), f, interleaved, backward=True)
    assert torch.allclose(back, q, atol=1e-14)


@pytest.mark.parametrize("interleaved", [False, True])
def test_reference_gradient_agrees_with_differences(interleaved):
    g = torch.Generator().manual_seed(1)
    x, dy = (torch.randn(3, 2, 10, generator=g, dtype=torch.float64) for _ in range(2))
    at, f = torch.tensor([0, 4, 33]), [1.0, 0.4, 0.05]
    dx, _ = CR.turn(dy, at, f, interleaved, 0.7, backward=True)
    for n in range(0, x.numel(), 7):
        h, got = 1e-6, []
        for step in (h, -h):
            y = x.clone()
            y.view(-1)[n] += step
            y, _ = CR.turn(y, at, f, interleaved, 0.7)
            got.append((y * dy).sum().item())
        assert abs((got[0] - got[1]) / (2 * h) - dx.reshape(-1)[n].item()) < 1e-8


def test_reference_scales():
    assert CR.scale_of(448.0) == 1.0 and CR.scale_of(448.0001) == 2.0 and CR.scale_of(224.0) == 0.5 and CR.scale_of(224.01) == 1.0
    assert CR.scale_of(0.0) == 2.0 ** -100 and CR.scale_of(3.0e38) == 2.0 ** 120


def test_reference_attention_is_a_softmax():
    g = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((4, 6), (9, 2, 6), (9, 2, 6)))
    o, _, lse = CR.attend(q, k, v, 0.3)
    for h in range(4):
        z = (k[:, h // 2] @ q[h]) * 0.3
        assert torch.allclose(o[h], torch.softmax(z, 0) @ v[:, h // 2], atol=1e-14) and abs(torch.logsumexp(z, 0) - lse[h]) < 1e-13
    o, _, lse = CR.attend(q, k[:0], v[:0], 0.3)
    assert not o.any() and (lse == -math.inf).all()


# ---- refusals: the context is never looked at, so a block of zeros stands for it ---------------------------------------------------------------

ADDR = 1 << 20        # an aligned address that nothing follows


def _ctx():
    return C.create_string_buffer(1 << 16)


def _rotary(**over):
    a = R._Rotary()
    for n in ("q", "k", "frequencies", "cu_seqlens", "d_num", "cu_prompts", "survivor_idx"):
        setattr(a, n, ADDR)
    a.q_out, a.k_out = 2 * ADDR, 3 * ADDR
    a.q_stride = a.k_stride = a.q_out_stride = a.k_out_stride = 8 * 64
    a.T_max, a.S_max, a.P, a.G, a.Hq, a.Hkv, a.D, a.R, a.factor = 100, 4, 2, 4, 8, 4, 64, 64, 1.0
    for n, x in over.items():
        setattr(a, n, x)
    return a


@pytest.mark.parametrize("call", ["arrol_rotary", "arrol_rotary_backward"])
@pytest.mark.parametrize("over,code", [
    (dict(q=None), -1), (dict(k=ADDR + 8), -1), (dict(q_out=None), -1), (dict(k_out=ADDR + 2), -1), (dict(q_stride=8 * 64 + 4), -1), (dict(k_stride=4 * 64 - 8), -1),
    (dict(q_out=ADDR, q_out_stride=8 * 64 + 8), -1), (dict(k_out=ADDR, k_out_stride=4 * 64), -1), (dict(frequencies=None), -1), (dict(frequencies=ADDR + 4), -1),
    (dict(cu_seqlens=None), -1), (dict(d_num=None), -1), (dict(cu_prompts=None), -1), (dict(P=0), -1), (dict(G=0), -1), (dict(S_max=-1), -1), (dict(T_max=-1), -1),
    (dict(R=0), -1), (dict(R=63), -1), (dict(R=66), -1), (dict(Hq=-1), -1), (dict(D=0), -1), (dict(factor=math.nan), -1), (dict(factor=math.inf), -1),
    (dict(D=68), -2), (dict(D=264), -2), (dict(T_max=(1 << 31) - 512), -2), (dict(Hq=65537), -2),
])
def test_rotary_refuses(lib, call, over, code):
    assert getattr(lib, call)(_ctx(), C.byref(_rotary(**over)), None) == code


def _pool(c):
    for n in ("k_cache", "v_cache", "k_scale", "v_scale"):
        setattr(c, n, ADDR)
    c.k_page_stride = c.v_page_stride = 4 * 32 * 64
    c.k_scale_stride = c.v_scale_stride = 4
    c.pages, c.page, c.Hkv, c.D = 50, 32, 4, 64


POOL_REFUSALS = [
    (dict(k_cache=None), -1), (dict(v_cache=ADDR + 8), -1), (dict(k_scale=None), -1), (dict(v_scale=ADDR + 2), -1), (dict(k_page_stride=4 * 32 * 64 - 16), -1),
    (dict(v_page_stride=4 * 32 * 64 + 8), -1), (dict(k_scale_stride=3), -1), (dict(v_scale_stride=0), -1), (dict(pages=-1), -1), (dict(Hkv=0), -1), (dict(page=0), -1),
    (dict(page=48), -2), (dict(page=256), -2), (dict(page=8), -2), (dict(D=72), -2), (dict(D=144), -2),
]


def _append(pool=None, **over):
    a = K._Append()
    _pool(a.cache)
    for n in ("q", "k", "v", "page_table", "lengths", "keep", "prompt_lengths", "frequencies"):
        setattr(a, n, ADDR)
    a.q_out, a.k_out = 2 * ADDR, 3 * ADDR
    a.q_stride = a.k_stride = a.v_stride = a.q_out_stride = a.k_out_stride = 8 * 64
    a.rows, a.table_pages, a.table_stride, a.N, a.P, a.G, a.Hq, a.R, a.factor = 8, 5, 5, 8, 2, 4, 8, 64, 1.0
    for n, x in (pool or {}).items():
        setattr(a.cache, n, x)
    for n, x in over.items():
        setattr(a, n, x)
    return a


@pytest.mark.parametrize("over,code", POOL_REFUSALS)
def test_append_refuses_pools(lib, over, code):
    if over in (dict(D=72), dict(D=144)):
        over = dict(over, k_page_stride=1 << 20, v_page_stride=1 << 20)
    assert lib.arrol_cache_append(_ctx(), C.byref(_append(pool=over)), None) == code


@pytest.mark.parametrize("over,code", [
    (dict(q=None), -1), (dict(q_out=None), -1), (dict(k=None), -1), (dict(v=ADDR + 4), -1), (dict(k_stride=8), -1), (dict(q_out_stride=8 * 64 + 1), -1),
    (dict(k_out=ADDR, k_out_stride=8 * 64 + 8), -1), (dict(q_out=ADDR, q_out_stride=8 * 72), -1), (dict(page_table=None), -1), (dict(table_pages=0), -1), (dict(table_stride=4), -1),
    (dict(lengths=None), -1), (dict(frequencies=None), -1), (dict(R=0), -1), (dict(R=7), -1), (dict(R=66), -1), (dict(factor=math.nan), -1), (dict(prompt_lengths=None), -1),
    (dict(P=0), -1), (dict(P=3), -1), (dict(G=0), -1), (dict(rows=9), -1), (dict(rows=-1), -1), (dict(N=-8), -1), (dict(Hq=0), -1),
    (dict(cu_new=ADDR, rows=(1 << 31) - 512), -2), (dict(N=(1 << 24) + 4, P=(1 << 22) + 1, rows=(1 << 24) + 4), -2),
])
def test_append_refuses(lib, over, code):
    assert lib.arrol_cache_append(_ctx(), C.byref(_append(**over)), None) == code


def _attend(pool=None, **over):
    a = K._Attend()
    _pool(a.cache)
    for n in ("q", "page_table", "lengths", "keep", "prompt_table", "prompt_lengths", "o", "lse", "workspace"):
        setattr(a, n, ADDR)
    a.q_stride = a.o_stride = 8 * 64
    a.table_pages = a.table_stride = a.prompt_table_pages = a.prompt_table_stride = 5
    a.N, a.P, a.G, a.Hq, a.scale = 8, 2, 4, 8, 0.125
    for n, x in (pool or {}).items():
        setattr(a.cache, n, x)
    for n, x in over.items():
        setattr(a, n, x)
    return a


@pytest.mark.parametrize("over,code", POOL_REFUSALS)
def test_attention_refuses_pools(lib, over, code):
    if over in (dict(D=72), dict(D=144)):
        over = dict(over, k_page_stride=1 << 20, v_page_stride=1 << 20)
    assert lib.arrol_cache_attention(_ctx(), C.byref(_attend(pool=over)), None) == code


@pytest.mark.parametrize("over,code", [
    (dict(q=None), -1), (dict(o=ADDR + 8), -1), (dict(q_stride=8 * 64 - 8), -1), (dict(o_stride=8 * 64 + 4), -1), (dict(lengths=None), -1), (dict(page_table=None), -1),
    (dict(table_stride=4), -1), (dict(table_pages=-1), -1), (dict(prompt_table=None), -1), (dict(prompt_lengths=None), -1), (dict(prompt_table_stride=4), -1), (dict(P=0), -1),
    (dict(P=1), -1), (dict(G=0), -1), (dict(N=-1), -1), (dict(Hq=6), -1), (dict(Hq=0), -1), (dict(scale=0.0), -1), (dict(scale=-1.0), -1), (dict(scale=math.nan), -1),
    (dict(scale=math.inf), -1), (dict(Hq=4 * 65), -2), (dict(G=2048, P=1, N=2048), -2), (dict(N=(1 << 24) + 4, P=(1 << 22) + 1), -2),
    (dict(workspace=None), -3), (dict(workspace=ADDR + 64), -3), (dict(workspace_bytes=255), -3),
    # tables whose tokens, all of them there, would be more pieces than 32 bits count
    (dict(table_pages=1 << 28, table_stride=1 << 28, workspace_bytes=1 << 40), -2), (dict(prompt_table_pages=1 << 28, prompt_table_stride=1 << 28, workspace_bytes=1 << 40), -2),
    (dict(table_pages=1 << 26, table_stride=1 << 26, workspace_bytes=1 << 40), -2), (dict(N=1 << 24, P=1 << 22, workspace_bytes=1 << 60), -2),
])
def test_attention_refuses(lib, over, code):
    assert lib.arrol_cache_attention(_ctx(), C.byref(_attend(**over)), None) == code


@pytest.mark.parametrize("Hq,Hkv,G,N", [(33, 1, 64, 256), (22, 1, 5, 40), (20, 2, 3, 30), (64, 1, 4, 64), (8, 4, 16, 512), (64, 8, 100, 400)])
def test_tables_up_to_the_limits_are_taken(lib, Hq, Hkv, G, N):
    """A prompt counts once for every floor(64 / (Hq / Hkv)) rollouts of its group, for these read it together.  Tables of own tokens and of prompts right below what the interface
    promises are taken, both at once; what is well above is refused.  Sizes are looked at before the workspace, which is missing here."""
    ratio, P = Hq // Hkv, N // G
    rollouts = 64 // ratio
    own = ((1 << (31 if ratio > 16 else 34)) - 1) // (N * Hkv) - 256
    prompts = ((1 << 31) - 1) // (P * -(-G // rollouts) * Hkv) - 256
    pool = dict(Hkv=Hkv, page=16, k_page_stride=1 << 24, v_page_stride=1 << 24, k_scale_stride=64, v_scale_stride=64)
    base = dict(N=N, P=P, G=G, Hq=Hq, q_stride=1 << 14, o_stride=1 << 14, workspace=None)

    def call(own, prompts):
        own, prompts = min(own, (1 << 31) - 16) // 16, min(prompts, (1 << 31) - 16) // 16
        return lib.arrol_cache_attention(_ctx(), C.byref(_attend(pool=pool, table_pages=own, table_stride=own, prompt_table_pages=prompts, prompt_table_stride=prompts, **base)), None)

    assert call(own, prompts) == call(own, 16) == call(16, prompts) == -3
    if 3 * prompts < 1 << 31:
        assert call(own, 3 * prompts) == call(16, 3 * prompts) == -2
    if 3 * own < 1 << 31:
        assert call(3 * own, 16) == -2


def test_null_contexts_and_empty_calls(lib):
    null = C.c_void_p()
    for call in ("arrol_rotary", "arrol_rotary_backward", "arrol_cache_append", "arrol_cache_attention"):
        assert getattr(lib, call)(null, None, None) == -1 and getattr(lib, call)(_ctx(), None, None) == -1
    assert lib.arrol_rotary(_ctx(), C.byref(_rotary(T_max=0)), None) == 0
    assert lib.arrol_rotary(_ctx(), C.byref(_rotary(Hq=0, Hkv=0)), None) == 0
    assert lib.arrol_cache_append(_ctx(), C.byref(_append(N=0, P=0, prompt_lengths=None, rows=0)), None) == 0
    assert lib.arrol_cache_append(_ctx(), C.byref(_append(cu_new=ADDR, rows=0)), None) == 0
    assert lib.arrol_cache_attention(_ctx(), C.byref(_attend(N=0, P=0, prompt_lengths=None, prompt_table=None)), None) == 0
    assert lib.arrol_cache_attention_workspace(null, 1, 0, 1, 8, 4, 64) == 0
    assert lib.arrol_cache_attention_workspace(_ctx(), 1, 0, 0, 8, 4, 64) == 0
    assert lib.arrol_cache_attention_workspace(_ctx(), 1, 0, 1, 8, 3, 64) == 0


class _NoContext:
    handle = None


def test_bindings_refuse_types_and_shapes():
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    f = torch.ones(4, dtype=torch.float64)
    with pytest.raises(TypeError):
        R.arrol_rotary(_NoContext, bf(3, 2, 8).float(), None, f, bf(3, 2, 8), None, positions=torch.zeros(3, dtype=torch.int32))
    for kw in (dict(), dict(positions=torch.zeros(2, dtype=torch.int32)), dict(positions=torch.zeros(3, dtype=torch.int64)),
               dict(positions=torch.zeros(3, dtype=torch.int32), cu_seqlens=torch.zeros(2, dtype=torch.int64))):
        with pytest.raises(ValueError):
            R.arrol_rotary(_NoContext, bf(3, 2, 8), None, f, bf(3, 2, 8), None, **kw)
    with pytest.raises(ValueError):
        R.arrol_rotary(_NoContext, bf(3, 2, 8), None, f.float(), bf(3, 2, 8), None, positions=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError):
        R.arrol_rotary(_NoContext, None, None, f, None, None, positions=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError):
        R.arrol_rotary(_NoContext, bf(3, 2, 8), None, f, None, None, positions=torch.zeros(3, dtype=torch.int32))
    pool = dict(k_cache=torch.zeros(5, 2, 16, 16, dtype=torch.uint8), v_cache=torch.zeros(5, 2, 16, 16, dtype=torch.uint8), k_scale=torch.zeros(5, 2), v_scale=torch.zeros(5, 2))
    table, lengths = torch.zeros(3, 2, dtype=torch.int32), torch.ones(3, dtype=torch.int32)
    k = bf(3, 2, 16)
    for name, value, error in (("k_cache", pool["k_cache"].float(), TypeError), ("v_cache", pool["v_cache"][:4], ValueError), ("k_scale", pool["k_scale"].double(), TypeError),
                               ("v_scale", pool["v_scale"].T.contiguous().T, ValueError), ("k_cache", pool["k_cache"].transpose(2, 3), ValueError)):
        with pytest.raises(error):
            K.arrol_cache_append(_NoContext, k, k, **(pool | {name: value}), page_table=table, lengths=lengths)
    for kw in (dict(page_table=table[:2]), dict(page_table=table.long()), dict(lengths=lengths.long()), dict(q=k), dict(keep=torch.ones(2, dtype=torch.uint8)),
               dict(cu_new=torch.zeros(3, dtype=torch.int64)), dict(lengths=lengths[:2], page_table=table[:2])):
        with pytest.raises(ValueError):
            K.arrol_cache_append(_NoContext, k, k, **pool, **(dict(page_table=table, lengths=lengths) | kw))
    for kw in (dict(q=bf(3, 2, 32)), dict(prompt_table=table), dict(prompt_lengths=lengths), dict(lse=torch.zeros(5))):
        with pytest.raises(ValueError):
            K.arrol_cache_attention(_NoContext, **(dict(q=k, o=bf(3, 2, 16), lse=None) | pool | dict(page_table=table, lengths=lengths, workspace=None) | kw))
