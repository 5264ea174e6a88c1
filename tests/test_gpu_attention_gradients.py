"""Norms of the attention gradients' errors, long sequences and large scores.  The bounds of attention_reference.py hold for every entry and add up all roundings
in absolute value, so they grow with the rows that are summed while the sums grow with their root: what they leave free where sequences are long, a norm
does not."""
import math

import pytest
import torch

from attention_reference import BF16
from paper_2603_24840_b200 import binding as B
from test_gpu_attention import SHAPES, SPLIT, Problem

pytestmark = pytest.mark.gpu

# Three roundings to bf16 stand between a gradient and its formula: ds (or p), the o that delta is taken from, and the result, each by half a step at most, of
# either sign and independent: 2^-8 / sqrt(3) of the norm each, 2^-8 together.  Twice that, for sums in which terms cancel.
NORM = 2 * BF16
NAMES = {"dq": "dq", "dk": "dk", "dv": "dv", "dprompt_k": "dpk", "dprompt_v": "dpv"}


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    c.close()


def _check_norms(p, out, res):
    for name, ref in NAMES.items():
        if name not in out:
            continue
        live = p.T if not name.startswith("dp") else p.cu_prompts[-1]
        x, y = out[name][:live].double(), res[ref][:live]
        assert ((x - y).norm() <= NORM * y.norm() + 1e-6 * y.numel() ** 0.5), (name, ((x - y).norm() / y.norm()).item())


@pytest.mark.parametrize("lens,prompts,index,G,Hq,Hkv,D", [x for x in SHAPES + SPLIT if sum(x[0]) > 100] + [
    ([700, 650, 720, 30], [200], [0, 1, 2, 3], 4, 8, 2, 64),            # a prompt whose tokens come in parts
    ([90] * 24, [300, 40, 513], [8 * p + i for p in range(3) for i in range(8)], 8, 8, 4, 128),
    ([1000, 30], [60], [0, 1], 2, 64, 1, 64),
    ([333, 900], [2000, 100], [0, 1], 1, 10, 2, 88),
])
def test_norms_of_the_gradients_errors(ctx, lens, prompts, index, G, Hq, Hkv, D):
    p = Problem(lens, prompts, index, G, Hq, Hkv, D, seed=40 + len(lens) + D)
    _check_norms(p, p.run(ctx), p.reference()[0])


@pytest.mark.parametrize("lens,prompts,index,G,Hq,Hkv,D", [
    ([8192], None, None, 1, 2, 1, 128),
    ([8191], None, None, 1, 1, 1, 64),
    ([4100, 77], [3001], [0, 1], 2, 2, 2, 64),
    ([5000], [2000], [0], 1, 3, 1, 96),
])
def test_long_sequences(ctx, lens, prompts, index, G, Hq, Hkv, D):
    p = Problem(lens, prompts, index, G, Hq, Hkv, D, seed=50 + D)
    out = p.run(ctx)
    p.check(out)
    _check_norms(p, out, p.reference()[0])


@pytest.mark.parametrize("D,Hq,Hkv", [(64, 4, 2), (128, 4, 1)])
@pytest.mark.parametrize("q_scale,scale", [(60.0, None), (1.5, 1e-6), (8.0, 1.0)])
def test_gradients_with_large_scores_and_small_scale(ctx, q_scale, scale, D, Hq, Hkv):
    """Scores of hundreds, and a scale that leaves none: p is taken again from the logarithm of the sum."""
    p = Problem([400, 150], [300], [0, 1], 2, Hq, Hkv, D, seed=45, q_scale=q_scale, scale=scale)
    out = p.run(ctx)
    res, tol = p.reference()
    # Relative error of every p by the exponent's, as in the forward's test (|z| 2^-20, which covers what lse loses as a natural logarithm in fp32), once from
    # the recomputed p, once more in o and the sum of it: each of the bounds' parts is at least 2^-8 of the p (ds) that it stands for, so they grow by this factor.
    zmax = (p.q.float().norm(dim=-1).max() * max(p.k.float().norm(dim=-1).max(), p.pk.float().norm(dim=-1).max()) * p.scale).item()
    grow = 1 + 3 * zmax * 2.0 ** -20 / BF16
    for name, ref in NAMES.items():
        live = p.T if not name.startswith("dp") else p.cu_prompts[-1]
        x, y, t = out[name][:live].double(), res[ref][:live], tol[ref][:live] * grow
        assert ((x - y).abs() <= t).all(), (name, ((x - y).abs() / t).max().item())
