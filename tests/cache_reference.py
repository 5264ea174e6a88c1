"""Rotary positions and the paged 8-bit cache in 64 bits, from the definition, one row and one page at a time; beside results how far a kernel may be from them that computes in
fp32 and rounds what the interface says it rounds."""
import math

import torch

F8 = torch.float8_e4m3fn
BF16, FP16, E4M3 = 2.0 ** -8, 2.0 ** -11, 2.0 ** -4        # half a step, relative
F32 = 2.0 ** -13                                           # sums over D and over keys, exponentials and logarithms in fp32
# A turned entry before it is rounded: cosine and sine to a few steps of fp32, the angle's rest rounded to fp32 (at most pi x 2^-24), factor, two products and a sum.
TURN = 2.0 ** -20


def turn(x, positions, frequencies, interleaved=False, factor=1.0, backward=False):
    """x [T, H, D] -> (turned, bound on the error before the last rounding), both in 64 bits."""
    y = x.double().clone()
    size = torch.zeros_like(y)
    n = len(frequencies)
    for i, f in enumerate(frequencies):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, n + i)
        angle = positions.double() * float(f) * (-1.0 if backward else 1.0)
        c, s = (factor * angle.cos())[:, None], (factor * angle.sin())[:, None]
        x1, x2 = x[..., a].double(), x[..., b].double()
        y[..., a], y[..., b] = x1 * c - x2 * s, x2 * c + x1 * s
        size[..., a] = size[..., b] = (x1.abs() + x2.abs()) * abs(factor)
    return y, TURN * size


def scale_of(amax):
    """The least power of two, from 2^-100 on, that brings amax to 448 or less."""
    e = -100
    while amax > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def read(cache, scale, table, n):
    """[n, Hkv, D] in 64 bits: the tokens of one sequence."""
    page = cache.shape[2]
    out = []
    for j in range(n):
        p = int(table[j // page])
        out.append(cache.view(torch.uint8)[p, :, j % page].view(F8).double() * scale[p].double()[:, None])
    return torch.stack(out) if out else torch.zeros(0, cache.shape[1], cache.shape[3], dtype=torch.float64, device=cache.device)


def read_many(cache, scale, table, lengths):
    """The same for all rows of a table, as one padded gather: a list."""
    page = cache.shape[2]
    out = []
    for i, n in enumerate(lengths):
        at = table[i, :-(-n // page)].long()
        x = cache.view(torch.uint8)[at].view(F8).double() * scale[at].double()[:, :, None, None]
        out.append(x.transpose(1, 2).reshape(-1, cache.shape[1], cache.shape[3])[:n])
    return out


def attend(q, keys, values, scale):
    """q [Hq, D], keys, values [n, Hkv, D] in 64 bits -> o, bound, lse."""
    q = q.double()
    (Hq, D), Hkv = q.shape, keys.shape[1]
    if keys.shape[0] == 0:
        return torch.zeros_like(q), torch.zeros_like(q), torch.full((Hq,), -math.inf, dtype=torch.float64, device=q.device)
    r = Hq // Hkv
    z = torch.einsum("grd,jgd->grj", q.view(Hkv, r, D), keys) * scale
    lse = torch.logsumexp(z, -1)
    p = torch.exp(z - lse[..., None])
    o = torch.einsum("grj,jgd->grd", p, values).reshape(Hq, D)
    spread = torch.einsum("grj,jgd->grd", p, values.abs()).reshape(Hq, D)
    # o is rounded to bf16, every probability to fp16 before its product with the value
    return o, BF16 * o.abs() + (FP16 + F32) * spread + 1e-30, lse.reshape(Hq)
