"""Plain 64-bit forms of the operators over a paged cache, written token by token from their definitions (torch on the
CPU), for the tests of the kernels."""
import math

import torch


def e4m3(x):
    """x in 64 bits to 4 significant bits, below 2^-6 to multiples of 2^-9; ties to even."""
    e = (torch.frexp(x)[1] - 1).clamp_min(-6)
    step = torch.ldexp(torch.ones_like(x), e - 3)
    return torch.round(x / step) * step


def held(x):
    """(what stands in a cache of e4m3, exponent) of rows x [..., dim]: x / 2^e, e the least integer >= -126 for which
    no finite entry passes 448; what is not finite is NaN."""
    last = 8 if x.dtype == torch.float16 else 120  # the exponent under which 256 2^e is beyond x's type, and 240 2^e is not
    x = x.double()
    fine = torch.isfinite(x)
    top = x.masked_fill(~fine, 0).abs().amax(-1)
    e = torch.full(top.shape, -126, dtype=torch.int32)
    for _ in range(260):
        over = top > torch.ldexp(torch.full_like(top, 448.0), e)
        if not bool(over.any()):
            break
        e = e + over.int()
    q = x / torch.ldexp(torch.ones_like(top), e)[..., None]
    limit = torch.where(e == last, torch.full_like(top, 240.0), torch.full_like(top, 448.0))[..., None]
    q = e4m3(torch.minimum(torch.maximum(q, -limit), limit))
    return torch.where(fine, q, torch.full_like(q, math.nan)), e


def place(table, lengths, starts, page, b, i):
    """(page, place) of row i of sequence b, or None before the first token."""
    p = int(lengths[b]) - (int(starts[b + 1]) - int(starts[b])) + i
    if p < 0:
        return None
    return (int(table[b, p // page]) if p // page < table.shape[1] else -1), p % page


def attend(q, k, v, p, scale, causal, window):
    """q [dim], k and v [tokens][dim] in 64 bits, token p of them: (result, lse, sum of weights times |v| over l,
    largest scale |q| . |k|)."""
    j = torch.arange(k.shape[0])
    sees = torch.ones_like(j, dtype=torch.bool)
    if causal:
        sees &= j <= p
    if window:
        sees &= j >= p - window + 1
    if not bool(sees.any()):
        return torch.zeros(k.shape[1], dtype=torch.float64), -math.inf, torch.zeros(k.shape[1], dtype=torch.float64), 0.0
    k, v = k[sees], v[sees]
    s = scale * (k @ q)
    w = torch.softmax(s, 0)
    return (w[:, None] * v).sum(0), float(torch.logsumexp(s, 0)), w @ v.abs(), float(scale * (k.abs() @ q.abs()).max())
