"""A cache of 8 bits read by the 16-bit type that did not write it.  bfloat16 has scales that float16's range does not hold: what is
held is rounded to float16 then, beyond its range to an infinity, below it to its smallest steps or zero.  bfloat16 holds whatever float16
wrote.

Bounds.  What is read back is one rounding of a defined value: equal.  The attention is that over the values so rounded, under the
bounds of test_gpu_block_attend and one term more.  These take the result's rounding as u |o|, which holds from float16's least normal
value 2^-14 on.  Below it float16 has the multiples of 2^-24 alone, so that a result is rounded by up to half of one, 2^-25, where
u |o| < 2^-11 2^-14 = 2^-25: with D = 2^-25 for float16 (bfloat16 has the range of 32 bits: D = 0)
    |out - o| <= u |o| + (u + E + 2^-16) A (1 + u) + Z + D.
"""
import math

import pytest
import torch

from tests import cache_ref as R
from tests.gpu_util import need_gpu, say
from tests.test_gpu_block_attend import U
from tests.test_gpu_block_cache import DT, filled, gen, layout

pytestmark = pytest.mark.gpu

PAGE, HEADS = 16, 2


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


def written(x, y, dim, g):
    """A cache that keys x and values y [T][HEADS][dim] were written to as one sequence, its table, and what it holds of
    them in 64 bits."""
    from paper_2504_00598_amd import block
    T = x.shape[0]
    table, starts, lens, pages = layout([T], [T], PAGE, g)
    cache = filled(block.KVCache.empty(pages, PAGE, HEADS, dim, torch.float8_e4m3fn), 0xff)
    block.cache_write(cache, x.cuda(), y.cuda(), block.Sequences(table.cuda(), starts.cuda(), lens.cuda()))
    value = lambda t: (lambda h, e: h * torch.pow(2.0, e.double())[..., None])(*R.held(t))  # noqa: E731
    return cache, table, value(x), value(y)


def paged(x, table, pages):
    """Rows [T][HEADS][dim] as [pages][HEADS][PAGE][dim]."""
    out = torch.zeros(pages, HEADS, PAGE, x.shape[2], dtype=x.dtype)
    for p in range(x.shape[0]):
        out[int(table[0, p // PAGE]), :, p % PAGE] = x[p]
    return out


def check(got, lse, q, k, v, table, length, scale, rows):
    """Rows of one sequence of the last tokens; k, v [pages][HEADS][PAGE][dim] in 64 bits."""
    n, hq, dim = q.shape
    u, half = U[q.dtype], q.dtype is torch.float16
    got, lse, q = got.cpu().double(), lse.cpu().double(), q.double()
    at = table[0, :-(-length // PAGE)].long()
    k, v = (t[at].transpose(0, 1).reshape(HEADS, -1, dim)[:, :length] for t in (k, v))
    for i in rows:
        for h in range(hq):
            kv = h // (hq // HEADS)
            o, ls, A, S = R.attend(q[i, h], k[kv], v[kv], length - n + i, scale, True, 0)
            Z, D = (2.0 ** -33 * v[kv].abs().sum(0), 2.0 ** -25) if half else (0.0, 0.0)
            E = 2 * (dim + 4) * 2.0 ** -24 * S
            off = (got[i, h] - o).abs() - (u * o.abs() + (u + E + 2.0 ** -16) * A * (1 + u) + Z + D + 1e-30)
            assert bool((off <= 0).all()), (i, h, float((got[i, h] - o).abs().max()), float(A.max()), float(off.max()))
            assert abs(float(lse[i, h]) - ls) <= E + 2.0 ** -16 + 2.0 ** -22 * abs(ls), (i, h, ls)


@pytest.mark.parametrize("wrote,reads", [("bf16", "f16"), ("f16", "bf16")])
def test_read_back_as_the_other_type(wrote, reads):
    from paper_2504_00598_amd import block
    g = gen(1)
    T, dim = 150, 64
    powers = torch.randint(-40, 40, (T, HEADS, 1), generator=g) if wrote == "bf16" else torch.randint(-14, 15, (T, HEADS, 1), generator=g)
    x, y = ((torch.randn(T, HEADS, dim, generator=g) * 2.0 ** powers).to(DT[wrote]) for _ in range(2))
    cache, table, k, v = written(x, y, dim, g)
    seqs = block.Sequences(table.cuda(), torch.tensor([0, T], dtype=torch.int32).cuda(), torch.tensor([T], dtype=torch.int32).cuda())
    got = block.cache_read(cache, seqs, T, dtype=DT[reads])
    for a, b in zip(got, (k, v)):
        assert torch.equal(a.cpu(), b.to(DT[reads]))
    if wrote == "bf16":
        assert bool(got[1].isinf().any()) and bool((got[1] == 0).any())


@pytest.mark.parametrize("new,group,dim", [(1, 1, 64), (3, 4, 96), (5, 4, 64), (70, 4, 128), (70, 4, 192), (5, 4, 256)])
@pytest.mark.parametrize("wrote,reads,low,high,scale", [
    ("bf16", "f16", -19, -13, 2.0 ** 12),  # below float16's normal range
    ("bf16", "f16", 8, 13, 2.0 ** -14), ("f16", "bf16", -13, -9, 2.0 ** 9), ("f16", "bf16", 8, 13, 2.0 ** -14)])
def test_attention_in_the_other_type(wrote, reads, low, high, scale, new, group, dim):
    from paper_2504_00598_amd import block
    say("other type", wrote, reads, low, new, group, dim)
    g = gen(dim + new)
    T = 150
    x, y = ((torch.randn(T, HEADS, dim, generator=g) * 2.0 ** torch.randint(low, high, (T, HEADS, 1), generator=g)).to(DT[wrote])
            for _ in range(2))
    cache, table, k, v = written(x, y, dim, g)
    k, v = (paged(t.to(DT[reads]).double(), table, cache.k.shape[0]) for t in (k, v))
    starts, lens = torch.tensor([0, new], dtype=torch.int32), torch.tensor([T], dtype=torch.int32)
    q = torch.randn(new, HEADS * group, dim, generator=g).to(DT[reads])
    seqs = block.Sequences(table.cuda(), starts.cuda(), lens.cuda())
    out = block.attend(q.cuda(), cache, seqs, scale=scale, with_lse=True)
    check(*out, q, k, v, table, T, scale, {0, new // 2, new - 1})


@pytest.mark.parametrize("new,group,dim", [(1, 1, 64), (3, 4, 96), (5, 4, 64), (70, 4, 128), (70, 4, 192)])
def test_tokens_beyond_float16(new, group, dim):
    """One token of bfloat16's range in its key or its value: rows that see it have no finite result, the others the same bits."""
    from paper_2504_00598_amd import block
    say("beyond float16", new, group, dim)
    g = gen(dim)
    T = 150
    x, y = (torch.randn(T, HEADS, dim, generator=g).bfloat16() for _ in range(2))
    q = torch.randn(new, HEADS * group, dim, generator=g).half().cuda()
    starts, lens = torch.tensor([0, new], dtype=torch.int32).cuda(), torch.tensor([T], dtype=torch.int32).cuda()
    got = []
    for what in (None, "key", "value"):
        a, b = x.clone(), y.clone()
        if what:
            (a if what == "key" else b)[T - 1] = 2.0 ** 60
        cache, table, _, _ = written(a, b, dim, gen(3))
        got.append(block.attend(q, cache, block.Sequences(table.cuda(), starts, lens, max_new=new), with_lse=True))
    for y2, lse2 in got[1:]:
        assert torch.equal(y2[:-1], got[0][0][:-1]) and torch.equal(lse2[:-1], got[0][1][:-1])
    assert not bool(torch.isfinite(got[2][0][-1]).any()) and torch.equal(got[2][1], got[0][1])
    last = got[1][0][-1]  # a score of infinity leaves no number, one of -infinity no trace
    s = q[-1].float().sum(1)
    assert bool(last[s > 1].isnan().all()) and math.isfinite(float(got[0][0].float().abs().max()))
