"""Infinities that rows see: scores of -infinity alone are as if nothing were seen, and an infinite value leaves its entry without
a finite result, whatever its weight.  No bounds: zeros, infinities and equal bits."""
import math

import pytest
import torch

from tests.gpu_util import need_gpu, say
from tests.test_gpu_block_attend import held_cache
from tests.test_gpu_block_cache import DT, gen, layout

pytestmark = pytest.mark.gpu

FORMS = [(1, 1, 64), (5, 4, 64), (70, 4, 64), (40, 2, 192)]


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


@pytest.mark.parametrize("length", [150, 2500])  # whole, and in parts
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("new,group,dim", FORMS)
def test_scores_of_minus_infinity(new, group, dim, dt, length):
    from paper_2504_00598_amd import block
    say("minus infinity", new, group, dim, dt, length)
    g = gen(dim + new)
    table, starts, lens, pages = layout([length], [new], 16, g)
    cache, _, _ = held_cache(pages, 16, 2, dim, dt, dt, g)
    q = torch.randn(new, 2 * group, dim, generator=g).to(DT[dt]).cuda()
    q[:, :, 0] = 1.0
    seqs = block.Sequences(table.cuda(), starts.cuda(), lens.cuda(), max_new=new)
    old = cache.k.clone()
    cache.k[..., 0] = -math.inf
    y, lse = block.attend(q, cache, seqs, with_lse=True)
    assert bool((y == 0).all()) and bool((lse == -math.inf).all())
    # beside one token that has a score, its value is the result
    only = (int(table[0, 1]), 3)
    cache.k[only[0], :, only[1]] = old[only[0], :, only[1]]
    y, lse = block.attend(q, cache, seqs, with_lse=True)
    v = cache.v[only[0], :, :, only[1]]
    assert torch.equal(y, v.repeat_interleave(group, 0).expand_as(y)) and bool(torch.isfinite(lse).all())


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("new,group,dim", FORMS)
def test_an_infinite_value_of_any_weight(new, group, dim, dt):
    from paper_2504_00598_amd import block
    say("infinite value", new, group, dim, dt)
    g = gen(dim + new)
    L = 200
    table, starts, lens, pages = layout([L], [new], 16, g)
    cache, _, _ = held_cache(pages, 16, 2, dim, dt, dt, g)
    q = torch.randn(new, 2 * group, dim, generator=g).to(DT[dt]).cuda()
    q[:, :, 0] = 1.0
    cache.k[..., 0] = 0.0
    seqs = block.Sequences(table.cuda(), starts.cuda(), lens.cuda(), max_new=new)
    keep = torch.arange(dim, device="cuda") != 5
    for p in (0, 70, L - new):  # in a tile that all rows see, and at the first row's own token
        at = int(table[0, p // 16]), p % 16
        for score in (0.0, -30000.0):
            old = cache.k.clone(), cache.v.clone()
            cache.k[at[0], :, at[1], 0] = score
            clean = block.attend(q, cache, seqs, scale=1.0)
            cache.v[at[0], :, 5, at[1]] = -math.inf
            y = block.attend(q, cache, seqs, scale=1.0)
            assert not bool(torch.isfinite(y[:, :, 5]).any()), (p, score)
            assert torch.equal(y[:, :, keep], clean[:, :, keep]), (p, score)
            cache.k.copy_(old[0]), cache.v.copy_(old[1])
