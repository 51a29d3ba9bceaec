"""Sequences whose rows lie behind ones that are not the call's: what starts outside the rows is no sequence, and those after it
are whole, cut into parts or not.  Compared with the 64-bit form under the bounds of test_gpu_block_attend."""
import pytest
import torch

from tests.gpu_util import need_gpu, say
from tests.test_gpu_block_attend import check, held_cache
from tests.test_gpu_block_cache import gen, layout

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


@pytest.mark.parametrize("first,dim", [([-4, 0], 64), ([-40, -1, 0], 128), ([-3, 5], 64), ([-200, 7], 192), ([3], 64), ([-1, 0], 64)])
@pytest.mark.parametrize("lengths,new", [([2477], [133]), ([2477, 30, 1999], [70, 1, 40])])
def test_sequences_behind_starts_before_the_rows(lengths, new, first, dim):
    from paper_2504_00598_amd import block
    say("starts", first, lengths, new, dim)
    g = gen(dim + len(first))
    none = len(first) - 1  # sequences in front that begin before the rows
    table, starts, lens, pages = layout([50] * none + lengths, [0] * none + new, 16, g)
    starts = torch.cat([torch.tensor(first[:-1], dtype=torch.int32), starts[none:] + first[-1]])
    cache, k, v = held_cache(pages, 16, 1, dim, "bf16", "bf16", g)
    T = int(starts[-1]) + 6
    q = torch.randn(T, 8, dim, generator=g).bfloat16()
    out = torch.full((T, 8, dim), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((T, 8), 7.0, device="cuda")
    y, lse = block.attend(q.cuda(), cache, block.Sequences(table.cuda(), starts.cuda(), lens.cuda()), with_lse=True, out=out)
    lo, hi = first[-1], int(starts[-1])
    rows = set(range(lo, lo + 8)) | set(range(lo, hi, 13)) | {hi - 1}
    check(y, lse, q, k, v, table[none:], starts[none:], lens[none:], dim ** -0.5, True, 0, first, rows)
    assert not bool((lse[lo:hi] == 7).any())
    for t in (y, lse):
        assert bool((t[:lo] == 7).all()) and bool((t[hi:] == 7).all())
