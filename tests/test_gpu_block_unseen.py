"""What no row sees of a cache of 8 bits has no effect, its scales among it: a fresh cache holds any byte behind a
sequence's end, in pages that no table names and in page 0, which stands for entries outside the cache.

No bounds: a result with other bytes in unseen places has the same bits.  The result itself is compared with the 64-bit form
under the bounds of test_gpu_block_attend.
"""
import pytest
import torch

from tests.gpu_util import need_gpu, say
from tests.test_gpu_block_attend import check, held_cache
from tests.test_gpu_block_cache import DT, gen

pytestmark = pytest.mark.gpu

L, PAGE, HEADS = 150, 16, 2


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


def make(dim, dt, g):
    """A cache whose page 0 is no sequence's, one sequence of L tokens in it and table entries of -1 behind its last page."""
    cache, k, v = held_cache(14, PAGE, HEADS, dim, dt, "e4m3", g)
    table = torch.full((1, 12), -1, dtype=torch.int32)
    table[0, :10] = torch.randperm(13, generator=g)[:10].int() + 1
    return cache, k, v, table


def places(table, tokens):
    """[pages][page] truth values: where the tokens lie."""
    at = torch.zeros(14, PAGE, dtype=torch.bool)
    for p in tokens:
        at[int(table[0, p // PAGE]), p % PAGE] = True
    return at


def fill(cache, at, entry, scale):
    """Bytes of the entries and of the scales of all heads at the places `at`."""
    at = at.cuda()
    cache.k.view(torch.uint8).masked_fill_(at[:, None, :, None], entry)
    cache.v.view(torch.uint8).masked_fill_(at[:, None, None, :], entry)
    for s in (cache.k_scale, cache.v_scale):
        s.masked_fill_(at[:, None, :], scale)


FILLS = [(0x31, 255), (0xff, 255), (0x00, 255), (0xfe, 200), (0x7e, 254), (0x01, 0)]


def unseen(new, group, dim, dt, window):
    from paper_2504_00598_amd import block
    say("unseen", new, group, dim, dt, window)
    g = gen(dim + new)
    cache, k, v, table = make(dim, dt, g)
    starts, lens = torch.tensor([0, new], dtype=torch.int32), torch.tensor([L], dtype=torch.int32)
    q = torch.randn(new, HEADS * group, dim, generator=g).to(DT[dt])
    seqs = block.Sequences(table.cuda(), starts.cuda(), lens.cuda(), max_new=new)
    clean = block.attend(q.cuda(), cache, seqs, window=window, with_lse=True)
    check(*clean, q, k, v, table, starts, lens, dim ** -0.5, True, window, "clean", {0, new - 1})
    other = ~places(table, range(max(L - new - window + 1, 0) if window else 0, L))
    for entry, scale in FILLS:
        fill(cache, other, entry, scale)
        y, lse = block.attend(q.cuda(), cache, seqs, window=window, with_lse=True)
        assert torch.equal(y, clean[0]) and torch.equal(lse, clean[1]), (entry, scale, int(y.isnan().sum()), y.numel())


@pytest.mark.parametrize("window", [0, 20])
@pytest.mark.parametrize("dim", [64, 96, 256])
@pytest.mark.parametrize("new,group", [(1, 1), (3, 4), (5, 4)])
def test_scales_that_no_row_sees_where_weights_take_them(new, group, dim, window):
    """Up to 32 rows a key head in bfloat16: a weight of zero is multiplied by the scale of what it masks."""
    unseen(new, group, dim, "bf16", window)
