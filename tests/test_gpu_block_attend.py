"""Attention over a paged cache against a plain 64-bit form (tests/cache_ref.py), row by row.

Bounds.  u is the unit roundoff of q's type (2^-8, 2^-11).  With w the weights over their sum and A = sum w |v|: a
weight is rounded to the type once before the product (u w |v| each), the result once (u |o|).  A score is a sum of dim
products in 32 bits, off by at most (dim + 4) 2^-24 S with S = scale |q| . |k|, and what a score is off by its weight is off
relatively: twice over (in the weight and in the sum of the weights) E = 2 (dim + 4) 2^-24 max S.  Powers of two, the
sum over n tokens and the rescaling of parts add less than 2^-16 for n up to 2^14 in the sums' usual growth (the
square root of n, 2^7 2^-24, with the exponentials' 2^-22).  float16's weights have no bits below 2^-24; they are held
times 2^8 or more over the largest, so each is off by half of 2^-24 2^-8 of it at most, and the sum of the weights is no less
than the largest: Z = 2^-33 sum |v| (bfloat16 has the range of 32 bits: Z = 0).  Together
    |out - o| <= u |o| + (u + E + 2^-16) A (1 + u) + Z,   |lse - exact| <= E + 2^-16 + 2^-22 |lse|.
"""
import math

import pytest
import torch

from tests import cache_ref as R
from tests.gpu_util import need_gpu, say
from tests.test_gpu_block_cache import DT, gen, layout

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


def held_cache(pages, page, heads, dim, dt, held, g, spread=1.0):
    """A full cache (KVCache) and its values (keys [pages][heads][page][dim], values alike, in 64 bits, CPU)."""
    from paper_2504_00598_amd import block
    k, v = (spread * torch.randn(pages, heads, page, dim, generator=g) for _ in range(2))
    if held != "e4m3":
        k, v = k.to(DT[held]), v.to(DT[held])
        return block.KVCache(k.cuda(), v.transpose(2, 3).contiguous().cuda()), k.double(), v.double()
    k = k * 2.0 ** torch.randint(-2, 3, (pages, heads, page, 1), generator=g)
    v = v * 2.0 ** torch.randint(-6, 7, (pages, heads, page, 1), generator=g)
    (k, ke), (v, ve) = R.held(k.to(DT[dt])), R.held(v.to(DT[dt]))
    byte = lambda t: t.float().to(torch.float8_e4m3fn)  # noqa: E731
    cache = block.KVCache(byte(k).cuda(), byte(v).view(pages, heads, page, dim).transpose(2, 3).contiguous().cuda(),
                          (ke + 127).to(torch.uint8).cuda(), (ve + 127).to(torch.uint8).cuda())
    return cache, k * torch.pow(2.0, ke.double())[..., None], v * torch.pow(2.0, ve.double())[..., None]


def check(got, lse, q, k, v, table, starts, lengths, scale, causal, window, what, rows=None):
    """Every row of every sequence (or those in `rows`); k, v [pages][heads][page][dim] in 64 bits."""
    T, hq, dim = q.shape
    heads, page = k.shape[1], k.shape[2]
    q_type, u = q.dtype, U[q.dtype]
    got, lse, q = got.cpu().double(), lse.cpu().double(), q.cpu().double()
    for b in range(lengths.numel()):
        L, n = int(lengths[b]), int(starts[b + 1]) - int(starts[b])
        used = -(-L // page)
        at = table[b, :used].long()
        kb = k[at].transpose(0, 1).reshape(heads, -1, dim)[:, :L]
        vb = v[at].transpose(0, 1).reshape(heads, -1, dim)[:, :L]
        for i in range(n):
            r = int(starts[b]) + i
            if rows is not None and r not in rows:
                continue
            for h in range(hq):
                kv = h // (hq // heads)
                o, ls, A, S = R.attend(q[r, h], kb[kv], vb[kv], L - n + i, scale, causal, window)
                Z = 2.0 ** -33 * vb[kv].abs().sum(0) if q_type is torch.float16 else 0.0
                E = 2 * (dim + 4) * 2.0 ** -24 * S
                off = (got[r, h] - o).abs() - (u * o.abs() + (u + E + 2.0 ** -16) * A * (1 + u) + Z + 1e-30)
                assert bool((off <= 0).all()), (what, b, i, h, float((got[r, h] - o).abs().max()), float(A.max()))
                if ls == -math.inf:
                    assert float(lse[r, h]) == -math.inf, (what, b, i, h)
                else:
                    assert abs(float(lse[r, h]) - ls) <= E + 2.0 ** -16 + 2.0 ** -22 * abs(ls), (what, b, i, h, ls)


CASES = [  # lengths, new tokens, query heads, key heads, dim, page, causal, window
    ([1], [1], 1, 1, 64, 16, True, 0),
    ([1], [1], 4, 1, 16, 16, True, 0),
    ([33], [1], 32, 8, 128, 16, True, 0),
    ([5, 16, 17, 100], [1, 1, 1, 1], 8, 2, 128, 16, True, 0),
    ([700, 3, 129], [1, 1, 1], 10, 2, 80, 32, True, 0),
    ([200, 64], [5, 3], 4, 4, 64, 32, True, 16),
    ([300], [8], 8, 2, 96, 64, False, 0),
    ([300], [8], 4, 2, 96, 16, False, 50),
    ([90, 0, 40], [70, 0, 40], 6, 3, 64, 16, True, 0),
    ([150, 77], [33, 77], 5, 1, 80, 16, True, 0),
    ([260], [40], 7, 1, 192, 128, True, 0),
    ([130, 9, 300], [100, 1, 2], 4, 1, 256, 64, True, 0),
    ([333], [129], 2, 2, 128, 256, True, 100),
    ([200], [200], 2, 1, 112, 32, False, 0),
    ([65], [65], 2, 1, 240, 16, True, 1),
    ([140, 150], [20, 150], 16, 1, 32, 16, True, 37),
    ([90], [1], 32, 1, 128, 16, True, 0),
    ([90, 50], [1, 30], 24, 1, 64, 32, True, 0),
    ([70, 44], [1, 1], 40, 1, 128, 16, True, 0),
    ([300, 270], [1, 6], 12, 4, 160, 16, True, 0),
    ([600, 90, 17], [300, 90, 17], 2, 1, 128, 64, True, 0),
]


@pytest.mark.parametrize("dt,held", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")])
@pytest.mark.parametrize("lengths,new,hq,heads,dim,page,causal,window", CASES)
def test_attend(lengths, new, hq, heads, dim, page, causal, window, dt, held):
    from paper_2504_00598_amd import block
    say("attend", lengths, new, hq, heads, dim, page, causal, window, dt, held)
    g = gen(dim + page + hq)
    table, starts, length, pages = layout(lengths, new, page, g)
    cache, k, v = held_cache(pages, page, heads, dim, dt, held, g)
    T = int(starts[-1])
    lead = 3 if dim == 80 else 0  # off 16 bytes
    qkv = torch.randn(T, (hq + 2) * dim + lead, generator=g).to(DT[dt])
    q = qkv[:, lead:lead + hq * dim].unflatten(1, (hq, dim))
    qd = qkv.cuda()[:, lead:lead + hq * dim].unflatten(1, (hq, dim))
    seqs = block.Sequences(table.cuda(), starts.cuda(), length.cuda(), max_new=max(new))
    y, lse = block.attend(qd, cache, seqs, causal=causal, window=window, with_lse=True)
    assert y.dtype == DT[dt] and y.shape == q.shape and lse.shape == (T, hq)
    check(y, lse, q, k, v, table, starts, length, dim ** -0.5, causal, window, (dt, held))
    # the same with no bound on the rows, which may take the other forms, and again: no order changes it
    free = block.Sequences(table.cuda(), starts.cuda(), length.cuda())
    y2, lse2 = block.attend(qd, cache, free, causal=causal, window=window, with_lse=True)
    check(y2, lse2, q, k, v, table, starts, length, dim ** -0.5, causal, window, (dt, held, "free"))
    assert torch.equal(y, block.attend(qd, cache, seqs, causal=causal, window=window))


@pytest.mark.parametrize("held", ["bf16", "e4m3"])
@pytest.mark.parametrize("length,new,hq,heads,dim,page", [
    (9001, 1, 8, 2, 128, 16), (16384, 4, 8, 1, 64, 64), (5000, 150, 4, 1, 128, 32), (6007, 40, 8, 2, 80, 16),
    (4100, 36, 2, 2, 256, 128)])
def test_long_contexts_in_parts(length, new, hq, heads, dim, page, held):
    from paper_2504_00598_amd import block
    say("parts", length, new, hq, heads, dim, page, held)
    g = gen(length)
    table, starts, lens, pages = layout([length, 700], [new, 1], page, g)
    cache, k, v = held_cache(pages, page, heads, dim, "bf16", held, g)
    q = torch.randn(new + 1, hq, dim, generator=g).bfloat16()
    seqs = block.Sequences(table.cuda(), starts.cuda(), lens.cuda(), max_new=new)
    rows = {0, new // 2, new - 1, new}
    for window in (0, 3001):
        y, lse = block.attend(q.cuda(), cache, seqs, scale=0.2, window=window, with_lse=True)
        check(y, lse, q, k, v, table, starts, lens, 0.2, True, window, (length, window), rows)


def test_scores_that_keep_growing():
    """The running maximum moves in every tile, by a little and by much; weights that vanish beside later ones."""
    from paper_2504_00598_amd import block
    g = gen(3)
    for step in (0.01, 0.3, 8.0, -0.3, -8.0):
        table, starts, lens, pages = layout([600, 600], [1, 64], 16, g)
        cache, k, v = held_cache(pages, 16, 1, 64, "bf16", "bf16", g)
        for b in range(2):
            for p in range(600):
                k[table[b, p // 16], 0, p % 16] = 0.05 * torch.randn(64, generator=g).double()
                k[table[b, p // 16], 0, p % 16, 0] = step * (p // 8)
        k = k.bfloat16()
        cache.k.copy_(k)
        q = 0.1 * torch.randn(65, 2, 64, generator=g)
        q[..., 0] = 1.0
        q = q.bfloat16()
        seqs = block.Sequences(table.cuda(), starts.cuda(), lens.cuda())
        y, lse = block.attend(q.cuda(), cache, seqs, scale=1.0, with_lse=True)
        check(y, lse, q, k.double(), v, table, starts, lens, 1.0, True, 0, step)


@pytest.mark.parametrize("dt,held", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3")])
@pytest.mark.parametrize("new", [1, 4, 70])
@pytest.mark.parametrize("window", [0, 20])
def test_what_is_masked_has_no_effect(new, window, dt, held):
    """NaN and infinities behind a row's token, before its window and behind the sequence's end; one that a row sees
    reaches it as arithmetic has it."""
    from paper_2504_00598_amd import block
    g = gen(11)
    page, heads, dim, hq, L = 32, 2, 64, 4, 150
    table, starts, lens, pages = layout([L], [new], page, g, width=5)
    cache, k, v = held_cache(pages, page, heads, dim, dt, held, g)
    q = torch.randn(new, hq, dim, generator=g).to(DT[dt])
    seqs = block.Sequences(table.cuda(), starts.cuda(), lens.cuda(), max_new=new)

    def put(to, scales, p, d, x):
        """x into entry d of token p's value (or key) of all heads."""
        pg, at = int(table[0, p // page]), p % page
        if to is cache.k:
            to[pg, :, at, d] = torch.tensor(x).to(to.dtype)
        else:
            to[pg, :, d, at] = torch.tensor(x).to(to.dtype)

    clean = block.attend(q.cuda(), cache, seqs, window=window, with_lse=True)
    check(*clean, q, k, v, table, starts, lens, dim ** -0.5, True, window, "clean")
    bad = [math.nan] if held == "e4m3" else [math.nan, math.inf, -math.inf]
    # behind the end, in the last page
    for i, p in enumerate(range(L, 160)):
        for d in range(dim):
            put(cache.k, None, p, d, bad[i % len(bad)])
            put(cache.v, None, p, d, bad[(i + d) % len(bad)])
    again = block.attend(q.cuda(), cache, seqs, window=window, with_lse=True)
    assert torch.equal(clean[0], again[0]) and torch.equal(clean[1], again[1])
    # token P is seen by the rows from P on, up to the window's end
    for P, x in [(L - 3, bad[0]), (L - 60, bad[-1]), (L - 2, bad[len(bad) // 2])]:
        old_k, old_v = cache.k.clone(), cache.v.clone()
        put(cache.v, None, P, 5, x)
        y, lse = block.attend(q.cuda(), cache, seqs, window=window, with_lse=True)
        assert torch.equal(lse, clean[1])
        tok = torch.arange(new) + L - new
        sees = (tok >= P) & ((tok - window < P) if window else (tok >= 0))
        for i in range(new):
            if sees[i]:
                want = math.nan if math.isnan(x) else x
                assert bool(y[i, :, 5].isnan().all()) if math.isnan(want) else bool((y[i, :, 5] == want).all()), (P, x, i)
            else:
                assert torch.equal(y[i], clean[0][i]), (P, x, i)
            keep = [d for d in range(dim) if d != 5]
            assert torch.equal(y[i][:, keep], clean[0][i][:, keep]), (P, x, i)
        put(cache.v, None, P, 5, 0.0)
        cache.v.copy_(old_v)
        put(cache.k, None, P, 5, math.nan)
        y, lse = block.attend(q.cuda(), cache, seqs, window=window, with_lse=True)
        for i in range(new):
            if sees[i]:
                assert bool(y[i].isnan().all()) and bool(lse[i].isnan().all()), (P, i)
            else:
                assert torch.equal(y[i], clean[0][i]) and torch.equal(lse[i], clean[1][i]), (P, i)
        cache.k.copy_(old_k)


def test_pages_outside_the_cache_and_sequences_that_do_not_fit():
    from paper_2504_00598_amd import block
    g = gen(12)
    page, heads, dim, hq = 16, 1, 64, 2
    for new in (1, 3, 40):
        cache, k, v = held_cache(8, page, heads, dim, "bf16", "bf16", g)
        table = torch.tensor([[0, 1, 2, 3, -5], [4, 99, 5, 6, 7], [0, 1, 2, 3, 2 ** 31 - 1], [0, 1, 2, 3, 4], [7, 1, 2, 3, 4]],
                             dtype=torch.int32)
        lens = torch.tensor([60, 60, 70, 81, 50], dtype=torch.int32)  # 81: longer than its table
        starts = (torch.arange(6) * new).int() + 2
        T = 5 * new + 5
        q = torch.randn(T, hq, dim, generator=g).bfloat16()
        seqs = block.Sequences(table.cuda(), starts.cuda(), lens.cuda(), max_new=new)
        out = torch.full((T, hq, dim), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((T, hq), 7.0, device="cuda")
        y, lse = block.attend(q.cuda(), cache, seqs, with_lse=True, out=out)
        assert y is out[0] and lse is out[1]
        assert bool((y[:2] == 7).all()) and bool((lse[:2] == 7).all()) and bool((y[5 * new + 2:] == 7).all())
        assert bool((lse[5 * new + 2:] == 7).all())
        part = lambda b: slice(2 + b * new, 2 + (b + 1) * new)  # noqa: E731
        check(y[part(0)], lse[part(0)], q[part(0)], k, v, table[:1].clamp_min(0), torch.tensor([0, new]), lens[:1],
              dim ** -0.5, True, 0, "pages that are not reached")
        sees = torch.arange(60 - new, 60) >= 16  # the second page
        for t in (y[part(1)], lse[part(1)].unsqueeze(2)):
            assert torch.equal(t.isnan().all(2).all(1).cpu(), sees) and torch.equal(t.isnan().any(2).any(1).cpu(), sees)
        sees = torch.arange(70 - new, 70) >= 64
        for t in (y[part(2)], lse[part(2)].unsqueeze(2)):
            assert torch.equal(t.isnan().all(2).all(1).cpu(), sees) and torch.equal(t.isnan().any(2).any(1).cpu(), sees)
        assert bool(y[part(3)].isnan().all()) and bool(lse[part(3)].isnan().all())
        check(y[part(4)], lse[part(4)], q[part(4)], k, v, table[4:], torch.tensor([0, new]), lens[4:], dim ** -0.5, True, 0, "last")
        # more rows than announced
        if new > 1:
            few = block.Sequences(table.cuda(), starts.cuda(), lens.cuda(), max_new=new - 1)
            assert bool(block.attend(q.cuda(), cache, few)[2:5 * new + 2].isnan().all())


def test_rows_that_see_nothing():
    """More rows than tokens, lengths of zero and below, and no rows at all."""
    from paper_2504_00598_amd import block
    g = gen(13)
    cache, k, v = held_cache(8, 16, 1, 64, "bf16", "bf16", g)
    table = torch.arange(8, dtype=torch.int32).view(4, 2)
    for new, lens in (([5, 2, 0, 3], [3, 0, 20, -7]), ([50, 40, 0, 0], [9, 0, 0, 0])):
        starts, lens = torch.tensor([0] + new).cumsum(0).int(), torch.tensor(lens, dtype=torch.int32)
        T = int(starts[-1])
        q = torch.randn(T, 2, 64, generator=g).bfloat16()
        seqs = block.Sequences(table.cuda(), starts.cuda(), lens.cuda())
        for causal in (True, False):
            y, lse = block.attend(q.cuda(), cache, seqs, causal=causal, with_lse=True)
            check(y, lse, q, k, v, table, starts, lens.clamp_min(0), 0.125, causal, 0, (new, causal))
    none = block.Sequences(table[:0].cuda(), torch.zeros(1, dtype=torch.int32).cuda(), lens[:0].cuda())
    assert block.attend(q[:0].cuda(), cache, seqs).shape == (0, 2, 64)
    assert block.attend(q.cuda(), cache, none, out=torch.full_like(q.cuda(), 3.0)).eq(3).all()


def test_starts_that_leave_the_rows_are_no_sequences():
    from paper_2504_00598_amd import block
    g = gen(14)
    cache, _, _ = held_cache(4, 16, 1, 64, "bf16", "bf16", g)
    q = torch.randn(80, 2, 64, generator=g).bfloat16().cuda()
    table = torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2)
    for starts in ([0, 81, 90], [-4, -1, 0], [80, 40, 2], [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1]):
        seqs = block.Sequences(table, torch.tensor(starts, dtype=torch.int32, device="cuda"),
                               torch.tensor([30, 30], dtype=torch.int32, device="cuda"))
        out = torch.full_like(q, 7.0), torch.full((80, 2), 7.0, device="cuda")
        block.attend(q, cache, seqs, out=out, with_lse=True)
        assert all(bool((o == 7).all()) for o in out), starts


def test_a_batch_of_tokens_and_chunks_in_many_sequences():
    from paper_2504_00598_amd import block
    g = gen(15)
    new = [1 if i % 7 else 45 for i in range(150)]
    lengths = [n + int(torch.randint(0, 60, (1,), generator=g)) for n in new]
    table, starts, lens, pages = layout(lengths, new, 16, g)
    cache, k, v = held_cache(pages, 16, 1, 32, "f16", "f16", g)
    q = torch.randn(int(starts[-1]), 2, 32, generator=g).half()
    seqs = block.Sequences(table.cuda(), starts.cuda(), lens.cuda())
    y, lse = block.attend(q.cuda(), cache, seqs, with_lse=True)
    rows = set(range(0, q.shape[0], 3)) | {int(s) - 1 for s in starts[1:]}
    check(y, lse, q, k, v, table, starts, lens, 32 ** -0.5, True, 0, "many", rows)


def test_more_sequences_than_lanes_in_parts():
    """Lengths from nothing to thousands, so that sequences have one part or many and some workgroups none."""
    from paper_2504_00598_amd import block
    g = gen(21)
    lengths = [0 if b % 11 == 3 else int(1.07 ** b) % 2500 + 1 for b in range(140)]
    new = [min(1 + b % 2, n) for b, n in enumerate(lengths)]
    table, starts, lens, pages = layout(lengths, new, 16, g)
    cache, k, v = held_cache(pages, 16, 1, 32, "bf16", "bf16", g)
    q = torch.randn(int(starts[-1]), 4, 32, generator=g).bfloat16()
    for most in (2, None):
        seqs = block.Sequences(table.cuda(), starts.cuda(), lens.cuda(), max_new=most)
        y, lse = block.attend(q.cuda(), cache, seqs, with_lse=True)
        check(y, lse, q, k, v, table, starts, lens, 32 ** -0.5, True, 0, most)


@pytest.mark.parametrize("dim,held", [(64, "bf16"), (96, "e4m3"), (192, "bf16")])
@pytest.mark.parametrize("lengths,new,hq,heads,causal,window", [
    ([2300, 900, 40, 1700], [70, 1, 1, 1], 8, 2, True, 0),  # a chunk among tokens
    ([2477, 1301, 333], [133, 90, 300], 8, 1, True, 0),  # chunks of unlike lengths
    ([2000, 30, 1999], [129, 20, 40], 4, 1, True, 700),  # windows over several parts
    ([1500, 1500], [40, 41], 8, 2, False, 100),
    ([700 + b % 3 * 350 if b % 9 == 4 else b for b in range(150)], [34 if b % 9 == 4 else min(b, 1) for b in range(150)], 2, 1, True, 0),
])
def test_chunks_that_are_cut_into_parts(lengths, new, hq, heads, causal, window, dim, held):
    from paper_2504_00598_amd import block
    g = gen(23)
    table, starts, lens, pages = layout(lengths, new, 16, g)
    cache, k, v = held_cache(pages, 16, heads, dim, "bf16", held, g)
    q = torch.randn(int(starts[-1]), hq, dim, generator=g).bfloat16()
    seqs = block.Sequences(table.cuda(), starts.cuda(), lens.cuda())
    y, lse = block.attend(q.cuda(), cache, seqs, causal=causal, window=window, with_lse=True)
    rows = set(range(0, q.shape[0], 13)) | {int(s) - 1 for s in starts[1:] if s > 0} | {int(s) for s in starts[:-1] if s < q.shape[0]}
    check(y, lse, q, k, v, table, starts, lens, dim ** -0.5, causal, window, "cut", rows)
    again = block.attend(q.cuda(), cache, seqs, causal=causal, window=window, with_lse=True)
    assert torch.equal(y, again[0]) and torch.equal(lse, again[1])


def test_pages_that_lie_apart_and_beyond_32_bits():
    from paper_2504_00598_amd import block
    heads, dim, page, layers = 2, 128, 64, 4
    pages = (1 << 32) // (layers * heads * dim * page) + 40
    whole = [torch.empty((pages, layers) + s, dtype=torch.bfloat16, device="cuda") for s in
             ((heads, page, dim), (heads, dim, page))]
    cache = block.KVCache(*(t[:, 3] for t in whole))
    g = gen(16)
    table = torch.tensor([[pages - 1, 1, pages - 2]], dtype=torch.int32)
    for new in (1, 100):
        small, k, v = held_cache(3, page, heads, dim, "bf16", "bf16", g)
        for i in range(3):
            cache.k[int(table[0, i])] = small.k[i]
            cache.v[int(table[0, i])] = small.v[i]
        starts, lens = torch.tensor([0, new], dtype=torch.int32), torch.tensor([170], dtype=torch.int32)
        q = torch.randn(new, 4, dim, generator=g).bfloat16()
        y, lse = block.attend(q.cuda(), cache, block.Sequences(table.cuda(), starts.cuda(), lens.cuda()), with_lse=True)
        check(y, lse, q, k, v, torch.tensor([[0, 1, 2]]), starts, lens, dim ** -0.5, True, 0, new, {0, new // 2, new - 1})


def test_results_over_parts_of_a_context_join():
    """As the parts of one sequence on two devices would: by their logarithms."""
    from paper_2504_00598_amd import block
    g = gen(17)
    table, starts, lens, pages = layout([320], [1], 16, g)
    cache, k, v = held_cache(pages, 16, 2, 64, "bf16", "bf16", g)
    q = torch.randn(1, 4, 64, generator=g).bfloat16()
    got = []
    for cut, n in ((slice(0, 10), 160), (slice(10, 20), 160)):
        seqs = block.Sequences(table[:, cut].cuda(), starts.cuda(), torch.tensor([n], dtype=torch.int32).cuda())
        got.append(block.attend(q.cuda(), cache, seqs, causal=False, with_lse=True))
    lse = torch.logsumexp(torch.stack([x[1].double() for x in got]), 0)
    y = sum(x[0].double() * (x[1].double() - lse).exp()[..., None] for x in got)
    whole, one = block.attend(q.cuda(), cache, block.Sequences(table.cuda(), starts.cuda(), lens.cuda()), with_lse=True)
    # three results, each within two roundings to bfloat16 of weighted means of |v| <= 6
    assert float((y - whole.double()).abs().max()) <= 4 * 2.0 ** -8 * 6 and float((lse - one).abs().max()) < 1e-4


def test_captured_calls_follow_the_sequences():
    """Replays with other lengths, other rows and eager work between them; two captured calls have workspaces of their own."""
    from paper_2504_00598_amd import block
    g = gen(18)
    page, heads, dim, hq = 16, 2, 64, 8
    cache, k, v = held_cache(600, page, heads, dim, "bf16", "bf16", g)
    table = torch.randperm(600, generator=g).int().view(3, 200)
    starts, lens = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    seqs = block.Sequences(table.cuda(), starts, lens)
    q = torch.zeros(60, hq, dim, dtype=torch.bfloat16, device="cuda")
    graphs, outs = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(block.attend(q, cache, seqs, with_lse=True))
        graphs.append(graph)
    for n, ln in (([1, 1, 1], [3000, 5, 700]), ([50, 0, 9], [3200, 20, 10]), ([2, 3, 1], [2, 3, 3200]), ([20, 20, 20], [900, 20, 64])):
        s, ln = torch.tensor([0] + n).cumsum(0).int(), torch.tensor(ln, dtype=torch.int32)
        x = torch.randn(60, hq, dim, generator=g).bfloat16()
        for to, t in ((starts, s), (lens, ln), (q, x)):
            to.copy_(t)
        T = int(s[-1])
        for graph in graphs:
            graph.replay()
        eager = block.attend(q, cache, seqs, with_lse=True)
        torch.cuda.synchronize()
        for y, lse in outs:
            assert torch.equal(y[:T], eager[0][:T]) and torch.equal(lse[:T], eager[1][:T])
        check(*eager, x, k, v, table, s, ln, dim ** -0.5, True, 0, n, {0, T - 1})


def test_named_streams():
    from paper_2504_00598_amd import block
    g = gen(19)
    table, starts, lens, pages = layout([3000, 40], [1, 1], 16, g)
    cache, k, v = held_cache(pages, 16, 1, 64, "bf16", "bf16", g)
    q = torch.randn(2, 4, 64, generator=g).bfloat16().cuda()
    seqs = block.Sequences(table.cuda(), starts.cuda(), lens.cuda(), max_new=1)
    want = block.attend(q, cache, seqs)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    y = block.attend(q, cache, seqs, stream=side)
    del q
    other = [torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda") for _ in range(8)]
    side.synchronize()
    assert torch.equal(y, want) and not any(bool(o.any()) for o in other)


@pytest.mark.parametrize("held", ["bf16", "e4m3"])
def test_a_block_token_by_token_is_the_block_at_once(held):
    """Norm and rotation, the cache's write and attention as they are used: a prompt in one chunk, in uneven chunks,
    and token by token leave one cache, and results that differ by what their sums' orders and roundings do."""
    from paper_2504_00598_amd import block
    g = gen(20)
    T, hq, heads, dim, page = 150, 8, 2, 64, 16
    x = torch.randn(T, (hq + 2 * heads) * dim, generator=g).bfloat16().cuda()
    wq, wk = (1 + 0.1 * torch.randn(dim, generator=g)).bfloat16().cuda(), (1 + 0.1 * torch.randn(dim, generator=g)).bfloat16().cuda()
    a = torch.arange(T, dtype=torch.float64)[:, None] * 10000.0 ** (-2.0 * torch.arange(dim // 2) / dim)
    cos, sin = a.cos().float().cuda(), a.sin().float().cuda()
    table = torch.randperm(12, generator=g).int()[None, :10].cuda()

    def run(cuts):
        cache = block.KVCache.empty(12, page, heads, dim, DT[held])
        for t in cache._tensors():
            if t is not None:
                t.view(torch.uint8).zero_()
        ys = []
        for lo, hi in zip(cuts[:-1], cuts[1:]):
            part = x[lo:hi].unflatten(1, (-1, dim))
            pos = torch.arange(lo, hi, dtype=torch.int32, device="cuda")
            q, k = block.qk_norm_rope(part[:, :hq], part[:, hq:hq + heads], wq, wk, cos, sin, pos)
            seqs = block.Sequences(table, torch.tensor([0, hi - lo], dtype=torch.int32, device="cuda"),
                                   torch.tensor([hi], dtype=torch.int32, device="cuda"), max_new=hi - lo)
            block.cache_write(cache, k, part[:, hq + heads:], seqs)
            ys.append(block.attend(q, cache, seqs))
        return torch.cat(ys), cache

    whole, cache = run([0, T])
    for cuts in ([0, 1, 40, 41, 127, T], list(range(T + 1))):
        y, other = run(cuts)
        for p, r in zip(cache._tensors(), other._tensors()):
            assert p is None or torch.equal(p.view(torch.uint8), r.view(torch.uint8))
        # each within u (|o| + A) of the exact value, A <= max |v| of about 4.5
        v = x.unflatten(1, (-1, dim))[:, hq + heads:].float().abs().max()
        assert float((y.float() - whole.float()).abs().max()) <= 4 * 2.0 ** -8 * float(v)


@pytest.mark.parametrize("new", [1, 40])
def test_rows_that_are_no_numbers_stay_alone(new):
    from paper_2504_00598_amd import block
    g = gen(22)
    table, starts, lens, pages = layout([200], [new], 16, g)
    cache, k, v = held_cache(pages, 16, 1, 64, "bf16", "bf16", g)
    q = torch.randn(new, 4, 64, generator=g).bfloat16()
    seqs = block.Sequences(table.cuda(), starts.cuda(), lens.cuda(), max_new=new)
    clean = block.attend(q.cuda(), cache, seqs, with_lse=True)
    q[0, 1, 7], q[new - 1, 3, 60] = math.nan, math.inf
    y, lse = block.attend(q.cuda(), cache, seqs, with_lse=True)
    bad = torch.zeros(new, 4, dtype=torch.bool)
    bad[0, 1] = bad[new - 1, 3] = True
    assert torch.equal(y.isnan().all(2).cpu(), bad) and torch.equal(y.isnan().any(2).cpu(), bad)
    for a, b in ((y, clean[0]), (lse, clean[1])):
        assert torch.equal(a[~bad.cuda()], b[~bad.cuda()])


def test_values_of_any_magnitude():
    """Scales from 2^-120 to 2^60 beside each other: what a token adds is as large as its value."""
    from paper_2504_00598_amd import block
    g = gen(23)
    for dt, held, low, high in (("bf16", "bf16", -120, 60), ("bf16", "e4m3", -110, 60), ("f16", "f16", -10, 12), ("f16", "e4m3", -8, 7)):
        table, starts, lens, pages = layout([90, 150], [1, 60], 16, g)
        cache, k, _ = held_cache(pages, 16, 1, 64, dt, held, g)
        v = (torch.randn(pages, 1, 16, 64, generator=g) * 2.0 ** torch.randint(low, high, (pages, 1, 16, 1), generator=g)).to(DT[dt])
        rows = torch.tensor([0, 90, 240], dtype=torch.int32)
        every = block.Sequences(table.cuda(), rows.cuda(), lens.cuda())
        at = [(int(table[b, p // 16]), p % 16) for b in range(2) for p in range(int(lens[b]))]
        kk, _ = block.cache_read(cache, every, 240, dtype=DT[dt])
        vv = torch.stack([v[pg, :, i] for pg, i in at])
        block.cache_write(cache, kk, vv.cuda(), every)
        _, vv = block.cache_read(cache, every, 240, dtype=DT[dt])
        v = v.double()
        k = k.clone()
        kk = kk.cpu().double()
        for (pg, i), x, y in zip(at, vv.cpu().double(), kk):
            v[pg, :, i], k[pg, :, i] = x, y
        q = torch.randn(61, 2, 64, generator=g).to(DT[dt])
        seqs = block.Sequences(table.cuda(), starts.cuda(), lens.cuda())
        y, lse = block.attend(q.cuda(), cache, seqs, with_lse=True)
        check(y, lse, q, k, v, table, starts, lens, 0.125, True, 0, (dt, held))


def test_refused_where_a_gradient_is_recorded():
    from paper_2504_00598_amd import block
    cache = block.KVCache.empty(2, 16, 1, 64, torch.bfloat16)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    seqs = block.Sequences(i32(0, 1)[None], i32(0, 3), i32(20))
    x = torch.zeros(3, 1, 64, dtype=torch.bfloat16, device="cuda", requires_grad=True)
    with pytest.raises(RuntimeError):
        block.attend(x, cache, seqs)
    with pytest.raises(RuntimeError):
        block.cache_write(cache, x, x, seqs)
    with torch.no_grad():
        block.cache_write(cache, x, x, seqs)
        assert block.attend(x, cache, seqs).shape == x.shape


def test_refusals_of_the_binding():
    from paper_2504_00598_amd import block
    from paper_2504_00598_amd._lib import CfpError
    bf, f16 = torch.bfloat16, torch.float16
    cache = block.KVCache.empty(4, 16, 2, 32, bf)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    seqs = block.Sequences(i32(0, 1)[None], i32(0, 3), i32(20))
    q = torch.zeros(3, 4, 32, dtype=bf, device="cuda")
    k = torch.zeros(3, 2, 32, dtype=bf, device="cuda")
    for bad in (dict(q=q.cpu()), dict(q=q.half()), dict(q=q.float()), dict(q=q[:, :3]), dict(q=q[..., :16]), dict(q=q[0]),
                dict(q=q[..., ::2].repeat(1, 1, 2)[..., ::1].transpose(1, 2)), dict(cache=cache.k), dict(seqs=(1, 2)),
                dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan), dict(window=-1),
                dict(out=q[:2]), dict(out=q.half()), dict(ws=torch.zeros(8, device="cuda"))):
        a = {"q": q, "cache": cache, "seqs": seqs, **bad}
        with pytest.raises((TypeError, ValueError, CfpError)):
            block.attend(a.pop("q"), a.pop("cache"), a.pop("seqs"), **a)
    for bad in ((k.half(), k), (k, k.half()), (k[:2], k), (q, q), (k.cpu(), k.cpu()), (k.float(), k.float())):
        with pytest.raises((TypeError, ValueError)):
            block.cache_write(cache, *bad, seqs)
    for how in (dict(dtype=f16), dict(dtype=torch.float32), dict(out=(k, k.half())), dict(out=(k, k[:2])), dict(out=(k,))):
        with pytest.raises((TypeError, ValueError)):
            block.cache_read(cache, seqs, 3, **how)
    with pytest.raises(ValueError):
        block.cache_read(cache, seqs, -1)
    kv = torch.zeros(4, 2, 16, 32, dtype=bf, device="cuda"), torch.zeros(4, 2, 32, 16, dtype=bf, device="cuda")
    sc = torch.zeros(4, 2, 16, dtype=torch.uint8, device="cuda")
    e = [t.to(torch.float8_e4m3fn) for t in kv]
    for bad in ((kv[0], kv[0]), (kv[0], kv[1].half()), (kv[0].float(), kv[1].float()), (*kv, sc, sc), (*e,), (*e, sc, sc[:3]),
                (kv[0].cpu(), kv[1].cpu()), (kv[0].transpose(1, 2), kv[1]), (*e, sc, sc.int()), (*e, sc, None)):
        with pytest.raises((TypeError, ValueError)):
            block.KVCache(*bad)
    for bad in ((i32(0, 1), i32(0, 3), i32(20)), (i32(0, 1)[None], i32(0), i32(20)), (i32(0, 1)[None], i32(0, 3), i32(20, 3)),
                (i32(0, 1)[None].long(), i32(0, 3), i32(20)), (i32(0, 1)[None], i32(0, 9, 3)[::2], i32(20))):
        with pytest.raises((TypeError, ValueError)):
            block.Sequences(*bad)
    with pytest.raises(ValueError):
        block.Sequences(i32(0, 1)[None], i32(0, 3), i32(20), max_new=-1)
    for odd in (block.KVCache.empty(4, 8, 2, 32, bf), block.KVCache.empty(4, 48, 2, 32, bf), block.KVCache.empty(4, 16, 2, 40, bf),
                block.KVCache.empty(4, 16, 2, 272, bf)):
        x = torch.zeros(3, 2, odd.k.shape[3], dtype=bf, device="cuda")
        with pytest.raises(CfpError):
            block.attend(x, odd, seqs)
        with pytest.raises(CfpError):
            block.cache_write(odd, x, x, seqs)
