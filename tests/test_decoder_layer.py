"""The decoder layer's blocks under each strategy: their shares put together are the whole block's results, and
the plan found from the times is the cheapest.

Bounds.  A head's and a token's values do not depend on what else a call holds, so shares of heads and tokens give
the same bits.  The experts' products may run in other tiles, in another order of 32-bit sums: whole and share
are each within 1.5 u of the exact value in the 2-norm (u = 2^-8, one operand and one result rounded to
bfloat16, see test_gpu_block.py), so whole and the sum of the shares differ by at most 1.5 u times the sum of all
their norms.  Sums of gains' and weights' gradients are in 32 bits; a gain's over 40 tokens of 4 heads and a
weight's over 64 entries, both with terms of magnitude at most the norms' product, are given 2^-14.
"""
import itertools

import pytest

from tests.gpu_util import need_gpu
from workloads import decoder_layer as D

SMALL = D.Layer(tokens=40, heads=4, key_heads=2, dim=32, experts=6, k=3, hidden=96, inner=64)


def cheapest(cost, edges, layers):
    rows = cost * layers
    best = [(c, (s,)) for s, c in enumerate(rows[0]) if c < 2 ** 31 - 1]
    for i, row in enumerate(rows[1:], 1):
        best = [min((b + edges[i % 3][plan[-1]][s] + c, plan + (s,)) for b, plan in best)
                for s, c in enumerate(row) if c < 2 ** 31 - 1]
    return min(best)[0]


def some_times(seed):
    return {(b, s): (i * 7919 + seed * 104729) % 50021 + 100 for i, (b, s) in
            enumerate(itertools.product(D.BLOCKS, D.STRATEGIES)) if D.available(SMALL, b, s, 2)}


def test_strategies_that_apply():
    layer = D.Layer(heads=8, key_heads=2, experts=6, inner=100)
    got = {(b, s) for b in D.BLOCKS for s in D.STRATEGIES if D.available(layer, b, s, 4)}
    assert got == {("qk", "tokens"), ("qk", "whole"), ("route", "tokens"), ("route", "whole"), ("experts", "tokens"),
                   ("experts", "width"), ("experts", "whole")}


@pytest.mark.parametrize("n,parts", [(10, 3), (1, 4), (8, 8), (7, 1)])
def test_shares_cover_everything_once(n, parts):
    seen = [i for p in range(parts) for i in range(n)[D._share(n, parts, p)]]
    assert seen == list(range(n))


def test_tables():
    times = some_times(1)
    cost, edges = D.tables(SMALL, 2, 1e9, times)
    assert [len(r) for r in cost] == [4, 4, 4] and cost[1][1] == cost[1][2] == 2 ** 31 - 1
    # 6 experts of 3 x 64 x 96 parameters of 2 bytes, half of them out and half in: that many ns at 1 GB/s
    assert cost[2][0] - times["experts", "tokens"] == 6 * 3 * 64 * 96 * 2
    assert cost[2][3] == times["experts", "whole"]
    assert all(e[s][s] == 0 for e in (edges[0], edges[1], edges[2]) for s in (0, 3))
    assert edges[1][0][2] == 2 * 40 * 96 * 2 // 2  # from tokens to experts: the other half, forward and back
    assert edges[1][1][0] * 2 == edges[1][0][2]    # from heads to tokens: half of that


@pytest.mark.gpu
@pytest.mark.parametrize("seed,layers,link", [(1, 1, 1e9), (2, 3, 1e8), (3, 7, 1e10)])
def test_plan_is_cheapest(seed, layers, link):
    need_gpu()
    times = some_times(seed)
    total, plan = D.plan_layers(SMALL, layers, 2, link, times)
    cost, edges = D.tables(SMALL, 2, link, times)
    assert total == cheapest(cost, edges, layers) and len(plan) == 3 * layers
    ids = [D.STRATEGIES.index(s) for s in plan]
    assert total == sum((cost * layers)[i][s] for i, s in enumerate(ids)) + sum(
        edges[i % 3][ids[i - 1]][ids[i]] for i in range(1, len(ids)))


@pytest.mark.gpu
def test_shares_are_the_whole():
    need_gpu()
    import torch

    u, data = 2.0 ** -8, D.Data(SMALL)

    def parts(name, strategy):
        return [D.shard(data, name, strategy, 2, p)() for p in range(2)]

    def close(whole, shares, joined, bound, what):
        off = (whole.double() - joined).norm()
        assert float(off) <= bound * (float(whole.double().norm()) + sum(float(s.double().norm()) for s in shares)), what

    whole = D.shard(data, "qk", "whole", 2)()
    for strategy, axis in (("tokens", 0), ("width", 1)):
        got = parts("qk", strategy)
        for i in range(4):
            assert torch.equal(whole[i], torch.cat([g[i] for g in got], axis)), (strategy, i)
        for i in (4, 5):
            close(whole[i], [g[i] for g in got], sum(g[i].double() for g in got), 2.0 ** -14, (strategy, i))

    whole = D.shard(data, "route", "whole", 2)()
    got = parts("route", "tokens")
    for i in (0, 1, 3):
        assert torch.equal(whole[i], torch.cat([g[i] for g in got])), i

    whole = D.shard(data, "experts", "whole", 2)()  # y, dx, dw1, dw2, dweight
    E, F, H = SMALL.experts, SMALL.inner, SMALL.hidden
    for strategy in ("tokens", "experts", "width"):
        got = parts("experts", strategy)
        for i in range(5):
            shares = [g[i] for g in got]
            if strategy == "tokens":
                joined = torch.cat(shares).double() if i in (0, 1, 4) else sum(s.double() for s in shares)
            elif i in (0, 1, 4):
                joined = sum(s.double() for s in shares)
            elif strategy == "experts":
                joined = torch.cat(shares).double()
            elif i == 2:
                joined = torch.cat([s.view(E, 2, F // 2, H) for s in shares], 2).view(E, 2 * F, H).double()
            else:
                joined = torch.cat(shares, 2).double()
            close(whole[i], shares, joined, 1.5 * u, (strategy, i))


@pytest.mark.gpu
def test_measure_and_plan():
    need_gpu()
    times = D.measure(D.Data(SMALL), 2, reps=3)
    assert set(times) == set(some_times(1)) and all(0 < t < 10 ** 9 for t in times.values())
    total, plan = D.plan_layers(SMALL, 2, 2, 64e9, times)
    assert 0 < total and all(s in D.APPLIES[b] for s, b in zip(plan, D.BLOCKS * 2))
