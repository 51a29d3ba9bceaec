"""A mixture-of-experts decoder layer's blocks, timed shard by shard on this card, and the plan found for them.

    python -m workloads.decoder_layer --parts 8 --layers 24

The chain has three blocks a layer: norm and rotation of queries and keys ("qk"), routing with the order of
assignments ("route"), and the experts ("experts").  A strategy says what one of `parts` equal devices holds:

    tokens    its share of the tokens, all heads, experts and their whole width
    width     all tokens; its share of the heads (qk) or of every expert's inner width (experts)
    experts   all tokens; its share of the experts, the assignments to the others dropped (experts)
    whole     everything

One device's share of a block, forward and backward, runs through paper_2504_00598_amd.block and is timed here;
that is p_n of Eq. T.  Its communication c_n (sums of partial outputs and input gradients, or of parameter
gradients) and the resharding R between blocks are counted in bytes and priced at `link` bytes per second, a
stated rate: one card cannot measure them.  All are in nanoseconds, as the int32 tables of the search.
"""
from __future__ import annotations

import argparse
import statistics
from dataclasses import dataclass

STRATEGIES = ("tokens", "width", "experts", "whole")
BLOCKS = ("qk", "route", "experts")
APPLIES = {"qk": ("tokens", "width", "whole"), "route": ("tokens", "whole"), "experts": STRATEGIES}


@dataclass(frozen=True)
class Layer:
    tokens: int = 4096
    heads: int = 32
    key_heads: int = 8
    dim: int = 128
    experts: int = 64
    k: int = 6
    hidden: int = 2048
    inner: int = 1024
    dtype: str = "bfloat16"


def _share(n: int, parts: int, part: int) -> slice:
    per = -(-n // parts)
    return slice(min(part * per, n), min((part + 1) * per, n))


def available(layer: Layer, block: str, strategy: str, parts: int) -> bool:
    """Whether the block can run so: heads and experts go to devices whole and in equal shares."""
    if strategy not in APPLIES[block]:
        return False
    if block == "qk" and strategy == "width":
        return layer.heads % parts == 0 and layer.key_heads % parts == 0
    if strategy == "experts":
        return layer.experts % parts == 0
    return strategy != "width" or layer.inner >= parts


class Data:
    """Synthetic inputs, parameters and output gradients of a whole layer on the GPU."""

    def __init__(self, layer: Layer, seed: int = 0):
        import torch

        from paper_2504_00598_amd import block

        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        dt = getattr(torch, layer.dtype)

        def normal(*shape, scale=1.0, dtype=dt):
            return torch.empty(shape, device="cuda", dtype=dtype).normal_(0.0, scale, generator=g)

        c = self.layer = layer
        T, half = c.tokens, c.dim // 2
        qk = normal(T, c.heads + c.key_heads, c.dim)  # as one projection leaves them
        self.q, self.k = qk[:, :c.heads], qk[:, c.heads:]
        self.dq, self.dk = normal(T, c.heads, c.dim), normal(T, c.key_heads, c.dim)
        self.wq, self.wk = normal(c.dim, scale=0.1) + 1, normal(c.dim, scale=0.1) + 1
        angle = torch.arange(T, device="cuda")[:, None] * 10000.0 ** (-torch.arange(half, device="cuda") / half)
        self.cos, self.sin = angle.cos(), angle.sin()
        self.x, self.dy = normal(T, c.hidden), normal(T, c.hidden)
        self.logits = self.x.float() @ normal(c.hidden, c.experts, scale=c.hidden ** -0.5, dtype=torch.float32)
        self.dweight = normal(T, c.k, dtype=torch.float32)
        self.w1 = normal(c.experts, 2 * c.inner, c.hidden, scale=c.hidden ** -0.5)
        self.w2 = normal(c.experts, c.hidden, c.inner, scale=c.inner ** -0.5)
        self.weight, self.index = block.route(self.logits, c.k, renormalise=True)


def shard(data: Data, name: str, strategy: str, parts: int, part: int = 0):
    """A function that runs device `part`'s share of a block, forward and backward, and returns its results.
    The shares of the parameters are laid out here, once, as a device would hold them."""
    from paper_2504_00598_amd import block

    c = data.layer
    t = _share(c.tokens, parts if strategy == "tokens" else 1, 0 if strategy != "tokens" else part)
    if name == "qk":
        n, m = (parts, part) if strategy == "width" else (1, 0)
        h, hk = _share(c.heads, n, m), _share(c.key_heads, n, m)
        args = (data.q[t, h], data.k[t, hk], data.wq, data.wk, data.cos[t], data.sin[t])
        dq, dk = data.dq[t, h], data.dk[t, hk]

        def qk():
            return block.qk_norm_rope(*args) + block.qk_norm_rope_bwd(dq, dk, *args)

        return qk
    if name == "route":
        logits, dweight = data.logits[t], data.dweight[t]

        def route():
            weight, index = block.route(logits, c.k, renormalise=True)
            plan = block.expert_plan(index, c.experts)
            return weight, index, plan, block.route_bwd(dweight, logits, index, renormalise=True)

        return route
    x, dy, weight = data.x[t], data.dy[t], data.weight[t]
    w1, w2, first = data.w1, data.w2, 0
    if strategy == "experts":
        e = _share(c.experts, parts, part)
        w1, w2, first = w1[e].contiguous(), w2[e].contiguous(), e.start
    elif strategy == "width":
        f = _share(c.inner, parts, part)
        w1 = w1.view(c.experts, 2, c.inner, c.hidden)[:, :, f].flatten(1, 2).contiguous()
        w2 = w2[:, :, f].contiguous()
    plan = block.expert_plan(data.index[t], w1.shape[0], first=first)

    def experts():
        y, kept = block.experts(x, w1, w2, weight, plan, keep=True)
        return (y,) + block.experts_bwd(dy, x, w1, w2, weight, plan, kept)

    return experts


def time_ns(run, reps: int = 7, calls: int = 5) -> int:
    """Time of one call on the card: the median of `reps` runs of `calls` in a row."""
    import torch

    run()
    times = []
    for _ in range(reps):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        for _ in range(calls):
            run()
        b.record()
        b.synchronize()
        times.append(a.elapsed_time(b) / calls * 1e6)
    return round(statistics.median(times))


def comm_bytes(layer: Layer, name: str, strategy: str, parts: int) -> int:
    """Bytes that a device sends for a block in one step: rings of reduce-scatter and all-gather."""
    c, ring = layer, 2 * (parts - 1) / parts
    if parts == 1 or strategy == "whole" or name == "route":
        return 0
    if name == "qk":  # the gains' gradients, from every device's tokens or heads
        return round(ring * 2 * c.dim * 4)
    if strategy == "tokens":  # the parameters' gradients
        return round(ring * c.experts * 3 * c.inner * c.hidden * 2)
    return round(ring * 2 * c.tokens * c.hidden * 2)  # y forward, dx backward


def reshard_bytes(layer: Layer, before: str, after: str, parts: int) -> int:
    """Bytes that a device receives between two blocks, forward and backward.  What is whole is only sliced; a
    block cut by experts or by inner width takes and leaves whole activations, one cut by heads leaves heads."""
    kinds = {"tokens": "tokens", "width": "heads", "experts": "whole", "whole": "whole"}
    a, b = kinds[before], kinds[after]
    if a == b or a == "whole" or parts == 1:
        return 0
    share = 1 if b == "whole" else 1 / parts  # an all-gather, or an all-to-all
    return round(2 * share * (parts - 1) / parts * layer.tokens * layer.hidden * 2)


def tables(layer: Layer, parts: int, link: float, times: dict):
    """One layer's c[3][strategies] and R[3][strategies][strategies] (the edge into each block) in nanoseconds,
    from times[block, strategy]; a strategy without a time is unavailable."""
    from paper_2504_00598_amd import CFP_COST_INF

    ns = 1e9 / link
    cost = [[times[b, s] + round(comm_bytes(layer, b, s, parts) * ns) if (b, s) in times else CFP_COST_INF
             for s in STRATEGIES] for b in BLOCKS]

    def edge(before, after):  # only a qk block cut by width leaves heads apart, and only it takes them so
        return [[round(reshard_bytes(layer, "experts" if s == "width" and before != "qk" else s,
                                     "experts" if t == "width" and after != "qk" else t, parts) * ns)
                 for t in STRATEGIES] for s in STRATEGIES]

    return cost, [edge(BLOCKS[i - 1], BLOCKS[i]) for i in range(3)]


def measure(data: Data, parts: int, reps: int = 7) -> dict:
    return {(b, s): time_ns(shard(data, b, s, parts), reps)
            for b in BLOCKS for s in STRATEGIES if available(data.layer, b, s, parts)}


def plan_layers(layer: Layer, layers: int, parts: int, link: float, times: dict):
    """The cheapest strategies of a chain of `layers` equal layers: (nanoseconds, [strategy of each block])."""
    import torch

    from paper_2504_00598_amd import CFP_ST_OK, search, status_string

    cost, edges = tables(layer, parts, link, times)
    res = search.dp_chain(torch.tensor([cost * layers], dtype=torch.int32, device="cuda"),
                          torch.tensor(edges, dtype=torch.int32, device="cuda"), [i % 3 for i in range(3 * layers)])
    status = int(res.status[0])
    if status != CFP_ST_OK:
        raise RuntimeError(f"search: {status_string(status)}")
    return int(res.opt[0]), [STRATEGIES[s] for s in res.plan[0].tolist()]


def main(argv=None):
    p = argparse.ArgumentParser(description="time a decoder layer's blocks under each strategy, and plan them")
    for name, default in Layer.__dataclass_fields__.items():
        p.add_argument("--" + name.replace("_", "-"), type=type(default.default), default=default.default)
    p.add_argument("--parts", type=int, default=8, help="devices")
    p.add_argument("--layers", type=int, default=24)
    p.add_argument("--link", type=float, default=64e9, help="bytes per second that a device sends to another")
    a = p.parse_args(argv)
    layer = Layer(**{n: getattr(a, n) for n in Layer.__dataclass_fields__})
    times = measure(Data(layer), a.parts)
    cost, _ = tables(layer, a.parts, a.link, times)
    print(f"{'block':10s}" + "".join(f"{s:>22s}" for s in STRATEGIES) + "   us measured + communication")
    for i, b in enumerate(BLOCKS):
        cells = (f"{times[b, s] / 1e3:.1f} + {(cost[i][j] - times[b, s]) / 1e3:.1f}" if (b, s) in times else "-"
                 for j, s in enumerate(STRATEGIES))
        print(f"{b:10s}" + "".join(f"{c:>22s}" for c in cells))
    total, plan = plan_layers(layer, a.layers, a.parts, a.link, times)
    print(f"plan: {total / 1e6:.3f} ms; first layer {', '.join(plan[:3])}; last {', '.join(plan[-3:])}")


if __name__ == "__main__":
    main()
