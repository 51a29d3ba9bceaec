"""Measured cases of the decoder-block operators: the norm and rotation of queries and
keys, the routing of tokens to experts with the order of their assignments, and the
experts' products, each with its gradient.

run() computes a case in its plain form, elementary torch operations in 32 bits, where
`own` is false, and calls the framework where it is true; exact() computes it in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda"
DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-6
P_TABLE = 32768  # rows of the rotation tables


def listed():
    return [
        # Queries and keys of four sequences that each take one token: a launch and its latency.
        {"name": "qk decode", "op": "qk", "T": 4, "hq": 32, "hk": 8, "d": 128, "r": 128, "pairs": "halves",
         "dtype": "bf16", "train": False},
        # A prompt of odd length, heads of 80 with half of each rotated, neighbouring pairs, half precision.
        {"name": "qk prompt odd", "op": "qk", "T": 1537, "hq": 20, "hk": 5, "d": 80, "r": 40, "pairs": "neighbours",
         "dtype": "f16", "train": False},
        # A training step over 16 sequences of 1024, hidden size 5120 in heads of 128, grouped keys.
        {"name": "qk train", "op": "qk", "T": 16384, "hq": 40, "hk": 8, "d": 128, "r": 128, "pairs": "halves",
         "dtype": "bf16", "train": True},
        # Routing of eight decoded tokens.
        {"name": "route decode", "op": "route", "T": 8, "E": 64, "k": 6, "score": "softmax", "bias": False, "groups": 1,
         "top_groups": 1, "group_score": "max", "renorm": True, "scale": 1.0, "masked": 0.0, "dtype": "bf16",
         "train": False},
        # A prompt's routing with the balance bias and groups: 8 of 256 experts, out of 4 of 8 groups.
        {"name": "route groups", "op": "route", "T": 16384, "E": 256, "k": 8, "score": "sigmoid", "bias": True,
         "groups": 8, "top_groups": 4, "group_score": "top2", "renorm": True, "scale": 2.5, "masked": 0.0,
         "dtype": "f32", "train": False},
        # A training step's routing: an odd number of tokens and of experts, some masked, some tokens all masked.
        {"name": "route train", "op": "route", "T": 32771, "E": 60, "k": 4, "score": "softmax", "bias": False,
         "groups": 1, "top_groups": 1, "group_score": "max", "renorm": False, "scale": 1.0, "masked": 0.1,
         "dtype": "bf16", "train": True},
        # One decoded token: the weights of the six experts it meets are read once.
        {"name": "experts token", "op": "experts", "T": 1, "E": 64, "first": 0, "all": 64, "k": 6, "H": 2048, "F": 1024,
         "skew": 0.0, "dtype": "bf16", "train": False},
        # A serving batch: every expert is met by a few tokens.
        {"name": "experts batch", "op": "experts", "T": 64, "E": 64, "first": 0, "all": 64, "k": 6, "H": 2048, "F": 1024,
         "skew": 0.5, "dtype": "bf16", "train": False},
        # One rank's window of the experts, uneven loads, ragged sizes, half precision.
        {"name": "experts window odd", "op": "experts", "T": 777, "E": 7, "first": 3, "all": 12, "k": 3, "H": 1000,
         "F": 364, "skew": 1.5, "dtype": "f16", "train": True},
        # An ordinary training step.
        {"name": "experts train", "op": "experts", "T": 4096, "E": 16, "first": 0, "all": 16, "k": 2, "H": 2048,
         "F": 1536, "skew": 0.3, "dtype": "bf16", "train": True},
        # A long prompt over many narrow experts.
        {"name": "experts prompt", "op": "experts", "T": 16384, "E": 64, "first": 0, "all": 64, "k": 8, "H": 2048,
         "F": 768, "skew": 0.5, "dtype": "bf16", "train": False},
        # A training step over 16 sequences of 1024.
        {"name": "experts train large", "op": "experts", "T": 16384, "E": 32, "first": 0, "all": 32, "k": 4, "H": 4096,
         "F": 1536, "skew": 0.3, "dtype": "bf16", "train": True},
    ]


def _spread(rng, low, high, step=1):
    """A multiple of `step` in [low, high], spread over the logarithm."""
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high))) / step)) * step
    return min(max(v, low), high)


def draw(rng):
    op = rng.choice(["qk", "route", "experts", "experts"])
    if op == "qk":
        hk = rng.choice([1, 2, 5, 8, 16])
        d = rng.choice([64, 80, 96, 112, 128, 192, 256])
        return {"op": op, "T": _spread(rng, 1, 16384), "hq": hk * rng.choice([1, 2, 4, 5]) if hk < 16 else hk, "hk": hk,
                "d": d, "r": rng.choice([d, d, d // 2, 2 * (d // 8)]), "pairs": rng.choice(["halves", "neighbours"]),
                "dtype": rng.choice(["bf16", "bf16", "f16", "f32"]) if d <= 128 else "bf16",
                "train": rng.random() < 0.5}
    if op == "route":
        groups = rng.choice([1, 1, 4, 8])
        bias = rng.random() < 0.5
        each = _spread(rng, 8, 256 if groups == 1 else 48)
        E = groups * each
        top_groups = max(1, groups // 2)
        renorm = rng.random() < 0.5  # of one weight alone is a constant, with no gradient to compare
        return {"op": op, "T": _spread(rng, 1, 32768), "E": E, "k": rng.randint(2 if renorm else 1, min(12, each)),
                "score": rng.choice(["softmax", "sigmoid"]), "bias": bias, "groups": groups, "top_groups": top_groups,
                "group_score": rng.choice(["max", "top2"]) if bias and groups > 1 else "max",
                "renorm": renorm, "scale": rng.choice([1.0, 2.5]), "masked": rng.choice([0.0, 0.0, 0.1]),
                "dtype": "f32" if bias else rng.choice(["f32", "bf16", "f16"]), "train": rng.random() < 0.5}
    E = _spread(rng, 4, 96)
    every = E if rng.random() < 0.6 else E + rng.randint(1, 2 * E)
    step = rng.choice([64, 64, 8, 8, 1])
    H, F = _spread(rng, 256, 4096, step), _spread(rng, 128, 2048, step)
    H = H - step if H == 3072 else H
    c = {"op": op, "T": _spread(rng, 1, 16384), "E": E, "first": rng.randint(0, every - E), "all": every,
         "k": rng.randint(1, min(8, E)), "H": H, "F": F, "skew": rng.choice([0.0, 0.5, 1.0]),
         "dtype": rng.choice(["bf16", "bf16", "f16"]), "train": rng.random() < 0.5}
    while c["E"] > 4 and c["E"] * H * F > 2.0e8:
        c["E"] //= 2
        c["all"] = max(c["E"], c["all"] // 2)
        c["first"] = min(c["first"] // 2, c["all"] - c["E"])
        c["k"] = min(c["k"], c["E"])
    while c["T"] * c["k"] * H * F > 4.0e11:
        c["T"] //= 2
    return c


# ---------------------------------------------------------------- inputs --

def _rotation(rows, r):
    """cos and sin [rows][r/2] of position p times 10000^(-2i/r)."""
    i = torch.arange(r // 2, device=DEVICE, dtype=torch.float64)
    a = torch.arange(rows, device=DEVICE, dtype=torch.float64)[:, None] * torch.pow(10000.0, -2.0 * i / max(r, 1))
    return a.cos().float(), a.sin().float()


def _prepare_qk(c, g):
    T, hq, hk, d, dt = c["T"], c["hq"], c["hk"], c["d"], DTYPE[c["dtype"]]
    rand = lambda *s: torch.randn(*s, generator=g, device=DEVICE)  # noqa: E731
    # one product makes queries, keys and values: the operator reads its first two parts
    qkv = (rand(T, (hq + 2 * hk) * d) * (0.5 + rand(T, 1).abs())).to(dt)
    s = {"q": qkv[:, :hq * d].view(T, hq, d), "k": qkv[:, hq * d:(hq + hk) * d].view(T, hk, d)}
    s["wq"], s["wk"] = (1 + 0.2 * rand(d)).to(dt), (1 + 0.2 * rand(d)).to(dt)
    s["cos"], s["sin"] = _rotation(P_TABLE, c["r"])
    s["pos"] = torch.randint(0, P_TABLE, (T,), generator=g, device=DEVICE, dtype=torch.int32) if T < 64 else (
        torch.arange(T, device=DEVICE, dtype=torch.int32) % 1024)
    if c["train"]:
        s["dq"], s["dk"] = rand(T, hq, d).to(dt), rand(T, hk, d).to(dt)
    return s


def _select_value(c, logits, bias):
    """(score, selection value) of every expert, in the type of `logits`; -inf: masked."""
    if c["score"] == "softmax":
        top = logits.amax(1, keepdim=True)
        e = torch.exp(logits - torch.where(top == -math.inf, torch.zeros_like(top), top))
        total = e.sum(1, keepdim=True)
        s = torch.where(total > 0, e / torch.where(total > 0, total, torch.ones_like(total)), torch.zeros_like(e))
    else:
        s = 1 / (1 + torch.exp(-logits))
    v = logits if bias is None else torch.where(logits == -math.inf, logits, s + bias)
    return s, v


def _prepare_route(c, g):
    T, E, k, dt = c["T"], c["E"], c["k"], DTYPE[c["dtype"]]
    bias = 0.1 * torch.randn(E, generator=g, device=DEVICE) if c["bias"] else None

    def logits():
        x = (1.5 * torch.randn(T, E, generator=g, device=DEVICE)).to(dt)
        if c["masked"] > 0:
            out = torch.rand(T, E, generator=g, device=DEVICE) < c["masked"]
            out |= torch.rand(T, 1, generator=g, device=DEVICE) < 0.01  # nothing left for this token
            x = x.masked_fill(out, -math.inf)
        return x

    x = logits()
    if c["bias"] or c["group_score"] == "top2":
        # Candidates nearer to each other than 32-bit sums can tell have no defined order: such rows are drawn again.
        for _ in range(6):
            _, v = _select_value(c, x.double(), None if bias is None else bias.double())
            gv = v.view(T, c["groups"], -1)
            two = gv.topk(2, dim=2)[0] if c["group_score"] == "top2" else gv.amax(2, keepdim=True)
            rank = two.sum(2).sort(dim=1, descending=True)
            near = torch.zeros(T, dtype=torch.bool, device=DEVICE)
            if c["top_groups"] < c["groups"]:
                edge = rank[0][:, c["top_groups"] - 1] - rank[0][:, c["top_groups"]]
                near |= edge.abs() < 4e-6
            kept = torch.zeros(T, c["groups"], dtype=torch.bool, device=DEVICE).scatter_(
                1, rank[1][:, :c["top_groups"]], True)
            v = torch.where(kept[:, :, None], gv, torch.full_like(gv, -math.inf)).view(T, E)
            top = v.sort(dim=1, descending=True)[0][:, :k + 1]
            near |= ((top[:, :-1] - top[:, 1:]).abs() < 4e-6).any(1)
            x = torch.where(near[:, None], logits(), x)
    s = {"logits": x, "bias": bias}
    if c["train"]:
        s["dw"] = torch.randn(T, k, generator=g, device=DEVICE)
    return s


def _prepare_experts(c, g):
    T, E, k, H, F, dt = c["T"], c["E"], c["k"], c["H"], c["F"], DTYPE[c["dtype"]]
    rand = lambda *s: torch.randn(*s, generator=g, device=DEVICE)  # noqa: E731
    load = c["skew"] * rand(c["all"])  # uneven popularity
    noise = -torch.log(-torch.log(torch.rand(T, c["all"], generator=g, device=DEVICE).clamp(1e-9, 1 - 1e-7)))
    chosen = (load + noise).topk(k, dim=1)[1].to(torch.int32)
    s = {"x": rand(T, H).to(dt), "index": chosen.contiguous(), "weight": torch.softmax(rand(T, k), 1)}
    s["w1"] = torch.randn(E, 2 * F, H, generator=g, device=DEVICE, dtype=dt) * (1 / math.sqrt(H))
    s["w2"] = torch.randn(E, H, F, generator=g, device=DEVICE, dtype=dt) * (1 / math.sqrt(F))
    if c["train"]:
        s["dy"] = rand(T, H).to(dt)
    return s


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    s = {"qk": _prepare_qk, "route": _prepare_route, "experts": _prepare_experts}[case["op"]](case, g)
    s["case"] = case
    return s


# ------------------------------------------------------------ plain forms --

def _rotate(z, cos, sin, r, pairs):
    if pairs == "halves":
        a, b, rest = z[..., :r // 2], z[..., r // 2:r], z[..., r:]
        return torch.cat((a * cos - b * sin, b * cos + a * sin, rest), -1)
    a, b, rest = z[..., 0:r:2], z[..., 1:r:2], z[..., r:]
    return torch.cat((torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2), rest), -1)


def _plain_norm(x, w, cos, sin, c):
    x = x.float()
    n = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return _rotate(n * w.float(), cos, sin, c["r"], c["pairs"])


def _plain_norm_bwd(dy, x, w, cos, sin, c):
    x = x.float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    n = x * r
    dz = _rotate(dy.float(), cos, -sin, c["r"], c["pairs"])  # the rotation by the opposite angle
    dn = dz * w.float()
    return r * (dn - n * (dn * n).mean(-1, keepdim=True)), (dz * n).sum((0, 1))


def _plain_qk(s):
    c = s["case"]
    dt = s["q"].dtype
    cos, sin = s["cos"][s["pos"].long()][:, None, :], s["sin"][s["pos"].long()][:, None, :]
    out = [_plain_norm(s["q"], s["wq"], cos, sin, c).to(dt), _plain_norm(s["k"], s["wk"], cos, sin, c).to(dt)]
    if c["train"]:
        dq, dwq = _plain_norm_bwd(s["dq"], s["q"], s["wq"], cos, sin, c)
        dk, dwk = _plain_norm_bwd(s["dk"], s["k"], s["wk"], cos, sin, c)
        out += [dq.to(dt), dk.to(dt), dwq, dwk]
    return out


def _order(index, first, n):
    """offsets [n+1] and the assignments in order of their expert (stable), -1 behind the last one kept."""
    e = index.reshape(-1).long() - first
    e = torch.where((e >= 0) & (e < n), e, torch.full_like(e, n))
    at = torch.sort(e, stable=True)[1]
    count = torch.zeros(n + 1, dtype=torch.int64, device=e.device).scatter_add_(0, e, torch.ones_like(e))
    offsets = torch.cat((torch.zeros(1, dtype=torch.int64, device=e.device), count[:n].cumsum(0)))
    rows = torch.where(torch.arange(e.numel(), device=e.device) < offsets[-1], at, torch.full_like(at, -1))
    return offsets.int(), rows.int()


def _plain_select(c, v, two):
    """The k experts of each row by selection value `v`, ties to the lowest index; -1 where none is left."""
    T, E = v.shape
    if c["top_groups"] < c["groups"]:
        by = two.view(T, c["groups"], -1)
        by = by.sort(dim=2, descending=True)[0][:, :, :2].sum(2) if c["group_score"] == "top2" else by.amax(2)
        kept = torch.sort(by, dim=1, descending=True, stable=True)[1][:, :c["top_groups"]]
        keep = torch.zeros(T, c["groups"], dtype=torch.bool, device=v.device).scatter_(1, kept, True)
        v = torch.where(keep.repeat_interleave(E // c["groups"], dim=1), v, torch.full_like(v, -math.inf))
    top, at = torch.sort(v, dim=1, descending=True, stable=True)
    return torch.where(top[:, :c["k"]] == -math.inf, torch.full_like(at[:, :c["k"]], -1), at[:, :c["k"]])


def _weights(c, s, index):
    w = torch.where(index < 0, torch.zeros((), dtype=s.dtype, device=s.device), s.gather(1, index.clamp_min(0)))
    if c["renorm"]:
        total = w.sum(1, keepdim=True)
        w = torch.where(total > 0, w / torch.where(total > 0, total, torch.ones_like(total)), torch.zeros_like(w))
    return w * c["scale"]


def _weights_bwd(c, s, index, dw):
    there = index >= 0
    at = index.clamp_min(0)
    chosen = torch.where(there, s.gather(1, at), torch.zeros((), dtype=s.dtype, device=s.device))
    dw = torch.where(there, dw * c["scale"], torch.zeros_like(dw))
    if c["renorm"]:
        total = chosen.sum(1, keepdim=True)
        safe = torch.where(total > 0, total, torch.ones_like(total))
        dw = torch.where(there & (total > 0), (dw - (dw * chosen).sum(1, keepdim=True) / safe) / safe, torch.zeros_like(dw))
    ds = torch.zeros_like(s).scatter_add_(1, at, dw)
    if c["score"] == "softmax":
        return s * (ds - (dw * chosen).sum(1, keepdim=True))
    return ds * s * (1 - s)


def _plain_route(s):
    c = s["case"]
    score, v = _select_value(c, s["logits"].float(), s["bias"])
    index = _plain_select(c, v, v)
    offsets, rows = _order(index, 0, c["E"])
    out = [_weights(c, score, index), index.int(), offsets, rows]
    if c["train"]:
        out.append(_weights_bwd(c, score, index, s["dw"]).to(s["logits"].dtype))
    return out


def _plain_experts(s):
    """The assignments padded to one batch of products over the experts that some token meets."""
    c, dt = s["case"], s["x"].dtype
    T, E, k, H, F = c["T"], c["E"], c["k"], c["H"], c["F"]
    e = s["index"].reshape(-1).long() - c["first"]
    kept = torch.nonzero((e >= 0) & (e < E)).flatten()
    weight = s["weight"].reshape(-1)
    grads = {"dx": torch.zeros(T * k, H, device=DEVICE), "dw1": torch.zeros_like(s["w1"]), "dw2": torch.zeros_like(s["w2"]),
             "dweight": torch.zeros_like(weight)} if c["train"] else {}
    y = torch.zeros(T * k, H, device=DEVICE)  # a row for each assignment, summed over a token's at the end
    if kept.numel():
        met, which = torch.unique(e[kept], return_inverse=True)
        at = torch.sort(which, stable=True)[1]
        count = torch.bincount(which, minlength=met.numel())
        start = count.cumsum(0) - count
        cap = int(count.max())
        group = which[at]
        place = group * cap + torch.arange(at.numel(), device=DEVICE) - start[group]  # in [met][cap]
        a = kept[at]
        token = a // k

        def lay(rows):
            return torch.zeros(met.numel() * cap, rows.shape[1], device=DEVICE).index_copy_(0, place, rows).view(
                met.numel(), cap, -1)

        w1, w2 = s["w1"][met].float(), s["w2"][met].float()
        x = lay(s["x"].float()[token])
        h = torch.matmul(x, w1.transpose(1, 2))
        gate, up = h[..., :F], h[..., F:]
        sig = 1 / (1 + torch.exp(-gate))
        act = gate * sig * up
        o = torch.matmul(act, w2.transpose(1, 2)).view(-1, H)[place]
        y.index_copy_(0, a, o * weight[a, None])
        if c["train"]:
            del o
            dy = lay(s["dy"].float()[token])
            p = torch.matmul(dy, w2)
            grads["dweight"].index_copy_(0, a, (p * act).sum(2).view(-1)[place])
            wt = lay(weight[a, None])
            grads["dw2"].index_copy_(0, met, torch.matmul(dy.transpose(1, 2), act * wt).to(dt))
            del dy, act
            p = p * wt
            dh = torch.cat((p * up * sig * (1 + gate * (1 - sig)), p * gate * sig), 2)
            grads["dw1"].index_copy_(0, met, torch.matmul(dh.transpose(1, 2), x).to(dt))
            grads["dx"].index_copy_(0, a, torch.matmul(dh, w1).view(-1, H)[place])
    out = [y.view(T, k, H).sum(1).to(dt)]
    if c["train"]:
        out += [grads["dx"].view(T, k, H).sum(1).to(dt), grads["dw1"], grads["dw2"], grads["dweight"].view(T, k)]
    return out


# ------------------------------------------------------- the framework's --

def _own_qk(s):
    from paper_2504_00598_amd import block

    c = s["case"]
    how = {"eps": EPS, "interleaved": c["pairs"] == "neighbours"}
    args = (s["q"], s["k"], s["wq"], s["wk"], s["cos"], s["sin"], s["pos"])
    out = list(block.qk_norm_rope(*args, **how))
    if c["train"]:
        out += block.qk_norm_rope_bwd(s["dq"], s["dk"], *args, **how)
    return out


def _own_route(s):
    from paper_2504_00598_amd import block

    c = s["case"]
    how = {"score": c["score"], "renormalise": c["renorm"], "scale": c["scale"]}
    weight, index = block.route(s["logits"], c["k"], bias=s["bias"], groups=c["groups"], top_groups=c["top_groups"],
                                group_score=c["group_score"], **how)
    plan = block.expert_plan(index, c["E"])
    out = [weight, index, plan.offsets, plan.rows]
    if c["train"]:
        out.append(block.route_bwd(s["dw"], s["logits"], index, **how))
    return out


def _own_experts(s):
    from paper_2504_00598_amd import block

    c = s["case"]
    plan = block.expert_plan(s["index"], c["E"], first=c["first"])
    if not c["train"]:
        return [block.experts(s["x"], s["w1"], s["w2"], s["weight"], plan)]
    y, h = block.experts(s["x"], s["w1"], s["w2"], s["weight"], plan, keep=True)
    return [y, *block.experts_bwd(s["dy"], s["x"], s["w1"], s["w2"], s["weight"], plan, h)]


def run(state):
    if own:
        return {"qk": _own_qk, "route": _own_route, "experts": _own_experts}[state["case"]["op"]](state)
    return {"qk": _plain_qk, "route": _plain_route, "experts": _plain_experts}[state["case"]["op"]](state)


# ------------------------------------------------------------------ work --

def work(case):
    """Inputs read once, outputs written once, and the products' operations.  An expert that no
    token is expected to meet is not read; a gradient is written for every expert."""
    c, size = case, SIZE[case["dtype"]]
    T = c["T"]
    if c["op"] == "qk":
        rows = T * (c["hq"] + c["hk"]) * c["d"]
        return {"bytes": rows * size * (2 + (3 if c["train"] else 0)) + T * (c["r"] * 4 + 4),
                "flops": rows * (8 + (16 if c["train"] else 0))}
    if c["op"] == "route":
        n = T * c["E"]
        kept = T * c["k"]
        return {"bytes": n * size * (3 if c["train"] else 1) + kept * (12 + (8 if c["train"] else 0)),
                "flops": n * (6 + (4 if c["train"] else 0))}
    kept = T * c["k"] * c["E"] / c["all"]
    met = c["E"] * (1 - (1 - c["k"] / c["all"]) ** T)
    weights = 3 * c["H"] * c["F"] * size
    b = met * weights + 2 * T * c["H"] * size + 8 * T * c["k"]
    if c["train"]:
        b += met * weights + c["E"] * weights + 3 * T * c["H"] * size + 8 * T * c["k"]
    return {"bytes": b, "flops": kept * c["H"] * c["F"] * (18 if c["train"] else 6)}


# ----------------------------------------------------------- in 64 bits --

def _exact_qk(c, s):
    T, r = c["T"], c["r"]
    cos, sin = s["cos"].double()[s["pos"].long()], s["sin"].double()[s["pos"].long()]
    half = r // 2
    first, second = (torch.arange(half), torch.arange(half) + half) if c["pairs"] == "halves" else (
        2 * torch.arange(half), 2 * torch.arange(half) + 1)

    def one(x, w, dy):
        x, w = x.double(), w.double()
        r1 = 1 / torch.sqrt(x.pow(2).sum(2) / c["d"] + EPS)
        n = x * r1[:, :, None]
        z = n * w
        y = z.clone()
        y[:, :, first] = z[:, :, first] * cos[:, None] - z[:, :, second] * sin[:, None]
        y[:, :, second] = z[:, :, second] * cos[:, None] + z[:, :, first] * sin[:, None]
        if dy is None:
            return y, None, None
        dy = dy.double()
        dz = dy.clone()
        dz[:, :, first] = dy[:, :, first] * cos[:, None] + dy[:, :, second] * sin[:, None]
        dz[:, :, second] = dy[:, :, second] * cos[:, None] - dy[:, :, first] * sin[:, None]
        dw = (dz * n).reshape(-1, c["d"]).sum(0)
        dn = dz * w
        dx = dn * r1[:, :, None] - x * ((dn * x).sum(2) * r1.pow(3) / c["d"])[:, :, None]
        return y, dx, dw

    yq, dq, dwq = one(s["q"], s["wq"], s.get("dq"))
    yk, dk, dwk = one(s["k"], s["wk"], s.get("dk"))
    return [yq, yk, dq, dk, dwq, dwk] if c["train"] else [yq, yk]


def _exact_route(c, s):
    x = s["logits"].double()
    T, E = x.shape
    masked = torch.isinf(x) & (x < 0)
    empty = masked.all(1, keepdim=True)
    if c["score"] == "softmax":
        p = torch.softmax(x.masked_fill(empty, 0.0), 1).masked_fill(masked, 0.0)
    else:
        p = torch.sigmoid(x)
    v = (x if s["bias"] is None else p + s["bias"].double()).masked_fill(masked, -math.inf)
    if c["top_groups"] < c["groups"]:
        gv = v.reshape(T, c["groups"], E // c["groups"])
        by = gv.topk(2, dim=2)[0].sum(2) if c["group_score"] == "top2" else gv.max(2)[0]
        out = torch.ones(T, c["groups"], dtype=torch.bool, device=x.device)
        out.scatter_(1, by.sort(dim=1, descending=True, stable=True)[1][:, :c["top_groups"]], False)
        v = gv.masked_fill(out[:, :, None], -math.inf).reshape(T, E)
    top, index = v.sort(dim=1, descending=True, stable=True)
    top, index = top[:, :c["k"]], index[:, :c["k"]]
    gone = torch.isinf(top) & (top < 0)
    w = p.gather(1, index).masked_fill(gone, 0.0)
    total = w.sum(1, keepdim=True) if c["renorm"] else torch.ones(T, 1, dtype=x.dtype, device=x.device)
    total = total.masked_fill(total == 0, 1.0)
    out = [w / total * c["scale"], None, None, None]
    if c["train"]:
        up = s["dw"].double().masked_fill(gone, 0.0) * c["scale"]
        if c["renorm"]:
            up = up / total - (up * w).sum(1, keepdim=True) / total ** 2
            up = up.masked_fill(gone | (w.sum(1, keepdim=True) == 0), 0.0)
        full = torch.zeros_like(p).scatter_add(1, index, up)
        dl = p * full - p * (p * full).sum(1, keepdim=True) if c["score"] == "softmax" else full * p * (1 - p)
        out.append(dl)
    return out


def _exact_experts(c, s):
    T, k, H, F = c["T"], c["k"], c["H"], c["F"]
    x, weight = s["x"].double(), s["weight"].double()
    y = torch.zeros(T, H, dtype=torch.float64, device=DEVICE)
    dx, dweight = torch.zeros_like(y), torch.zeros_like(weight)
    dw1 = torch.zeros(s["w1"].shape, dtype=torch.float64, device=DEVICE) if c["train"] else None
    dw2 = torch.zeros(s["w2"].shape, dtype=torch.float64, device=DEVICE) if c["train"] else None
    for e in range(c["E"]):
        t, j = torch.nonzero(s["index"] == e + c["first"], as_tuple=True)
        if t.numel() == 0:
            continue
        w1, w2, xe, we = s["w1"][e].double(), s["w2"][e].double(), x[t], weight[t, j][:, None]
        gate, up = xe @ w1[:F].T, xe @ w1[F:].T
        sig = torch.sigmoid(gate)
        act = gate * sig * up
        y.index_add_(0, t, (act @ w2.T) * we)
        if c["train"]:
            dye = s["dy"].double()[t]
            dact = dye @ w2
            dweight[t, j] = (dact * act).sum(1)
            dw2[e] = (dye * we).T @ act
            dact = dact * we
            dgate = dact * up * (sig + gate * sig * (1 - sig))
            dup = dact * gate * sig
            dw1[e, :F], dw1[e, F:] = dgate.T @ xe, dup.T @ xe
            dx.index_add_(0, t, dgate @ w1[:F] + dup @ w1[F:])
    return [y, dx, dw1, dw2, dweight] if c["train"] else [y]


def exact(case, seed):
    s = prepare(case, seed)
    return {"qk": _exact_qk, "route": _exact_route, "experts": _exact_experts}[case["op"]](case, s)
