"""Plain 64-bit forms of the decoder-block operators, written token by token from their
definitions (torch on the CPU), for the tests of the kernels."""
import math

import torch


def qk_rows(x, w, cos, sin, pos, eps, interleaved):
    """x [T][heads][D] and everything else in float64."""
    T, h, D = x.shape
    half = cos.shape[1]
    a = torch.arange(half) * 2 if interleaved else torch.arange(half)
    b = a + 1 if interleaved else a + half
    z = x / torch.sqrt((x * x).mean(2, keepdim=True) + eps) * (w if w is not None else 1.0)
    y = z.clone()
    c, s = cos[pos][:, None], sin[pos][:, None]
    y[:, :, a] = z[:, :, a] * c - z[:, :, b] * s
    y[:, :, b] = z[:, :, b] * c + z[:, :, a] * s
    return y


def scores(l, score):
    """Scores of rows of logits; a row of -inf alone has zeros."""
    if score == "sigmoid":
        return torch.sigmoid(l)
    none = (l == -math.inf).all(1, keepdim=True)
    return torch.softmax(l.masked_fill(none, 0.0), 1).masked_fill(none, 0.0)


def route(l, k, score, bias, groups, top_groups, group_score, renorm, scale):
    T, E = l.shape
    p = scores(l, score)
    w, idx = torch.zeros(T, k, dtype=torch.float64), torch.full((T, k), -1, dtype=torch.int64)
    per = E // groups
    for t in range(T):
        v = [float(x) for x in (l[t] if bias is None else p[t] + bias)]
        left = [e for e in range(E) if float(l[t, e]) != -math.inf]
        if top_groups < groups:
            best = []
            for g in range(groups):
                use = v if bias is not None or group_score == "max" else [float(x) for x in p[t]]
                own = sorted((use[e] for e in left if e // per == g), reverse=True)
                if group_score == "top2":
                    val = own[0] + own[1] if len(own) > 1 else -math.inf
                else:
                    val = own[0] if own else -math.inf
                best.append((-val, g))
            keep = {g for _, g in sorted(best)[:top_groups]}
            left = [e for e in left if e // per in keep]
        left.sort(key=lambda e: (-v[e], e))
        for j, e in enumerate(left[:k]):
            idx[t, j], w[t, j] = e, p[t, e]
        if renorm:
            s = float(w[t].sum())
            w[t] = w[t] / s if s else 0.0
    return w * scale, idx


def route_weights(l, idx, score, renorm, scale):
    """The weights as a function of the logits for a given choice (for gradients)."""
    p = scores(l, score)
    there = idx >= 0
    w = torch.where(there, p.gather(1, idx.clamp_min(0)), torch.zeros((), dtype=p.dtype))
    if renorm:
        s = w.sum(1, keepdim=True)
        w = torch.where(s > 0, w / torch.where(s > 0, s, torch.ones_like(s)), torch.zeros_like(w))
    return w * scale


def plan(idx, E, first):
    T, k = idx.shape
    by = [[] for _ in range(E)]
    for a, e in enumerate(idx.reshape(-1).tolist()):
        if first <= e < first + E:
            by[e - first].append(a)
    rows = [a for b in by for a in b]
    offsets = [0]
    for b in by:
        offsets.append(offsets[-1] + len(b))
    slot = [-1] * (T * k)
    for p, a in enumerate(rows):
        slot[a] = p
    return offsets, rows + [-1] * (T * k - len(rows)), slot


def experts(x, w1, w2, weight, idx, first):
    """y as a differentiable function (float64)."""
    T, H = x.shape
    E, F = w2.shape[0], w2.shape[2]
    y = torch.zeros(T, H, dtype=torch.float64)
    for e in range(E):
        t, j = torch.nonzero(idx == e + first, as_tuple=True)
        if t.numel():
            g, u = x[t] @ w1[e, :F].T, x[t] @ w1[e, F:].T
            y = y.index_add(0, t, (torch.sigmoid(g) * g * u) @ w2[e].T * weight[t, j][:, None])
    return y
