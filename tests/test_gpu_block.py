"""The decoder-block operators on the GPU against plain 64-bit forms (tests/block_ref.py).

Bounds.  u is the unit roundoff of a type: 2^-8 for the 8 significant bits of bfloat16,
2^-11 for the 11 of float16, 2^-24 for the 24 of float32.  A result that is computed in 32 bits and rounded
once is within u of its value, relative, beside the 32-bit error: a sum of n terms
in any order is within n 2^-24 of the sum of the terms' magnitudes, so 2^-24 times
a few hundred is allowed for rows of up to 512.  The experts' products round one
operand to 16 bits on the way (at most u of each of its entries, hence at most u of the
result in the 2-norm as the entries' errors are independent) and the result once; a
rounding's root mean square is u / sqrt(3) at most, two of them 0.82 u: 1.5 u in the 2-norm,
and 20 u of the larger of the value and the root mean square for one entry.
"""
import math

import pytest
import torch

from tests import block_ref as R
from tests.gpu_util import need_gpu, say

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def near(got, want, u, what, floor=2.0 ** -16):
    """Every entry within u relative, and within `floor` of the root mean square."""
    got, want = got.detach().cpu().double(), want.detach().double()
    assert got.shape == want.shape, what
    fin = torch.isfinite(want)
    assert torch.equal(fin, torch.isfinite(got)), what
    got, want = got[fin], want[fin]
    if want.numel() == 0:
        return
    rms = want.square().mean().sqrt()
    bad = (got - want).abs() - (u * want.abs() + floor * rms + 1e-30)
    assert float(bad.max()) <= 0, (what, float((got - want).abs().max()), float(rms))


def near_product(got, want, u, what):
    got, want = got.detach().cpu().double(), want.detach().double()
    assert got.shape == want.shape, what
    norm = want.norm()
    assert float((got - want).norm()) <= 1.5 * u * float(norm) + 1e-30, (what, float((got - want).norm() / norm))
    rms = norm / math.sqrt(max(1, want.numel()))
    off = (got - want).abs() / torch.maximum(want.abs(), rms.expand_as(want)).clamp_min(1e-30)
    assert want.numel() == 0 or float(off.max()) <= 20 * u, (what, float(off.max()))


# -------------------------------------------------------- queries and keys --

def tables(P, rot):
    i = torch.arange(rot // 2, dtype=torch.float64)
    a = torch.arange(P, dtype=torch.float64)[:, None] * 10000.0 ** (-2.0 * i / max(rot, 1))
    return a.cos().float(), a.sin().float()


QK = [  # T, query heads, key heads, D, rotated, interleaved, type, gain type (None: none)
    (1, 1, 1, 2, 2, False, "bf16", "bf16"),
    (1, 32, 8, 128, 128, False, "bf16", "bf16"),
    (3, 5, 0, 128, 128, True, "f16", "f32"),
    (3, 0, 5, 96, 32, True, "bf16", None),
    (37, 20, 5, 80, 40, True, "f16", "f16"),
    (17, 4, 2, 80, 20, False, "bf16", "bf16"),
    (130, 6, 3, 64, 16, False, "f32", "f32"),
    (5, 3, 1, 33, 10, True, "f32", "f32"),
    (5, 3, 1, 33, 10, False, "bf16", "f32"),
    (9, 2, 1, 512, 512, False, "bf16", "bf16"),
    (4, 2, 2, 511, 510, True, "f16", "f16"),
    (4, 2, 2, 510, 2, False, "f16", "f16"),
    (300, 7, 1, 192, 48, True, "bf16", "bf16"),
    (6, 2, 1, 7, 0, False, "bf16", "bf16"),
    (2000, 3, 2, 256, 256, False, "bf16", "bf16"),
]


@pytest.mark.parametrize("T,hq,hk,D,rot,inter,dt,wdt", QK)
@pytest.mark.parametrize("view", ["fused", "whole"])
def test_qk_norm_rope_and_gradient(T, hq, hk, D, rot, inter, dt, wdt, view):
    from paper_2504_00598_amd import block
    say("qk", T, hq, hk, D, rot, inter, dt, wdt, view)
    g = gen(T * 7 + D)
    dtype = DT[dt]
    cos, sin = tables(64, rot)
    pos = torch.randint(0, 64, (T,), generator=g, dtype=torch.int32)
    qkv = torch.randn(T, (hq + 2 * hk) * D + 3, generator=g).to(dtype)
    lead = 3 if view == "fused" else 0  # a view that starts off 16 bytes
    q = qkv[:, lead:lead + hq * D].unflatten(1, (hq, D)) if hq else torch.empty(T, 0, D, dtype=dtype)
    k = qkv[:, lead + hq * D:lead + (hq + hk) * D].unflatten(1, (hk, D)) if hk else torch.empty(T, 0, D, dtype=dtype)
    dev = qkv.cuda()
    qd = dev[:, lead:lead + hq * D].unflatten(1, (hq, D)) if hq else q.cuda()
    kd = dev[:, lead + hq * D:lead + (hq + hk) * D].unflatten(1, (hk, D)) if hk else k.cuda()
    if view == "whole":
        qd, kd = qd.contiguous(), kd.contiguous()
    wq = wk = None
    if wdt:
        wq, wk = (1 + torch.randn(D, generator=g)).to(DT[wdt]), (1 + torch.randn(D, generator=g)).to(DT[wdt])
    dy = [torch.randn(T, h, D, generator=g).to(dtype) for h in (hq, hk)]
    cu = lambda t: None if t is None else t.cuda()  # noqa: E731
    args = (qd, kd, cu(wq), cu(wk), cos.cuda(), sin.cuda(), pos.cuda())
    yq, yk = block.qk_norm_rope(*args, eps=1e-5, interleaved=inter)
    dq, dk, dwq, dwk = block.qk_norm_rope_bwd(dy[0].cuda(), dy[1].cuda(), *args, eps=1e-5, interleaved=inter)
    torch.cuda.synchronize()
    u = U[dtype] * 1.01 + 2.0 ** -20
    for x, w, y, d, dx, dw, name in ((q, wq, yq, dy[0], dq, dwq, "q"), (k, wk, yk, dy[1], dk, dwk, "k")):
        xr = x.double().clone().requires_grad_()
        wr = None if w is None else w.double().clone().requires_grad_()
        ref = R.qk_rows(xr, wr, cos.double(), sin.double(), pos.long(), 1e-5, inter)
        near(y, ref, u, name)
        (ref * d.double()).sum().backward()
        near(dx, xr.grad, u, "d" + name)
        if w is None:
            assert dw is None
        elif x.numel():
            near(dw, wr.grad, 2.0 ** -18, "dw" + name)
        else:
            assert not dw.any()


def test_qk_positions_default_and_outside():
    from paper_2504_00598_amd import block
    cos, sin = tables(8, 4)
    q = torch.randn(6, 2, 8, generator=gen(0))
    args = (q.cuda(), q[:, :1].cuda(), None, None, cos.cuda(), sin.cuda())
    a = block.qk_norm_rope(*args)
    b = block.qk_norm_rope(*args, torch.arange(6, dtype=torch.int32).cuda())
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    y, _ = block.qk_norm_rope(*args, torch.tensor([0, -1, 2, 8, 2 ** 31 - 1, 5], dtype=torch.int32).cuda())
    bad = torch.tensor([False, True, False, True, True, False])
    assert torch.equal(y.isnan().any(2).all(1).cpu(), bad)
    assert not y[:, :, 4:].isnan().any() and torch.equal(y[0], a[0][0])


def test_qk_gradient_against_differences():
    """dq along a direction against the 64-bit form's difference quotient (its error is h^2 of the third derivative)."""
    from paper_2504_00598_amd import block
    g = gen(5)
    cos, sin = tables(16, 8)
    q, v, w = (torch.randn(4, 3, 12, generator=g), torch.randn(4, 3, 12, generator=g), torch.randn(12, generator=g))
    d, pos = torch.randn(4, 3, 12, generator=g), torch.arange(4)
    dq, _, dw, _ = block.qk_norm_rope_bwd(d.cuda(), d[:, :0].cuda(), q.cuda(), q[:, :0].cuda(), w.cuda(), None, cos.cuda(),
                                          sin.cuda())
    f = lambda x, ww: float((R.qk_rows(x, ww, cos.double(), sin.double(), pos, 1e-6, False) * d.double()).sum())  # noqa: E731
    h = 1e-4
    num = (f(q.double() + h * v.double(), w.double()) - f(q.double() - h * v.double(), w.double())) / (2 * h)
    assert abs(num - float((dq.cpu().double() * v).sum())) <= 1e-4 * (dq.cpu().double().norm() * v.double().norm())
    numw = (f(q.double(), w.double() + h) - f(q.double(), w.double() - h)) / (2 * h)
    assert abs(numw - float(dw.cpu().double().sum())) <= 1e-4 * float(dw.cpu().abs().sum())


# ----------------------------------------------------------------- routing --

ROUTE = [  # T, E, k, score, bias, groups, top_groups, group_score, renorm, type, masked share
    (1, 1, 1, "softmax", False, 1, 1, "max", False, "f32", 0.0),
    (1, 64, 6, "softmax", False, 1, 1, "max", True, "bf16", 0.0),
    (7, 60, 4, "softmax", False, 1, 1, "max", False, "bf16", 0.5),
    (65, 257, 32, "sigmoid", True, 1, 1, "max", True, "f32", 0.1),
    (33, 256, 8, "sigmoid", True, 8, 4, "top2", True, "f32", 0.0),
    (33, 96, 5, "softmax", False, 12, 3, "max", True, "f16", 0.6),
    (20, 96, 12, "softmax", False, 8, 1, "top2", False, "f32", 0.0),
    (20, 160, 6, "softmax", True, 8, 3, "max", False, "f32", 0.3),
    (9, 1024, 32, "sigmoid", False, 1, 1, "max", False, "bf16", 0.0),
    (9, 1000, 7, "softmax", True, 125, 9, "top2", True, "f32", 0.0),
    (5, 17, 17, "sigmoid", False, 1, 1, "max", True, "f32", 0.3),
    (300, 128, 2, "softmax", False, 1, 1, "max", True, "f16", 0.0),
]


@pytest.mark.parametrize("T,E,k,score,bias,groups,top,gs,renorm,dt,masked", ROUTE)
def test_route_and_gradient(T, E, k, score, bias, groups, top, gs, renorm, dt, masked):
    from paper_2504_00598_amd import block
    say("route", T, E, k, score, bias, groups, top, gs, renorm, dt, masked)
    g = gen(E + k)
    l = torch.randn(T, E + 5, generator=g)[:, :E]
    if bias or gs == "top2":  # values apart by far more than a 32-bit sum's error: a shuffled ladder
        l = torch.stack([torch.randperm(E, generator=g) for _ in range(T)]).float() * (6.0 / E) - 3.0
        l = torch.nn.functional.pad(l, (0, 5))[:, :E]
    l = l.to(DT[dt])
    out = torch.rand(T, E, generator=g) < masked
    l = l.masked_fill(out, -math.inf)
    if masked and T > 2:
        l[1] = -math.inf
        l[2, 1:] = -math.inf
    full = torch.zeros(T, E + 5, dtype=l.dtype)
    full[:, :E] = l
    ld = full.cuda()[:, :E]
    b = (torch.arange(E) % 3).float() if bias else None  # 0, 1, 2: ties only between equal scores
    w, idx = block.route(ld, k, score=score, bias=None if b is None else b.cuda(), groups=groups, top_groups=top,
                         group_score=gs, renormalise=renorm, scale=1.5)
    rw, ridx = R.route(l.double(), k, score, None if b is None else b.double(), groups, top, gs, renorm, 1.5)
    assert torch.equal(idx.cpu().long(), ridx)
    near(w, rw, 2.0 ** -18, "weight")
    assert not w[idx < 0].any()
    dw = torch.randn(T, k, generator=g)
    dl = block.route_bwd(dw.cuda(), ld, idx, score=score, renormalise=renorm, scale=1.5)
    lr = l.double().clone().requires_grad_()
    (R.route_weights(lr, ridx, score, renorm, 1.5) * dw.double()).sum().backward()
    want = torch.nan_to_num(lr.grad, nan=0.0)
    # a sum of n terms that cancel: 2^-20 of the largest gradient that goes in
    lim = U[DT[dt]] * 1.01 * want.abs() + 2.0 ** -18 * 1.5 * float(dw.abs().max())
    assert bool(((dl.cpu().double() - want).abs() <= lim).all())


def test_route_ties_infinities_and_nan():
    from paper_2504_00598_amd import block
    l = torch.zeros(4, 70)
    l[1] = torch.finfo(torch.float32).min          # the type's lowest value is an ordinary logit
    l[2, 3:] = -math.inf
    l[3, 10], l[3, 11:] = math.nan, -math.inf
    w, idx = block.route(l.cuda(), 12, score="softmax")
    idx = idx.cpu()
    assert torch.equal(idx[0], torch.arange(12, dtype=torch.int32)) and torch.equal(idx[1], idx[0])
    assert idx[2].tolist() == [0, 1, 2] + [-1] * 9 and not w[2, 3:].any()
    assert torch.allclose(w[:2], torch.full((2, 12), 1 / 70.0).cuda())
    assert idx[3].tolist() == list(range(10)) + [10, -1]  # not a number: behind every other that is not masked
    assert w[3, :11].isnan().all() and w[3, 11] == 0
    z = torch.tensor([[-0.0, 0.0, -0.0, 0.0]])
    assert block.route(z.cuda(), 4)[1].tolist() == [[0, 1, 2, 3]]


def test_route_gradient_against_differences():
    from paper_2504_00598_amd import block
    g = gen(3)
    l, v, dw = torch.randn(6, 20, generator=g), torch.randn(6, 20, generator=g), torch.randn(6, 5, generator=g)
    for score in ("softmax", "sigmoid"):
        for renorm in (False, True):
            _, idx = block.route(l.cuda(), 5, score=score, renormalise=renorm)
            dl = block.route_bwd(dw.cuda(), l.cuda(), idx, score=score, renormalise=renorm).cpu().double()
            f = lambda x: float((R.route_weights(x, idx.cpu().long(), score, renorm, 1.0) * dw.double()).sum())  # noqa: E731
            h = 1e-4
            num = (f(l.double() + h * v.double()) - f(l.double() - h * v.double())) / (2 * h)
            assert abs(num - float((dl * v).sum())) <= 1e-4 * float(dl.norm() * v.double().norm())


@pytest.mark.parametrize("T,k,E,first,every", [(1, 1, 1, 0, 1), (5, 3, 4, 2, 9), (0, 2, 7, 0, 7), (700, 6, 64, 0, 64),
                                               (2000, 8, 60, 100, 256), (4097, 1, 1024, 0, 1024), (3000, 5, 3, 0, 3)])
def test_expert_plan(T, k, E, first, every):
    from paper_2504_00598_amd import block
    say("plan", T, k, E, first, every)
    idx = torch.randint(-1, every, (T, k), generator=gen(T + E), dtype=torch.int32)
    p = block.expert_plan(idx.cuda(), E, first=first)
    offsets, rows, slot = R.plan(idx, E, first)
    assert p.offsets.tolist() == offsets and p.rows.tolist() == rows and p.slot.tolist() == slot


# ----------------------------------------------------------------- experts --

EXPERTS = [  # T, H, F, E, first, all, k, type
    (1, 64, 32, 4, 0, 4, 2, "bf16"),
    (3, 8, 8, 2, 0, 2, 2, "bf16"),
    (5, 1, 1, 3, 0, 3, 1, "f16"),
    (1, 2048, 264, 8, 0, 8, 4, "bf16"),
    (16, 520, 136, 5, 0, 5, 3, "f16"),
    (70, 100, 37, 3, 1, 6, 4, "bf16"),
    (129, 130, 66, 7, 0, 7, 1, "bf16"),
    (300, 256, 128, 4, 0, 4, 2, "bf16"),
    (300, 264, 200, 6, 3, 12, 6, "f16"),
    (1000, 192, 320, 2, 0, 2, 2, "bf16"),
    (40, 24, 16, 100, 0, 100, 3, "bf16"),
]


def expert_inputs(T, H, F, E, first, every, k, dtype, seed=0):
    g = gen(seed + T + H)
    idx = torch.rand(T, every, generator=g).topk(k, 1)[1].to(torch.int32)
    if T > 4:
        idx[3] = -1       # a token without experts
        idx[4, 1:] = -1
    x, dy = torch.randn(T, H, generator=g).to(dtype), torch.randn(T, H, generator=g).to(dtype)
    w1 = (torch.randn(E, 2 * F, H, generator=g) / math.sqrt(H)).to(dtype)
    w2 = (torch.randn(E, H, F, generator=g) / math.sqrt(F)).to(dtype)
    return idx, x, dy, w1, w2, torch.rand(T, k, generator=g) + 0.1


@pytest.mark.parametrize("T,H,F,E,first,every,k,dt", EXPERTS)
def test_experts_and_gradient(T, H, F, E, first, every, k, dt):
    from paper_2504_00598_amd import block
    say("experts", T, H, F, E, first, every, k, dt)
    dtype = DT[dt]
    idx, x, dy, w1, w2, weight = expert_inputs(T, H, F, E, first, every, k, dtype)
    plan = block.expert_plan(idx.cuda(), E, first=first)
    dev = [t.cuda() for t in (x, w1, w2, weight)]
    y = block.experts(*dev, plan)
    yk, kept = block.experts(*dev, plan, keep=True)
    torch.cuda.synchronize()
    grads = block.experts_bwd(dy.cuda(), *dev, plan, kept)
    torch.cuda.synchronize()
    ref = [t.double().clone().requires_grad_() for t in (x, w1, w2, weight)]
    want = R.experts(*ref, idx, first)
    (want * dy.double()).sum().backward()
    u = U[dtype]
    near_product(y, want, u, "y")
    near_product(yk, want, u, "y kept")
    for name, got, r in zip(("dx", "dw1", "dw2", "dweight"), grads, ref):
        near_product(got, r.grad if r.grad is not None else torch.zeros_like(r), u if name != "dweight" else 2.0 ** -16, name)
    if T > 4:
        assert not y[3].any() and not grads[0][3].any() and not grads[3][3].any()
    # experts without tokens
    none = plan.offsets[1:] == plan.offsets[:-1]
    assert not grads[1][none].any() and not grads[2][none].any()


@pytest.mark.parametrize("H,F,off", [(64, 32, 0), (64, 32, 1), (96, 40, 4)])
def test_experts_rows_apart(H, F, off):
    """x and dy as views of wider tensors, also off 16 bytes: the results of contiguous copies."""
    from paper_2504_00598_amd import block
    idx, x, dy, w1, w2, weight = expert_inputs(50, H, F, 4, 0, 4, 2, torch.bfloat16)
    plan = block.expert_plan(idx.cuda(), 4)
    wide = lambda t: torch.nn.functional.pad(t, (off, 13)).cuda()[:, off:off + H]  # noqa: E731
    w = [t.cuda() for t in (w1, w2, weight)]
    y, kept = block.experts(x.cuda(), *w, plan, keep=True)
    y2, kept2 = block.experts(wide(x), *w, plan, keep=True)
    assert torch.equal(y, y2)
    for a, b in zip(block.experts_bwd(dy.cuda(), x.cuda(), *w, plan, kept),
                    block.experts_bwd(wide(dy), wide(x), *w, plan, kept2)):
        assert torch.equal(a, b)


def test_experts_same_bits_every_time_and_on_another_stream():
    from paper_2504_00598_amd import block
    idx, x, dy, w1, w2, weight = expert_inputs(400, 128, 96, 6, 0, 6, 3, torch.bfloat16)
    dev = [t.cuda() for t in (x, w1, w2, weight)]
    plan = block.expert_plan(idx.cuda(), 6)
    y, kept = block.experts(*dev, plan, keep=True)
    first = [y, *block.experts_bwd(dy.cuda(), *dev, plan, kept)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    d = dy.cuda()
    side.wait_stream(torch.cuda.current_stream())
    p2 = block.expert_plan(plan.rows.new_tensor(idx.tolist()), 6, stream=side)
    torch.cuda.synchronize()
    y, kept = block.experts(*dev, p2, keep=True, stream=side)
    again = [y, *block.experts_bwd(d, *dev, p2, kept, stream=side)]
    side.synchronize()
    for a, b in zip(first, again):
        assert torch.equal(a, b)


def test_no_tokens():
    from paper_2504_00598_amd import block
    bf = torch.bfloat16
    z = lambda *s, dtype=bf: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
    cos, sin = (t.cuda() for t in tables(4, 8))
    g = torch.ones(8, dtype=bf, device="cuda")
    q, k = block.qk_norm_rope(z(0, 2, 8), z(0, 1, 8), g, g, cos, sin)
    assert q.shape == (0, 2, 8) and k.shape == (0, 1, 8)
    out = block.qk_norm_rope_bwd(z(0, 2, 8), z(0, 1, 8), z(0, 2, 8), z(0, 1, 8), g, g, cos, sin)
    assert not out[2].any() and not out[3].any()
    w, idx = block.route(z(0, 6), 2)
    assert w.shape == idx.shape == (0, 2)
    assert block.route_bwd(w, z(0, 6), idx).shape == (0, 6)
    plan = block.expert_plan(idx, 6)
    assert plan.offsets.tolist() == [0] * 7
    w1, w2 = torch.ones(6, 32, 24, dtype=bf, device="cuda"), torch.ones(6, 24, 16, dtype=bf, device="cuda")
    y, kept = block.experts(z(0, 24), w1, w2, w, plan, keep=True)
    dx, dw1, dw2, dweight = block.experts_bwd(z(0, 24), z(0, 24), w1, w2, w, plan, kept)
    assert y.shape == dx.shape == (0, 24) and dweight.shape == (0, 2) and not dw1.any() and not dw2.any()


def test_experts_infinities_stay_in_their_token():
    from paper_2504_00598_amd import block
    idx, x, _, w1, w2, weight = expert_inputs(200, 64, 32, 3, 0, 3, 2, torch.bfloat16)
    dev = [t.cuda() for t in (w1, w2, weight)]
    plan = block.expert_plan(idx.cuda(), 3)
    y = block.experts(x.cuda(), *dev, plan)
    bad = x.clone()
    bad[7, 5], bad[90] = math.inf, math.nan
    z = block.experts(bad.cuda(), *dev, plan)
    other = [t for t in range(200) if t not in (7, 90)]
    assert torch.equal(y[other], z[other]) and z[90].isnan().all() and not z[7].isfinite().any()


def test_captured_graph_replays():
    """Routing, order, products and their gradients in one graph, replayed on new inputs between eager work."""
    from paper_2504_00598_amd import block
    idx, x, dy, w1, w2, _ = expert_inputs(150, 64, 48, 5, 0, 5, 2, torch.bfloat16)
    x, dy, w1, w2 = (t.cuda() for t in (x, dy, w1, w2))
    logits = torch.randn(150, 5, generator=gen(1)).cuda()

    def step():
        w, i = block.route(logits, 2)
        plan = block.expert_plan(i, 5)
        y, kept = block.experts(x, w1, w2, w, plan, keep=True)
        dx, dw1, dw2, dw = block.experts_bwd(dy, x, w1, w2, w, plan, kept)
        return [w, i, y, dx, dw1, dw2, dw, block.route_bwd(dw, logits, i)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for r in range(4):
        x.copy_(torch.randn(150, 64, generator=gen(10 + r)).to(torch.bfloat16))
        logits.copy_(torch.randn(150, 5, generator=gen(20 + r)))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        for a, b in zip(got, step()):
            assert torch.equal(a, b), r
        torch.cuda.synchronize()
