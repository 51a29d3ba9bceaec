"""Norm and rotation by positions of several axes against a plain 64-bit form: every pair turned by itself.

Bounds as for one axis (test_gpu_block.py): a result is within its type's roundoff of its value beside the error in 32
bits, a gain's gradient within 2^-18."""
import pytest
import torch

from tests.gpu_util import need_gpu, say
from tests.test_gpu_block import DT, U, gen, near, tables

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


def rows(x, w, cos, sin, pos, axes, eps, interleaved):
    """x [T][heads][D] in 64 bits, pos [axes][T]."""
    half = len(axes)
    z = x / torch.sqrt((x * x).mean(2, keepdim=True) + eps) * (w if w is not None else 1.0)
    out = [None] * x.shape[2]
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        c, s = cos[pos[axes[i]], i][:, None], sin[pos[axes[i]], i][:, None]
        out[a], out[b] = z[..., a] * c - z[..., b] * s, z[..., b] * c + z[..., a] * s
    return torch.stack([z[..., j] if o is None else o for j, o in enumerate(out)], 2)


def sections(*n):
    return [a for a, m in enumerate(n) for _ in range(m)]


CASES = [  # T, query heads, key heads, D, axis of each pair, axes, interleaved, type, gain type
    (1, 1, 1, 2, [0], 1, False, "bf16", "bf16"),
    (1, 32, 8, 128, sections(16, 24, 24), 3, False, "bf16", "bf16"),
    (9, 4, 2, 128, [i % 3 for i in range(64)], 3, False, "bf16", "bf16"),
    (37, 5, 1, 80, sections(5, 10, 5), 3, True, "f16", "f32"),
    (17, 3, 0, 64, [i % 2 for i in range(32)], 2, True, "f32", "f32"),
    (17, 3, 2, 64, sections(9, 14, 1), 4, False, "bf16", None),
    (130, 2, 1, 96, [3, 2, 1, 0] * 6, 4, True, "bf16", "bf16"),
    (5, 3, 1, 33, [1, 0, 0, 2, 2], 3, False, "bf16", "f32"),
    (6, 2, 1, 512, [(i // 5) % 4 for i in range(256)], 4, False, "bf16", "bf16"),
    (6, 2, 1, 510, [(i * 7 // 3) % 4 for i in range(255)], 4, True, "f16", "f16"),
    (2000, 3, 2, 256, sections(64, 32, 32), 3, False, "bf16", "bf16"),
    (3, 2, 1, 16, [], 2, False, "bf16", "bf16"),
]


@pytest.mark.parametrize("T,hq,hk,D,axes,n,inter,dt,wdt", CASES)
@pytest.mark.parametrize("lead", [0, 3])
def test_axes_and_gradient(T, hq, hk, D, axes, n, inter, dt, wdt, lead):
    from paper_2504_00598_amd import block
    say("axes", T, hq, hk, D, axes, n, inter, dt, wdt, lead)
    g = gen(T + D)
    dtype = DT[dt]
    cos, sin = tables(64, 2 * len(axes))
    pos = torch.randint(0, 64, (n, T), generator=g, dtype=torch.int32)
    x = torch.randn(T, (hq + hk) * D + 3, generator=g).to(dtype)
    cut = lambda t: (t[:, lead:lead + hq * D].unflatten(1, (hq, D)),  # noqa: E731
                     t[:, lead + hq * D:lead + (hq + hk) * D].reshape(T, hk, D))
    q, k = cut(x)
    qd, kd = cut(x.cuda())
    wq = wk = None
    if wdt:
        wq, wk = (1 + torch.randn(D, generator=g)).to(DT[wdt]), (1 + torch.randn(D, generator=g)).to(DT[wdt])
    dy = [torch.randn(T, h, D, generator=g).to(dtype) for h in (hq, hk)]
    cu = lambda t: None if t is None else t.cuda()  # noqa: E731
    args = (qd, kd, cu(wq), cu(wk), cos.cuda(), sin.cuda(), pos.cuda())
    how = dict(eps=1e-5, interleaved=inter, axes=axes)
    yq, yk = block.qk_norm_rope(*args, **how)
    dq, dk, dwq, dwk = block.qk_norm_rope_bwd(dy[0].cuda(), dy[1].cuda(), *args, **how)
    u = U[dtype] * 1.01 + 2.0 ** -20
    for x, w, y, d, dx, dw, name in ((q, wq, yq, dy[0], dq, dwq, "q"), (k, wk, yk, dy[1], dk, dwk, "k")):
        if not x.numel():
            continue
        xr = x.double().clone().requires_grad_()
        wr = None if w is None else w.double().clone().requires_grad_()
        ref = rows(xr, wr, cos.double(), sin.double(), pos.long(), axes, 1e-5, inter)
        near(y, ref, u, name)
        (ref * d.double()).sum().backward()
        near(dx, xr.grad, u, "d" + name)
        if w is not None:
            near(dw, wr.grad, 2.0 ** -18, "dw" + name)


def test_equal_axes_are_one():
    from paper_2504_00598_amd import block
    g = gen(1)
    cos, sin = (t.cuda() for t in tables(64, 64))
    q, k = torch.randn(20, 4, 64, generator=g).bfloat16().cuda(), torch.randn(20, 2, 64, generator=g).bfloat16().cuda()
    pos = torch.randint(0, 64, (20,), generator=g, dtype=torch.int32).cuda()
    one = block.qk_norm_rope(q, k, None, None, cos, sin, pos)
    for axes in ([0] * 32, [i % 3 for i in range(32)], sections(8, 12, 12)):
        got = block.qk_norm_rope(q, k, None, None, cos, sin, pos.expand(3, 20).contiguous(), axes=axes)
        assert torch.equal(one[0], got[0]) and torch.equal(one[1], got[1])


@pytest.mark.parametrize("axes", [sections(2, 3, 3), [0, 1, 2, 0, 1, 2, 0, 1]])
def test_positions_outside_the_tables(axes):
    from paper_2504_00598_amd import block
    cos, sin = (t.cuda() for t in tables(8, 16))
    q = torch.randn(4, 2, 20, generator=gen(2)).cuda()
    pos = torch.tensor([[0, 8, 1, 2], [1, 1, -1, 2], [2, 2, 2, 2 ** 31 - 1]], dtype=torch.int32).cuda()
    y, _ = block.qk_norm_rope(q, q[:, :1], None, None, cos, sin, pos, axes=axes)
    dq, _, _, _ = block.qk_norm_rope_bwd(q, q[:, :1], q, q[:, :1], None, None, cos, sin, pos, axes=axes)
    for t in range(4):
        bad = torch.tensor([t == axes[i % 8] + 1 for i in range(16)] + [False] * 4)
        assert torch.equal(y[t].isnan().cpu(), bad.expand(2, 20)), t
        assert bool(dq[t].isnan().any()) == (t > 0)


def test_gradient_against_differences():
    """dq along a direction against the 64-bit form's difference quotient (its error is h^2 of the third derivative)."""
    from paper_2504_00598_amd import block
    g = gen(3)
    cos, sin = tables(16, 8)
    q, v, d = (torch.randn(4, 3, 12, generator=g) for _ in range(3))
    pos, axes = torch.randint(0, 16, (2, 4), generator=g, dtype=torch.int32), [1, 0, 0, 1]
    dq, _, _, _ = block.qk_norm_rope_bwd(d.cuda(), d[:, :0].cuda(), q.cuda(), q[:, :0].cuda(), None, None, cos.cuda(), sin.cuda(),
                                         pos.cuda(), axes=axes)
    f = lambda x: float((rows(x, None, cos.double(), sin.double(), pos.long(), axes, 1e-6, False) * d.double()).sum())  # noqa: E731
    h = 1e-4
    num = (f(q.double() + h * v.double()) - f(q.double() - h * v.double())) / (2 * h)
    assert abs(num - float((dq.cpu().double() * v).sum())) <= 1e-4 * (dq.cpu().double().norm() * v.double().norm())


def test_recorded_calls():
    from paper_2504_00598_amd import block
    g = gen(4)
    cos, sin = (t.cuda() for t in tables(40, 32))
    x = torch.randn(37, 8, 64, generator=g).bfloat16().cuda().requires_grad_()
    w = torch.randn(64, generator=g).bfloat16().cuda().requires_grad_()
    pos = torch.randint(0, 40, (3, 37), generator=g, dtype=torch.int32).cuda()
    axes = [i % 3 for i in range(16)]
    dq, dk = (torch.randn(37, n, 64, generator=g).bfloat16().cuda() for n in (5, 3))
    q, k = block.qk_norm_rope(x[:, :5], x[:, 5:], w, w, cos, sin, pos, axes=axes)
    axes_then, axes[0] = list(axes), 2  # what the caller does with its list afterwards changes nothing
    torch.autograd.backward([q, k], [dq, dk])
    with torch.no_grad():
        args = (x[:, :5], x[:, 5:], w, w, cos, sin, pos)
        plain = block.qk_norm_rope(*args, axes=axes_then)
        want = block.qk_norm_rope_bwd(dq, dk, *args, axes=axes_then)
    assert torch.equal(q, plain[0]) and torch.equal(k, plain[1])
    assert torch.equal(x.grad, torch.cat(want[:2], 1))
    assert torch.equal(w.grad, want[2].bfloat16() + want[3].bfloat16())


def test_captured_calls_follow_the_positions():
    from paper_2504_00598_amd import block
    g = gen(5)
    cos, sin = (t.cuda() for t in tables(40, 32))
    q, k = (torch.randn(7, n, 32, generator=g).bfloat16().cuda() for n in (4, 2))
    pos = torch.zeros(2, 7, dtype=torch.int32, device="cuda")
    axes = [0, 1] * 8
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = block.qk_norm_rope(q, k, None, None, cos, sin, pos, axes=axes)
        grad = block.qk_norm_rope_bwd(q, k, q, k, None, None, cos, sin, pos, axes=axes)
    axes[:] = [0] * 16
    for _ in range(3):
        pos.copy_(torch.randint(0, 40, (2, 7), generator=g, dtype=torch.int32))
        graph.replay()
        want = block.qk_norm_rope(q, k, None, None, cos, sin, pos, axes=[0, 1] * 8)
        dwant = block.qk_norm_rope_bwd(q, k, q, k, None, None, cos, sin, pos, axes=[0, 1] * 8)
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
        assert torch.equal(grad[0], dwant[0]) and torch.equal(grad[1], dwant[1])


def test_refusals():
    from paper_2504_00598_amd import block
    cos, sin = (t.cuda() for t in tables(8, 8))
    q = torch.randn(3, 2, 16).cuda()
    pos = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    for p, axes in ((None, [0] * 4), (pos[0], [0] * 4), (pos, None), (pos, [0] * 3), (pos, [0] * 5), (pos, [0, 1, 2, 0]),
                    (pos, [0, -1, 0, 0]), (pos, [300, 0, 0, 0]), (pos.long(), [0] * 4), (pos[:, :2], [0] * 4), (pos.cpu(), [0] * 4),
                    (pos.t().contiguous().t(), [0] * 4), (pos[:0], [0] * 4), (torch.cat([pos] * 3), [0] * 4), (pos, 4), (pos, [0.0] * 4)):
        with pytest.raises((TypeError, ValueError)):
            block.qk_norm_rope(q, q, None, None, cos, sin, p, axes=axes)
        with pytest.raises((TypeError, ValueError)):
            block.qk_norm_rope_bwd(q, q, q, q, None, None, cos, sin, p, axes=axes)
