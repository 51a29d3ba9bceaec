"""The operators inside a recorded program: backward() reaches their inputs with what the *_bwd calls give."""
import pytest
import torch

from tests.gpu_util import need_gpu
from tests.test_gpu_block import expert_inputs, gen, tables

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


def leaf(t):
    return t.cuda().requires_grad_()


def test_queries_and_keys():
    from paper_2504_00598_amd import block
    g = gen(0)
    cos, sin = (t.cuda() for t in tables(40, 32))
    qkv = leaf(torch.randn(37, 8, 64, generator=g).bfloat16())
    wq, wk = leaf(torch.randn(64, generator=g).bfloat16()), leaf(torch.randn(64, generator=g).bfloat16())
    dq, dk = torch.randn(37, 5, 64, generator=g).cuda().bfloat16(), torch.randn(37, 3, 64, generator=g).cuda().bfloat16()
    q, k = block.qk_norm_rope(qkv[:, :5], qkv[:, 5:], wq, wk, cos, sin, eps=1e-5, interleaved=True)
    torch.autograd.backward([q, k], [dq, dk])
    with torch.no_grad():
        args = (qkv[:, :5], qkv[:, 5:], wq, wk, cos, sin)
        plain = block.qk_norm_rope(*args, eps=1e-5, interleaved=True)
        want = block.qk_norm_rope_bwd(dq, dk, *args, eps=1e-5, interleaved=True)
    assert torch.equal(q, plain[0]) and torch.equal(k, plain[1]) and not plain[0].requires_grad
    assert torch.equal(qkv.grad, torch.cat(want[:2], 1))
    assert torch.equal(wq.grad, want[2].bfloat16()) and torch.equal(wk.grad, want[3].bfloat16())
    # one result alone, through a broadcast gradient, without gains
    x = leaf(torch.randn(4, 2, 64, generator=g))
    block.qk_norm_rope(x, x[:, :1].detach(), None, None, cos, sin)[0].sum().backward()
    ones = torch.ones(4, 2, 64, device="cuda")
    assert torch.equal(x.grad, block.qk_norm_rope_bwd(ones, ones[:, :1], x.detach(), x[:, :1].detach(), None, None, cos,
                                                      sin)[0])
    with pytest.raises(ValueError):
        block.qk_norm_rope(x, x[:, :1], None, None, cos.clone().requires_grad_(), sin)


@pytest.mark.parametrize("stream", [False, True])
def test_a_layer_of_experts(stream):
    from paper_2504_00598_amd import block
    _, x, dy, w1, w2, _ = expert_inputs(90, 64, 48, 5, 0, 5, 2, torch.bfloat16)
    x, w1, w2, dy = leaf(x), leaf(w1), leaf(w2), dy.cuda()
    logits = leaf(torch.randn(90, 5, generator=gen(1)))
    bias = torch.randn(5, generator=gen(2)).cuda()
    side = torch.cuda.Stream() if stream else None
    torch.cuda.synchronize()
    how = dict(score="sigmoid", renormalise=True, scale=2.0)
    weight, index = block.route(logits, 2, bias=bias, stream=side, **how)
    assert weight.requires_grad and not index.requires_grad
    plan = block.expert_plan(index, 5, stream=side)
    y = block.experts(x, w1, w2, weight, plan, stream=side)
    if stream:
        torch.cuda.current_stream().wait_stream(side)
    y.backward(dy)
    torch.cuda.synchronize()
    with torch.no_grad():
        again, kept = block.experts(x, w1, w2, weight, plan, keep=True)
        dx, dw1, dw2, dweight = block.experts_bwd(dy, x, w1, w2, weight, plan, kept)
        dlogits = block.route_bwd(dweight, logits, index, **how)
    for a, b in ((y, again), (x.grad, dx), (w1.grad, dw1), (w2.grad, dw2), (logits.grad, dlogits)):
        assert torch.equal(a, b)


def test_only_what_is_asked_for():
    from paper_2504_00598_amd import block
    idx, x, dy, w1, w2, weight = expert_inputs(90, 64, 48, 5, 0, 5, 2, torch.bfloat16)
    dev = [t.cuda() for t in (x, w1, w2, weight)]
    plan = block.expert_plan(idx.cuda(), 5)
    y, kept = block.experts(*dev, plan, keep=True)
    assert y.grad_fn is None
    dev[3].requires_grad_()
    y, kept = block.experts(*dev, plan, keep=True)
    assert y.requires_grad and not kept.requires_grad
    y.sum().backward()
    ones = torch.ones_like(y)
    with torch.no_grad():
        want = block.experts_bwd(ones, *dev, plan, kept)
    assert torch.equal(dev[3].grad, want[3]) and dev[0].grad is None and dev[1].grad is None
    # an explicit call still takes inputs that require a gradient
    assert torch.equal(block.experts_bwd(ones, *dev, plan, kept)[1], want[1])


def test_inputs_outlive_their_stream():
    """What only the recorded program holds is not handed out again while the call's stream still reads it."""
    from paper_2504_00598_amd import block
    idx, _, dy, w1, w2, weight = expert_inputs(4096, 64, 48, 5, 0, 5, 2, torch.bfloat16)
    w1, w2, dy, weight, idx = leaf(w1), leaf(w2), dy.cuda(), weight.cuda(), idx.cuda()
    side = torch.cuda.Stream()
    x = torch.randn(4096, 64, device="cuda").bfloat16()
    at, size = x.data_ptr(), x.shape
    side.wait_stream(torch.cuda.current_stream())
    plan = block.expert_plan(idx, 5, stream=side)
    y = block.experts(x, w1, w2, weight, plan, stream=side)
    del x
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)  # cycles of a kernel that only waits
        y.backward(dy)
    del y
    others = [torch.empty(size, dtype=torch.bfloat16, device="cuda") for _ in range(64)]
    assert at not in [t.data_ptr() for t in others]
    torch.cuda.synchronize()
    assert bool(w1.grad.isfinite().all())
