"""Calls with so many rows that a launch's threads in one dimension would pass 2^32."""
import pytest
import torch

from tests.gpu_util import need_gpu, say

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()
    yield
    torch.cuda.empty_cache()


def test_qk_rows():
    from paper_2504_00598_amd import block
    T, heads = 65537, 1024  # rows of 65 entries, which 64 lanes hold
    say("qk", T, heads)
    base = torch.randn(1, 1, 65, generator=torch.Generator().manual_seed(0)).cuda().bfloat16()
    q, none = base.expand(T, heads, 65), base.expand(T, heads, 65)[:, :0]
    empty = torch.empty(T, 0, device="cuda")
    y, _ = block.qk_norm_rope(q, none, None, None, empty, empty)
    one, _ = block.qk_norm_rope(base.expand(1, 1, 65), none[:1], None, None, empty[:1], empty[:1])
    for part in y.split(4096):
        assert bool((part == one).all())


def test_route_tokens():
    from paper_2504_00598_amd import block
    T = (1 << 28) + 3  # 16 lanes a token
    say("route", T)
    logits = torch.empty(T, 2, device="cuda", dtype=torch.bfloat16)
    for part in logits.split(1 << 26):
        part.normal_()
    logits[-1] = torch.tensor([1.0, 3.0])
    weight, index = block.route(logits, 1)
    grad = block.route_bwd(torch.ones_like(weight), logits, index)
    for l, w, i, d in zip(*(t.split(1 << 24) for t in (logits, weight, index, grad))):
        first = l[:, 0] >= l[:, 1]
        assert bool((i[:, 0] == (~first).int()).all())
        p = torch.sigmoid((l[:, 0].float() - l[:, 1].float()).abs())
        assert bool(((w[:, 0] - p).abs() <= 2.0 ** -20).all())
        ds = p * (1 - p)
        assert float((d[:, 0].float() - torch.where(first, ds, -ds)).abs().max()) <= 2.0 ** -9


def test_experts_tokens():
    from paper_2504_00598_amd import block
    T = (1 << 24) + 5  # a workgroup a token in the sums over a token's experts
    say("experts", T)
    g = torch.Generator().manual_seed(1)
    w1, w2 = torch.randn(1, 16, 8, generator=g).cuda().bfloat16(), torch.randn(1, 8, 8, generator=g).cuda().bfloat16()
    few = torch.randn(4099, 8, generator=g).cuda().bfloat16()
    at = torch.arange(T, device="cuda") % 4099
    x = few[at]
    idx, weight = torch.zeros(T, 1, dtype=torch.int32, device="cuda"), torch.ones(T, 1, device="cuda")
    y = block.experts(x, w1, w2, weight, block.expert_plan(idx, 1))
    want = block.experts(few, w1, w2, weight[:4099], block.expert_plan(idx[:4099], 1))
    # the same 8 terms of a sum in any tile
    assert bool(((y.float() - want[at].float()).abs() <= 2.0 ** -7 * want[at].float().abs() + 2.0 ** -12).all())
