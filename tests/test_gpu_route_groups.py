"""A group's value without a bias: of two definitions that rank groups differently, the scores' one."""
import pytest
import torch

from tests import block_ref as R
from tests.gpu_util import need_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("score,want", [("softmax", [0, 1]), ("sigmoid", [2, 3])])
def test_two_largest_scores_of_a_group(score, want):
    """Logits (5, -5) and (1, 1) sum to 0 and 2.  Their probabilities sum to 0.965 and 0.035, their sigmoids to 1 and 1.46."""
    from paper_2504_00598_amd import block
    need_gpu()
    logits = torch.tensor([[5.0, -5.0, 1.0, 1.0]])
    how = dict(score=score, groups=2, top_groups=1, group_score="top2")
    assert R.route(logits.double(), 2, score, None, 2, 1, "top2", False, 1.0)[1].tolist() == [want]
    for bias in (None, torch.zeros(4).cuda()):  # none is the same as zeros
        assert block.route(logits.cuda(), 2, bias=bias, **how)[1].tolist() == [want]


@pytest.mark.parametrize("E,groups,top", [(96, 8, 3), (60, 5, 2), (256, 8, 4)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_no_bias_is_a_bias_of_zeros(E, groups, top, score):
    from paper_2504_00598_amd import block
    need_gpu()
    g = torch.Generator()
    g.manual_seed(E)
    logits = torch.stack([torch.randperm(E, generator=g) for _ in range(40)]).float() * (6.0 / E) - 3.0
    how = dict(score=score, groups=groups, top_groups=top, group_score="top2")
    a = block.route(logits.cuda(), 6, **how)
    b = block.route(logits.cuda(), 6, bias=torch.zeros(E).cuda(), **how)
    want = R.route(logits.double(), 6, score, None, groups, top, "top2", False, 1.0)[1]
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and torch.equal(a[1].cpu().long(), want)
