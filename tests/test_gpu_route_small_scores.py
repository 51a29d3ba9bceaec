"""The gradient of weights over their sum, where the chosen scores are so small that one over their sum is no float.

Bound.  A score of 2^-130 holds 19 bits as a 32-bit float: 2^-16 of the largest incoming gradient for a few such
factors and the sums over them."""
import pytest
import torch

from tests import block_ref as R
from tests.gpu_util import need_gpu

pytestmark = pytest.mark.gpu


def test_renormalised_weights_of_small_scores():
    from paper_2504_00598_amd import block
    need_gpu()
    logits = torch.tensor([[0.0, -90.0, -91.0, -90.5, 0.5], [1.0, -88.5, -89.0, -2.0, -88.0]])
    bias = torch.tensor([0.0, 3.0, 2.0, 0.0, 0.0])  # the choice is experts 1 and 2
    weight, index = block.route(logits.cuda(), 2, bias=bias.cuda(), renormalise=True)
    assert index.tolist() == [[1, 2], [1, 2]]
    dw = torch.tensor([[1.0, -0.5], [0.25, 2.0]])
    dl = block.route_bwd(dw.cuda(), logits.cuda(), index, renormalise=True).cpu().double()
    lr = logits.double().requires_grad_()
    w = R.route_weights(lr, index.cpu().long(), "softmax", True, 1.0)
    assert bool(((weight.cpu().double() - w.detach()).abs() <= 2.0 ** -16).all())
    (w * dw.double()).sum().backward()
    assert bool(((dl - lr.grad).abs() <= 2.0 ** -16 * 2).all()), (dl, lr.grad)
