"""The experts' products where what lies between two products is far larger or smaller than its inputs and results,
against the formulas in 64 bits.

Bounds.  Powers of two on inputs change no mantissa, so the bounds are those of test_gpu_block.py: 1.5 u in the
2-norm and 20 u for an entry, u the unit roundoff of the type, taken for the entries of one magnitude.  A result
in float16 below 2^-14 is a multiple of 2^-24: 2^-25 for an entry is allowed beside.
"""
import math

import pytest
import torch

from tests.gpu_util import need_gpu, say
from tests.test_gpu_block import U, near_product
from tests.test_gpu_block_large import formulas

pytestmark = pytest.mark.gpu

SIZES = [(5, 72, 40, 3, 2), (150, 96, 72, 4, 2), (3001, 520, 264, 5, 1)]  # few tokens; small and larger tiles


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


def inputs(T, H, F, E, k, dtype, x=1.0, w1=1.0, w2=1.0, dy=1.0, weight=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(T + H)

    def normal(*shape, scale):
        return torch.empty(shape, device="cuda").normal_(0.0, 1.0, generator=g) * scale

    idx = torch.rand(T, E, device="cuda", generator=g).topk(k, 1)[1].to(torch.int32)
    t = [normal(T, H, scale=x), normal(E, 2 * F, H, scale=w1 / math.sqrt(H)), normal(E, H, F, scale=w2 / math.sqrt(F)),
         normal(T, H, scale=dy)]
    x, w1, w2, dy = (a.to(dtype) for a in t)
    return x, w1, w2, (torch.rand(T, k, device="cuda", generator=g) + 0.5) * weight, idx, dy


def results(x, w1, w2, weight, idx, dy):
    from paper_2504_00598_amd import block
    plan = block.expert_plan(idx, w1.shape[0])
    y, kept = block.experts(x, w1, w2, weight, plan, keep=True)
    return (y,) + block.experts_bwd(dy, x, w1, w2, weight, plan, kept)


@pytest.mark.parametrize("T,H,F,E,k", SIZES)
def test_features_of_other_magnitudes(T, H, F, E, k):
    """A feature's result does not depend on how large the features beside it are."""
    say("features", T, H, F, E, k)
    x, w1, w2, weight, idx, dy = inputs(T, H, F, E, k, torch.bfloat16)
    s = torch.full((H,), 2.0 ** -25, device="cuda")
    s[::32] = 2.0 ** 20
    # y and dx are s times the ones without s, feature by feature, dw1 and dw2 one s-th
    args = ((x / s).bfloat16(), (w1 * s).bfloat16(), (w2 * s[:, None]).bfloat16(), weight, idx, (dy / s).bfloat16())
    want = formulas(*(t.double() for t in (x, w1, w2, weight)), idx, dy.double())
    got = results(*args)
    back = (got[0].double() / s, got[1].double() / s, got[2].double() * s, got[3].double() * s[:, None], got[4])
    for name, a, b in zip(("y", "dx", "dw1", "dw2", "dweight"), back, want):
        near_product(a, b.cpu(), U[torch.bfloat16] if name != "dweight" else 2.0 ** -16, name)


@pytest.mark.parametrize("T", [60, 349])
def test_activation_at_any_gate(T):
    """dweight = s . p with one term: silu of the gate, in 32 bits, within eight roundings of it (below 2^-116: 0)."""
    say("gate", T)
    far = torch.tensor([-2.0 ** 127, -2.0 ** 14, -256, -96, 256, 2.0 ** 14, 2.0 ** 127], device="cuda")
    gate = torch.cat((torch.arange(T, device="cuda") * 0.5 - 87, far))
    T = len(gate)
    x = torch.zeros(T, 8, device="cuda")
    x[:, 0], x[:, 1] = gate, 1
    w1, w2, dy = torch.zeros(1, 16, 8, device="cuda"), torch.zeros(1, 8, 8, device="cuda"), torch.zeros(T, 8, device="cuda")
    w1[0, 0, 0] = w1[0, 8, 1] = w2[0, 0, 0] = 1
    dy[:, 0] = 1
    idx, weight = torch.zeros(T, 1, dtype=torch.int32, device="cuda"), torch.ones(T, 1, device="cuda")
    x16 = x.bfloat16()
    assert torch.equal(x16.float(), x)
    dweight = results(x16, w1.bfloat16(), w2.bfloat16(), weight, idx, dy.bfloat16())[4][:, 0].double()
    want = gate.double() * torch.sigmoid(gate.double())
    assert bool(((dweight - want).abs() <= 2.0 ** -21 * want.abs() + 2.0 ** -116).all()), float(((dweight - want) / want).abs().nan_to_num().max())
