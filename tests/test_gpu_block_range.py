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


HALF = [  # scales of x, w1, w2, dy and the weights
    dict(x=2.0 ** 4, w1=2.0 ** 4, w2=2.0 ** -8, dy=2.0 ** -10),                        # s above 65504
    dict(x=2.0 ** -8, w2=2.0 ** 8),                                                    # s below 2^-14
    dict(x=2.0 ** 10, w1=2.0 ** -4, w2=2.0 ** -3, dy=2.0 ** 12),                       # the gradients of gate and up above 65504
    dict(x=2.0 ** -9, w1=2.0 ** 9, dy=2.0 ** -9, weight=2.0 ** -12),                   # and below 2^-14
    dict(x=2.0 ** -4, w1=2.0 ** -1, w2=2.0 ** -4, dy=2.0 ** 6, weight=2.0 ** -14),     # w s below 2^-14
]


@pytest.mark.parametrize("scales", range(len(HALF)))
@pytest.mark.parametrize("T,H,F,E,k", SIZES)
def test_float16_between_the_products(T, H, F, E, k, scales):
    """float16 inputs and results in range, what lies between them not."""
    say("float16", T, H, F, E, k, HALF[scales])
    args = inputs(T, H, F, E, k, torch.float16, **HALF[scales])
    want = formulas(*(t.double() for t in args[:4]), args[4], args[5].double())
    u = U[torch.float16]
    for name, a, b in zip(("y", "dx", "dw1", "dw2", "dweight"), results(*args), want):
        if name == "dweight":
            near_product(a, b.cpu(), 2.0 ** -16, name)
            continue
        step, rms = 2.0 ** -25, b.square().mean().sqrt()
        entry = 20 * u * torch.maximum(b.abs(), rms) + step
        # a result of float16 ends at 65504: infinite where it is past it by more than the bound
        fits, past = b.abs() + entry < 65504, b.abs() - entry > 65520
        assert bool(a[past].isinf().all()), name
        off = (a.double() - b).abs()
        assert bool((off <= entry)[fits].all()), (name, float(off[fits].max()), float(rms))
        assert name not in ("y", "dx") or bool(fits.all()), name
        if bool(fits.all()):
            assert float(off.norm()) <= 1.5 * u * float(b.norm()) + step * math.sqrt(b.numel()), (name, float(off.norm() / b.norm()))


def test_float16_tokens_of_other_magnitudes():
    """A token's results do not depend on how large the other tokens of its expert are."""
    args = list(inputs(150, 96, 72, 2, 1, torch.float16, x=2.0 ** -6, w1=2.0 ** 6))
    small = results(*args)
    large = torch.arange(150, device="cuda") % 3 == 0
    args[0], args[5] = args[0].clone(), args[5].clone()
    args[0][large] *= 2.0 ** 9
    args[5][large] *= 2.0 ** 6
    both = results(*args)
    for a, b in zip((small[0], small[1], small[4]), (both[0], both[1], both[4])):
        assert torch.equal(a[~large], b[~large])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("T", [0, 40, 700])
def test_nothing_kept(T, dtype):
    """No tokens, or a window that drops every assignment: zeros, whatever the workspace held."""
    from paper_2504_00598_amd import block
    say("nothing kept", T, dtype)
    x, w1, w2, weight, idx, dy = inputs(T, 96, 72, 4, 2, dtype)
    plan = block.expert_plan(idx, 4, first=7)
    ws = torch.full((1 << 24,), 255, dtype=torch.uint8, device="cuda")
    y, kept = block.experts(x, w1, w2, weight, plan, keep=True, ws=ws)
    ws.fill_(255)
    for t in (y,) + block.experts_bwd(dy, x, w1, w2, weight, plan, kept, ws=ws):
        assert not t.any()
