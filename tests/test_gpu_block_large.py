"""The experts' products at sizes that take the large tiles, with edges inside a tile, widths that are padded, and
an expert without tokens, against the formulas in 64 bits.  Bounds as in test_gpu_block.py: 1.5 u in the 2-norm and 20 u
for an entry, u the unit roundoff of the type; dweight, whose sums are in 32 bits throughout, with 2^-16 for u."""
import pytest
import torch

from tests.gpu_util import need_gpu, say
from tests.test_gpu_block import DT, U, near_product

pytestmark = pytest.mark.gpu


def formulas(x, w1, w2, weight, idx, dy):
    """(y, dx, dw1, dw2, dweight), float64 on the GPU."""
    F = w2.shape[2]
    y, dx = torch.zeros_like(x), torch.zeros_like(x)
    dw1, dw2, dweight = torch.zeros_like(w1), torch.zeros_like(w2), torch.zeros_like(weight)
    for e in range(w1.shape[0]):
        t, j = torch.nonzero(idx == e, as_tuple=True)
        xe, dye, w = x[t], dy[t], weight[t, j][:, None]
        g, u = (xe @ w1[e].T).split(F, 1)
        sg = torch.sigmoid(g)
        s, p = g * sg * u, dye @ w2[e]
        dgu = torch.cat((w * p * u * sg * (1 + g * (1 - sg)), w * p * g * sg), 1)
        y.index_add_(0, t, w * (s @ w2[e].T))
        dx.index_add_(0, t, dgu @ w1[e])
        dw1[e], dw2[e] = dgu.T @ xe, dye.T @ (w * s)
        dweight[t, j] = (s * p).sum(1)
    return y, dx, dw1, dw2, dweight


@pytest.mark.parametrize("T,H,F,E,k", [(12001, 2056, 1548, 4, 2), (8000, 1031, 390, 6, 2), (3001, 520, 264, 5, 1)])
@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_experts_large(T, H, F, E, k, dt):
    from paper_2504_00598_amd import block
    need_gpu()
    say("experts large", T, H, F, E, k, dt)
    g = torch.Generator(device="cuda")
    g.manual_seed(T + H)

    def normal(*shape, scale=1.0):
        return torch.empty(shape, device="cuda").normal_(0.0, scale, generator=g).to(DT[dt])

    x, dy = normal(T, H), normal(T, H)
    w1, w2 = normal(E, 2 * F, H, scale=H ** -0.5), normal(E, H, F, scale=F ** -0.5)
    weight = torch.rand(T, k, device="cuda", generator=g) + 0.1
    # the last expert has none; the others' shares differ
    idx = torch.stack([torch.randperm(E - 1, device="cuda", generator=g)[:k] for _ in range(97)])
    idx = idx[torch.arange(T, device="cuda") ** 2 % 97].to(torch.int32)
    plan = block.expert_plan(idx, E)
    y, kept = block.experts(x, w1, w2, weight, plan, keep=True)
    got = (y,) + block.experts_bwd(dy, x, w1, w2, weight, plan, kept)
    want = formulas(*(t.double() for t in (x, w1, w2, weight)), idx, dy.double())
    u = U[DT[dt]]
    for name, a, b in zip(("y", "dx", "dw1", "dw2", "dweight"), got, want):
        near_product(a, b.cpu(), u if name != "dweight" else 2.0 ** -16, name)
    assert not got[2][-1].any() and not got[3][-1].any()
    again = (block.experts(x, w1, w2, weight, plan),) + block.experts_bwd(dy, x, w1, w2, weight, plan, kept)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
