"""The order of very many assignments: its counts, of which every workgroup reads all, stay few."""
import ctypes

import pytest

from paper_2504_00598_amd import block as B


@pytest.mark.parametrize("n", [1 << 12, 1 << 20, 1 << 23, (1 << 31) - 1])
@pytest.mark.parametrize("experts", [8, 256, 1024])
def test_counts_do_not_grow_with_the_assignments(n, experts):
    need = B.lib().cfp_expert_plan_workspace_bytes(ctypes.byref(B.cfp_plan_desc(n, 1, experts, 0, 0x1000)))
    assert need <= 512 * (experts + 1) * 4


@pytest.mark.gpu
@pytest.mark.parametrize("T,k,E,first,every", [(262144, 4, 64, 0, 64), (262145, 4, 64, 0, 64), (1100003, 8, 250, 3, 256)])
def test_many_assignments(T, k, E, first, every):
    import torch

    from tests.gpu_util import need_gpu, say
    need_gpu()
    say("plan", T, k, E)
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    idx = torch.randint(-1, every, (T, k), generator=g, device="cuda", dtype=torch.int32)
    plan = B.expert_plan(idx, E, first=first)
    e = idx.flatten().long() - first
    e = torch.where((e >= 0) & (e < E), e, E)
    order = torch.sort(e, stable=True)[1]
    count = torch.bincount(e, minlength=E + 1)
    offsets = torch.cat((count.new_zeros(1), count[:E].cumsum(0)))
    n = int(offsets[-1])
    assert torch.equal(plan.offsets.long(), offsets)
    assert torch.equal(plan.rows[:n].long(), order[:n]) and bool((plan.rows[n:] == -1).all())
    slot = torch.full_like(e, -1)
    slot[order[:n]] = torch.arange(n, device="cuda")
    assert torch.equal(plan.slot.long(), slot)
