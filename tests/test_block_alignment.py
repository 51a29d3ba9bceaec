"""Workspaces and what the experts keep: pointers off their alignment are refused before any launch."""
import ctypes

import pytest

from paper_2504_00598_amd import _lib as L
from paper_2504_00598_amd import block as B
from tests.test_block_host import P, experts, qk


@pytest.mark.parametrize("off", [1, 2, 4, 8])
def test_experts_refuse_what_is_not_on_16_bytes(off):
    d = ctypes.byref(experts())
    lib, n = B.lib(), 1 << 30
    assert lib.cfp_experts(d, P, None, P + off, n, None) == L.CFP_ERR_ARG
    assert lib.cfp_experts(d, P, P + off, P, n, None) == L.CFP_ERR_ARG
    assert lib.cfp_experts_bwd(d, P, 16, P, P, P, P, P, P + off, n, None) == L.CFP_ERR_ARG
    assert lib.cfp_experts_bwd(d, P, 16, P + off, P, P, P, P, P, n, None) == L.CFP_ERR_ARG


@pytest.mark.parametrize("off", [1, 2])
def test_the_others_refuse_what_is_not_on_4_bytes(off):
    lib, n = B.lib(), 1 << 30
    assert lib.cfp_qk_norm_rope_bwd(ctypes.byref(qk()), P, 24, 8, P, 24, 8, P, P, P, P, P + off, n, None) == L.CFP_ERR_ARG
    plan = B.cfp_plan_desc(1 << 20, 4, 64, 0, P)
    assert lib.cfp_expert_plan(ctypes.byref(plan), P, P, P, P + off, n, None) == L.CFP_ERR_ARG


@pytest.mark.gpu
def test_the_binding_refuses_them():
    import torch

    from tests.gpu_util import need_gpu
    from tests.test_gpu_block import expert_inputs
    need_gpu()
    idx, x, dy, w1, w2, weight = expert_inputs(50, 64, 32, 4, 0, 4, 2, torch.bfloat16)
    dev = [t.cuda() for t in (x, w1, w2, weight)]
    plan = B.expert_plan(idx.cuda(), 4)
    arena = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    y, kept = B.experts(*dev, plan, keep=True, ws=arena[16:])
    grads = B.experts_bwd(dy.cuda(), *dev, plan, kept, ws=arena[32:])
    assert torch.equal(y, B.experts(*dev, plan))
    for a, b in zip(grads, B.experts_bwd(dy.cuda(), *dev, plan, kept)):
        assert torch.equal(a, b)
    for off in (1, 4, 8):
        with pytest.raises(ValueError):
            B.experts(*dev, plan, ws=arena[off:])
        with pytest.raises(ValueError):
            B.experts_bwd(dy.cuda(), *dev, plan, kept, ws=arena[off:])
        moved = torch.empty(kept.numel() + off, dtype=torch.uint8, device="cuda")[off:]
        with pytest.raises(ValueError):
            B.experts_bwd(dy.cuda(), *dev, plan, moved.copy_(kept))
    with pytest.raises(TypeError):
        B.experts_bwd(dy.cuda(), *dev, plan, None)
