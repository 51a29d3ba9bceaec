"""The decoder-block library on the CPU: it exports what include/cfp_block.h declares and refuses bad
arguments before it touches a device."""
import ctypes
import os
import re
import subprocess

import pytest

from paper_2504_00598_amd import _lib as L
from paper_2504_00598_amd import block as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x1000  # a pointer that no refused call follows


def test_header_binding_and_exports_agree():
    text = open(os.path.join(ROOT, "include", "cfp_block.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    assert sorted(set(re.findall(r"\b(cfp_[a-z_]+)\s*\(", text))) == sorted(B.EXPORTED)
    B.lib()
    out = subprocess.check_output(["nm", "-D", "--defined-only", B.LIB_PATH], text=True)
    assert {ln.split()[-1] for ln in out.splitlines() if " T " in ln} == set(B.EXPORTED)


def test_packed_descriptors_have_the_structures_layout():
    for pack, c in ((B._QK, B.cfp_qk_desc), (B._ROUTE, B.cfp_route_desc), (B._PLAN, B.cfp_plan_desc),
                    (B._EXPERTS, B.cfp_experts_desc)):
        values = [i + 1 for i, _ in enumerate(c._fields_)]
        got = c.from_buffer_copy(pack(*values).ljust(ctypes.sizeof(c), b"\0"))
        assert [getattr(got, f) for f, _ in c._fields_] == values


def qk(**kw):
    d = dict(n_tokens=4, n_q=2, n_k=1, dim=8, rot=8, interleaved=0, dtype=2, wdtype=2, eps=1e-6, n_pos=16, q=P, k=P,
             q_token_stride=24, q_head_stride=8, k_token_stride=24, k_head_stride=8, wq=P, wk=P, cos=P, sin=P, pos=P)
    d.update(kw)
    return B.cfp_qk_desc(**d)


@pytest.mark.parametrize("bad,code", [
    (dict(n_tokens=-1), L.CFP_ERR_ARG), (dict(dim=0), L.CFP_ERR_ARG), (dict(rot=3), L.CFP_ERR_ARG),
    (dict(rot=10), L.CFP_ERR_ARG), (dict(dtype=3), L.CFP_ERR_ARG), (dict(wdtype=-1), L.CFP_ERR_ARG),
    (dict(eps=-1.0), L.CFP_ERR_ARG), (dict(eps=float("nan")), L.CFP_ERR_ARG), (dict(q=None), L.CFP_ERR_ARG),
    (dict(cos=None), L.CFP_ERR_ARG), (dict(pos=None, n_pos=3), L.CFP_ERR_ARG), (dict(dim=513, rot=0), L.CFP_ERR_UNSUPPORTED),
    (dict(n_tokens=2 ** 31), L.CFP_ERR_UNSUPPORTED), (dict(n_tokens=2 ** 30), L.CFP_ERR_UNSUPPORTED)])
def test_qk_refusals(bad, code):
    d = qk(**bad)
    assert B.lib().cfp_qk_norm_rope(ctypes.byref(d), P, P, None) == code
    assert B.lib().cfp_qk_norm_rope_bwd(ctypes.byref(d), P, 24, 8, P, 24, 8, P, P, P, P, P, 1 << 20, None) == code
    assert B.lib().cfp_qk_workspace_bytes(ctypes.byref(d)) == 0


def test_qk_missing_outputs_and_workspace():
    d = qk()
    assert B.lib().cfp_qk_norm_rope(None, P, P, None) == L.CFP_ERR_ARG
    assert B.lib().cfp_qk_norm_rope(ctypes.byref(d), None, P, None) == L.CFP_ERR_ARG
    need = B.lib().cfp_qk_workspace_bytes(ctypes.byref(d))
    assert need > 0
    for ws, n in ((None, need), (P, need - 1)):
        assert B.lib().cfp_qk_norm_rope_bwd(ctypes.byref(d), P, 24, 8, P, 24, 8, P, P, P, P, ws, n,
                                            None) == L.CFP_ERR_WORKSPACE


@pytest.mark.parametrize("bad,code", [
    (dict(n_experts=0), L.CFP_ERR_ARG), (dict(k=0), L.CFP_ERR_ARG), (dict(k=17), L.CFP_ERR_ARG),
    (dict(groups=3), L.CFP_ERR_ARG), (dict(groups=4, top_groups=5), L.CFP_ERR_ARG), (dict(top_groups=0), L.CFP_ERR_ARG),
    (dict(score=2), L.CFP_ERR_ARG), (dict(group_score=2), L.CFP_ERR_ARG),
    (dict(groups=16, top_groups=2, group_score=1), L.CFP_ERR_ARG), (dict(dtype=9), L.CFP_ERR_ARG),
    (dict(logits=None), L.CFP_ERR_ARG), (dict(stride=15), L.CFP_ERR_ARG),
    (dict(n_experts=1025, stride=1025), L.CFP_ERR_UNSUPPORTED), (dict(n_experts=64, k=33, stride=64), L.CFP_ERR_UNSUPPORTED),
    (dict(n_tokens=2 ** 31), L.CFP_ERR_UNSUPPORTED)])
def test_route_refusals(bad, code):
    a = dict(n_tokens=4, n_experts=16, k=2, score=0, groups=1, top_groups=1, group_score=0, renormalise=0, dtype=0,
             scale=1.0, logits=P, stride=16, bias=None)
    a.update(bad)
    d = B.cfp_route_desc(**a)
    assert B.lib().cfp_route(ctypes.byref(d), P, P, None) == code
    assert B.lib().cfp_route_bwd(ctypes.byref(d), P, P, P, None) == code


@pytest.mark.parametrize("bad,code", [
    (dict(n_tokens=-1), L.CFP_ERR_ARG), (dict(k=0), L.CFP_ERR_ARG), (dict(n_experts=0), L.CFP_ERR_ARG),
    (dict(first=-1), L.CFP_ERR_ARG), (dict(index=None), L.CFP_ERR_ARG), (dict(k=65), L.CFP_ERR_UNSUPPORTED),
    (dict(n_experts=1025), L.CFP_ERR_UNSUPPORTED), (dict(n_tokens=2 ** 30, k=2), L.CFP_ERR_UNSUPPORTED)])
def test_plan_refusals(bad, code):
    a = dict(n_tokens=4, k=2, n_experts=8, first=0, index=P)
    a.update(bad)
    d = B.cfp_plan_desc(**a)
    assert B.lib().cfp_expert_plan(ctypes.byref(d), P, P, P, P, 1 << 20, None) == code


def test_plan_workspace():
    d = B.cfp_plan_desc(1 << 20, 4, 64, 0, P)
    need = B.lib().cfp_expert_plan_workspace_bytes(ctypes.byref(d))
    assert need > 0
    assert B.lib().cfp_expert_plan(ctypes.byref(d), P, P, P, P, need - 1, None) == L.CFP_ERR_WORKSPACE
    assert B.lib().cfp_expert_plan(ctypes.byref(d), None, P, P, P, need, None) == L.CFP_ERR_ARG


def experts(**kw):
    a = dict(n_tokens=4, k=2, n_experts=3, hidden=16, inner=8, dtype=2, x=P, x_stride=16, w1=P, w2=P, weight=P, offsets=P,
             rows=P, slot=P)
    a.update(kw)
    return B.cfp_experts_desc(**a)


@pytest.mark.parametrize("bad,code", [
    (dict(n_tokens=-1), L.CFP_ERR_ARG), (dict(hidden=0), L.CFP_ERR_ARG), (dict(inner=0), L.CFP_ERR_ARG),
    (dict(dtype=0), L.CFP_ERR_ARG), (dict(x=None), L.CFP_ERR_ARG), (dict(w1=None), L.CFP_ERR_ARG),
    (dict(offsets=None), L.CFP_ERR_ARG), (dict(slot=None), L.CFP_ERR_ARG), (dict(x_stride=15), L.CFP_ERR_ARG),
    (dict(hidden=32769, x_stride=32769), L.CFP_ERR_UNSUPPORTED), (dict(inner=32769), L.CFP_ERR_UNSUPPORTED),
    (dict(k=65), L.CFP_ERR_UNSUPPORTED), (dict(n_tokens=2 ** 30), L.CFP_ERR_UNSUPPORTED)])
def test_experts_refusals(bad, code):
    d = experts(**bad)
    assert B.lib().cfp_experts(ctypes.byref(d), P, None, P, 1 << 40, None) == code
    assert B.lib().cfp_experts_bwd(ctypes.byref(d), P, 16, P, P, P, P, P, P, 1 << 40, None) == code
    assert B.lib().cfp_experts_workspace_bytes(ctypes.byref(d), 0) == 0


def test_experts_workspace_and_outputs():
    d = experts()
    for bwd in (0, 1):
        need = B.lib().cfp_experts_workspace_bytes(ctypes.byref(d), bwd)
        assert need > 0
        for ws, n in ((None, need), (P, need - 1)):
            rc = (B.lib().cfp_experts_bwd(ctypes.byref(d), P, 16, P, P, P, P, P, ws, n, None) if bwd else
                  B.lib().cfp_experts(ctypes.byref(d), P, None, ws, n, None))
            assert rc == L.CFP_ERR_WORKSPACE
    assert B.lib().cfp_experts(ctypes.byref(d), None, None, P, 1 << 30, None) == L.CFP_ERR_ARG
    assert B.lib().cfp_experts_bwd(ctypes.byref(d), P, 8, P, P, P, P, P, P, 1 << 30, None) == L.CFP_ERR_ARG
    assert B.lib().cfp_experts_bwd(ctypes.byref(d), P, 16, None, P, P, P, P, P, 1 << 30, None) == L.CFP_ERR_ARG


def test_the_binding_refuses_cpu_tensors_and_wrong_types():
    import torch
    x = torch.zeros(2, 3, 8)
    with pytest.raises(TypeError):
        B.qk_norm_rope(x, x, None, None, x[0], x[0])
    with pytest.raises(TypeError):
        B.route(torch.zeros(2, 4), 1)
    with pytest.raises(TypeError):
        B.expert_plan(torch.zeros(2, 4, dtype=torch.int32), 4)
    with pytest.raises(TypeError):
        B.experts(x[0], x, x, x[0], None)
