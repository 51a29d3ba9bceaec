"""Operators of a decoder block: what the blocks of a searched chain run.

    from paper_2504_00598_amd import block
    q, k = block.qk_norm_rope(q, k, wq, wk, cos, sin, positions)
    weight, index = block.route(logits, 8, score="sigmoid", bias=bias, groups=8, top_groups=4, group_score="top2")
    plan = block.expert_plan(index, n_experts)
    y = block.experts(x, w1, w2, weight, plan)

Each has its gradient beside it (`*_bwd`).  Argument marshalling only: the work is
the HIP kernels' behind the C ABI of include/cfp_block.h, enqueued on the current
stream or on `stream`; nothing synchronises.  Results and workspaces are allocated
for the stream that the work runs on.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
from dataclasses import dataclass

from ._lib import CFP_OK, CfpError, _stream

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libcfp_block.so")

CFP_DT_F32, CFP_DT_F16, CFP_DT_BF16 = 0, 1, 2
SCORES = {"softmax": 0, "sigmoid": 1}
CFP_PLAN_PAD = 16  # entries behind the last of a plan's rows
GROUP_SCORES = {"max": 0, "top2": 1}

EXPORTED = ("cfp_qk_norm_rope", "cfp_qk_workspace_bytes", "cfp_qk_norm_rope_bwd", "cfp_route", "cfp_route_bwd",
            "cfp_expert_plan_workspace_bytes", "cfp_expert_plan", "cfp_experts_kept_bytes",
            "cfp_experts_workspace_bytes", "cfp_experts", "cfp_experts_bwd")

_P, _I32, _I64, _F32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float


class cfp_qk_desc(ctypes.Structure):
    _fields_ = [("n_tokens", _I64), ("n_q", _I32), ("n_k", _I32), ("dim", _I32), ("rot", _I32), ("interleaved", _I32),
                ("dtype", _I32), ("wdtype", _I32), ("eps", _F32), ("n_pos", _I64), ("q", _P), ("k", _P),
                ("q_token_stride", _I64), ("q_head_stride", _I64), ("k_token_stride", _I64), ("k_head_stride", _I64),
                ("wq", _P), ("wk", _P), ("cos", _P), ("sin", _P), ("pos", _P)]


class cfp_route_desc(ctypes.Structure):
    _fields_ = [("n_tokens", _I64), ("n_experts", _I32), ("k", _I32), ("score", _I32), ("groups", _I32),
                ("top_groups", _I32), ("group_score", _I32), ("renormalise", _I32), ("dtype", _I32), ("scale", _F32),
                ("logits", _P), ("stride", _I64), ("bias", _P)]


class cfp_plan_desc(ctypes.Structure):
    _fields_ = [("n_tokens", _I64), ("k", _I32), ("n_experts", _I32), ("first", _I32), ("index", _P)]


class cfp_experts_desc(ctypes.Structure):
    _fields_ = [("n_tokens", _I64), ("k", _I32), ("n_experts", _I32), ("hidden", _I32), ("inner", _I32), ("dtype", _I32),
                ("x", _P), ("x_stride", _I64), ("w1", _P), ("w2", _P), ("weight", _P), ("offsets", _P), ("rows", _P),
                ("slot", _P)]


_lib = None


def lib() -> ctypes.CDLL:
    """Load libcfp_block.so (raises OSError if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise OSError(f"{LIB_PATH} is missing: build it with `python -m paper_2504_00598_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        Q, R, N, X = (ctypes.POINTER(t) for t in (cfp_qk_desc, cfp_route_desc, cfp_plan_desc, cfp_experts_desc))
        SZ = ctypes.c_size_t
        for name, args in (("cfp_qk_workspace_bytes", [Q]), ("cfp_expert_plan_workspace_bytes", [N]),
                           ("cfp_experts_kept_bytes", [X]), ("cfp_experts_workspace_bytes", [X, _I32])):
            getattr(L, name).argtypes, getattr(L, name).restype = args, SZ
        for name, args in (("cfp_qk_norm_rope", [Q, _P, _P, _P]),
                           ("cfp_qk_norm_rope_bwd", [Q, _P, _I64, _I64, _P, _I64, _I64, _P, _P, _P, _P, _P, SZ, _P]),
                           ("cfp_route", [R, _P, _P, _P]), ("cfp_route_bwd", [R, _P, _P, _P, _P]),
                           ("cfp_expert_plan", [N, _P, _P, _P, _P, SZ, _P]),
                           ("cfp_experts", [X, _P, _P, _P, SZ, _P]),
                           ("cfp_experts_bwd", [X, _P, _I64, _P, _P, _P, _P, _P, _P, SZ, _P])):
            getattr(L, name).argtypes, getattr(L, name).restype = args, ctypes.c_int
        _lib = L
    return _lib


# ------------------------------------------------------------- marshalling --

_DT = {}


def _torch():
    import torch

    if not _DT:
        _DT.update({torch.float32: CFP_DT_F32, torch.float16: CFP_DT_F16, torch.bfloat16: CFP_DT_BF16})
    return torch


def _check(fn, rc):
    if rc != CFP_OK:
        raise CfpError(fn, rc)


def _tensor(name, t, torch, dtypes=None, dim=None):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a torch tensor on the GPU")
    if t.dtype not in (dtypes or _DT):
        raise TypeError(f"{name}: type {t.dtype} is not supported")
    if dim is not None and t.dim() != dim:
        raise ValueError(f"{name} must have {dim} dimensions")
    return t


def _same_device(first, *others):
    for t in others:
        if t is not None and t.device != first.device:
            raise ValueError("all tensors must be on one device")


def _on(torch, device, stream):
    """Context whose allocations and current stream are the call's; none where both are current."""
    if stream is None:
        return contextlib.nullcontext() if device.index == torch.cuda.current_device() else torch.cuda.device(device)
    if stream.device != device:
        raise ValueError("the stream is of another device than the tensors")
    return torch.cuda.stream(stream)


def _rows(name, t):
    """Row stride of a matrix whose rows are contiguous."""
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}: rows must be contiguous")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _ws(torch, nbytes, device, ws):
    if ws is None:
        return torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device)
    if ws.dtype != torch.uint8 or not ws.is_contiguous() or ws.device != device:
        raise TypeError("ws must be a contiguous uint8 tensor on the tensors' device")
    return ws


# -------------------------------------------------------- queries and keys --

def _heads(name, t, torch):
    _tensor(name, t, torch, dim=3)
    if t.shape[2] > 1 and t.stride(2) != 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    return t.stride(0), t.stride(1)


def _qk_desc(q, k, wq, wk, cos, sin, positions, eps, interleaved, torch):
    (qt, qh), (kt, kh) = _heads("q", q, torch), _heads("k", k, torch)
    T, hq, D = q.shape
    if k.shape[0] != T or k.shape[2] != D or k.dtype != q.dtype:
        raise ValueError("q is [T][heads][D] and k is [T][key heads][D], of one type")
    for name, w in (("wq", wq), ("wk", wk)):
        if w is not None:
            _tensor(name, w, torch, dim=1)
            if w.shape[0] != D or not w.is_contiguous():
                raise ValueError(f"{name} must be contiguous [D]")
    if wq is not None and wk is not None and wq.dtype != wk.dtype:
        raise ValueError("wq and wk must be of one type")
    for name, t in (("cos", cos), ("sin", sin)):
        _tensor(name, t, torch, (torch.float32,), 2)
        if not t.is_contiguous() or t.shape != cos.shape:
            raise ValueError("cos and sin must be contiguous [positions][rotated / 2]")
    if positions is not None:
        _tensor("positions", positions, torch, (torch.int32,), 1)
        if positions.shape[0] != T or not positions.is_contiguous():
            raise ValueError("positions must be contiguous [T]")
    elif cos.shape[1] and T > cos.shape[0]:
        raise ValueError("without positions the tables must hold a row for every token")
    _same_device(q, k, wq, wk, cos, sin, positions)
    w = wq if wq is not None else wk
    return cfp_qk_desc(T, hq, k.shape[1], D, 2 * cos.shape[1], int(bool(interleaved)), _DT[q.dtype],
                       _DT[w.dtype] if w is not None else CFP_DT_F32, float(eps), cos.shape[0], q.data_ptr(),
                       k.data_ptr(), qt, qh, kt, kh, wq.data_ptr() if wq is not None else None,
                       wk.data_ptr() if wk is not None else None, cos.data_ptr(), sin.data_ptr(),
                       positions.data_ptr() if positions is not None else None)


def qk_norm_rope(q, k, wq, wk, cos, sin, positions=None, *, eps=1e-6, interleaved=False, stream=None):
    """Norm and rotation of queries and keys in one pass.

    q [T][heads][D] and k [T][key heads][D] may be views of a larger product (last
    dimension contiguous).  Each head is divided by sqrt(mean(x^2) + eps), times its
    gain wq or wk [D] (None: ones), and its first 2 * cos.shape[1] entries are rotated by
    the angles of row positions[t] of the tables cos, sin [positions][rotated / 2]
    (None: row t): pairs (i, i + rotated / 2), or with `interleaved` (2i, 2i + 1).  A position outside
    the tables makes its rotated entries NaN.  Returns contiguous (q, k) of q's type."""
    torch = _torch()
    d = _qk_desc(q, k, wq, wk, cos, sin, positions, eps, interleaved, torch)
    with _on(torch, q.device, stream):
        yq, yk = torch.empty(q.shape, dtype=q.dtype, device=q.device), torch.empty(k.shape, dtype=q.dtype, device=q.device)
        _check("cfp_qk_norm_rope", lib().cfp_qk_norm_rope(ctypes.byref(d), yq.data_ptr(), yk.data_ptr(), _stream(stream)))
    return yq, yk


def qk_norm_rope_bwd(dyq, dyk, q, k, wq, wk, cos, sin, positions=None, *, eps=1e-6, interleaved=False, ws=None,
                     stream=None):
    """Gradients of qk_norm_rope in q, k, wq and wk from those of its results (the inputs
    as they were given to it).  Returns (dq, dk, dwq, dwk); dwq and dwk are float32, None for a gain of None."""
    torch = _torch()
    d = _qk_desc(q, k, wq, wk, cos, sin, positions, eps, interleaved, torch)
    (qt, qh), (kt, kh) = _heads("dyq", dyq, torch), _heads("dyk", dyk, torch)
    if dyq.shape != q.shape or dyk.shape != k.shape or dyq.dtype != q.dtype or dyk.dtype != q.dtype:
        raise ValueError("dyq and dyk must have the shapes and the type of q and k")
    _same_device(q, dyq, dyk)
    with _on(torch, q.device, stream):
        dq, dk = torch.empty(q.shape, dtype=q.dtype, device=q.device), torch.empty(k.shape, dtype=q.dtype, device=q.device)
        dwq = torch.empty(q.shape[2], dtype=torch.float32, device=q.device) if wq is not None else None
        dwk = torch.empty(q.shape[2], dtype=torch.float32, device=q.device) if wk is not None else None
        ws = _ws(torch, lib().cfp_qk_workspace_bytes(ctypes.byref(d)), q.device, ws)
        _check("cfp_qk_norm_rope_bwd", lib().cfp_qk_norm_rope_bwd(
            ctypes.byref(d), dyq.data_ptr(), qt, qh, dyk.data_ptr(), kt, kh, dq.data_ptr(), dk.data_ptr(),
            dwq.data_ptr() if dwq is not None else None, dwk.data_ptr() if dwk is not None else None, ws.data_ptr(),
            ws.numel(), _stream(stream)))
    return dq, dk, dwq, dwk


# ----------------------------------------------------------------- routing --

def _route_desc(logits, k, score, bias, groups, top_groups, group_score, renormalise, scale, torch):
    _tensor("logits", logits, torch, dim=2)
    if score not in SCORES:
        raise ValueError(f"score must be one of {sorted(SCORES)}")
    if group_score not in GROUP_SCORES:
        raise ValueError(f"group_score must be one of {sorted(GROUP_SCORES)}")
    if bias is not None:
        _tensor("bias", bias, torch, (torch.float32,), 1)
        if bias.shape[0] != logits.shape[1] or not bias.is_contiguous():
            raise ValueError("bias must be contiguous [experts]")
        _same_device(logits, bias)
    return cfp_route_desc(logits.shape[0], logits.shape[1], int(k), SCORES[score], int(groups), int(top_groups),
                          GROUP_SCORES[group_score], int(bool(renormalise)), _DT[logits.dtype], float(scale),
                          logits.data_ptr(), _rows("logits", logits), bias.data_ptr() if bias is not None else None)


def route(logits, k, *, score="softmax", bias=None, groups=1, top_groups=1, group_score="max", renormalise=False,
          scale=1.0, stream=None):
    """The k experts of every token and their weights.

    logits [T][experts] (rows may lie apart).  score "softmax" or "sigmoid"; `bias`
    [experts] float32 is added to the scores for the choice alone.  With groups > top_groups
    only the experts of the `top_groups` best of `groups` equal runs take part (a run's largest
    value, or with group_score "top2" the sum of its two largest).  Weights are the scores, over
    their sum with `renormalise`, times `scale`.  Returns (weight [T][k] float32, index [T][k]
    int32), best first, equal values by the lowest index.  A logit of -inf masks its expert;
    a place with no expert left has index -1 and weight 0."""
    torch = _torch()
    d = _route_desc(logits, k, score, bias, groups, top_groups, group_score, renormalise, scale, torch)
    with _on(torch, logits.device, stream):
        weight = torch.empty((logits.shape[0], int(k)), dtype=torch.float32, device=logits.device)
        index = torch.empty((logits.shape[0], int(k)), dtype=torch.int32, device=logits.device)
        _check("cfp_route", lib().cfp_route(ctypes.byref(d), weight.data_ptr(), index.data_ptr(), _stream(stream)))
    return weight, index


def route_bwd(dweight, logits, index, *, score="softmax", renormalise=False, scale=1.0, stream=None):
    """Gradient of route's weights in the logits [T][experts], from dweight [T][k] float32 and the index it returned."""
    torch = _torch()
    k = index.shape[1] if index.dim() == 2 else 0
    d = _route_desc(logits, k, score, None, 1, 1, "max", renormalise, scale, torch)
    _tensor("index", index, torch, (torch.int32,), 2)
    _tensor("dweight", dweight, torch, (torch.float32,), 2)
    if tuple(index.shape) != (logits.shape[0], k) or index.shape != dweight.shape:
        raise ValueError("index and dweight are [T][k]")
    _same_device(logits, index, dweight)
    with _on(torch, logits.device, stream):
        index, dweight = index.contiguous(), dweight.contiguous()
        dlogits = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        _check("cfp_route_bwd", lib().cfp_route_bwd(ctypes.byref(d), index.data_ptr(), dweight.data_ptr(),
                                                    dlogits.data_ptr(), _stream(stream)))
    return dlogits


# ----------------------------------------------------------------- experts --

@dataclass
class ExpertPlan:
    """Order of the assignments a = token * k + place by expert."""

    offsets: object   # [experts + 1] int32: the positions of each expert
    rows: object      # [T * k] int32: the assignment at each position, -1 behind the last one kept
    slot: object      # [T * k] int32: the position of each assignment, -1 where it is dropped
    n_tokens: int
    k: int
    n_experts: int
    first: int


def expert_plan(index, n_experts, *, first=0, stream=None) -> ExpertPlan:
    """Stable order of the assignments in index [T][k] int32 by expert.  The plan is for the
    experts first .. first + n_experts - 1 (a device's share of them); assignments to others, and negative ones, are dropped."""
    torch = _torch()
    _tensor("index", index, torch, (torch.int32,), 2)
    T, k = index.shape
    with _on(torch, index.device, stream):
        index = index.contiguous()
        d = cfp_plan_desc(T, k, int(n_experts), int(first), index.data_ptr())
        n, e = T * k, int(n_experts)
        need = int(lib().cfp_expert_plan_workspace_bytes(ctypes.byref(d)))
        r, s = max(e, 0) + 1, max(e, 0) + 1 + n + CFP_PLAN_PAD  # where rows and slot begin
        buf = torch.empty(s + n + need // 4, dtype=torch.int32, device=index.device)
        plan = ExpertPlan(buf[:r], buf[r:r + n], buf[s:s + n], T, k, e, int(first))
        at = buf.data_ptr()
        _check("cfp_expert_plan", lib().cfp_expert_plan(
            ctypes.byref(d), at, at + 4 * r, at + 4 * s, at + 4 * (s + n), need, _stream(stream)))
    return plan


def _experts_desc(x, w1, w2, weight, plan, torch):
    half = (torch.float16, torch.bfloat16)
    _tensor("x", x, torch, half, 2)
    _tensor("w1", w1, torch, half, 3)
    _tensor("w2", w2, torch, half, 3)
    _tensor("weight", weight, torch, (torch.float32,), 2)
    T, H = x.shape
    E, F = w2.shape[0], w2.shape[2]
    if tuple(w1.shape) != (E, 2 * F, H) or w2.shape[1] != H:
        raise ValueError("w1 is [experts][2 * inner][hidden] and w2 is [experts][hidden][inner]")
    if w1.dtype != x.dtype or w2.dtype != x.dtype:
        raise TypeError("x, w1 and w2 must be of one type")
    if not (w1.is_contiguous() and w2.is_contiguous() and weight.is_contiguous()):
        raise ValueError("w1, w2 and weight must be contiguous")
    if not isinstance(plan, ExpertPlan) or (plan.n_tokens, plan.n_experts) != (T, E) or tuple(weight.shape) != (T, plan.k):
        raise ValueError("the plan is of another number of tokens, experts or places than x, w1 and weight")
    _same_device(x, w1, w2, weight, plan.offsets)
    return cfp_experts_desc(T, plan.k, E, H, F, _DT[x.dtype], x.data_ptr(), _rows("x", x), w1.data_ptr(), w2.data_ptr(),
                            weight.data_ptr(), plan.offsets.data_ptr(), plan.rows.data_ptr(), plan.slot.data_ptr())


def experts(x, w1, w2, weight, plan, *, keep=False, ws=None, stream=None):
    """y [T][hidden]: for every token the sum over its assignments in `plan` of
    weight * W2 (silu(gate) * up), [gate up] = W1 x.

    x [T][hidden] (rows may lie apart), w1 [experts][2 * inner][hidden] (gate rows, then
    up rows), w2 [experts][hidden][inner], float16 or bfloat16; weight [T][k] float32.  A token
    without assignments gets zeros.  With `keep` returns (y, kept): kept is what experts_bwd needs."""
    torch = _torch()
    d = _experts_desc(x, w1, w2, weight, plan, torch)
    ref = ctypes.byref(d)
    with _on(torch, x.device, stream):
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        ws = _ws(torch, lib().cfp_experts_workspace_bytes(ref, 0), x.device, ws)
        kept = _ws(torch, lib().cfp_experts_kept_bytes(ref), x.device, None) if keep else None
        _check("cfp_experts", lib().cfp_experts(ref, y.data_ptr(), kept.data_ptr() if keep else None, ws.data_ptr(),
                                                ws.numel(), _stream(stream)))
    return (y, kept) if keep else y


def experts_bwd(dy, x, w1, w2, weight, plan, kept, *, ws=None, stream=None):
    """Gradients of experts from dy [T][hidden] and what it kept: (dx, dw1, dw2, dweight).
    An expert without assignments gets zeros, and a dropped assignment's weight 0."""
    torch = _torch()
    d = _experts_desc(x, w1, w2, weight, plan, torch)
    ref = ctypes.byref(d)
    _tensor("dy", dy, torch, (x.dtype,), 2)
    if dy.shape != x.shape:
        raise ValueError("dy must have the shape of x")
    _same_device(x, dy, kept)
    if kept.dtype != torch.uint8 or kept.numel() < lib().cfp_experts_kept_bytes(ref) or not kept.is_contiguous():
        raise ValueError("kept is not what experts returned for these sizes")
    with _on(torch, x.device, stream):
        dx, dw1, dw2 = torch.empty(x.shape, dtype=x.dtype, device=x.device), torch.empty_like(w1), torch.empty_like(w2)
        dweight = torch.empty_like(weight)
        ws = _ws(torch, lib().cfp_experts_workspace_bytes(ref, 1), x.device, ws)
        _check("cfp_experts_bwd", lib().cfp_experts_bwd(
            ref, dy.data_ptr(), _rows("dy", dy), kept.data_ptr(), dx.data_ptr(), dw1.data_ptr(), dw2.data_ptr(),
            dweight.data_ptr(), ws.data_ptr(), ws.numel(), _stream(stream)))
    return dx, dw1, dw2, dweight
