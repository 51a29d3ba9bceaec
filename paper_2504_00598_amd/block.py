"""Operators of a decoder block: what the blocks of a searched chain run.

    from paper_2504_00598_amd import block
    q, k = block.qk_norm_rope(q, k, wq, wk, cos, sin, positions)
    weight, index = block.route(logits, 8, score="sigmoid", bias=bias, groups=8, top_groups=4, group_score="top2")
    plan = block.expert_plan(index, n_experts)
    y = block.experts(x, w1, w2, weight, plan)

Each has its gradient beside it (`*_bwd`), and where gradients are recorded and an input requires one, backward()
reaches it through that (block_grad).  What a `*_bwd` returns has no gradient of its own.  Argument marshalling only: the work is
the HIP kernels' behind the C ABI of include/cfp_block.h, enqueued on the current
stream or on `stream`; nothing synchronises.  Results and workspaces are allocated
for the stream that the work runs on.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import struct

from ._lib import CFP_OK, CfpError

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


# The same layouts for struct.pack: filling a ctypes structure of 21 fields takes 3 us, packing it 0.6 (a small
# launch takes 3).  A packed descriptor is passed by the address of its bytes.
_CODES = {_I64: "q", _I32: "i", _F32: "f", _P: "P"}
_QK, _ROUTE, _PLAN, _EXPERTS = (struct.Struct("@" + "".join(_CODES[t] for _, t in c._fields_)).pack
                                for c in (cfp_qk_desc, cfp_route_desc, cfp_plan_desc, cfp_experts_desc))

_lib = None


def lib() -> ctypes.CDLL:
    """Load libcfp_block.so (raises OSError if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise OSError(f"{LIB_PATH} is missing: build it with `python -m paper_2504_00598_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        SZ = ctypes.c_size_t
        for name, args in (("cfp_qk_workspace_bytes", [_P]), ("cfp_expert_plan_workspace_bytes", [_P]),
                           ("cfp_experts_kept_bytes", [_P]), ("cfp_experts_workspace_bytes", [_P, _I32])):
            getattr(L, name).argtypes, getattr(L, name).restype = args, SZ
        for name, args in (("cfp_qk_norm_rope", [_P, _P, _P, _P]),
                           ("cfp_qk_norm_rope_bwd", [_P, _P, _I64, _I64, _P, _I64, _I64, _P, _P, _P, _P, _P, SZ, _P]),
                           ("cfp_route", [_P, _P, _P, _P]), ("cfp_route_bwd", [_P, _P, _P, _P, _P]),
                           ("cfp_expert_plan", [_P, _P, _P, _P, _P, SZ, _P]),
                           ("cfp_experts", [_P, _P, _P, _P, SZ, _P]),
                           ("cfp_experts_bwd", [_P, _P, _I64, _P, _P, _P, _P, _P, _P, SZ, _P])):
            getattr(L, name).argtypes, getattr(L, name).restype = args, ctypes.c_int
        _lib = L
    return _lib


# ------------------------------------------------------------- marshalling --

_DT = {}


def _torch():
    import torch

    if not _DT:
        _DT.update({torch.float32: CFP_DT_F32, torch.float16: CFP_DT_F16, torch.bfloat16: CFP_DT_BF16})
        lib()
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


def _same_device(first, *others):
    for t in others:
        if t is not None and t.device != first.device:
            raise ValueError("all tensors must be on one device")


_HERE = contextlib.nullcontext()


def _on(torch, device, stream):
    """Context whose current device and stream, and so whose allocations, are the call's."""
    if stream is None:
        return _HERE if device.index == torch._C._cuda_getDevice() else torch.cuda.device(device)
    if stream.device != device:
        raise ValueError("the stream is of another device than the tensors")
    return torch.cuda.stream(stream)


def _raw(torch, device):
    """The current stream's handle, inside _on."""
    return torch._C._cuda_getCurrentRawStream(device.index)


def _rows(name, t):
    """Row stride of a matrix whose rows are contiguous."""
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}: rows must be contiguous")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _ws(torch, nbytes, device, ws, align=16):
    if ws is None:
        return torch.empty(max(nbytes, 1), dtype=torch.uint8, device=device)
    if not isinstance(ws, torch.Tensor) or ws.dtype != torch.uint8 or not ws.is_contiguous() or ws.device != device:
        raise TypeError("ws must be a contiguous uint8 tensor on the tensors' device")
    if ws.data_ptr() % align:
        raise ValueError(f"ws must start on {align} bytes")
    return ws


def _like(torch, t):
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def _recorded(torch, *inputs):
    """Whether backward() has to reach one of the inputs through this call."""
    if torch.is_grad_enabled():
        for t in inputs:
            if t is not None and t.requires_grad:
                return True
    return False


def _ptr(t):
    return 0 if t is None else t.data_ptr()


# -------------------------------------------------------- queries and keys --

def _qk_refuse(q, k, wq, wk, cos, sin, positions, torch):
    """Raises what is wrong with the arguments."""
    for name, t in (("q", q), ("k", k)):
        _tensor(name, t, torch, dim=3)
        if t.shape[2] > 1 and t.stride(2) != 1:
            raise ValueError(f"{name}: the last dimension must be contiguous")
    T, _, D = q.shape
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


def _qk_desc(q, k, wq, wk, cos, sin, positions, eps, interleaved, torch):
    # one pass over what has to hold, on the way of every call; what does not hold is said by _qk_refuse
    try:
        at, half = q.get_device(), cos.shape[1]
        (T, hq, D), (qt, qh, qd), (kt, kh, kd) = q.shape, q.stride(), k.stride()
        ok = (at >= 0 and k.shape[0] == T and k.shape[2] == D and k.dtype is q.dtype and k.get_device() == at and
              (D == 1 or (qd == 1 and kd == 1)) and cos.dtype is torch.float32 and sin.dtype is torch.float32 and
              cos.is_contiguous() and sin.is_contiguous() and sin.shape == cos.shape and cos.get_device() == at and
              sin.get_device() == at)
        for w in (wq, wk):
            ok = ok and (w is None or (w.numel() == D and w.dim() == 1 and w.get_device() == at and w.is_contiguous()))
        ok = ok and (wq is None or wk is None or wq.dtype is wk.dtype)
        if positions is None:
            ok = ok and (T <= cos.shape[0] or half == 0)
        else:
            ok = ok and (positions.dtype is torch.int32 and positions.numel() == T and positions.dim() == 1 and
                         positions.get_device() == at and positions.is_contiguous())
        w = wq if wq is not None else wk
        types = _DT[q.dtype], CFP_DT_F32 if w is None else _DT[w.dtype]
    except (AttributeError, KeyError, IndexError, TypeError, ValueError):
        ok = False
    if not ok:
        _qk_refuse(q, k, wq, wk, cos, sin, positions, torch)
        raise ValueError("unsupported arguments")
    return _QK(T, hq, k.shape[1], D, 2 * half, 1 if interleaved else 0, *types, eps, cos.shape[0], q.data_ptr(),
               k.data_ptr(), qt, qh, kt, kh, _ptr(wq), _ptr(wk), cos.data_ptr(), sin.data_ptr(), _ptr(positions))


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
    if _recorded(torch, q, k, wq, wk, cos, sin):
        from . import block_grad
        with _on(torch, q.device, stream):
            return block_grad.qk_norm_rope(q, k, wq, wk, cos, sin, positions, eps, interleaved, stream)
    with _on(torch, q.device, stream):
        yq, yk = _like(torch, q), _like(torch, k)
        rc = _lib.cfp_qk_norm_rope(d, yq.data_ptr(), yk.data_ptr(), _raw(torch, q.device))
    if rc:
        _check("cfp_qk_norm_rope", rc)
    return yq, yk


def qk_norm_rope_bwd(dyq, dyk, q, k, wq, wk, cos, sin, positions=None, *, eps=1e-6, interleaved=False, ws=None,
                     stream=None):
    """Gradients of qk_norm_rope in q, k, wq and wk from those of its results (the inputs
    as they were given to it).  Returns (dq, dk, dwq, dwk); dwq and dwk are float32, None for a gain of None."""
    torch = _torch()
    d = _qk_desc(q, k, wq, wk, cos, sin, positions, eps, interleaved, torch)
    for name, t, of in (("dyq", dyq, q), ("dyk", dyk, k)):
        _tensor(name, t, torch, (q.dtype,), 3)
        if t.shape != of.shape or (t.shape[2] > 1 and t.stride(2) != 1):
            raise ValueError(f"{name} must have the shape of its input, the last dimension contiguous")
    _same_device(q, dyq, dyk)
    with _on(torch, q.device, stream):
        dq, dk = _like(torch, q), _like(torch, k)
        dwq = torch.empty(q.shape[2], dtype=torch.float32, device=q.device) if wq is not None else None
        dwk = torch.empty(q.shape[2], dtype=torch.float32, device=q.device) if wk is not None else None
        ws = _ws(torch, _lib.cfp_qk_workspace_bytes(d), q.device, ws, 4)
        _check("cfp_qk_norm_rope_bwd", _lib.cfp_qk_norm_rope_bwd(
            d, dyq.data_ptr(), dyq.stride(0), dyq.stride(1), dyk.data_ptr(), dyk.stride(0), dyk.stride(1),
            dq.data_ptr(), dk.data_ptr(), _ptr(dwq), _ptr(dwk), ws.data_ptr(), ws.numel(), _raw(torch, q.device)))
    return dq, dk, dwq, dwk


# ----------------------------------------------------------------- routing --

def _route_desc(logits, k, score, bias, groups, top_groups, group_score, renormalise, scale, torch):
    if not (isinstance(logits, torch.Tensor) and logits.is_cuda and logits.dtype in _DT and logits.dim() == 2):
        _tensor("logits", logits, torch, dim=2)
    if score not in SCORES:
        raise ValueError(f"score must be one of {sorted(SCORES)}")
    if group_score not in GROUP_SCORES:
        raise ValueError(f"group_score must be one of {sorted(GROUP_SCORES)}")
    T, E = logits.shape
    if bias is not None:
        _tensor("bias", bias, torch, (torch.float32,), 1)
        if bias.shape[0] != E or not bias.is_contiguous():
            raise ValueError("bias must be contiguous [experts]")
        _same_device(logits, bias)
    return _ROUTE(T, E, k, SCORES[score], groups, top_groups, GROUP_SCORES[group_score], 1 if renormalise else 0,
                  _DT[logits.dtype], scale, logits.data_ptr(), _rows("logits", logits), _ptr(bias))


def route(logits, k, *, score="softmax", bias=None, groups=1, top_groups=1, group_score="max", renormalise=False,
          scale=1.0, stream=None):
    """The k experts of every token and their weights.

    logits [T][experts] (rows may lie apart).  score "softmax" or "sigmoid"; `bias`
    [experts] float32 is added to the scores for the choice alone.  With groups > top_groups
    only the experts of the `top_groups` best of `groups` equal runs take part (a run's largest
    value, or with group_score "top2" the sum of its two largest scores, each with its bias).  Weights are the scores, over
    their sum with `renormalise`, times `scale`.  Returns (weight [T][k] float32, index [T][k]
    int32), best first, equal values by the lowest index.  A logit of -inf masks its expert;
    a place with no expert left has index -1 and weight 0."""
    torch = _torch()
    d = _route_desc(logits, k, score, bias, groups, top_groups, group_score, renormalise, scale, torch)
    device = logits.device
    if _recorded(torch, logits):
        from . import block_grad
        with _on(torch, device, stream):
            return block_grad.route(logits, k, {"bias": bias, "groups": groups, "top_groups": top_groups,
                                                "group_score": group_score},
                                    {"score": score, "renormalise": renormalise, "scale": scale}, stream)
    with _on(torch, device, stream):
        weight = torch.empty((logits.shape[0], k), dtype=torch.float32, device=device)
        index = torch.empty((logits.shape[0], k), dtype=torch.int32, device=device)
        rc = _lib.cfp_route(d, weight.data_ptr(), index.data_ptr(), _raw(torch, device))
    if rc:
        _check("cfp_route", rc)
    return weight, index


def route_bwd(dweight, logits, index, *, score="softmax", renormalise=False, scale=1.0, stream=None):
    """Gradient of route's weights in the logits [T][experts], from dweight [T][k] float32 and the index it returned."""
    torch = _torch()
    _tensor("index", index, torch, (torch.int32,), 2)
    _tensor("dweight", dweight, torch, (torch.float32,), 2)
    d = _route_desc(logits, index.shape[1], score, None, 1, 1, "max", renormalise, scale, torch)
    if index.shape[0] != logits.shape[0] or index.shape != dweight.shape:
        raise ValueError("index and dweight are [T][k]")
    _same_device(logits, index, dweight)
    with _on(torch, logits.device, stream):
        index, dweight = index.contiguous(), dweight.contiguous()
        dlogits = _like(torch, logits)
        _check("cfp_route_bwd", _lib.cfp_route_bwd(d, index.data_ptr(), dweight.data_ptr(), dlogits.data_ptr(),
                                                   _raw(torch, logits.device)))
    return dlogits


# ----------------------------------------------------------------- experts --

class ExpertPlan:
    """Order of the assignments a = token * k + place by expert.

    offsets [experts + 1] int32: the positions of each expert; rows [T * k] int32: the assignment at
    each position, -1 behind the last one kept; slot [T * k] int32: the position of each
    assignment, -1 where it is dropped."""

    __slots__ = ("_buf", "n_tokens", "k", "n_experts", "first")

    def __init__(self, buf, n_tokens, k, n_experts, first):
        self._buf, self.n_tokens, self.k, self.n_experts, self.first = buf, n_tokens, k, n_experts, first

    # places in the buffer: offsets, rows and CFP_PLAN_PAD entries, slot
    @property
    def offsets(self):
        return self._buf[:self.n_experts + 1]

    @property
    def rows(self):
        return self._buf[self.n_experts + 1:self.n_experts + 1 + self.n_tokens * self.k]

    @property
    def slot(self):
        at = self.n_experts + 1 + self.n_tokens * self.k + CFP_PLAN_PAD
        return self._buf[at:at + self.n_tokens * self.k]

    def _pointers(self):
        at, n = self._buf.data_ptr(), self.n_tokens * self.k
        rows = at + 4 * (self.n_experts + 1)
        return at, rows, rows + 4 * (n + CFP_PLAN_PAD)


def expert_plan(index, n_experts, *, first=0, stream=None) -> ExpertPlan:
    """Stable order of the assignments in index [T][k] int32 by expert.  The plan is for the
    experts first .. first + n_experts - 1 (a device's share of them); assignments to others, and negative ones, are dropped."""
    torch = _torch()
    _tensor("index", index, torch, (torch.int32,), 2)
    T, k = index.shape
    device = index.device
    with _on(torch, device, stream):
        index = index.contiguous()
        d = _PLAN(T, k, n_experts, first, index.data_ptr())
        need = _lib.cfp_expert_plan_workspace_bytes(d)
        size = max(n_experts, 0) + 1 + 2 * T * k + CFP_PLAN_PAD
        plan = ExpertPlan(torch.empty(size + need // 4, dtype=torch.int32, device=device), T, k, n_experts, first)
        offsets, rows, slot = plan._pointers()
        rc = _lib.cfp_expert_plan(d, offsets, rows, slot, offsets + 4 * size, need, _raw(torch, device))
    if rc:
        _check("cfp_expert_plan", rc)
    return plan


def _experts_refuse(x, w1, w2, weight, plan, torch):
    """Raises what is wrong with the arguments."""
    half = (torch.float16, torch.bfloat16)
    _tensor("x", x, torch, half, 2)
    _tensor("w1", w1, torch, half, 3)
    _tensor("w2", w2, torch, half, 3)
    _tensor("weight", weight, torch, (torch.float32,), 2)
    T, H = x.shape
    E, _, F = w2.shape
    if w1.shape != (E, 2 * F, H) or w2.shape[1] != H:
        raise ValueError("w1 is [experts][2 * inner][hidden] and w2 is [experts][hidden][inner]")
    if w1.dtype != x.dtype or w2.dtype != x.dtype:
        raise TypeError("x, w1 and w2 must be of one type")
    if not (w1.is_contiguous() and w2.is_contiguous() and weight.is_contiguous()):
        raise ValueError("w1, w2 and weight must be contiguous")
    if not isinstance(plan, ExpertPlan) or (plan.n_tokens, plan.n_experts) != (T, E) or weight.shape != (T, plan.k):
        raise ValueError("the plan is of another number of tokens, experts or places than x, w1 and weight")
    _same_device(x, w1, w2, weight, plan._buf)
    _rows("x", x)


def _experts_desc(x, w1, w2, weight, plan, torch):
    # one pass over what has to hold, on the way of every call; what does not hold is said by _experts_refuse
    try:
        at, dt = x.get_device(), x.dtype
        (T, H), (E, H2, F), (ld, one) = x.shape, w2.shape, x.stride()
        ok = (at >= 0 and dt is not torch.float32 and w1.dtype is dt and w2.dtype is dt and weight.dtype is torch.float32 and
              w1.shape == (E, 2 * F, H) and H2 == H and weight.shape == (T, plan.k) and plan.n_tokens == T and
              plan.n_experts == E and w1.get_device() == at and w2.get_device() == at and weight.get_device() == at and
              plan._buf.get_device() == at and w1.is_contiguous() and w2.is_contiguous() and weight.is_contiguous() and
              (one == 1 or H == 1))
        kind = _DT[dt]
    except (AttributeError, KeyError, TypeError, ValueError):
        ok = False
    if not ok:
        _experts_refuse(x, w1, w2, weight, plan, torch)
        raise ValueError("unsupported arguments")
    return _EXPERTS(T, plan.k, E, H, F, kind, x.data_ptr(), ld if T > 1 else H, w1.data_ptr(), w2.data_ptr(),
                    weight.data_ptr(), *plan._pointers())


def experts(x, w1, w2, weight, plan, *, keep=False, ws=None, stream=None):
    """y [T][hidden]: for every token the sum over its assignments in `plan` of
    weight * W2 (silu(gate) * up), [gate up] = W1 x.

    x [T][hidden] (rows may lie apart), w1 [experts][2 * inner][hidden] (gate rows, then
    up rows), w2 [experts][hidden][inner], float16 or bfloat16; weight [T][k] float32.  A token
    without assignments gets zeros.  With `keep` returns (y, kept): kept is what experts_bwd needs, and is kept as well
    where gradients are recorded."""
    torch = _torch()
    d = _experts_desc(x, w1, w2, weight, plan, torch)
    if _recorded(torch, x, w1, w2, weight):
        from . import block_grad
        with _on(torch, x.device, stream):
            return block_grad.experts(x, w1, w2, weight, plan, keep, ws, stream)
    with _on(torch, x.device, stream):
        y = _like(torch, x)
        ws = _ws(torch, _lib.cfp_experts_workspace_bytes(d, 0), x.device, ws)
        kept = _ws(torch, _lib.cfp_experts_kept_bytes(d), x.device, None) if keep else None
        rc = _lib.cfp_experts(d, y.data_ptr(), _ptr(kept), ws.data_ptr(), ws.numel(), _raw(torch, x.device))
    if rc:
        _check("cfp_experts", rc)
    return (y, kept) if keep else y


def experts_bwd(dy, x, w1, w2, weight, plan, kept, *, ws=None, stream=None):
    """Gradients of experts from dy [T][hidden] and what it kept: (dx, dw1, dw2, dweight).
    An expert without assignments gets zeros, and a dropped assignment's weight 0."""
    torch = _torch()
    d = _experts_desc(x, w1, w2, weight, plan, torch)
    _tensor("dy", dy, torch, (x.dtype,), 2)
    if dy.shape != x.shape:
        raise ValueError("dy must have the shape of x")
    _same_device(x, dy)
    if not isinstance(kept, torch.Tensor) or kept.dtype != torch.uint8:
        raise TypeError("kept must be what experts returned")
    if kept.device != x.device or not kept.is_contiguous() or kept.numel() < _lib.cfp_experts_kept_bytes(d):
        raise ValueError("kept is not what experts returned for these sizes")
    if kept.data_ptr() % 16:
        raise ValueError("kept must start on 16 bytes")
    with _on(torch, x.device, stream):
        dx, dw1, dw2 = _like(torch, x), torch.empty_like(w1), torch.empty_like(w2)
        dweight = torch.empty_like(weight)
        ws = _ws(torch, _lib.cfp_experts_workspace_bytes(d, 1), x.device, ws)
        _check("cfp_experts_bwd", _lib.cfp_experts_bwd(
            d, dy.data_ptr(), _rows("dy", dy), kept.data_ptr(), dx.data_ptr(), dw1.data_ptr(), dw2.data_ptr(),
            dweight.data_ptr(), ws.data_ptr(), ws.numel(), _raw(torch, x.device)))
    return dx, dw1, dw2, dweight
