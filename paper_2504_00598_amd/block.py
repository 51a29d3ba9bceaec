"""Operators of a decoder block: what the blocks of a searched chain run.

    from paper_2504_00598_amd import block
    q, k = block.qk_norm_rope(q, k, wq, wk, cos, sin, positions)
    weight, index = block.route(logits, 8, score="sigmoid", bias=bias, groups=8, top_groups=4, group_score="top2")
    plan = block.expert_plan(index, n_experts)
    y = block.experts(x, w1, w2, weight, plan)

    cache = block.KVCache.empty(pages, 64, key_heads, dim, torch.float8_e4m3fn)
    seqs = block.Sequences(table, starts, lengths, max_new=1)
    block.cache_write(cache, k, v, seqs)
    y = block.attend(q, cache, seqs)

The first three have their gradient beside them (`*_bwd`), and where gradients are recorded and an input requires one, backward()
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

CFP_DT_F32, CFP_DT_F16, CFP_DT_BF16, CFP_DT_E4M3 = 0, 1, 2, 3
CFP_QK_MAX_AXES = 4
SCORES = {"softmax": 0, "sigmoid": 1}
CFP_PLAN_PAD = 16  # entries behind the last of a plan's rows
GROUP_SCORES = {"max": 0, "top2": 1}

EXPORTED = ("cfp_qk_norm_rope", "cfp_qk_workspace_bytes", "cfp_qk_norm_rope_bwd", "cfp_route", "cfp_route_bwd",
            "cfp_expert_plan_workspace_bytes", "cfp_expert_plan", "cfp_experts_kept_bytes",
            "cfp_experts_workspace_bytes", "cfp_experts", "cfp_experts_bwd", "cfp_qk_norm_rope_axes",
            "cfp_qk_norm_rope_axes_bwd", "cfp_cache_write", "cfp_cache_read", "cfp_attend_workspace_bytes", "cfp_attend")

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


class cfp_cache_desc(ctypes.Structure):
    _fields_ = [("n_pages", _I64), ("page", _I32), ("heads", _I32), ("dim", _I32), ("dtype", _I32), ("k", _P), ("v", _P),
                ("k_scale", _P), ("v_scale", _P), ("k_page_stride", _I64), ("v_page_stride", _I64),
                ("k_scale_page_stride", _I64), ("v_scale_page_stride", _I64)]


class cfp_sequences_desc(ctypes.Structure):
    _fields_ = [("n_seqs", _I32), ("width", _I32), ("table", _P), ("table_stride", _I64), ("starts", _P), ("lengths", _P),
                ("max_new", _I32)]


class cfp_attend_desc(ctypes.Structure):
    _fields_ = [("n_tokens", _I64), ("n_q", _I32), ("dtype", _I32), ("q", _P), ("q_token_stride", _I64),
                ("q_head_stride", _I64), ("scale", _F32), ("causal", _I32), ("window", _I32)]


# The same layouts for struct.pack: filling a ctypes structure of 21 fields takes 3 us, packing it 0.6 (a small
# launch takes 3).  A packed descriptor is passed by the address of its bytes.
_CODES = {_I64: "q", _I32: "i", _F32: "f", _P: "P"}
_QK, _ROUTE, _PLAN, _EXPERTS, _CACHE, _SEQUENCES, _ATTEND = (
    struct.Struct("@" + "".join(_CODES[t] for _, t in c._fields_) + "0q").pack
    for c in (cfp_qk_desc, cfp_route_desc, cfp_plan_desc, cfp_experts_desc, cfp_cache_desc, cfp_sequences_desc,
              cfp_attend_desc))

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
                           ("cfp_experts_kept_bytes", [_P]), ("cfp_experts_workspace_bytes", [_P, _I32]),
                           ("cfp_attend_workspace_bytes", [_P, _P, _P])):
            getattr(L, name).argtypes, getattr(L, name).restype = args, SZ
        for name, args in (("cfp_qk_norm_rope", [_P, _P, _P, _P]),
                           ("cfp_qk_norm_rope_bwd", [_P, _P, _I64, _I64, _P, _I64, _I64, _P, _P, _P, _P, _P, SZ, _P]),
                           ("cfp_route", [_P, _P, _P, _P]), ("cfp_route_bwd", [_P, _P, _P, _P, _P]),
                           ("cfp_expert_plan", [_P, _P, _P, _P, _P, SZ, _P]),
                           ("cfp_experts", [_P, _P, _P, _P, SZ, _P]),
                           ("cfp_experts_bwd", [_P, _P, _I64, _P, _P, _P, _P, _P, _P, SZ, _P]),
                           ("cfp_qk_norm_rope_axes", [_P, _P, _I32, _P, _P, _P]),
                           ("cfp_qk_norm_rope_axes_bwd", [_P, _P, _I32, _P, _I64, _I64, _P, _I64, _I64, _P, _P, _P, _P, _P,
                                                          SZ, _P]),
                           ("cfp_cache_write", [_P, _P, _I64, _I32, _P, _I64, _I64, _P, _I64, _I64, _P]),
                           ("cfp_cache_read", [_P, _P, _I64, _I32, _P, _P, _P]),
                           ("cfp_attend", [_P, _P, _P, _P, _P, _P, SZ, _P])):
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

def _qk_refuse(q, k, wq, wk, cos, sin, positions, axes, torch):
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
    if axes is not None:
        if positions is None:
            raise ValueError("axes need positions of each axis")
        _tensor("positions", positions, torch, (torch.int32,), 2)
        if positions.shape[1] != T or not positions.is_contiguous() or not 1 <= positions.shape[0] <= CFP_QK_MAX_AXES:
            raise ValueError(f"positions must be contiguous [axes][T], of at most {CFP_QK_MAX_AXES} axes")
        if len(axes) != cos.shape[1] or any(a not in range(positions.shape[0]) for a in axes):
            raise ValueError("axes must name an axis of positions for each rotated pair")
    elif positions is not None:
        _tensor("positions", positions, torch, (torch.int32,), 1)
        if positions.shape[0] != T or not positions.is_contiguous():
            raise ValueError("positions must be contiguous [T]")
    elif cos.shape[1] and T > cos.shape[0]:
        raise ValueError("without positions the tables must hold a row for every token")
    _same_device(q, k, wq, wk, cos, sin, positions)


def _qk_desc(q, k, wq, wk, cos, sin, positions, eps, interleaved, axes, torch):
    """The packed descriptor, and with axes that of each pair in a byte."""
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
        pairs = None
        if positions is None:
            ok = ok and axes is None and (T <= cos.shape[0] or half == 0)
        elif axes is not None:
            pairs = bytes([*axes])
            ok = ok and (positions.dtype is torch.int32 and positions.dim() == 2 and positions.shape[1] == T and
                         positions.get_device() == at and positions.is_contiguous() and len(pairs) == half and
                         1 <= positions.shape[0] <= CFP_QK_MAX_AXES and max(pairs, default=0) < positions.shape[0])
        else:
            ok = ok and (positions.dtype is torch.int32 and positions.numel() == T and positions.dim() == 1 and
                         positions.get_device() == at and positions.is_contiguous())
        w = wq if wq is not None else wk
        types = _DT[q.dtype], CFP_DT_F32 if w is None else _DT[w.dtype]
    except (AttributeError, KeyError, IndexError, TypeError, ValueError):
        ok = False
    if not ok:
        _qk_refuse(q, k, wq, wk, cos, sin, positions, axes, torch)
        raise ValueError("unsupported arguments")
    return _QK(T, hq, k.shape[1], D, 2 * half, 1 if interleaved else 0, *types, eps, cos.shape[0], q.data_ptr(),
               k.data_ptr(), qt, qh, kt, kh, _ptr(wq), _ptr(wk), cos.data_ptr(), sin.data_ptr(), _ptr(positions)), pairs


def qk_norm_rope(q, k, wq, wk, cos, sin, positions=None, *, eps=1e-6, interleaved=False, axes=None, stream=None):
    """Norm and rotation of queries and keys in one pass.

    q [T][heads][D] and k [T][key heads][D] may be views of a larger product (last
    dimension contiguous).  Each head is divided by sqrt(mean(x^2) + eps), times its
    gain wq or wk [D] (None: ones), and its first 2 * cos.shape[1] entries are rotated by
    the angles of row positions[t] of the tables cos, sin [positions][rotated / 2]
    (None: row t): pairs (i, i + rotated / 2), or with `interleaved` (2i, 2i + 1).  With `axes`, the axis of each pair
    (a sequence of rotated / 2 numbers), pair i turns by row positions[axes[i]][t], positions [axes][T].  A position outside
    the tables makes the entries that it rotates NaN.  Returns contiguous (q, k) of q's type."""
    torch = _torch()
    d, pairs = _qk_desc(q, k, wq, wk, cos, sin, positions, eps, interleaved, axes, torch)
    if _recorded(torch, q, k, wq, wk, cos, sin):
        from . import block_grad
        with _on(torch, q.device, stream):
            return block_grad.qk_norm_rope(q, k, wq, wk, cos, sin, positions, eps, interleaved, stream, axes)
    with _on(torch, q.device, stream):
        yq, yk = _like(torch, q), _like(torch, k)
        if pairs is None:
            rc = _lib.cfp_qk_norm_rope(d, yq.data_ptr(), yk.data_ptr(), _raw(torch, q.device))
        else:
            rc = _lib.cfp_qk_norm_rope_axes(d, pairs, positions.shape[0], yq.data_ptr(), yk.data_ptr(),
                                            _raw(torch, q.device))
    if rc:
        _check("cfp_qk_norm_rope", rc)
    return yq, yk


def qk_norm_rope_bwd(dyq, dyk, q, k, wq, wk, cos, sin, positions=None, *, eps=1e-6, interleaved=False, axes=None,
                     ws=None, stream=None):
    """Gradients of qk_norm_rope in q, k, wq and wk from those of its results (the inputs
    as they were given to it).  Returns (dq, dk, dwq, dwk); dwq and dwk are float32, None for a gain of None."""
    torch = _torch()
    d, pairs = _qk_desc(q, k, wq, wk, cos, sin, positions, eps, interleaved, axes, torch)
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
        rest = (dyq.data_ptr(), dyq.stride(0), dyq.stride(1), dyk.data_ptr(), dyk.stride(0), dyk.stride(1),
                dq.data_ptr(), dk.data_ptr(), _ptr(dwq), _ptr(dwk), ws.data_ptr(), ws.numel(), _raw(torch, q.device))
        _check("cfp_qk_norm_rope_bwd", _lib.cfp_qk_norm_rope_bwd(d, *rest) if pairs is None else
               _lib.cfp_qk_norm_rope_axes_bwd(d, pairs, positions.shape[0], *rest))
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


# --------------------------------------------- past tokens and attention --

class KVCache:
    """Keys and values of past tokens in pages.

    k [pages][heads][page][dim] and v [pages][heads][dim][page], float16, bfloat16 or float8_e4m3fn; the last with
    k_scale, v_scale [pages][heads][page] uint8: an entry stands for itself times 2^(scale - 127), scales from 1 to 254.  Pages may lie apart (a
    view of a larger tensor), what is in one is contiguous.  page is 16, 32, 64, 128 or 256, dim a multiple of 16 up to 256."""

    __slots__ = ("k", "v", "k_scale", "v_scale", "_desc", "_held", "_heads", "_dim", "_at")

    def __init__(self, k, v, k_scale=None, v_scale=None):
        torch = _torch()
        byte = getattr(k, "dtype", None) is torch.float8_e4m3fn
        held = {torch.float16: CFP_DT_F16, torch.bfloat16: CFP_DT_BF16, torch.float8_e4m3fn: CFP_DT_E4M3}
        for name, t in (("k", k), ("v", v)):
            _tensor(name, t, torch, held, 4)
        (n, h, page, d), device = k.shape, k.device
        if v.dtype != k.dtype or v.shape != (n, h, d, page):
            raise ValueError("k is [pages][heads][page][dim] and v is [pages][heads][dim][page], of one type")
        if byte != (k_scale is not None) or byte != (v_scale is not None):
            raise ValueError("k_scale and v_scale go with float8_e4m3fn")
        strides = []
        for name, t in (("k", k), ("v", v)) + ((("k_scale", k_scale), ("v_scale", v_scale)) if byte else ()):
            if name in ("k_scale", "v_scale"):
                _tensor(name, t, torch, (torch.uint8,), 3)
                if t.shape != (n, h, page):
                    raise ValueError(f"{name} must be [pages][heads][page]")
            if n and not t[0].is_contiguous():
                raise ValueError(f"{name}: what is in a page must be contiguous")
            strides.append(t.stride(0) if n > 1 else t[0].numel() if n else 0)
        _same_device(k, v, k_scale, v_scale)
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self._held, self._heads, self._dim, self._at = k.dtype, h, d, k.get_device()
        self._desc = _CACHE(n, page, h, d, held[k.dtype], k.data_ptr(), v.data_ptr(), _ptr(k_scale), _ptr(v_scale),
                            *(strides + [0, 0])[:4])

    @classmethod
    def empty(cls, pages, page, heads, dim, dtype, device="cuda"):
        """A cache of its own; what its pages hold is unspecified until it is written."""
        import torch

        k = torch.empty((pages, heads, page, dim), dtype=dtype, device=device)
        v = torch.empty((pages, heads, dim, page), dtype=dtype, device=device)
        if dtype is not torch.float8_e4m3fn:
            return cls(k, v)
        return cls(k, v, *(torch.empty((pages, heads, page), dtype=torch.uint8, device=device) for _ in range(2)))

    def _tensors(self):
        return self.k, self.v, self.k_scale, self.v_scale


class Sequences:
    """Which rows of a call are which tokens of which sequence, and where these lie in a cache.

    Rows starts[b] .. starts[b + 1] - 1 are the last tokens of sequence b, which has lengths[b] with them; its token p is in
    page table[b][p // page].  table [sequences][width], starts [sequences + 1] and lengths [sequences] are
    int32 on the GPU and are read when the kernels run: a captured call follows what a program writes into them.  starts
    ascends; rows outside it belong to no sequence.  max_new: the most rows that a sequence has, or
    more (None: any number); attend lays its work out for it, and for table's width."""

    __slots__ = ("table", "starts", "lengths", "max_new", "_desc", "_at")

    def __init__(self, table, starts, lengths, *, max_new=None):
        torch = _torch()
        _tensor("table", table, torch, (torch.int32,), 2)
        _tensor("starts", starts, torch, (torch.int32,), 1)
        _tensor("lengths", lengths, torch, (torch.int32,), 1)
        n, width = table.shape
        if starts.shape[0] != n + 1 or lengths.shape[0] != n:
            raise ValueError("table is [sequences][width], starts [sequences + 1] and lengths [sequences]")
        if not starts.is_contiguous() or not lengths.is_contiguous():
            raise ValueError("starts and lengths must be contiguous")
        _same_device(table, starts, lengths)
        if max_new is not None and max_new < 0:
            raise ValueError("max_new must not be negative")
        self.table, self.starts, self.lengths, self.max_new, self._at = table, starts, lengths, max_new, table.get_device()
        most = 0x7FFFFFFF if max_new is None else min(max_new, 0x7FFFFFFF)
        self._desc = _SEQUENCES(n, width, table.data_ptr(), _rows("table", table), starts.data_ptr(), lengths.data_ptr(), most)

    def _tensors(self):
        return self.table, self.starts, self.lengths


def _paged(torch, cache, seqs):
    """Checks what the operators over a cache share."""
    if not isinstance(cache, KVCache):
        raise TypeError("cache must be a KVCache")
    if not isinstance(seqs, Sequences):
        raise TypeError("seqs must be Sequences")
    if seqs._at != cache._at:
        raise ValueError("all tensors must be on one device")


def _rows_fit(t, cache):
    """Whether t is rows of heads of the cache's dim and a type that it takes, on its device."""
    return (t.get_device() == cache._at and t.dim() == 3 and t.shape[2] == cache._dim and t.stride(2) == 1 and
            (t.dtype is cache._held or (cache._held not in _DT and t.dtype in _DT and _DT[t.dtype] != CFP_DT_F32)))


def _rows_refuse(name, t, torch, cache):
    """Raises what is wrong with such rows."""
    _tensor(name, t, torch, (torch.float16, torch.bfloat16), 3)
    if t.shape[2] != cache._dim or t.stride(2) != 1:
        raise ValueError(f"{name} must be [T][heads][dim] with the cache's dim, the last dimension contiguous")
    if cache._held in _DT and t.dtype is not cache._held:
        raise TypeError(f"{name} must be of the cache's type")
    _same_device(cache.k, t)


def _no_gradient(torch, name, *inputs):
    if _recorded(torch, *inputs):
        raise RuntimeError(f"{name} has no gradient: call it under torch.no_grad()")


def _used_on(stream, *tensors):
    """The caching allocator hands memory out again in the order of the stream it was allocated on."""
    if stream is not None:
        for t in tensors:
            if t is not None:
                t.record_stream(stream)


def cache_write(cache, k, v, seqs, *, stream=None):
    """Writes k and v [T][heads][dim] (views with a contiguous last dimension) to their sequences' places in the cache.

    A cache of 16 bits is of their type.  One of float8_e4m3fn gets for each token and head the least power of two under
    which no finite entry passes 448, and every entry over it rounded to the nearest; infinities and NaN become NaN.  A token
    whose page is not one of the cache's is not written.  Two rows must not have one place."""
    torch = _torch()
    _paged(torch, cache, seqs)
    for name, t in (("k", k), ("v", v)):
        if not isinstance(t, torch.Tensor) or not _rows_fit(t, cache):
            _rows_refuse(name, t, torch, cache)
            raise ValueError("unsupported arguments")
    T, heads, _ = k.shape
    if heads != cache._heads or v.shape != k.shape or v.dtype is not k.dtype:
        raise ValueError("k and v are [T][the cache's heads][dim], of one type")
    _no_gradient(torch, "cache_write", k, v)
    if stream is not None:
        _used_on(stream, k, v, *cache._tensors(), *seqs._tensors())
    (kt, kh, _), (vt, vh, _), device = k.stride(), v.stride(), k.device
    with _on(torch, device, stream):
        rc = _lib.cfp_cache_write(cache._desc, seqs._desc, T, _DT[k.dtype], k.data_ptr(), kt, kh, v.data_ptr(), vt, vh,
                                  _raw(torch, device))
    if rc:
        _check("cfp_cache_write", rc)


def cache_read(cache, seqs, n_tokens, *, dtype=None, out=None, stream=None):
    """The tokens of `seqs` back from the cache, as the values that they stand for: (k, v) [n_tokens][heads][dim] of the
    cache's type, or of `dtype` (float8_e4m3fn: bfloat16, or float16, to which what bfloat16 rows wrote is rounded, beyond its
    range to an infinity).  With starts as the sums of lengths these are whole sequences.  A token whose page is not one of the cache's reads as NaN.  Rows of no sequence are left as they
    are: unspecified, or with out=(k, v) what these held."""
    torch = _torch()
    _paged(torch, cache, seqs)
    held, device = cache._held, cache.k.device
    if dtype is None:
        dtype = held if held in _DT else torch.bfloat16
    if dtype is not held and (held in _DT or dtype not in (torch.float16, torch.bfloat16)):
        raise TypeError("dtype must be the cache's, or float16 or bfloat16 of float8_e4m3fn")
    if n_tokens < 0:
        raise ValueError("n_tokens must not be negative")
    shape = (n_tokens, cache._heads, cache._dim)
    if out is not None:
        for name, t in zip(("k", "v"), out, strict=True):
            _tensor(name, t, torch, (dtype,), 3)
            if t.shape != shape or not t.is_contiguous():
                raise ValueError("out must be contiguous [n_tokens][heads][dim]")
        _same_device(cache.k, *out)
        _used_on(stream, *out)
    if stream is not None:
        _used_on(stream, *cache._tensors(), *seqs._tensors())
    with _on(torch, device, stream):
        k, v = out if out is not None else (torch.empty(shape, dtype=dtype, device=device) for _ in range(2))
        rc = _lib.cfp_cache_read(cache._desc, seqs._desc, n_tokens, _DT[dtype], k.data_ptr(), v.data_ptr(), _raw(torch, device))
    if rc:
        _check("cfp_cache_read", rc)
    return k, v


def attend(q, cache, seqs, *, scale=None, causal=True, window=0, with_lse=False, out=None, ws=None, stream=None):
    """Attention of new tokens over a cache that holds them and those before them.

    q [T][heads][dim] (a view with a contiguous last dimension), heads a multiple of the cache's: head h reads head
    h // (heads / cache heads).  A row that is token p of its sequence sees the tokens up to p, or all without `causal`, and with a
    window > 0 none before p - window + 1.  Its result is the mean of their values weighted by exp(scale q . k)
    (scale > 0; None: 1 / sqrt(dim)).  Returns [T][heads][dim] of q's type, or with `with_lse` also the logarithm of the
    sum of the weights, [T][heads] float32, by which results over parts of a context are joined.  A row that sees nothing, or only scores
    of -infinity, gets zeros and -inf; what it does not see has no effect on it, whatever its memory holds.  An infinite value that it sees
    leaves the entry infinite or NaN.  Keys and values of float8_e4m3fn are those that cache_read gives in q's type.  A row that sees a page outside the cache, a sequence
    longer than its table and one with more rows than max_new get NaN.  Rows of no sequence are left as they are: unspecified,
    or what `out` (or out=(y, lse) with `with_lse`) held."""
    torch = _torch()
    _paged(torch, cache, seqs)
    if not isinstance(q, torch.Tensor) or not _rows_fit(q, cache):
        _rows_refuse("q", q, torch, cache)
        raise ValueError("unsupported arguments")
    T, hq, dim = q.shape
    if hq == 0 or cache._heads == 0 or hq % cache._heads:
        raise ValueError("q's heads must be a multiple of the cache's")
    if scale is None:
        scale = dim ** -0.5
    _no_gradient(torch, "attend", q)
    device = q.device
    y, lse = out if with_lse and out is not None else (out, None)
    if out is not None:
        _tensor("out", y, torch, (q.dtype,), 3)
        if y.shape != q.shape or not y.is_contiguous():
            raise ValueError("out must be contiguous, of q's shape")
        if with_lse:
            _tensor("lse", lse, torch, (torch.float32,), 2)
            if lse.shape != (T, hq) or not lse.is_contiguous():
                raise ValueError("lse must be contiguous [T][heads]")
        _same_device(q, y, lse)
        _used_on(stream, y, lse)
    tok, head, _ = q.stride()
    d = _ATTEND(T, hq, _DT[q.dtype], q.data_ptr(), tok, head, scale, 1 if causal else 0,
                window if 0 <= window < 1 << 31 else -1 if window < 0 else 0x7FFFFFFF)
    if stream is not None:
        _used_on(stream, q, ws, *cache._tensors(), *seqs._tensors())
    with _on(torch, device, stream):
        if out is None:
            y = torch.empty(q.shape, dtype=q.dtype, device=device)
            lse = torch.empty((T, hq), dtype=torch.float32, device=device) if with_lse else None
        need = _lib.cfp_attend_workspace_bytes(d, cache._desc, seqs._desc)
        if need or ws is not None:
            ws = _ws(torch, need, device, ws)
        rc = _lib.cfp_attend(d, cache._desc, seqs._desc, y.data_ptr(), _ptr(lse), _ptr(ws), 0 if ws is None else ws.numel(),
                             _raw(torch, device))
    if rc:
        _check("cfp_attend", rc)
    return (y, lse) if with_lse else y
