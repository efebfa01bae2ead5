"""The operators of a transformer block around its int8 linears (C ABI in include/nmspmm.h).

* `quantize_rows`: int8 codes of activation rows with a scale for each token.
* `norm_residual`, `norm_residual_i8`, `norm_residual_backward`: the norm after a block, its gate and residual scale,
  and the norm before the next block in one pass; with int8 codes in place of the normalised rows; and the gradients.

Tensors are device tensors of float16, bfloat16 or float32, [..., channels] with consecutive channels; two-dimensional
inputs may have any row stride.  Parameters are float32.  Every call enqueues its kernels on `stream` (a
torch.cuda.Stream; the current one without it) and returns; outputs that are not given are allocated for that stream.
There is no fallback: a missing library raises.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

from .nmspmm import NmError, _check, _need, _ptr, _stream, _torch, lib  # noqa: F401 (NmError: raised to callers)

NM_TYPE_F16, NM_TYPE_BF16, NM_TYPE_F32 = 1, 2, 3
NM_NORM_NONE, NM_NORM_RMS, NM_NORM_LAYER = 0, 1, 2
_NORMS = {"none": NM_NORM_NONE, "rms": NM_NORM_RMS, "layer": NM_NORM_LAYER}
_types = None


def _type_of(t, name: str) -> int:
    global _types
    if _types is None:
        torch = _torch()
        _types = {torch.float16: NM_TYPE_F16, torch.bfloat16: NM_TYPE_BF16, torch.float32: NM_TYPE_F32}
    code = _types.get(t.dtype)
    if code is None:
        raise ValueError(f"{name}: dtype {t.dtype}, expected float16, bfloat16 or float32")
    return code


def _rows(t, name: str, width: Optional[int] = None):
    """(t as [rows x channels], its row stride); refuses what has no such view."""
    if t.dim() != 2:
        if t.dim() == 0 or not t.is_contiguous():
            raise ValueError(f"{name}: must be two-dimensional, or contiguous with channels last")
        t = t.view(-1, t.shape[-1])
    m, k = t.shape
    if width is not None and k != width:
        raise ValueError(f"{name}: {k} channels, expected {width}")
    if k > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}: channels must be consecutive")
    return t, (t.stride(0) if m > 1 else max(k, 1))


def _same(t, name: str, like):
    if t.dtype != like.dtype:
        raise ValueError(f"{name}: dtype {t.dtype}, expected {like.dtype}")
    if t.device != like.device:
        raise ValueError(f"{name}: on {t.device}, expected {like.device}")


def _on_current_device(t, name: str):
    if not t.is_cuda:
        raise ValueError(f"{name}: must be a device tensor")
    if t.get_device() != _torch().cuda.current_device():
        raise ValueError(f"{name}: on {t.device}, but the current device is {_torch().cuda.current_device()}")


def _empty(shape, dtype, like, stream):
    """Memory of the call's stream: torch's allocator orders its reuse there."""
    torch = _torch()
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=like.device)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(stream.cuda_stream, device=like.device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=like.device)


def _output(given, name: str, shape, dtype, like, stream):
    if given is None:
        return _empty(shape, dtype, like, stream)
    _need(given, name, (dtype,), shape)
    if given.device != like.device:
        raise ValueError(f"{name}: on {given.device}, expected {like.device}")
    return given


def padded(k: int) -> int:
    """Row length of int8 codes of k channels: a multiple of 16."""
    return (k + 15) & ~15


# ---------------------------------------------------------------- row codes

def quantize_rows(x, xq=None, scale=None, stream=None):
    """nm_quantize_rows: (codes int8 [rows x padded(k)], scales float32 [rows]) of x."""
    _on_current_device(x, "x")
    code = _type_of(x, "x")
    x, ld = _rows(x, "x")
    m, k = x.shape
    torch = _torch()
    xq = _output(xq, "xq", (m, padded(k)), torch.int8, x, stream)
    scale = _output(scale, "scale", (m,), torch.float32, x, stream)
    _check(lib().nm_quantize_rows(x.data_ptr(), ld, code, m, k, xq.data_ptr(), scale.data_ptr(), _stream(stream)),
           "nm_quantize_rows")
    return xq, scale


# ---------------------------------------------------------------- norms around a block

class NmNorm(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("eps", ctypes.c_float), ("weight", ctypes.c_void_p),
                ("bias", ctypes.c_void_p)]


class NmNormArgs(ctypes.Structure):
    _fields_ = [("y", ctypes.c_void_p), ("r", ctypes.c_void_p), ("ldy", ctypes.c_int64), ("ldr", ctypes.c_int64),
                ("type", ctypes.c_int32), ("m", ctypes.c_int32), ("d", ctypes.c_int32), ("groups", ctypes.c_int32),
                ("gate", ctypes.c_void_p), ("alpha", ctypes.c_float), ("post", NmNorm), ("pre", NmNorm),
                ("res", ctypes.c_void_p), ("z", ctypes.c_void_p), ("zq", ctypes.c_void_p), ("zs", ctypes.c_void_p)]


class NmNormGradArgs(ctypes.Structure):
    _fields_ = [("y", ctypes.c_void_p), ("res", ctypes.c_void_p), ("dz", ctypes.c_void_p), ("dres", ctypes.c_void_p),
                ("ldy", ctypes.c_int64), ("ldres", ctypes.c_int64), ("lddz", ctypes.c_int64),
                ("lddres", ctypes.c_int64), ("type", ctypes.c_int32), ("m", ctypes.c_int32), ("d", ctypes.c_int32),
                ("groups", ctypes.c_int32), ("gate", ctypes.c_void_p), ("alpha", ctypes.c_float), ("post", NmNorm),
                ("pre", NmNorm), ("dy", ctypes.c_void_p), ("dr", ctypes.c_void_p), ("dgate", ctypes.c_void_p),
                ("dpre_weight", ctypes.c_void_p), ("dpre_bias", ctypes.c_void_p), ("dpost_weight", ctypes.c_void_p),
                ("dpost_bias", ctypes.c_void_p)]


class Norm:
    """A norm of the channels: kind "rms" or "layer", float32 weight and bias [d] (None: 1 and 0), eps."""

    def __init__(self, kind: str, weight=None, bias=None, eps: float = 1e-6):
        if kind not in ("rms", "layer"):
            raise ValueError(f"norm: kind {kind!r}, expected 'rms' or 'layer'")
        if not eps > 0:
            raise ValueError("norm: eps must be positive")
        self.kind, self.weight, self.bias, self.eps = kind, weight, bias, float(eps)

    def _args(self, d: int, like, name: str) -> NmNorm:
        torch = _torch()
        for t, what in ((self.weight, "weight"), (self.bias, "bias")):
            if t is not None:
                _need(t, f"{name}.{what}", (torch.float32,), (d,))
                if t.device != like.device:
                    raise ValueError(f"{name}.{what}: on {t.device}, expected {like.device}")
        return NmNorm(_NORMS[self.kind], self.eps, _ptr(self.weight), _ptr(self.bias))


def _norm_args(norm: Optional[Norm], d, like, name) -> NmNorm:
    return NmNorm() if norm is None else norm._args(d, like, name)


def _gate(gate, m: int, d: int, like) -> int:
    """Checks the gate [groups x d] (or [d]) and returns groups."""
    if gate is None:
        return 1
    torch = _torch()
    groups = gate.shape[0] if gate.dim() == 2 else 1
    _need(gate, "gate", (torch.float32,), (groups, d) if gate.dim() == 2 else (d,))
    if gate.device != like.device:
        raise ValueError(f"gate: on {gate.device}, expected {like.device}")
    if groups < 1 or m % groups:
        raise ValueError(f"gate: {groups} groups do not divide {m} tokens")
    return groups


def _around(y, r, pre, post, gate, alpha, res, stream):
    like, name = (y, "y") if y is not None else (r, "r")
    if like is None:
        raise ValueError("y and r: at least one is needed")
    _on_current_device(like, name)
    a = NmNormArgs()
    a.type = _type_of(like, name)
    shape, m, d = like.shape, 0, 0
    if y is not None:
        y2, a.ldy = _rows(y, "y")
        a.y = y2.data_ptr()
        m, d = y2.shape
    if r is not None:
        _same(r, "r", like)
        r2, a.ldr = _rows(r, "r", d if y is not None else None)
        if y is not None and r2.shape[0] != m:
            raise ValueError(f"r: {r2.shape[0]} tokens, expected {m}")
        a.r = r2.data_ptr()
        m, d = r2.shape
    a.m, a.d, a.groups, a.gate, a.alpha = m, d, _gate(gate, m, d, like), _ptr(gate), alpha
    a.post, a.pre = _norm_args(post, d, like, "post"), _norm_args(pre, d, like, "pre")
    res = _output(res, "res", shape, like.dtype, like, stream)
    a.res = res.data_ptr()
    return a, like, res


def norm_residual(y, r, pre: Optional[Norm] = None, post: Optional[Norm] = None, gate=None, alpha: float = 1.0,
                  res=None, z=None, stream=None):
    """nm_norm_residual: (res, z) with u = post(y), res = alpha r + gate u, z = pre(res).

    y (the block's output) or r (the residual stream) may be None.  gate: float32 [d], or [groups x d] with a row
    for each of `groups` equal runs of tokens.  Without `pre` there is no z (None)."""
    a, like, res = _around(y, r, pre, post, gate, alpha, res, stream)
    if pre is not None:
        z = _output(z, "z", res.shape, like.dtype, like, stream)
        a.z = z.data_ptr()
    elif z is not None:
        raise ValueError("z: given without a norm for it")
    _check(lib().nm_norm_residual(ctypes.byref(a), _stream(stream)), "nm_norm_residual")
    return res, z


def norm_residual_i8(y, r, pre: Norm, post: Optional[Norm] = None, gate=None, alpha: float = 1.0, res=None, zq=None,
                     zs=None, stream=None):
    """norm_residual with the codes of z and their scales in its place: (res, zq int8 [rows x padded(d)], zs)."""
    if pre is None:
        raise ValueError("pre: the codes are those of a norm's rows")
    a, like, res = _around(y, r, pre, post, gate, alpha, res, stream)
    torch = _torch()
    zq = _output(zq, "zq", (a.m, padded(a.d)), torch.int8, like, stream)
    zs = _output(zs, "zs", (a.m,), torch.float32, like, stream)
    a.zq, a.zs = zq.data_ptr(), zs.data_ptr()
    _check(lib().nm_norm_residual(ctypes.byref(a), _stream(stream)), "nm_norm_residual")
    return res, zq, zs


class NormGrads(NamedTuple):
    """Gradients of norm_residual's inputs; None where there is no such input."""
    dy: object
    dr: object
    dgate: object
    dpre_weight: object
    dpre_bias: object
    dpost_weight: object
    dpost_bias: object


def norm_residual_backward(dz, dres, y, res, pre: Optional[Norm] = None, post: Optional[Norm] = None, gate=None,
                           alpha: float = 1.0, stream=None) -> NormGrads:
    """nm_norm_residual_backward: the gradients at y and res (as norm_residual returned it) from dz and dres, either
    of which may be None.  Without y (a pass that had none) only the residual's side is computed."""
    like, name = (dz, "dz") if dz is not None else (dres, "dres")
    if like is None:
        raise ValueError("dz and dres: at least one is needed")
    if dz is not None and pre is None:
        raise ValueError("dz: given without its norm")
    _on_current_device(like, name)
    a = NmNormGradArgs()
    a.type = _type_of(like, name)
    flat, _ = _rows(like, name)
    m, d = flat.shape
    for t, what, ld in ((dz, "dz", "lddz"), (dres, "dres", "lddres"), (y, "y", "ldy"), (res, "res", "ldres")):
        if t is None:
            continue
        _same(t, what, like)
        t2, stride = _rows(t, what, d)
        if t2.shape[0] != m:
            raise ValueError(f"{what}: {t2.shape[0]} tokens, expected {m}")
        setattr(a, what, t2.data_ptr())
        setattr(a, ld, stride)
    if pre is not None and res is None:
        raise ValueError("res: needed for the gradient of its norm")
    if y is None and (post is not None or gate is not None):
        raise ValueError("y: needed for the gradients of its norm and gate")
    a.m, a.d, a.groups, a.gate, a.alpha = m, d, _gate(gate, m, d, like), _ptr(gate), alpha
    a.post, a.pre = _norm_args(post, d, like, "post"), _norm_args(pre, d, like, "pre")
    torch = _torch()
    f32 = torch.float32
    dy = _empty(like.shape, like.dtype, like, stream) if y is not None else None
    dr = _empty(like.shape, like.dtype, like, stream)
    dgate = _empty(gate.shape, f32, like, stream) if gate is not None else None
    params = []
    for norm in (pre, post):
        for t in (norm.weight, norm.bias) if norm is not None else (None, None):
            params.append(_empty((d,), f32, like, stream) if t is not None else None)
    a.dy, a.dr, a.dgate = _ptr(dy), _ptr(dr), _ptr(dgate)
    a.dpre_weight, a.dpre_bias, a.dpost_weight, a.dpost_bias = (_ptr(p) for p in params)
    need = ctypes.c_size_t()
    _check(lib().nm_norm_residual_backward_workspace(m, d, a.groups, ctypes.byref(need)),
           "nm_norm_residual_backward_workspace")
    ws = _empty((need.value,), torch.uint8, like, stream) if need.value else None
    _check(lib().nm_norm_residual_backward(ctypes.byref(a), _ptr(ws), need.value, _stream(stream)),
           "nm_norm_residual_backward")
    return NormGrads(dy, dr, dgate, *params)
