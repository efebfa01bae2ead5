"""The operators of a transformer block around its int8 linears (C ABI in include/nmspmm.h).

* `quantize_rows`: int8 codes of activation rows with a scale for each token.
* `linear_i8`, `gemm_i8_scaled`: the int8 product (dense or N:M weights) with scales for each token and channel, of
  activations or of codes already made; `ScaledWeight` holds its weight.
* `gated_ffn`, `gated_ffn_i8`, `gated_ffn_backward`: both projections of a gated feed-forward block, the activation and
  their product in one kernel, and the gradients; `GatedWeight` holds both weights.
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

from .nmspmm import (NM_LAYOUT_DENSE, DeviceWeight, NmDesc, NmError, _check, _need, _ptr, _stream, _torch,  # noqa: F401
                     compress, compress_size, lib)

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


# ---------------------------------------------------------------- scaled int8 products

NM_ACT_SILU, NM_ACT_GELU, NM_ACT_GELU_TANH, NM_ACT_RELU, NM_ACT_SIGMOID = range(1, 6)
_ACTS = {"silu": NM_ACT_SILU, "gelu": NM_ACT_GELU, "gelu_tanh": NM_ACT_GELU_TANH, "relu": NM_ACT_RELU,
         "sigmoid": NM_ACT_SIGMOID}


class NmScaledWeight(ctypes.Structure):
    _fields_ = [("desc", ctypes.POINTER(NmDesc)), ("vals", ctypes.c_void_p), ("meta", ctypes.c_void_p),
                ("scale", ctypes.c_void_p), ("bias", ctypes.c_void_p), ("n", ctypes.c_int32), ("k", ctypes.c_int32)]


class NmGatedGradArgs(ctypes.Structure):
    _fields_ = [("xq", ctypes.c_void_p), ("sx", ctypes.c_void_p), ("dh", ctypes.c_void_p), ("lddh", ctypes.c_int64),
                ("m", ctypes.c_int32), ("act", ctypes.c_int32), ("type", ctypes.c_int32), ("dx", ctypes.c_void_p),
                ("dw_gate", ctypes.c_void_p), ("dw_up", ctypes.c_void_p), ("dbias_gate", ctypes.c_void_p),
                ("dbias_up", ctypes.c_void_p)]


def _device_i8(W, name: str, device):
    torch = _torch()
    if not torch.is_tensor(W):
        W = torch.from_numpy(W)
    if W.dtype != torch.int8 or W.dim() != 2:
        raise ValueError(f"{name}: expected a two-dimensional int8 matrix")
    return W.to(device) if device is not None else W if W.is_cuda else W.cuda()


def _vector(v, name: str, n: int, like):
    torch = _torch()
    v = torch.as_tensor(v, dtype=torch.float32, device=like.device)
    if v.shape != (n,):
        raise ValueError(f"{name}: shape {tuple(v.shape)}, expected ({n},)")
    return v


def _pad(t, rows: int, cols: Optional[int] = None):
    """t with zeros up to `rows` (and `cols`), in memory of its own."""
    out = t.new_zeros((rows,) if cols is None else (rows, cols))
    if cols is None:
        out[:t.shape[0]] = t
    else:
        out[:t.shape[0], :t.shape[1]] = t
    return out


class ScaledWeight:
    """An int8 weight [n x k], dense or N:M, with a scale for each channel and optionally a bias, laid out for the
    kernels: made once, used by every call."""

    def __init__(self, weight: DeviceWeight, scale, bias, n: int, k: int):
        self.weight, self.scale, self.bias, self.n, self.k = weight, scale, bias, n, k
        self.device = weight.vals.device
        self._c = NmScaledWeight(ctypes.pointer(weight.desc), _ptr(weight.vals),
                                 _ptr(weight.meta) if weight.desc.meta_bytes else None, _ptr(scale), _ptr(bias), n, k)
        self._ref = ctypes.byref(self._c)
        self._needs = {}

    @staticmethod
    def _pack(W, rows: int, N: int, M: int) -> DeviceWeight:
        """W (a device matrix) packed with zeros up to `rows` rows and a multiple of 16 columns."""
        cols = padded(W.shape[1])
        desc = compress_size(rows, cols, N, M)
        if desc.layout == NM_LAYOUT_DENSE:
            return DeviceWeight(_pad(W, rows, cols).view(-1), W.new_empty(0).view(_torch().uint8), desc)
        return DeviceWeight.from_packed(compress(_pad(W, rows, cols).cpu().numpy(), N, M), W.device)

    @classmethod
    def from_int8(cls, W, scale, bias=None, N: int = 8, M: int = 8, device=None):
        """W int8 [n x k] (tensor or array) whose windows of M hold at most N nonzeros; scale and bias [n]."""
        W = _device_i8(W, "W", device)
        n, k = W.shape
        rows = (n + 15) & ~15
        return cls(cls._pack(W, rows, N, M), _pad(_vector(scale, "scale", n, W), rows),
                   None if bias is None else _pad(_vector(bias, "bias", n, W), rows), n, k)

    @classmethod
    def from_float(cls, W, bias=None):
        """A dense weight of codes of the rows of W (a device matrix), each channel with its own scale."""
        q, scale = quantize_rows(W)
        return cls.from_int8(q[:, :W.shape[1]], scale, bias)

    def _workspace(self, m: int, xtype: int, like, stream):
        need = self._needs.get((m, xtype))
        if need is None:      # a size by tokens and type: not a buffer
            size = ctypes.c_size_t()
            _check(lib().nm_linear_workspace(self._ref, m, xtype, ctypes.byref(size)), "nm_linear_workspace")
            if len(self._needs) > 256:
                self._needs.clear()
            need = self._needs[m, xtype] = size.value
        if not need:
            return None, 0
        return _empty((need,), _torch().uint8, like, stream), need


class GatedWeight(ScaledWeight):
    """Both projections of a gated block as one int8 weight, 16 gate channels and the same 16 up channels in turn."""

    def __init__(self, weight, scale, bias, n, k, act: str):
        if act not in _ACTS:
            raise ValueError(f"act: {act!r}, expected one of {tuple(_ACTS)}")
        super().__init__(weight, scale, bias, n, k)
        self.act, self._act = act, _ACTS[act]

    @staticmethod
    def _interleave(gate, up):
        rows = (gate.shape[0] + 31) & ~31
        shape = (rows // 16, 16) + tuple(gate.shape[1:])
        pads = [_pad(t, rows, *t.shape[1:]).view(shape) for t in (gate, up)]
        return _torch().stack(pads, 1).view(2 * rows, *gate.shape[1:])

    @classmethod
    def from_int8(cls, Wg, scale_gate, Wu, scale_up, bias_gate=None, bias_up=None, act: str = "silu", N: int = 8,
                  M: int = 8, trainable: bool = False, device=None):
        """Wg, Wu int8 [n x k] with scales [n]; both biases or neither.  trainable: refuse layouts that the backward
        pass does not take (the compact N:M ones)."""
        Wg, Wu = _device_i8(Wg, "Wg", device), _device_i8(Wu, "Wu", device)
        if Wg.shape != Wu.shape or Wg.device != Wu.device:
            raise ValueError(f"Wg and Wu: {tuple(Wg.shape)} and {tuple(Wu.shape)}, expected the same")
        if (bias_gate is None) != (bias_up is None):
            raise ValueError("bias_gate and bias_up: both or neither")
        n, k = Wg.shape
        W = cls._interleave(Wg, Wu)
        weight = cls._pack(W, W.shape[0], N, M)
        if trainable and weight.desc.layout != NM_LAYOUT_DENSE:
            raise ValueError(f"the backward pass takes dense layouts, not {N}:{M}")
        scale = cls._interleave(_vector(scale_gate, "scale_gate", n, W), _vector(scale_up, "scale_up", n, W))
        bias = None if bias_gate is None else cls._interleave(_vector(bias_gate, "bias_gate", n, W),
                                                              _vector(bias_up, "bias_up", n, W))
        return cls(weight, scale, bias, n, k, act)

    @classmethod
    def from_float(cls, Wg, Wu, bias_gate=None, bias_up=None, act: str = "silu"):
        (qg, sg), (qu, su) = quantize_rows(Wg), quantize_rows(Wu)
        k = Wg.shape[1]
        return cls.from_int8(qg[:, :k], sg, qu[:, :k], su, bias_gate, bias_up, act=act, trainable=True)


def _product_out(out, shape, dtype, like, stream):
    """(output, its row stride): rows may lie apart in a given one."""
    if out is None:
        return _empty(shape, dtype, like, stream), shape[-1]
    if out.dtype != dtype or tuple(out.shape) != tuple(shape) or out.device != like.device:
        raise ValueError(f"out: {out.dtype} {tuple(out.shape)} on {out.device}, expected {dtype} {tuple(shape)} on "
                         f"{like.device}")
    flat, ld = _rows(out, "out")
    return out, ld


def _of_rows(x, w: ScaledWeight, out, out_dtype, stream, gated: bool):
    _on_current_device(x, "x")
    if x.device != w.device:
        raise ValueError(f"x: on {x.device}, expected {w.device}")
    xtype = _type_of(x, "x")
    flat, ld = _rows(x, "x", w.k)
    m = flat.shape[0]
    dtype = x.dtype if out_dtype is None else out_dtype
    out, ldo = _product_out(out, (*x.shape[:-1], w.n), dtype, x, stream)
    ws, need = w._workspace(m, xtype, x, stream)
    wp = None if ws is None else ws.data_ptr()
    if gated:
        _check(lib().nm_gated(flat.data_ptr(), ld, xtype, m, w._ref, w._act, out.data_ptr(), ldo, _type_of(out, "out"),
                              wp, need, _stream(stream)), "nm_gated")
    else:
        _check(lib().nm_linear_i8(flat.data_ptr(), ld, xtype, m, w._ref, out.data_ptr(), ldo, _type_of(out, "out"), wp,
                                  need, _stream(stream)), "nm_linear_i8")
    return out


def _codes_in(xq, sx, w: ScaledWeight) -> int:
    torch = _torch()
    _on_current_device(xq, "xq")
    if xq.dim() != 2:
        raise ValueError(f"xq: {xq.dim()}-D, expected [tokens x {padded(w.k)}]")
    m = xq.shape[0]
    _need(xq, "xq", (torch.int8,), (m, padded(w.k)))
    _need(sx, "sx", (torch.float32,), (m,))
    for t, name in ((xq, "xq"), (sx, "sx")):
        if t.device != w.device:
            raise ValueError(f"{name}: on {t.device}, expected {w.device}")
    return m


def _of_codes(xq, sx, w: ScaledWeight, out, out_dtype, stream, gated: bool):
    m = _codes_in(xq, sx, w)
    out, ldo = _product_out(out, (m, w.n), out.dtype if out is not None else out_dtype, xq, stream)
    ws, need = w._workspace(m, 0, xq, stream)
    wp = None if ws is None else ws.data_ptr()
    if gated:
        _check(lib().nm_gated_i8(xq.data_ptr(), sx.data_ptr(), m, w._ref, w._act, out.data_ptr(), ldo,
                                 _type_of(out, "out"), wp, need, _stream(stream)), "nm_gated_i8")
    else:
        _check(lib().nm_gemm_i8_scaled(xq.data_ptr(), sx.data_ptr(), m, w._ref, out.data_ptr(), ldo,
                                       _type_of(out, "out"), wp, need, _stream(stream)), "nm_gemm_i8_scaled")
    return out


def linear_i8(x, w: ScaledWeight, out=None, out_dtype=None, stream=None):
    """nm_linear_i8: x [..., k] in int8 codes by token times w, scaled back: [..., n] of x's type (or out_dtype)."""
    if isinstance(w, GatedWeight):
        raise ValueError("w: a gated block's weight")
    return _of_rows(x, w, out, out_dtype, stream, False)


def gemm_i8_scaled(xq, sx, w: ScaledWeight, out=None, out_dtype=None, stream=None):
    """nm_gemm_i8_scaled: the product of codes and scales as quantize_rows or norm_residual_i8 give them; of
    out_dtype (float16 without it)."""
    if isinstance(w, GatedWeight):
        raise ValueError("w: a gated block's weight")
    return _of_codes(xq, sx, w, out, out_dtype or _torch().float16, stream, False)


def gated_ffn(x, w: GatedWeight, out=None, out_dtype=None, stream=None):
    """nm_gated: act(x Wg^T + bg) * (x Wu^T + bu) with x in int8 codes by token: [..., n]."""
    if not isinstance(w, GatedWeight):
        raise ValueError("w: not a gated block's weight")
    return _of_rows(x, w, out, out_dtype, stream, True)


def gated_ffn_i8(xq, sx, w: GatedWeight, out=None, out_dtype=None, stream=None):
    """nm_gated_i8: the same of codes and scales; of out_dtype (float16 without it)."""
    if not isinstance(w, GatedWeight):
        raise ValueError("w: not a gated block's weight")
    return _of_codes(xq, sx, w, out, out_dtype or _torch().float16, stream, True)


class GatedGrads(NamedTuple):
    """Gradients of the gated block: of the dequantised x and weights, in dh's type; of the biases in float32."""
    dx: object
    dw_gate: object
    dw_up: object
    dbias_gate: object
    dbias_up: object


def gated_ffn_backward(xq, sx, w: GatedWeight, dh, stream=None) -> GatedGrads:
    """nm_gated_backward: from dh [tokens x n] (float16 or bfloat16) at the codes that the forward pass used; the
    gradients pass straight through the rounding to codes.  w must be of a dense layout."""
    if not isinstance(w, GatedWeight):
        raise ValueError("w: not a gated block's weight")
    if w.weight.desc.layout != NM_LAYOUT_DENSE:
        raise ValueError("w: the backward pass takes dense layouts")
    torch = _torch()
    m = _codes_in(xq, sx, w)
    if dh.dtype not in (torch.float16, torch.bfloat16):
        raise ValueError(f"dh: dtype {dh.dtype}, expected float16 or bfloat16")
    if dh.device != w.device:
        raise ValueError(f"dh: on {dh.device}, expected {w.device}")
    flat, ld = _rows(dh, "dh", w.n)
    if flat.shape[0] != m:
        raise ValueError(f"dh: {flat.shape[0]} tokens, expected {m}")
    T, f32 = dh.dtype, torch.float32
    dx = _empty((m, w.k), T, dh, stream)
    dwg, dwu = _empty((w.n, w.k), T, dh, stream), _empty((w.n, w.k), T, dh, stream)
    dbg = dbu = None
    if w.bias is not None:
        dbg, dbu = _empty((w.n,), f32, dh, stream), _empty((w.n,), f32, dh, stream)
    need = ctypes.c_size_t()
    _check(lib().nm_gated_backward_workspace(w._ref, m, ctypes.byref(need)), "nm_gated_backward_workspace")
    ws = _empty((need.value,), torch.uint8, dh, stream) if need.value else None
    a = NmGatedGradArgs(xq.data_ptr(), sx.data_ptr(), flat.data_ptr(), ld, m, w._act, _type_of(dh, "dh"), _ptr(dx),
                        _ptr(dwg), _ptr(dwu), _ptr(dbg), _ptr(dbu))
    _check(lib().nm_gated_backward(ctypes.byref(a), w._ref, _ptr(ws), need.value, _stream(stream)),
           "nm_gated_backward")
    return GatedGrads(dx, dwg, dwu, dbg, dbu)
