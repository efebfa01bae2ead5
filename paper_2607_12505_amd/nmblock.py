"""The operators of a transformer block around its int8 linears (C ABI in include/nmspmm.h).

* `quantize_rows`: int8 codes of activation rows with a scale for each token; `pad_codes`: codes made elsewhere, as the
  products read them (which take rows of an odd number of codes and pad them, or padded rows).
* `linear_i8`, `gemm_i8_scaled`: the int8 product (dense or N:M weights) with scales for each token and channel, of
  activations or of codes already made; `ScaledWeight` holds its weight.
* `gated_ffn`, `gated_ffn_i8`, `gated_ffn_backward`: both projections of a gated feed-forward block, the activation and
  their product in one kernel, and the gradients; `GatedWeight` holds both weights.
* `norm_residual`, `norm_residual_i8`, `norm_residual_backward`: the norm after a block, its gate and residual scale,
  and the norm before the next block in one pass; with int8 codes in place of the normalised rows; and the gradients.

Tensors are device tensors of float16, bfloat16 or float32, [..., channels] with consecutive channels; two-dimensional
inputs may have any row stride.  Parameters are float32.  Every call enqueues its kernels on `stream` (a
torch.cuda.Stream; the current one without it) and returns; outputs that are not given are allocated for that stream.
Tensors are used as they are: no call records an autograd graph, and outputs never require gradients (the gradients are
the `_backward` functions' to give).  A given output counts as modified in place, so that torch refuses to go back through
what it held.  There is no fallback: a missing library raises.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

from .nmspmm import (NM_ERR_WORKSPACE, NM_LAYOUT_DENSE, NM_OK, DeviceWeight, NmDesc, NmError, _check, compress,
                     compress_size, lib)

NM_TYPE_F16, NM_TYPE_BF16, NM_TYPE_F32 = 1, 2, 3
NM_NORM_NONE, NM_NORM_RMS, NM_NORM_LAYER = 0, 1, 2
_NORMS = {"rms": NM_NORM_RMS, "layer": NM_NORM_LAYER}


class _Runtime:
    """What every call looks up, looked up once: a call of one token takes a few microseconds of host time, which
    imports inside functions and Stream objects would double."""

    def __init__(self):
        import torch
        L = lib()
        self.torch = torch
        self.f32, self.i8, self.u8 = torch.float32, torch.int8, torch.uint8
        self.types = {torch.float16: NM_TYPE_F16, torch.bfloat16: NM_TYPE_BF16, torch.float32: NM_TYPE_F32}
        self.device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        self.raw_stream = raw or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)
        self.quantize, self.norm, self.norm_grad = L.nm_quantize_rows, L.nm_norm_residual, L.nm_norm_residual_backward
        self.linear, self.linear_codes = L.nm_linear_i8, L.nm_gemm_i8_scaled
        self.gated, self.gated_codes, self.gated_grad = L.nm_gated, L.nm_gated_i8, L.nm_gated_backward


_rt: Optional[_Runtime] = None


def _runtime() -> _Runtime:
    global _rt
    if _rt is None:
        _rt = _Runtime()
    return _rt


def _index(t, name: str, rt: _Runtime) -> int:
    """The device of a call: the first tensor's, which has to be the current one (kernels go to its streams)."""
    if not t.is_cuda:
        raise ValueError(f"{name}: must be a device tensor")
    dev = t.get_device()
    if dev != rt.device():
        raise ValueError(f"{name}: on cuda:{dev}, but the current device is cuda:{rt.device()}")
    return dev


def _on(t, name: str, dev: int):
    if t.get_device() != dev:
        raise ValueError(f"{name}: on {t.device}, expected cuda:{dev}")


def _type_of(t, name: str, rt: _Runtime) -> int:
    code = rt.types.get(t.dtype)
    if code is None:
        raise ValueError(f"{name}: dtype {t.dtype}, expected float16, bfloat16 or float32")
    return code


def _rows(t, name: str):
    """(rows, channels, row stride) of [..., channels]; refuses what has no such view."""
    if t.dim() == 2:
        m, k = t.shape
        s0, s1 = t.stride()
        if s1 != 1 and k > 1:
            raise ValueError(f"{name}: channels must be consecutive")
        return m, k, (s0 if m > 1 else k)
    if t.dim() == 0 or not t.is_contiguous():
        raise ValueError(f"{name}: must be two-dimensional, or contiguous with channels last")
    k = t.shape[-1]
    return (t.numel() // k if k else 0), k, k


def _param(t, name: str, shape, dtype, dev: int):
    if t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous():
        raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)}, expected contiguous {dtype} {shape}")
    _on(t, name, dev)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _handle(stream, dev: int, rt: _Runtime) -> int:
    return rt.raw_stream(dev) if stream is None else stream.cuda_stream


def _empty(shape, dtype, like, stream, rt: _Runtime):
    """Memory of the call's stream: torch's allocator orders its reuse there.  (Sizes one by one: torch reads a tuple
    of them half a microsecond slower.)"""
    if stream is None:
        return like.new_empty(*shape, dtype=dtype)
    torch = rt.torch
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(stream.cuda_stream, device=like.device)
    with torch.cuda.stream(stream):
        return like.new_empty(*shape, dtype=dtype)


def _like(t, stream, rt: _Runtime):
    """Memory of t's shape and type, without gaps."""
    if stream is None and t.is_contiguous():
        return rt.torch.empty_like(t)
    return _empty(t.shape, t.dtype, t, stream, rt)


def _written(t, rt: _Runtime):
    """t, its version moved as torch's own in-place operations move it."""
    rt.torch.autograd.graph.increment_version(t)
    return t


def _output(given, name: str, shape, dtype, like, stream, rt: _Runtime):
    if given is None:
        return _empty(shape, dtype, like, stream, rt)
    _param(given, name, tuple(shape), dtype, like.get_device())
    return _written(given, rt)


def padded(k: int) -> int:
    """Row length of int8 codes of k channels: a multiple of 16."""
    return (k + 15) & ~15


# ---------------------------------------------------------------- row codes

def quantize_rows(x, xq=None, scale=None, stream=None):
    """nm_quantize_rows: (codes int8 [rows x padded(k)], scales float32 [rows]) of x."""
    rt = _rt or _runtime()
    dev = _index(x, "x", rt)
    code = _type_of(x, "x", rt)
    m, k, ld = _rows(x, "x")
    xq = _output(xq, "xq", (m, padded(k)), rt.i8, x, stream, rt)
    scale = _output(scale, "scale", (m,), rt.f32, x, stream, rt)
    _check(rt.quantize(x.data_ptr(), ld, code, m, k, xq.data_ptr(), scale.data_ptr(), _handle(stream, dev, rt)),
           "nm_quantize_rows")
    return xq, scale


def pad_codes(q, out=None, stream=None):
    """nm_pad_codes: codes int8 [rows x k] of any row stride as the products read them, [rows x padded(k)]."""
    rt = _rt or _runtime()
    dev = _index(q, "q", rt)
    if q.dtype != rt.i8 or q.dim() != 2:
        raise ValueError(f"q: {q.dtype} {tuple(q.shape)}, expected two-dimensional {rt.i8}")
    m, k, ld = _rows(q, "q")
    out = _output(out, "out", (m, padded(k)), rt.i8, q, stream, rt)
    _check(lib().nm_pad_codes(q.data_ptr(), ld, m, k, out.data_ptr(), _handle(stream, dev, rt)), "nm_pad_codes")
    return out


# ---------------------------------------------------------------- norms around a block

class NmNorm(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("eps", ctypes.c_float), ("weight", ctypes.c_void_p),
                ("bias", ctypes.c_void_p)]


_NO_NORM = NmNorm()


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
    """A norm of the channels: kind "rms" or "layer", float32 weight and bias [d] (None: 1 and 0), eps.

    The tensors are checked here, once, and read at every call: change their values in place."""

    def __init__(self, kind: str, weight=None, bias=None, eps: float = 1e-6):
        if kind not in _NORMS:
            raise ValueError(f"norm: kind {kind!r}, expected 'rms' or 'layer'")
        if not eps > 0:
            raise ValueError("norm: eps must be positive")
        import torch
        for t, name in ((weight, "weight"), (bias, "bias")):
            if t is not None and (t.dtype != torch.float32 or t.dim() != 1 or not t.is_contiguous() or not t.is_cuda):
                raise ValueError(f"norm: {name} must be a contiguous float32 vector on the device")
        if weight is not None and bias is not None and (weight.shape != bias.shape or weight.device != bias.device):
            raise ValueError("norm: weight and bias differ in size or device")
        one = weight if weight is not None else bias
        self.kind, self.eps = kind, float(eps)
        # aliases: their memory stays even if the caller's tensors are given other data
        self.weight = None if weight is None else weight.detach()
        self.bias = None if bias is None else bias.detach()
        self._d = None if one is None else one.shape[0]
        self._dev = None if one is None else one.get_device()
        self._args = NmNorm(_NORMS[kind], self.eps, _ptr(self.weight), _ptr(self.bias))

    def _for(self, d: int, dev: int, name: str) -> NmNorm:
        if self._d is not None and (self._d != d or self._dev != dev):
            raise ValueError(f"{name}: of {self._d} channels on cuda:{self._dev}, expected {d} on cuda:{dev}")
        return self._args


def _gate(gate, m: int, d: int, dev: int, rt: _Runtime) -> int:
    """Checks the gate [groups x d] (or [d]) and returns groups."""
    if gate is None:
        return 1
    groups = gate.shape[0] if gate.dim() == 2 else 1
    if gate.dtype != rt.f32 or gate.dim() not in (1, 2) or gate.shape[-1] != d or not gate.is_contiguous():
        raise ValueError(f"gate: {gate.dtype} {tuple(gate.shape)}, expected contiguous float32 [{d}] or [groups x {d}]")
    _on(gate, "gate", dev)
    if groups < 1 or m % groups:
        raise ValueError(f"gate: {groups} groups do not divide {m} tokens")
    return groups


def _around(y, r, pre, post, gate, alpha, res, stream, rt):
    like, name = (y, "y") if y is not None else (r, "r")
    if like is None:
        raise ValueError("y and r: at least one is needed")
    dev = _index(like, name, rt)
    code = _type_of(like, name, rt)
    yp = rp = None
    ldy = ldr = 0
    if y is not None:
        m, d, ldy = _rows(y, "y")
        yp = y.data_ptr()
    if r is not None:
        mr, dr, ldr = _rows(r, "r")
        if y is not None and (mr != m or dr != d or r.dtype != y.dtype):
            raise ValueError(f"r: {r.dtype} [{mr} x {dr}], expected {y.dtype} [{m} x {d}]")
        _on(r, "r", dev)
        rp, m, d = r.data_ptr(), mr, dr
    groups, gp = (1, None) if gate is None else (_gate(gate, m, d, dev, rt), gate.data_ptr())
    res = _like(like, stream, rt) if res is None else _output(res, "res", like.shape, like.dtype, like, stream, rt)
    a = NmNormArgs(yp, rp, ldy, ldr, code, m, d, groups, gp, alpha,
                   _NO_NORM if post is None else post._for(d, dev, "post"),
                   _NO_NORM if pre is None else pre._for(d, dev, "pre"), res.data_ptr())
    return a, like, res, _handle(stream, dev, rt)


def norm_residual(y, r, pre: Optional[Norm] = None, post: Optional[Norm] = None, gate=None, alpha: float = 1.0,
                  res=None, z=None, stream=None):
    """nm_norm_residual: (res, z) with u = post(y), res = alpha r + gate u, z = pre(res).

    y (the block's output; post and gate go with it) or r (the residual stream) may be None.  gate: float32 [d], or
    [groups x d] with a row for each of `groups` equal runs of tokens.  Without `pre` there is no z (None).  res may be y
    or r itself; no output may overlap an input otherwise."""
    rt = _rt or _runtime()
    a, like, res, at = _around(y, r, pre, post, gate, alpha, res, stream, rt)
    if pre is not None:
        z = _like(res, stream, rt) if z is None else _output(z, "z", res.shape, like.dtype, like, stream, rt)
        a.z = z.data_ptr()
    elif z is not None:
        raise ValueError("z: given without a norm for it")
    _check(rt.norm(ctypes.byref(a), at), "nm_norm_residual")
    return res, z


def norm_residual_i8(y, r, pre: Norm, post: Optional[Norm] = None, gate=None, alpha: float = 1.0, res=None, zq=None,
                     zs=None, stream=None):
    """norm_residual with the codes of z and their scales in its place: (res, zq int8 [rows x padded(d)], zs)."""
    if pre is None:
        raise ValueError("pre: the codes are those of a norm's rows")
    rt = _rt or _runtime()
    a, like, res, at = _around(y, r, pre, post, gate, alpha, res, stream, rt)
    zq = _output(zq, "zq", (a.m, padded(a.d)), rt.i8, like, stream, rt)
    zs = _output(zs, "zs", (a.m,), rt.f32, like, stream, rt)
    a.zq, a.zs = zq.data_ptr(), zs.data_ptr()
    _check(rt.norm(ctypes.byref(a), at), "nm_norm_residual")
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
    if pre is not None and res is None:
        raise ValueError("res: needed for the gradient of its norm")
    if y is None and (post is not None or gate is not None):
        raise ValueError("y: needed for the gradients of its norm and gate")
    rt = _rt or _runtime()
    dev = _index(like, name, rt)
    code = _type_of(like, name, rt)
    m, d, _ = _rows(like, name)

    def given(t, what):
        if t is None:
            return None, 0
        mt, dt, ld = _rows(t, what)
        if mt != m or dt != d or t.dtype != like.dtype:
            raise ValueError(f"{what}: {t.dtype} [{mt} x {dt}], expected {like.dtype} [{m} x {d}]")
        _on(t, what, dev)
        return t.data_ptr(), ld

    (zp, ldz), (sp, lds), (yp, ldy), (rp, ldr) = given(dz, "dz"), given(dres, "dres"), given(y, "y"), given(res, "res")
    groups, gp = (1, None) if gate is None else (_gate(gate, m, d, dev, rt), gate.data_ptr())
    dr = _like(like, stream, rt)
    dy = _like(like, stream, rt) if y is not None else None
    # the parameters' gradients are rows of one buffer: the gate's, then the norms' weights and biases
    wanted = [t is not None for n in (pre, post) for t in ((n.weight, n.bias) if n is not None else (None, None))]
    rows = (groups if gate is not None else 0) + sum(wanted)
    dgate, params, dgp = None, [None] * 4, None
    if rows:
        sums = _empty((rows, d), rt.f32, like, stream, rt)
        each = sums.unbind(0) if gate is None or groups == 1 else sums[groups:].unbind(0)
        if gate is not None:
            dgate = sums[:groups] if gate.dim() == 2 else each[0]
            dgp = dgate.data_ptr()
        left = iter(each[1:] if gate is not None and groups == 1 else each)
        params = [next(left) if want else None for want in wanted]
    a = NmNormGradArgs(yp, rp, zp, sp, ldy, ldr, ldz, lds, code, m, d, groups, gp, alpha,
                       _NO_NORM if post is None else post._for(d, dev, "post"),
                       _NO_NORM if pre is None else pre._for(d, dev, "pre"), _ptr(dy), dr.data_ptr(), dgp,
                       *[_ptr(t) for t in params])
    need = ctypes.c_size_t()
    _check(lib().nm_norm_residual_backward_workspace(m, d, a.groups, ctypes.byref(need)),
           "nm_norm_residual_backward_workspace")
    ws = _empty((need.value,), rt.u8, like, stream, rt) if need.value else None
    _check(rt.norm_grad(ctypes.byref(a), _ptr(ws), need.value, _handle(stream, dev, rt)), "nm_norm_residual_backward")
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
    torch = _runtime().torch
    if not torch.is_tensor(W):
        W = torch.from_numpy(W)
    if W.dtype != torch.int8 or W.dim() != 2:
        raise ValueError(f"{name}: expected a two-dimensional int8 matrix")
    return W.to(device) if device is not None else W if W.is_cuda else W.cuda()


def _vector(v, name: str, n: int, like):
    torch = _runtime().torch
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
        self.device, self._dev, self._kp = weight.vals.device, weight.vals.get_device(), padded(k)
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
            return DeviceWeight(_pad(W, rows, cols).view(-1), W.new_empty(0, dtype=_runtime().u8), desc)
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

    def _need(self, m: int, xtype: int) -> int:
        """Workspace bytes of a product: a size by tokens and type, not a buffer."""
        need = self._needs.get((m, xtype))
        if need is None:
            size = ctypes.c_size_t()
            _check(lib().nm_linear_workspace(self._ref, m, xtype, ctypes.byref(size)), "nm_linear_workspace")
            if len(self._needs) > 256:
                self._needs.clear()
            need = self._needs[m, xtype] = size.value
        return need


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
        return _runtime().torch.stack(pads, 1).view(2 * rows, *gate.shape[1:])

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


def _product_out(out, m: int, shape, dtype, like, stream, rt):
    """(output, its type, its row stride): rows may lie apart in a given one."""
    if out is None:
        code = rt.types.get(dtype)
        if code is None:
            raise ValueError(f"out_dtype: {dtype}, expected float16, bfloat16 or float32")
        return _empty(shape, dtype, like, stream, rt), code, shape[-1]
    if out.dtype != dtype or tuple(out.shape) != tuple(shape):
        raise ValueError(f"out: {out.dtype} {tuple(out.shape)}, expected {dtype} {tuple(shape)}")
    _on(out, "out", like.get_device())
    code, ld = _type_of(out, "out", rt), _rows(out, "out")[2]
    return _written(out, rt), code, ld


_FEW = 16      # most tokens of a call that makes its codes in the product's own launch


def _of_rows(x, w: ScaledWeight, out, out_dtype, stream, gated: bool):
    rt = _rt or _runtime()
    dev = _index(x, "x", rt)
    if dev != w._dev:
        raise ValueError(f"x: on {x.device}, expected {w.device}")
    xtype = _type_of(x, "x", rt)
    m, k, ld = _rows(x, "x")
    if k != w.k:
        raise ValueError(f"x: {k} channels, expected {w.k}")
    shape = (m, w.n) if x.dim() == 2 else (*x.shape[:-1], w.n)
    out, otype, ldo = _product_out(out, m, shape, out_dtype or x.dtype, x, stream, rt)
    at = _handle(stream, dev, rt)
    act = (w._act,) if gated else ()
    call, args = rt.gated if gated else rt.linear, (x.data_ptr(), ld, xtype, m, w._ref, *act, out.data_ptr(), ldo, otype)
    st = NM_ERR_WORKSPACE
    if m <= _FEW:       # needs no workspace where the kernel makes the codes itself
        st = call(*args, None, 0, at)
    if st == NM_ERR_WORKSPACE:
        need = w._need(m, xtype)
        ws = _empty((need,), rt.u8, x, stream, rt)
        st = call(*args, ws.data_ptr(), need, at)
    if st != NM_OK:
        raise NmError(st, "nm_gated" if gated else "nm_linear_i8")
    return out


def _codes_in(xq, sx, w: ScaledWeight, stream, rt):
    """(codes, tokens, device) of codes and scales for w: rows of w.k codes, which get their padding here, or padded."""
    dev = _index(xq, "xq", rt)
    m = xq.shape[0] if xq.dim() else 0
    _param(sx, "sx", (m,), rt.f32, w._dev)
    if w.k != w._kp and xq.dim() == 2 and xq.shape[1] == w.k:
        _on(xq, "xq", w._dev)
        return pad_codes(xq, stream=stream), m, dev
    _param(xq, "xq", (m, w._kp), rt.i8, w._dev)
    return xq, m, dev


def _of_codes(xq, sx, w: ScaledWeight, out, out_dtype, stream, gated: bool):
    rt = _rt or _runtime()
    xq, m, dev = _codes_in(xq, sx, w, stream, rt)
    dtype = out.dtype if out is not None else out_dtype or rt.torch.float16
    out, otype, ldo = _product_out(out, m, (m, w.n), dtype, xq, stream, rt)
    need = w._need(m, 0)
    ws = _empty((need,), rt.u8, xq, stream, rt) if need else None
    at = _handle(stream, dev, rt)
    if gated:
        _check(rt.gated_codes(xq.data_ptr(), sx.data_ptr(), m, w._ref, w._act, out.data_ptr(), ldo, otype, _ptr(ws),
                              need, at), "nm_gated_i8")
    else:
        _check(rt.linear_codes(xq.data_ptr(), sx.data_ptr(), m, w._ref, out.data_ptr(), ldo, otype, _ptr(ws), need,
                               at), "nm_gemm_i8_scaled")
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
    return _of_codes(xq, sx, w, out, out_dtype, stream, False)


def gated_ffn(x, w: GatedWeight, out=None, out_dtype=None, stream=None):
    """nm_gated: act(x Wg^T + bg) * (x Wu^T + bu) with x in int8 codes by token: [..., n]."""
    if not isinstance(w, GatedWeight):
        raise ValueError("w: not a gated block's weight")
    return _of_rows(x, w, out, out_dtype, stream, True)


def gated_ffn_i8(xq, sx, w: GatedWeight, out=None, out_dtype=None, stream=None):
    """nm_gated_i8: the same of codes and scales; of out_dtype (float16 without it)."""
    if not isinstance(w, GatedWeight):
        raise ValueError("w: not a gated block's weight")
    return _of_codes(xq, sx, w, out, out_dtype, stream, True)


class GatedGrads(NamedTuple):
    """Gradients of the gated block: of the dequantised x and weights, in dh's type; of the biases in float32."""
    dx: object
    dw_gate: object
    dw_up: object
    dbias_gate: object
    dbias_up: object


def gated_ffn_backward(xq, sx, w: GatedWeight, dh, stream=None) -> GatedGrads:
    """nm_gated_backward: from dh [tokens x n] (float16 or bfloat16) at the codes that the forward pass used; the
    gradients pass straight through the rounding to codes.  The gradients of g and u are rounded to dh's type before
    their products with x and the weights.  w must be of a dense layout."""
    if not isinstance(w, GatedWeight):
        raise ValueError("w: not a gated block's weight")
    if w.weight.desc.layout != NM_LAYOUT_DENSE:
        raise ValueError("w: the backward pass takes dense layouts")
    rt = _rt or _runtime()
    xq, m, dev = _codes_in(xq, sx, w, stream, rt)
    T, f32 = dh.dtype, rt.f32
    code = _type_of(dh, "dh", rt)
    if code == NM_TYPE_F32:
        raise ValueError(f"dh: dtype {T}, expected float16 or bfloat16")
    mh, n, ld = _rows(dh, "dh")
    if mh != m or n != w.n:
        raise ValueError(f"dh: [{mh} x {n}], expected [{m} x {w.n}]")
    _on(dh, "dh", dev)
    dx = _empty((m, w.k), T, dh, stream, rt)
    dwg, dwu = _empty((w.n, w.k), T, dh, stream, rt), _empty((w.n, w.k), T, dh, stream, rt)
    dbg = dbu = None
    if w.bias is not None:
        dbg, dbu = _empty((w.n,), f32, dh, stream, rt), _empty((w.n,), f32, dh, stream, rt)
    need = ctypes.c_size_t()
    _check(lib().nm_gated_backward_workspace(w._ref, m, ctypes.byref(need)), "nm_gated_backward_workspace")
    ws = _empty((need.value,), rt.u8, dh, stream, rt) if need.value else None
    a = NmGatedGradArgs(xq.data_ptr(), sx.data_ptr(), dh.data_ptr(), ld, m, w._act, code, dx.data_ptr(),
                        dwg.data_ptr(), dwu.data_ptr(), _ptr(dbg), _ptr(dbu))
    _check(rt.gated_grad(ctypes.byref(a), w._ref, _ptr(ws), need.value, _handle(stream, dev, rt)),
           "nm_gated_backward")
    return GatedGrads(dx, dwg, dwu, dbg, dbu)
