"""The attention half of a transformer block (C ABI in include/nmspmm.h).

* `rotary`, `rotary_qk`, `rotary_backward`: rotary positions with several axes (time, height, width) on queries and keys;
  `RotaryAxes` holds the frequency and axis of every pair of channels.
* `diff_attention`, `diff_attention_train`, `diff_attention_backward`: differential attention, the difference of two softmax
  maps with a learned weight (`DiffWeight`); causal or windowed, of padded or packed sequences, of single tokens over a
  cache (the keys are then split over the device), and the gradients.

Tensors are device tensors with consecutive channels; their other dimensions may have any strides (not negative), so queries,
keys and values may lie inside the rows of one product, or in a cache.  Streams, outputs, devices and errors are as in
nmblock: every call enqueues its kernels on `stream` (the current one without it) and returns; nothing records an
autograd graph; a given output counts as modified in place.  There is no fallback: a missing library raises.
"""
from __future__ import annotations

import ctypes
import math
import struct
from typing import NamedTuple, Optional

from . import nmblock
from .nmblock import NM_TYPE_F32, _empty, _handle, _index, _on, _ptr, _runtime, _type_of, _written
from .nmspmm import NM_OK, NmError, _check, lib


def _packer(structure) -> struct.Struct:
    """A C structure's values, one after the other, as its bytes: a call passes some forty, which ctypes would set one by
    one at twice the host time of a small call's kernels."""
    codes = {ctypes.c_void_p: "Q", ctypes.c_int64: "q", ctypes.c_int32: "i", ctypes.c_float: "f"}
    parts, end = ["="], 0

    def add(kind, at):
        nonlocal end
        if kind in codes:
            parts.append(f"{at - end}x{codes[kind]}")
            end = at + ctypes.sizeof(kind)
        elif issubclass(kind, ctypes.Array):
            for i in range(kind._length_):
                add(kind._type_, at + i * ctypes.sizeof(kind._type_))
        else:
            for name, field in kind._fields_:
                add(field, at + getattr(kind, name).offset)

    add(structure, 0)
    parts.append(f"{ctypes.sizeof(structure) - end}x")
    return struct.Struct("".join(parts))


class _Calls:
    """What every call looks up, looked up once."""

    def __init__(self):
        L = lib()
        self.rotary, self.forward, self.forward_size = L.nm_rotary, L.nm_diff_attention, L.nm_diff_attention_workspace
        self.backward, self.backward_size = L.nm_diff_attention_backward, L.nm_diff_attention_backward_workspace
        self.sizes = {}       # workspace bytes by shapes: sizes, not buffers


_calls: Optional[_Calls] = None


def _library() -> _Calls:
    global _calls
    if _calls is None:
        _calls = _Calls()
    return _calls


def _size(query, key, args) -> int:
    sizes = _calls.sizes
    need = sizes.get(key)
    if need is None:
        size = ctypes.c_size_t()
        _check(query(args, ctypes.byref(size)), "workspace")
        if len(sizes) > 512:
            sizes.clear()
        need = sizes[key] = size.value
    return need


def _heads(t, name: str, rt, dims=(3,)):
    """Refuses what is no tensor of heads: [.., tokens, heads, channels] with consecutive channels."""
    if t.dim() not in dims:
        raise ValueError(f"{name}: {t.dim()} dimensions, expected {' or '.join(str(n) for n in dims)}")
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: channels must be consecutive")


def _apart(t, name: str):
    """Refuses an output of which several places are one."""
    if 0 in t.stride() and any(s == 0 and n > 1 for s, n in zip(t.stride(), t.shape)):
        raise ValueError(f"{name}: an expanded tensor cannot be written")


# ---------------------------------------------------------------- rotary positions

class NmRotaryPart(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("out", ctypes.c_void_p), ("x_token", ctypes.c_int64),
                ("x_head", ctypes.c_int64), ("out_token", ctypes.c_int64), ("out_head", ctypes.c_int64),
                ("heads", ctypes.c_int32)]


class NmRotaryArgs(ctypes.Structure):
    _fields_ = [("part", NmRotaryPart * 2), ("pos", ctypes.c_void_p), ("ld_pos", ctypes.c_int64),
                ("freq", ctypes.c_void_p), ("axis", ctypes.c_void_p), ("tokens", ctypes.c_int64),
                ("type", ctypes.c_int32), ("pos_float", ctypes.c_int32), ("pairs", ctypes.c_int32),
                ("d", ctypes.c_int32), ("axes", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("back", ctypes.c_int32)]


class RotaryAxes:
    """The frequency (radians a unit of position) and the axis of every pair of channels, laid out once.

    style "halves": pair i is channels i and pairs + i of a head; "pairs": channels 2 i and 2 i + 1."""

    def __init__(self, freqs, axis, style: str = "halves", device="cuda"):
        import torch
        if style not in ("halves", "pairs"):
            raise ValueError(f"style: {style!r}, expected 'halves' or 'pairs'")
        freqs, axis = [float(f) for f in freqs], [int(a) for a in axis]
        if not freqs or len(freqs) != len(axis):
            raise ValueError(f"freqs and axis: {len(freqs)} and {len(axis)}, expected as many of both")
        if min(axis) < 0:
            raise ValueError("axis: must not be negative")
        if not all(math.isfinite(f) for f in freqs):
            raise ValueError("freqs: must be finite")
        self.pairs, self.axes, self.style = len(freqs), max(axis) + 1, style
        self.freqs = torch.tensor(freqs, dtype=torch.float64, device=device)
        self.axis = torch.tensor(axis, dtype=torch.int32, device=device)
        self._dev, self._interleaved = self.freqs.get_device(), style == "pairs"
        self._freqs_at, self._axis_at = self.freqs.data_ptr(), self.axis.data_ptr()

    @classmethod
    def of_sections(cls, sections, theta: float = 10000.0, own_ladders: bool = False, style: str = "halves",
                    device="cuda"):
        """sections: pairs of each axis, in their order.  Frequencies are powers of 1 / theta: one ladder over all pairs,
        or (own_ladders) one for each axis."""
        freqs, axis = [], []
        for a, n in enumerate(sections):
            for j in range(n):
                freqs.append(theta ** (-j / n if own_ladders else -len(freqs) / sum(sections)))
                axis.append(a)
        return cls(freqs, axis, style, device)


def _tokens_of(t, name: str):
    """(tokens, token stride) of [tokens, heads, channels] or [sequences, tokens, heads, channels]."""
    if t.dim() == 3:
        return t.shape[0], t.stride(0)
    b, n = t.shape[:2]
    if b > 1 and n > 1 and t.stride(0) != n * t.stride(1):
        raise ValueError(f"{name}: tokens of all sequences must lie at one stride")
    return b * n, t.stride(1) if n > 1 else t.stride(0)


_ROTARY = _packer(NmRotaryArgs)
_NO_PART = (0, 0, 0, 0, 0, 0, 0)


def _rotary(parts, positions, axes: RotaryAxes, back: bool, stream):
    """parts: (x, out or None, name) of one or two tensors; the outputs."""
    rt = nmblock._rt or _runtime()
    C = _calls or _library()
    torch = rt.torch
    x = parts[0][0]
    dev = _index(x, parts[0][2], rt)
    code = _type_of(x, parts[0][2], rt)
    if axes._dev != dev:
        raise ValueError(f"axes: on cuda:{axes._dev}, expected cuda:{dev}")
    d = x.shape[-1] if x.dim() else 0
    values, outs, tokens, heads = [], [], None, 0
    for t, out, name in parts:
        _heads(t, name, rt, (3, 4))
        if t is not x:
            _on(t, name, dev)
            if t.dtype != x.dtype or t.shape[-1] != d:
                raise ValueError(f"{name}: {t.dtype} of {t.shape[-1]} channels, expected {x.dtype} of {d}")
        n, stride = _tokens_of(t, name)
        if tokens not in (None, n):
            raise ValueError(f"{name}: {n} tokens, expected {tokens}")
        tokens = n
        if out is None:
            out = _empty(t.shape, t.dtype, t, stream, rt)
        else:
            if out.dtype != t.dtype or out.shape != t.shape:
                raise ValueError(f"out of {name}: {out.dtype} {tuple(out.shape)}, expected {t.dtype} {tuple(t.shape)}")
            _heads(out, f"out of {name}", rt, (3, 4))
            _apart(out, f"out of {name}")
            _on(out, f"out of {name}", dev)
            _written(out, rt)
        heads += t.shape[-2]
        values += (t.data_ptr(), out.data_ptr(), stride, t.stride(-2), _tokens_of(out, f"out of {name}")[1],
                   out.stride(-2), t.shape[-2])
        outs.append(out)
    if d < 2 * axes.pairs:
        raise ValueError(f"{parts[0][2]}: {d} channels, fewer than those of {axes.pairs} pairs")
    real = positions.dtype == torch.float32
    if not real and positions.dtype != torch.int32:
        raise ValueError(f"positions: {positions.dtype}, expected int32 or float32")
    if positions.dim() == 1 and axes.axes == 1:
        positions = positions.unsqueeze(0)
    if positions.dim() != 2 or positions.shape[0] < axes.axes or positions.shape[1] != tokens:
        raise ValueError(f"positions: {tuple(positions.shape)}, expected ({axes.axes}, {tokens})")
    if tokens > 1 and positions.stride(1) != 1:
        raise ValueError("positions: tokens must be consecutive")
    _on(positions, "positions", dev)
    if tokens == 0 or heads == 0:
        return outs
    if len(parts) == 1:
        values += _NO_PART
    args = _ROTARY.pack(*values, positions.data_ptr(), positions.stride(0), axes._freqs_at, axes._axis_at, tokens, code, real,
                        axes.pairs, d, axes.axes, axes._interleaved, back)
    st = C.rotary(args, _handle(stream, dev, rt))
    if st != NM_OK:
        raise NmError(st, "nm_rotary")
    return outs


def rotary(x, positions, axes: RotaryAxes, out=None, stream=None):
    """nm_rotary: x [tokens, heads, d] or [sequences, tokens, heads, d] with its pairs of channels turned by the positions,
    int32 or float32 [axes, tokens of all sequences].  out may be x."""
    return _rotary([(x, out, "x")], positions, axes, False, stream)[0]


def rotary_qk(q, k, positions, axes: RotaryAxes, out_q=None, out_k=None, stream=None):
    """rotary of queries and keys of the same tokens in one launch: (q, k)."""
    return tuple(_rotary([(q, out_q, "q"), (k, out_k, "k")], positions, axes, False, stream))


def rotary_backward(dy, positions, axes: RotaryAxes, out=None, stream=None):
    """The gradient of rotary's input from that of its output: the rotation back.  out may be dy."""
    return _rotary([(dy, out, "dy")], positions, axes, True, stream)[0]


# ---------------------------------------------------------------- differential attention

class NmHeads(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("batch", ctypes.c_int64), ("token", ctypes.c_int64), ("head", ctypes.c_int64)]


class NmTokens(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("tq", ctypes.c_int32), ("tk", ctypes.c_int32), ("left", ctypes.c_int32),
                ("right", ctypes.c_int32), ("q_offsets", ctypes.c_void_p), ("k_offsets", ctypes.c_void_p),
                ("q_lens", ctypes.c_void_p), ("k_lens", ctypes.c_void_p), ("total_q", ctypes.c_int64),
                ("total_k", ctypes.c_int64)]


class NmDiffWeight(ctypes.Structure):
    _fields_ = [("value", ctypes.c_void_p), ("q1", ctypes.c_void_p), ("k1", ctypes.c_void_p), ("q2", ctypes.c_void_p),
                ("k2", ctypes.c_void_p), ("init", ctypes.c_float), ("n", ctypes.c_int32), ("per_head", ctypes.c_int32)]


class NmDiffArgs(ctypes.Structure):
    _fields_ = [("q", NmHeads), ("k", NmHeads), ("v", NmHeads), ("o", NmHeads), ("kept", ctypes.c_void_p),
                ("stats", ctypes.c_void_p), ("tokens", NmTokens), ("weight", NmDiffWeight), ("type", ctypes.c_int32),
                ("H", ctypes.c_int32), ("Hk", ctypes.c_int32), ("d", ctypes.c_int32), ("dv", ctypes.c_int32),
                ("scale", ctypes.c_float)]


class NmDiffGradArgs(ctypes.Structure):
    _fields_ = [("q", NmHeads), ("k", NmHeads), ("v", NmHeads), ("grad_o", NmHeads), ("dq", NmHeads),
                ("dk", NmHeads), ("dv", NmHeads), ("kept", ctypes.c_void_p), ("stats", ctypes.c_void_p),
                ("dlam", ctypes.c_void_p), ("dq1", ctypes.c_void_p), ("dk1", ctypes.c_void_p), ("dq2", ctypes.c_void_p),
                ("dk2", ctypes.c_void_p), ("tokens", NmTokens), ("weight", NmDiffWeight), ("type", ctypes.c_int32),
                ("H", ctypes.c_int32), ("Hk", ctypes.c_int32), ("d", ctypes.c_int32), ("dv_width", ctypes.c_int32),
                ("scale", ctypes.c_float)]


class DiffWeight:
    """The weight of the second map: float32 [heads], or made from learned vectors (`of_vectors`).

    The tensors are checked here and at the calls' heads, and read at every call: change their values in place."""

    def __init__(self, value):
        import torch
        if value.dtype != torch.float32 or value.dim() != 1 or not value.is_contiguous() or not value.is_cuda:
            raise ValueError("value: must be a contiguous float32 vector on the device, one for each head")
        self.value, self.vectors, self.init = value.detach(), None, 0.0
        self._heads, self._dev = value.shape[0], value.get_device()
        self._args = (_ptr(self.value), 0, 0, 0, 0, 0.0, 0, 0)

    @classmethod
    def of_vectors(cls, q1, k1, q2, k2, init: float):
        """exp(q1 . k1) - exp(q2 . k2) + init of vectors float32 [n] that all heads share, or [heads x n]."""
        import torch
        vectors = (q1, k1, q2, k2)
        for t, name in zip(vectors, ("q1", "k1", "q2", "k2")):
            if t.dtype != torch.float32 or t.dim() not in (1, 2) or not t.is_contiguous() or not t.is_cuda or \
                    t.numel() == 0:
                raise ValueError(f"{name}: must be contiguous float32 [n] or [heads x n] on the device")
            if t.shape != q1.shape or t.device != q1.device:
                raise ValueError(f"{name}: {tuple(t.shape)} on {t.device}, expected {tuple(q1.shape)} on {q1.device}")
        self = cls.__new__(cls)
        self.value, self.vectors, self.init = None, tuple(t.detach() for t in vectors), float(init)
        self._heads, self._dev = (q1.shape[0] if q1.dim() == 2 else None), q1.get_device()
        self._args = (0, *(_ptr(t) for t in self.vectors), self.init, q1.shape[-1], int(q1.dim() == 2))
        return self

    def _for(self, heads: int, dev: int) -> tuple:
        if (self._heads is not None and self._heads != heads) or self._dev != dev:
            raise ValueError(f"weight: of {self._heads} heads on cuda:{self._dev}, expected {heads} on cuda:{dev}")
        return self._args


class _Shape(NamedTuple):
    """What a call's tensors say: heads, widths, the rows of q, and the values of the C structure of its tokens."""
    H: int
    Hk: int
    d: int
    dv: int
    rows: int
    packed: bool
    tokens: tuple
    code: int
    dev: int


def _lens(t, name: str, n: int, rt, dev: int):
    if t is None:
        return 0
    if t.dtype != rt.torch.int32 or t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)}, expected contiguous torch.int32 ({n},)")
    _on(t, name, dev)
    return t.data_ptr()


def _shape(q, k, v, causal, window, q_lens, k_lens, q_offsets, k_offsets, max_q, max_k, rt) -> _Shape:
    dev = _index(q, "q", rt)
    code = _type_of(q, "q", rt)
    if code == NM_TYPE_F32:
        raise ValueError(f"q: dtype {q.dtype}, expected float16 or bfloat16")
    packed = q_offsets is not None
    dims = 3 if packed else 4
    for t, name in ((q, "q"), (k, "k"), (v, "v")):
        if t.dim() != dims:
            raise ValueError(f"{name}: {t.dim()} dimensions, expected {dims} of "
                             f"{'packed' if packed else 'padded'} sequences")
        if t.shape[-1] > 1 and t.stride(-1) != 1:
            raise ValueError(f"{name}: channels must be consecutive")
        if t.dtype != q.dtype:
            raise ValueError(f"{name}: dtype {t.dtype}, expected {q.dtype}")
        if t.get_device() != dev:
            _on(t, name, dev)
    H2, d = q.shape[-2:]
    Hk, dv = v.shape[-2:]
    H = H2 // 2
    if H2 % 2 or H == 0 or k.shape[-2] != 2 * Hk or Hk == 0 or H % Hk:
        raise ValueError(f"q, k and v: {H2}, {k.shape[-2]} and {Hk} heads, expected 2 H, 2 Hk and Hk with Hk dividing H")
    if k.shape[-1] != d or k.shape[:-2] != v.shape[:-2]:
        raise ValueError(f"k and v: {tuple(k.shape)} and {tuple(v.shape)}, expected {d} channels of k and the same tokens")
    if causal and window is not None:
        raise ValueError("causal and window: one of them")
    left, right = (-1, 0) if causal else (-1, -1) if window is None else (min(int(w), 1 << 30) for w in window)
    if left < 0 or right < 0:
        left, right = max(left, -1), max(right, -1)
    if packed:
        if q_lens is not None or k_lens is not None:
            raise ValueError("q_lens and k_lens: of padded sequences, not of packed ones")
        batch = q_offsets.shape[0] - 1 if q_offsets.dim() == 1 else -1
        if batch < 0:
            raise ValueError(f"q_offsets: {tuple(q_offsets.shape)}, expected (sequences + 1,)")
        if max_q is None:
            raise ValueError("max_q: needed with q_offsets")
        if k_offsets is None:
            k_offsets, max_k = q_offsets, max_q
        elif max_k is None:
            raise ValueError("max_k: needed with k_offsets")
        qo, ko = _lens(q_offsets, "q_offsets", batch + 1, rt, dev), _lens(k_offsets, "k_offsets", batch + 1, rt, dev)
        rows = q.shape[0]
        tokens = (batch, min(int(max_q), rows), min(int(max_k), k.shape[0]), left, right, qo, ko, 0, 0, rows,
                  k.shape[0])
    else:
        if k_offsets is not None or max_q is not None or max_k is not None:
            raise ValueError("k_offsets, max_q and max_k: of packed sequences, with q_offsets")
        batch, tq = q.shape[:2]
        if k.shape[0] != batch:
            raise ValueError(f"k: {k.shape[0]} sequences, expected {batch}")
        rows = batch * tq
        tokens = (batch, tq, k.shape[1], left, right, 0, 0, _lens(q_lens, "q_lens", batch, rt, dev),
                  _lens(k_lens, "k_lens", batch, rt, dev), 0, 0)
    return _Shape(H, Hk, d, dv, rows, packed, tokens, code, dev)


def _strided(t, packed: bool) -> tuple:
    """The values of NmHeads."""
    if packed:
        s0, s1, _ = t.stride()
        return t.data_ptr(), 0, s0, s1
    s0, s1, s2, _ = t.stride()
    return t.data_ptr(), s0, s1, s2


_FORWARD, _BACKWARD = _packer(NmDiffArgs), _packer(NmDiffGradArgs)


def _into(t, name: str, shape, like, stream, rt):
    """A given output of heads, or a new one without gaps."""
    if t is None:
        return _empty(shape, like.dtype, like, stream, rt)
    if t.dtype != like.dtype or tuple(t.shape) != tuple(shape) or (t.shape[-1] > 1 and t.stride(-1) != 1):
        raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)}, expected {like.dtype} {tuple(shape)} with consecutive "
                         "channels")
    _apart(t, name)
    _on(t, name, like.get_device())
    return _written(t, rt)


def _scale(scale, d: int) -> float:
    if scale is None:
        return d ** -0.5
    if not (scale > 0 and math.isfinite(scale)):
        raise ValueError(f"scale: {scale}, expected a positive number")
    return scale


def _forward(q, k, v, weight, scale, causal, window, q_lens, k_lens, q_offsets, k_offsets, max_q, max_k, out, train,
             stream):
    rt = nmblock._rt or _runtime()
    C = _calls or _library()
    s = _shape(q, k, v, causal, window, q_lens, k_lens, q_offsets, k_offsets, max_q, max_k, rt)
    out = _into(out, "out", (*q.shape[:-2], s.H, s.dv), q, stream, rt)
    kept = stats = None
    if train:
        kept = _empty((s.rows, s.H, 2, s.dv), rt.torch.int16, q, stream, rt)
        stats = _empty((2 * s.H, _stat_rows(s.dv), s.rows), rt.f32, q, stream, rt)
    p = s.packed
    args = _FORWARD.pack(*_strided(q, p), *_strided(k, p), *_strided(v, p), *_strided(out, p),
                         0 if kept is None else kept.data_ptr(), 0 if stats is None else stats.data_ptr(), *s.tokens,
                         *weight._for(s.H, s.dev), s.code, s.H, s.Hk, s.d, s.dv, _scale(scale, s.d))
    need = _size(C.forward_size, (*s.tokens[:3], s.H, s.Hk, s.d, s.dv, s.dev, s.tokens[6] != 0 or s.tokens[8] != 0), args)
    ws = _empty((need,), rt.u8, q, stream, rt) if need else None
    st = C.forward(args, _ptr(ws), need, _handle(stream, s.dev, rt))
    if st != NM_OK:
        raise NmError(st, "nm_diff_attention")
    return out, kept, stats


def diff_attention(q, k, v, weight: DiffWeight, scale: Optional[float] = None, causal: bool = False, window=None,
                   q_lens=None, k_lens=None, q_offsets=None, k_offsets=None, max_q=None, max_k=None, out=None,
                   stream=None):
    """nm_diff_attention: o [.., H, dv] of q [.., 2 H, d], k [.., 2 Hk, d] and v [.., Hk, dv].

    Head h has the maps of q's heads 2 h and 2 h + 1; H / Hk heads share a key head.  Sequences are padded, [sequences, tokens,
    heads, channels] with q_lens and k_lens (int32 [sequences] on the device; None: all tokens), or packed, [tokens of all,
    heads, channels] with q_offsets (int32 [sequences + 1]) and max_q, no less than the longest; k_offsets and max_k
    where the keys have others.  A row r of nq with nk keys sees key j where -left <= j - (r + nk - nq) <= right:
    window = (left, right), negative for no bound; causal is (-1, 0).  scale: d ** -0.5 without it."""
    return _forward(q, k, v, weight, scale, causal, window, q_lens, k_lens, q_offsets, k_offsets, max_q, max_k, out,
                    False, stream)[0]


def _stat_rows(dv: int) -> int:
    return 1 + (dv + 127) // 128


class DiffForward(NamedTuple):
    """The output o, and what the backward pass reads: int16 codes of both maps' products with v [rows, H, 2, dv], and
    float32 [2 H, 1 + scales, rows]: the base-2 logarithms of the maps' sums and the codes' scales, one for 128 channels."""
    o: object
    kept: object
    stats: object


def diff_attention_train(q, k, v, weight: DiffWeight, scale: Optional[float] = None, causal: bool = False, window=None,
                         q_lens=None, k_lens=None, q_offsets=None, k_offsets=None, max_q=None, max_k=None, out=None,
                         stream=None) -> DiffForward:
    """diff_attention that also keeps what diff_attention_backward reads."""
    return DiffForward(*_forward(q, k, v, weight, scale, causal, window, q_lens, k_lens, q_offsets, k_offsets, max_q,
                                 max_k, out, True, stream))


class DiffGrads(NamedTuple):
    """Gradients of diff_attention's inputs: of q, k, v in their type; of the weight by head and (where it is made from
    them) of its vectors, in float32."""
    dq: object
    dk: object
    dv: object
    dlam: object
    dq1: object
    dk1: object
    dq2: object
    dk2: object


def diff_attention_backward(grad_o, forward: DiffForward, q, k, v, weight: DiffWeight, scale: Optional[float] = None,
                            causal: bool = False, window=None, q_lens=None, k_lens=None, q_offsets=None, k_offsets=None,
                            max_q=None, max_k=None, dq=None, dk=None, dv=None, stream=None) -> DiffGrads:
    """nm_diff_attention_backward: from grad_o (of o's shape), at what diff_attention_train returned for the same
    arguments.  Rows behind a sequence's end are left as they were in given dq, dk and dv."""
    rt = nmblock._rt or _runtime()
    C = _calls or _library()
    s = _shape(q, k, v, causal, window, q_lens, k_lens, q_offsets, k_offsets, max_q, max_k, rt)
    _, kept, stats = forward
    shape = (*q.shape[:-2], s.H, s.dv)
    if grad_o.dtype != q.dtype or tuple(grad_o.shape) != shape or (s.dv > 1 and grad_o.stride(-1) != 1):
        raise ValueError(f"grad_o: {grad_o.dtype} {tuple(grad_o.shape)}, expected {q.dtype} {shape} with consecutive "
                         "channels")
    _on(grad_o, "grad_o", s.dev)
    for t, name, dtype, want in ((kept, "kept", rt.torch.int16, (s.rows, s.H, 2, s.dv)),
                                 (stats, "stats", rt.f32, (2 * s.H, _stat_rows(s.dv), s.rows))):
        if t is None or t.dtype != dtype or tuple(t.shape) != want or not t.is_contiguous():
            raise ValueError(f"{name}: expected contiguous {dtype} {want}, as diff_attention_train gives it")
        _on(t, name, s.dev)
    w = weight._for(s.H, s.dev)
    dq, dk, dv = (_into(t, name, x.shape, x, stream, rt) for t, name, x in ((dq, "dq", q), (dk, "dk", k), (dv, "dv", v)))
    dlam, vectors = _empty((s.H,), rt.f32, q, stream, rt), [None] * 4
    if weight.vectors is not None:
        each = _empty((4, *weight.vectors[0].shape), rt.f32, q, stream, rt)
        vectors = list(each.unbind(0))
    p = s.packed
    args = _BACKWARD.pack(*(x for t in (q, k, v, grad_o, dq, dk, dv) for x in _strided(t, p)), kept.data_ptr(),
                          stats.data_ptr(), dlam.data_ptr(), *(_ptr(t) or 0 for t in vectors), *s.tokens, *w, s.code, s.H,
                          s.Hk, s.d, s.dv, _scale(scale, s.d))
    key = ("backward", *s.tokens[:3], s.rows, s.H, s.Hk, s.d, s.dv, s.dev)
    need = _size(C.backward_size, key, args)
    ws = _empty((need,), rt.u8, q, stream, rt) if need else None
    st = C.backward(args, _ptr(ws), need, _handle(stream, s.dev, rt))
    if st != NM_OK:
        raise NmError(st, "nm_diff_attention_backward")
    return DiffGrads(dq, dk, dv, dlam, *vectors)
