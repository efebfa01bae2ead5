"""Plain 64-bit forms of the transformer-block operators, and the error bounds that their tests use.

Bounds are derived, not fitted.  u(T) is half a unit in the last place of the output type (2^-11 binary16, 2^-8
bfloat16, 2^-24 binary32), e = 2^-24 that of binary32.  A value that is computed in binary32 by a chain of additions and
products over terms of total magnitude M is within K e M, K the longest chain: at most 16 terms in a lane, 6 steps in
a wave, 16 waves, and a dozen operations around them: K = 64.  Column sums over m tokens add at most
16 + m / 16 terms in a row: K = 64 + m / 16.  Where a row is centred, rounding of the inputs is relative to the values
before: M carries the factor max|v| / deviation."""
import numpy as np
import torch

E = 2.0 ** -24
UNIT = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
TINY = {torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133, torch.float32: 2.0 ** -149}
TYPES = [torch.float16, torch.bfloat16, torch.float32]
K = 64


def close(got, want, dtype, magnitude, k=K):
    """|got - want| <= u |want| + k e magnitude (+ one subnormal step), element by element; exact where not finite."""
    g, w = got.detach().double().cpu(), want.double().cpu()
    assert g.shape == w.shape, (g.shape, w.shape)
    odd = ~torch.isfinite(w)
    assert torch.equal(torch.isnan(g), torch.isnan(w))
    assert torch.equal(g[odd & ~torch.isnan(w)], w[odd & ~torch.isnan(w)])
    mag = torch.as_tensor(magnitude, dtype=torch.float64).expand_as(w)
    room = UNIT[dtype] * w.abs() + k * E * mag * (1 + UNIT[dtype]) + TINY[dtype]
    off = (g - w).abs()
    bad = (off > room) & ~odd
    assert not bad.any(), (int(bad.sum()), float((off / room)[~odd].max()))


def codes(x):
    """Codes and scales of rows, decided in binary32 as the operator defines them (numpy: correctly rounded)."""
    x = x.detach().float().cpu().numpy()
    with np.errstate(all="ignore"):
        top = np.abs(x).max(1)
        inv = (np.float32(127) / top).astype(np.float32)
        scale = (top / np.float32(127)).astype(np.float32)
        tiny, odd = top < np.float32(2.0 ** -100), ~np.isfinite(top)
        inv[tiny | odd], scale[tiny], scale[odd] = 0, 0, np.nan
        q = np.rint((x * inv[:, None]).astype(np.float32))
    q[odd] = 0
    return torch.from_numpy(q.astype(np.int8)), torch.from_numpy(scale)


def hat(v, norm):
    """(normalised rows, 1 / deviation) in 64 bits; norm: (kind, weight, bias, eps) or None."""
    kind, _, _, eps = norm
    mu = v.mean(1, keepdim=True) if kind == "layer" else 0.0
    inv = 1 / torch.sqrt(((v - mu) ** 2).mean(1, keepdim=True) + eps)
    return (v - mu) * inv, inv


def affine(h, norm):
    _, w, b, _ = norm
    h = h if w is None else h * w.double().cpu()
    return h if b is None else h + b.double().cpu()


def norm_residual(y, r, pre, post, gate, alpha):
    """(res, z, magnitude of res, magnitude of z) of [m x d] inputs (None: absent), 64 bits."""
    m, d = (y if y is not None else r).shape
    rows = torch.ones(1, d, dtype=torch.float64) if gate is None else gate.double().cpu().reshape(-1, d)
    rows = rows.repeat_interleave(m // rows.shape[0], 0)
    term, mag = torch.zeros(m, d, dtype=torch.float64), torch.zeros(m, d, dtype=torch.float64)
    if y is not None:
        v = y.double().cpu()
        u, um = v, v.abs()
        if post is not None:
            h, inv = hat(v, post)
            u = affine(h, post)
            um = affine(torch.ones_like(h), tuple(None if t is None else t.abs() if torch.is_tensor(t) else t
                                                  for t in post)) * (1 + v.abs().amax(1, keepdim=True) * inv)
        term, mag = rows * u, rows.abs() * um
    if r is not None:
        term, mag = term + alpha * r.double().cpu(), mag + abs(alpha) * r.double().cpu().abs()
    if pre is None:
        return term, None, mag, None
    h, inv = hat(term, pre)
    wide = affine(torch.ones_like(h), tuple(None if t is None else t.abs() if torch.is_tensor(t) else t for t in pre))
    return term, affine(h, pre), mag, wide * (1 + (mag.amax(1, keepdim=True)) * inv) * (1 + h.abs())


def norm_grads(dz, dres, y, res, pre, post, gate, alpha):
    """{name: (gradient, magnitude)} in 64 bits, by the formulas."""
    like = dz if dz is not None else dres
    m, d = like.shape
    dt = torch.zeros(m, d, dtype=torch.float64) if dres is None else dres.double().cpu()
    tm = dt.abs()
    out = {}

    def through(v, g, gm, norm, name):
        h, inv = hat(v, norm)
        kind, w, b, _ = norm
        amp = 1 + v.abs().amax(1, keepdim=True) * inv
        if w is not None:
            out[f"d{name}_weight"] = ((g * h).sum(0), (gm * (1 + h.abs()) * amp).sum(0))
        if b is not None:
            out[f"d{name}_bias"] = (g.sum(0), gm.sum(0))
        wd = torch.ones(d, dtype=torch.float64) if w is None else w.double().cpu()
        t, a = g * wd, gm * wd.abs()
        mean = t.mean(1, keepdim=True) if kind == "layer" else 0.0
        back = inv * (t - mean - h * (t * h).mean(1, keepdim=True))
        size = inv * (a + a.mean(1, keepdim=True) + (1 + h.abs()) * (a * (1 + h.abs())).mean(1, keepdim=True)) * amp
        return back, size

    if pre is not None and dz is not None:
        back, size = through(res.double().cpu(), dz.double().cpu(), dz.double().cpu().abs(), pre, "pre")
        dt, tm = dt + back, tm + size
    out["dr"] = (alpha * dt, abs(alpha) * tm)
    if y is None:
        return out
    groups = 1 if gate is None or gate.dim() == 1 else gate.shape[0]
    rows = torch.ones(1, d, dtype=torch.float64) if gate is None else gate.double().cpu().reshape(-1, d)
    rows = rows.repeat_interleave(m // groups, 0)
    v = y.double().cpu()
    if post is None:
        u, um = v, v.abs()
        out["dy"] = (dt * rows, tm * rows.abs())
    else:
        h, inv = hat(v, post)
        u = affine(h, post)
        um = (u.abs() + h.abs() + 1) * (1 + v.abs().amax(1, keepdim=True) * inv)
        out["dy"] = through(v, dt * rows, tm * rows.abs(), post, "post")
    if gate is not None:
        out["dgate"] = tuple(t.reshape(groups, m // groups, d).sum(1).reshape(gate.shape) for t in (dt * u, tm * um))
    return out
