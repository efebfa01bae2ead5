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


def weight(g, n, k, N=8, M=8):
    """Random int8 weight [n x k] (CPU) with at most N nonzeros in each window of M, and its scales."""
    w = torch.randint(-127, 128, (n, k), generator=g, dtype=torch.int64)
    if N < M:
        keep = torch.rand(n, k // M, M, generator=g).argsort(2).argsort(2) < N
        w = w * keep.view(n, k)
    return w.to(torch.int8), torch.exp(torch.randn(n, generator=g)) * 1e-3


def product(q, s, w, c, b):
    """(y, magnitude) of the scaled product in 64 bits; q holds k codes a row.  Magnitude: each of its terms once,
    for the four roundings in binary32 (the sum's conversion, two products, the addition)."""
    sums = q.double().cpu() @ w.double().cpu().t()
    y = sums * s.double().cpu()[:, None] * c.double().cpu()
    mag = y.abs()
    if b is not None:
        y, mag = y + b.double().cpu(), mag + b.double().cpu().abs()
    return y, mag


def act(g, name):
    """act(g) and its derivative in 64 bits."""
    s = torch.sigmoid(g)
    if name == "silu":
        return g * s, s * (1 + g * (1 - s))
    if name == "sigmoid":
        return s, s * (1 - s)
    if name == "relu":
        return torch.where(g > 0, g, torch.zeros_like(g)), (g > 0).double()
    if name == "gelu":
        p = 0.5 * torch.erfc(-g / 2 ** 0.5)
        return g * p, p + g * torch.exp(-g * g / 2) / (2 * torch.pi) ** 0.5
    a = (2 / torch.pi) ** 0.5
    t = torch.tanh(a * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * a * (1 + 3 * 0.044715 * g * g)


def gated(q, s, wg, cg, bg, wu, cu, bu, name):
    """(h, magnitude) in 64 bits: with the errors of g and u (4 e of their magnitudes; slopes of act are below 1.2)
    and of act itself: the exponential's argument and result are within 2 e (1 + |g|), so act(g) is within
    8 e (1 + g^2) of its value."""
    g, gm = product(q, s, wg, cg, bg)
    u, um = product(q, s, wu, cu, bu)
    f, _ = act(g, name)
    return f * u, u.abs() * (1.2 * gm + 2 * (1 + g * g)) + f.abs() * um


def gated_grads(q, s, wg, cg, bg, wu, cu, bu, name, dh, dtype):
    """{name: (gradient, room)} in 64 bits; room: what the operands' one rounding to dtype and the sums in binary32
    may add to the gradient's own rounding."""
    g, gm = product(q, s, wg, cg, bg)
    u, um = product(q, s, wu, cu, bu)
    f, df = act(g, name)
    dh = dh.double().cpu()
    dg, du = dh * u * df, dh * f
    # errors of dg and du in binary32 (second derivatives of act are below 1.2, slopes within 8 e (1 + |g|^3))
    eg = dh.abs() * 4 * E * (um * (df.abs() + 1) + u.abs() * (1.2 * gm + 2 * (1 + g.abs() ** 3)))
    eu = dh.abs() * 4 * E * (1.2 * gm + 2 * (1 + g * g))
    x = q.double().cpu() * s.double().cpu()[:, None]
    wg, wu = wg.double().cpu() * cg.double().cpu()[:, None], wu.double().cpu() * cu.double().cpu()[:, None]
    m, n = dg.shape
    unit = UNIT[dtype] + (K + n / 16) * E
    out = {"dx": (dg @ wg + du @ wu,
                  (dg.abs() * unit + eg) @ wg.abs() + (du.abs() * unit + eu) @ wu.abs()
                  + TINY[dtype] * (wg.abs() / cg.double().cpu()[:, None] + wu.abs() / cu.double().cpu()[:, None]).sum(0))}
    unit = UNIT[dtype] + (K + m / 16) * E
    sub = TINY[dtype] * q.double().cpu().abs().sum(0)       # codes times a power of two, beside d's subnormal step
    out["dw_gate"] = (dg.t() @ x, (dg.abs() * unit + eg).t() @ x.abs() + sub)
    out["dw_up"] = (du.t() @ x, (du.abs() * unit + eu).t() @ x.abs() + sub)
    if bg is not None:
        out["dbias_gate"] = (dg.sum(0), (dg.abs() * (K + m / 16) * E + eg).sum(0))
        out["dbias_up"] = (du.sum(0), (du.abs() * (K + m / 16) * E + eu).sum(0))
    return out
