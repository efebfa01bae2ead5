"""64-bit forms of rotary positions and differential attention, and the error bounds that their tests use.

Bounds are derived, not fitted.  u is half a unit in the last place of the type (2^-11 binary16, 2^-8 bfloat16), e = 2^-24.

Rotary: the angle in turns is made in 64 bits (three roundings of 2^-53, times the number of turns) and reduced to 32
bits within half a turn: 2^-25 of a turn, 2 pi 2^-25 < 4 e of an angle.  Sine and cosine add at most 4 e, the rotation two
products and a sum: 2 e.  |out - want| <= u |want| + (12 e + 8 |a| 2^-53) (|u| + |w|).

Attention.  A score's chain of d products is within (d + 8) e S, S the largest sum of |q||k| times scale, and is the exponent
of a map's value, which the hardware's exponential makes to 2 e: a value of a map is within eta = (2 (d + 8) S + 16) e of
itself (twice: the sum that divides it has the same error).  The product with v adds at most n / 16 + 32 roundings of a chain
over n keys.  Before that product the map's values are rounded: u each, and half a subnormal step of binary16 (2^-25) of
values whose largest is 1 or more.  So with A = p1 |v| + |lam| p2 |v|:
  |o - want| <= u |want| + (u + eta + (n / 16 + 32) e) A + 2^-25 sum |v| (binary16)
The backward pass rounds ds and p1 - lam p2 the same way (u; absolute 2^-25, its values being at most 1 there) and takes
D1 and D2 from codes of p_i v: half a step of 1 / 32767 of the largest, besides the bound above (and 4 e for making and
taking a code); all of it goes through the same products.  The sums of p2 dp for dlam have no 16-bit rounding."""
import math

import torch

E = 2.0 ** -24
UNIT = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150}


def within(got, want, room, what=""):
    g, w = got.detach().double().cpu(), want.double().cpu()
    assert g.shape == w.shape, (what, g.shape, w.shape)
    assert torch.isfinite(g).all(), (what, "not finite", int((~torch.isfinite(g)).sum()))
    off = (g - w).abs()
    bad = off > torch.as_tensor(room, dtype=torch.float64).cpu().expand_as(w)
    assert not bad.any(), (what, int(bad.sum()), w.numel(), float((off / room.cpu()).max()))


def rotary(x, pos, freqs, axis, style, back=False):
    """(out, room without the output's rounding) of x [tokens, heads, d] in 64 bits."""
    n = len(freqs)
    at = pos.double().cpu()[list(axis)].t() * torch.tensor(freqs, dtype=torch.float64)
    c, s = torch.cos(at)[:, None], torch.sin(at)[:, None] * (-1 if back else 1)
    x = x.double().cpu()
    y, room = x.clone(), torch.zeros_like(x)
    iu, iw = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if style == "pairs" else (slice(0, n), slice(n, 2 * n))
    u, w = x[..., iu], x[..., iw]
    y[..., iu], y[..., iw] = u * c - w * s, u * s + w * c
    k = (12 * E + 8 * at.abs()[:, None] * 2.0 ** -53) * (u.abs() + w.abs())
    room[..., iu], room[..., iw] = k, k
    return y, room


def seen(nq, nk, left, right):
    off = torch.arange(nk)[None] - (torch.arange(nq)[:, None] + nk - nq)
    ok = torch.ones(nq, nk, dtype=torch.bool)
    if left >= 0:
        ok &= off >= -left
    if right >= 0:
        ok &= off <= right
    return ok


def head(q, k, v, lam, scale, ok, T, do=None):
    """One head of one sequence: q, k pairs of [n x d], v [nk x dv], all 64 bits.  A dict of (value, room)."""
    nk, d, u = v.shape[0], q[0].shape[1], UNIT[T]
    n, half = max(1, nk), T == torch.float16
    p, lse, S = [], [], 0.0
    for i in (0, 1):
        z = (q[i] @ k[i].t() * scale).masked_fill(~ok, -math.inf)
        if nk and q[i].shape[0]:
            S = max(S, float((q[i].abs() @ k[i].abs().t()).max()) * scale)
        total = torch.logsumexp(z, 1, keepdim=True) if nk else torch.full((q[i].shape[0], 1), -math.inf,
                                                                          dtype=torch.float64)
        p.append(torch.where(ok, torch.exp(z - torch.where(total == -math.inf, 0.0, total)), 0.0))
        lse.append(torch.where(total == -math.inf, math.inf, total / math.log(2))[:, 0])
    eta = (2 * (d + 8) * S + 16) * E
    kappa = eta + (n / 16 + 32) * E
    al = abs(lam)
    o1, o2 = p[0] @ v, p[1] @ v
    A1, A2 = p[0] @ v.abs(), p[1] @ v.abs()
    tiny = TINY[T] * v.abs().sum(0) if half else 0.0 * v.abs().sum(0)
    o = o1 - lam * o2
    e1, e2 = (u + kappa) * A1 + tiny, (u + kappa) * A2 + tiny         # of o1 and o2 before their rounding
    step = [e + x.abs().amax(1, keepdim=True) * (2.0 ** -16 * 1.01 + 4 * E) if x.numel() else e
            for x, e in ((o1, e1), (o2, e2))]
    out = dict(o=(o, u * o.abs() + (e1 + al * e2) + TINY[T]), kept=(torch.stack((o1, o2), 1), torch.stack(step, 1)),
               lse=(torch.stack(lse), torch.full((2, 1), 2 * eta + 32 * E, dtype=torch.float64)))
    if do is None:
        return out
    both = p[0] - lam * p[1]
    dp, dpm = do @ v.t(), do.abs() @ v.abs().t()
    m = max(1, q[0].shape[0])
    kap = eta + (m / 16 + 32) * E
    mags = p[0] + al * p[1]
    dv = both.t() @ do
    dvr = (u + kap) * (mags.t() @ do.abs()) + (TINY[T] * do.abs().sum(0) if half else 0.0)
    out["dv"] = (dv, dvr)
    D = [(p[i] * dp).sum(1, keepdim=True) for i in (0, 1)]
    # the codes' errors, through do
    r1, r2 = ((do.abs() * (s + 300 * E * x.abs())).sum(1, keepdim=True) for s, x in zip(step, (o1, o2)))
    out["dlam"] = (-D[1].sum(), (kappa + 400 * E + (m / 16 + 64) * E) * float((p[1] * dpm).sum()) + 1e-30)
    for i, (r, f, amp) in enumerate(((r1, 1.0, 1.0), (r2, -lam, al))):
        ds = f * p[i] * (dp - D[i])
        room = amp * p[i] * (r + 300 * E * dpm + (u + eta) * (dp - D[i]).abs()) + (TINY[T] * max(1.0, amp) if half else
                                                                                  0.0)
        out[f"dq{i}"] = (scale * ds @ k[i], scale * (room @ k[i].abs()) + kappa * scale * (ds.abs() @ k[i].abs()))
        out[f"dk{i}"] = (scale * ds.t() @ q[i], scale * (room.t() @ q[i].abs()) + kap * scale * (ds.abs().t() @
                                                                                                q[i].abs()))
    return out


def attention(q, k, v, lam, scale, spans, left, right, T, do=None):
    """spans: (rows of q, rows of k) of each sequence as slices of flattened tokens.  q [rows, 2 H, d] ... flattened, in
    their 16-bit type.  {name: (value, room)} in flattened layouts; untouched rows are NaN."""
    q, k, v = (t.detach().double().cpu() for t in (q, k, v))
    do = None if do is None else do.detach().double().cpu()
    H, Hk, u = q.shape[1] // 2, v.shape[1], UNIT[T]
    nan = lambda *s: torch.full(s, math.nan, dtype=torch.float64)  # noqa: E731
    R = q.shape[0]
    res = dict(o=[nan(R, H, v.shape[2]), nan(R, H, v.shape[2])],
               kept=[nan(R, H, 2, v.shape[2]), nan(R, H, 2, v.shape[2])],
               lse=[nan(2 * H, R), nan(2 * H, R)])
    if do is not None:
        res.update(dq=[nan(*q.shape), nan(*q.shape)], dk=[nan(*k.shape), nan(*k.shape)], dv=[nan(*v.shape), nan(*v.shape)],
                   dlam=[torch.zeros(H, dtype=torch.float64), torch.zeros(H, dtype=torch.float64)])
    for rows, keys in spans:
        nq, nk = len(range(*rows.indices(R))), len(range(*keys.indices(k.shape[0])))
        ok = seen(nq, nk, left, right)
        if do is not None:
            for x in (0, 1):
                res["dk"][x][keys] = 0
                res["dv"][x][keys] = 0
        for h in range(H):
            g = h // (H // Hk)
            one = head([q[rows, 2 * h + i] for i in (0, 1)], [k[keys, 2 * g + i] for i in (0, 1)], v[keys, g],
                       float(lam[h]), scale, ok, T, None if do is None else do[rows, h])
            for x in (0, 1):
                res["o"][x][rows, h], res["kept"][x][rows, h] = one["o"][x], one["kept"][x]
                for i in (0, 1):
                    res["lse"][x][2 * h + i, rows] = one["lse"][x][i]
            if do is None:
                continue
            for x in (0, 1):
                for i in (0, 1):
                    res["dq"][x][rows, 2 * h + i] = one[f"dq{i}"][x]
                    res["dk"][x][keys, 2 * g + i] += one[f"dk{i}"][x]
                res["dv"][x][keys, g] += one["dv"][x]
                res["dlam"][x][h] += one["dlam"][x]
    for name in ("dq", "dk", "dv"):
        if name in res:     # and the outputs' own rounding
            res[name][1] = res[name][1] + u * res[name][0].abs() + TINY[T]
    return res
