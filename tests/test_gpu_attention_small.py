"""Differential attention in binary16 where values are small: its exponents end at 2^-14, its steps at 2^-24, and maps
over thousands of keys and the gradients of scores lie far below.

Bounds, with u = 2^-11, E = 2^-24 and the names of attention_util (a 16-bit rounding besides u costs half a step of 2^-24 in
its scaled place).  dp = do v^T; top = |do| of a row (for dk: of the rows, times max(1, |lam|)) times the largest |v|:
  ds for dq is scaled so that top is 2^13 or more:      2^-25 / 2^13 top = 2^-38 top
  ds for dk is scaled so that top is 2^12 or more:      2^-37 top (the rows' tops are known to a factor of 2)
  maps in the forward pass are 2^7 or more where their scores are largest: 2^-32 for each |v|
  p0 - lam p1 for dv is scaled so that 1 + |lam| (the largest of the heads that share it) is 2^14 or more: 2^-39 (1 + |lam|)
A row's own bits: every operation but the last rounding scales by powers of two, so gradients of 2^-s do are those of do
times 2^-s, to one rounding of each (2 steps of 2^-24 where they leave the normal range, else none).  (The sum over
heads of dk's bounds has their roundings of the output once each: more than there are.)"""
import math

import pytest
import torch

import attention_util as au
from paper_2607_12505_amd import nmattention as na

pytestmark = pytest.mark.gpu
T, U, E = torch.float16, 2.0 ** -11, 2.0 ** -24
WIDTHS = [(32, 64), (64, 128), (61, 107), (128, 128), (128, 256)]


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(g, *shape):
    return torch.randn(*shape, generator=g)


def maps(q, k, scale, ok):
    """p_i [2, rows, keys] of one head in 64 bits, and the largest sum of |q||k| scale."""
    z = torch.stack([q[:, i] @ k[:, i].t() for i in (0, 1)]) * scale
    S = max(float((q[:, i].abs() @ k[:, i].abs().t()).max()) for i in (0, 1)) * scale
    return torch.softmax(z.masked_fill(~ok, -math.inf), -1), S


def case(g, Tq, Tk, d, dv, do, wide):
    """One head, widened by powers of two so that dq (wide "q") or dk ("k") are of the size of do; scores are those of
    N(0, 1) rows."""
    q, k, v = randn(g, 1, Tq, 2, d), randn(g, 1, Tk, 2, d), randn(g, 1, Tk, 1, dv)
    f = 2.0 ** -8
    q, k = (q * f, k) if wide == "q" else (q, k * f)
    return [t.to(T).cuda() for t in (q, k, v)], d ** -0.5 / f, (do * randn(g, 1, Tq, 1, dv)).to(T).cuda()


def exact(q, k, v, do, lam, scale, window, head=0, group=1):
    """dq and dk of one head in 64 bits, and their bounds: (dq0, dk0, dq1, dk1, dlam)."""
    q, k, v, do = (t.double().cpu()[0] for t in (q, k, v, do))
    g = head // group
    q, k, v, do = q[:, 2 * head:2 * head + 2], k[:, 2 * g:2 * g + 2], v[:, g], do[:, head]
    (n, d), m = (q.shape[0], q.shape[2]), k.shape[0]
    scale = float(torch.tensor(scale, dtype=torch.float32))
    p, S = maps(q, k, scale, au.seen(n, m, *window))
    eta = (2 * (d + 8) * S + 16) * E
    kappa, kap = eta + (m / 16 + 32) * E, eta + (n / 16 + 32) * E
    dp, dpm = do @ v.t(), do.abs() @ v.abs().t()
    top = do.norm(dim=1, keepdim=True) * v.norm(dim=1).max()
    all_top = float(top.max()) * max(1.0, abs(lam))
    out = []
    for i, amp in ((0, 1.0), (1, abs(lam))):
        f = 1.0 if i == 0 else -lam
        o, A = p[i] @ v, p[i] @ v.abs()
        step = (U + kappa) * A + 2.0 ** -25 * v.abs().sum(0) + o.abs().amax(1, keepdim=True) * (2.0 ** -16 * 1.01 + 4 * E)
        r = (do.abs() * (step + 300 * E * o.abs())).sum(1, keepdim=True)
        D = (p[i] * dp).sum(1, keepdim=True)
        ds = f * p[i] * (dp - D)
        room = amp * p[i] * (r + 300 * E * dpm + (U + eta) * (dp - D).abs())
        for x, y, tiny, chain in ((ds, k[:, i], amp * 2.0 ** -38 * top, kappa),
                                  (ds.t(), q[:, i], torch.full((1, 1), 2.0 ** -37 * all_top, dtype=torch.float64), kap)):
            w = scale * x @ y
            e = room if x is ds else room.t()
            out.append((w, scale * ((e + tiny) @ y.abs() + chain * (x.abs() @ y.abs())) + U * w.abs() + 2.0 ** -25))
    out.append((-D.sum(), (kappa + 400 * E + (n / 16 + 64) * E) * float((p[1] * dpm).sum()) + 1e-30))
    return out


# few rows of few keys for dq (a sum over keys hides what each of them loses), few rows of many keys for dk
@pytest.mark.parametrize("d,dv", WIDTHS)
@pytest.mark.parametrize("size", [1e-2, 1e-4, 1e-5, 1e-6])
@pytest.mark.parametrize("Tq,Tk,wide", [(40, 3, "q"), (3, 40, "q"), (1, 4100, "k"), (2, 4100, "k"), (33, 2049, "k")])
def test_gradients_of_scores_keep_their_bits(d, dv, size, Tq, Tk, wide):
    g, lam = gen(Tk + d), 0.6
    (q, k, v), scale, do = case(g, Tq, Tk, d, dv, size, wide)
    weight = na.DiffWeight(torch.tensor([lam], device="cuda"))
    f = na.diff_attention_train(q, k, v, weight, scale=scale)
    got = na.diff_attention_backward(do, f, q, k, v, weight, scale=scale)
    want = exact(q, k, v, do, float(weight.value), scale, (-1, -1))
    for i in (0, 1):
        for name, t, (w, room) in (("dq", got.dq[0, :, i], want[2 * i]), ("dk", got.dk[0, :, i], want[2 * i + 1])):
            au.within(t, w, room, (name, i))


def steps(g, *shape):
    """Values of at most 7 bits down to 2^-5: times 2^-19 they are still binary16."""
    return torch.randint(-128, 129, shape, generator=g).float() / 32


@pytest.mark.parametrize("d,dv", WIDTHS)
@pytest.mark.parametrize("Tq,Tk,H,Hk,window", [(300, 300, 2, 1, (-1, 0)), (200, 1000, 2, 2, (-1, -1)), (40, 4096, 4, 1, (-1, 0)),
                                               (1500, 130, 1, 1, (60, 5))])
def test_gradients_scale_with_the_output_s(d, dv, Tq, Tk, H, Hk, window):
    g = gen(d + Tq)
    for wide in ("q", "k"):
        q, k = randn(g, 1, Tq, 2 * H, d), randn(g, 1, Tk, 2 * Hk, d)
        f = 2.0 ** -10
        q, k = ((q * f, k) if wide == "q" else (q, k * f))
        q, k, v = (t.to(T).cuda() for t in (q, k, randn(g, 1, Tk, Hk, dv)))
        weight, do = na.DiffWeight((0.2 + torch.rand(H, generator=g)).cuda()), steps(g, 1, Tq, H, dv)
        how = dict(scale=d ** -0.5 / f, window=window)
        fw = na.diff_attention_train(q, k, v, weight, **how)
        one = na.diff_attention_backward(do.to(T).cuda(), fw, q, k, v, weight, **how)
        for s in (7, 13):
            got = na.diff_attention_backward((do * 2.0 ** -s).to(T).cuda(), fw, q, k, v, weight, **how)
            assert torch.equal(got.dlam * 2.0 ** s, one.dlam)
            for name in ("dv", "dq" if wide == "q" else "dk"):
                a, b = getattr(got, name).double(), getattr(one, name).double() * 2.0 ** -s
                far = torch.isfinite(b) & (b.abs() >= 2.0 ** -14)      # normal in both
                assert torch.equal(a[far], b[far]), (name, s, int((a[far] != b[far]).sum()), int(far.sum()))
                assert ((a - b)[torch.isfinite(b)].abs() <= 2.0 ** -23).all()
        # do below 2^-16: the matrix instruction adds products of subnormal values less exactly, within the bounds still
        # (|a - b| <= |a - w| + |b - w|, w the formula's value, each within its room)
        small = (do * 2.0 ** -19).to(T).cuda()
        got = na.diff_attention_backward(small, fw, q, k, v, weight, **how)
        sums = {}
        for h in range(H):
            res = exact(q, k, v, small, float(weight.value[h]), how["scale"], window, h, H // Hk)
            for i in (0, 1):
                sums[("dq", 2 * h + i)] = res[2 * i]
                key = ("dk", 2 * (h // (H // Hk)) + i)
                sums[key] = res[2 * i + 1] if key not in sums else tuple(x + y for x, y in zip(sums[key], res[2 * i + 1]))
            au.within(got.dlam[h] * 1.0, res[4][0], res[4][1], "dlam")
        for (name, at), (w, room) in sums.items():
            au.within(getattr(got, name)[0, :, at], w, room, (name, at))


@pytest.mark.parametrize("d,dv", [(32, 64), (64, 128), (128, 256)])
def test_rows_of_all_sizes_beside_each_other(d, dv):
    # a row's dq does not depend on the sizes of the rows beside it; a row that is not finite spoils none of the others
    g, n = gen(d), 200
    (q, k, v), scale, _ = case(g, n, n, d, dv, 1.0, "q")
    weight, do = na.DiffWeight(torch.tensor([0.4], device="cuda")), steps(g, 1, n, 1, dv)
    shift = torch.randint(0, 20, (1, n, 1, 1), generator=g)
    fw = na.diff_attention_train(q, k, v, weight, scale=scale)
    one = na.diff_attention_backward(do.to(T).cuda(), fw, q, k, v, weight, scale=scale)
    got = na.diff_attention_backward((do * 2.0 ** -shift).to(T).cuda(), fw, q, k, v, weight, scale=scale)
    a, b = got.dq.double(), one.dq.double() * 2.0 ** -shift.cuda()
    far = (b.abs() >= 2.0 ** -14) & (shift.cuda() <= 13)               # (smaller rows: as above)
    assert torch.equal(a[far], b[far]) and int(far.sum()) > far.numel() // 4
    res = exact(q, k, v, (do * 2.0 ** -shift).to(T), float(weight.value), scale, (-1, -1))
    for i in (0, 1):
        au.within(got.dq[0, :, i], *res[2 * i], ("dq", i))
        au.within(got.dk[0, :, i], *res[2 * i + 1], ("dk", i))
    for bad in (math.inf, math.nan):
        do2 = do.to(T).cuda()
        do2[0, 37, 0, 5] = bad
        dq = na.diff_attention_backward(do2, fw, q, k, v, weight, scale=scale).dq
        keep = torch.arange(n) != 37
        assert torch.equal(dq[0, keep], one.dq[0, keep]) and dq[0, 37].isnan().any()


def test_large_gradients_and_weights_stay_finite():
    # ds of 2^17 and more, whose sums with small keys (queries) binary16 holds
    g, n, d, dv = gen(3), 70, 64, 128
    for lam in (0.5, 300.0):
        q, k, v = randn(g, 1, n, 2, d) * 2.0 ** -9, randn(g, 1, n, 2, d) * 2.0 ** -9, randn(g, 1, n, 1, dv) * 64
        q, k, v, do = (t.to(T).cuda() for t in (q, k, v, 512 * randn(g, 1, n, 1, dv)))
        weight = na.DiffWeight(torch.tensor([lam], device="cuda"))
        f = na.diff_attention_train(q, k, v, weight, scale=0.125, causal=True)
        got = na.diff_attention_backward(do, f, q, k, v, weight, scale=0.125, causal=True)
        want = exact(q, k, v, do, lam, 0.125, (-1, 0))
        for i in (0, 1):
            for name, t, (w, room) in (("dq", got.dq[0, :, i], want[2 * i]), ("dk", got.dk[0, :, i], want[2 * i + 1])):
                if float(w.abs().max()) < 60000:
                    au.within(t, w, room, (name, i, lam))


# one row, so that no sum hides what a key loses; maps of 2^-16 and far below
@pytest.mark.parametrize("d,dv", WIDTHS)
@pytest.mark.parametrize("Tq,Tk,lams", [(1, 70000, (0.6,)), (1, 70000, (0.3, 40.0)), (2, 50001, (0.8,)), (3, 9000, (0.0,)),
                                        (1, 5, (2e5,)), (40, 300, (1e4, 0.5))])
def test_gradients_of_values_keep_their_bits(d, dv, Tq, Tk, lams):
    g, H = gen(Tk + d), len(lams)
    q, k, v = randn(g, 1, Tq, 2 * H, d), randn(g, 1, Tk, 2, d), 0.01 * randn(g, 1, Tk, 1, dv)
    q, k, v = (t.to(T).cuda() for t in (q, k, v))
    # outputs of about 1: off the last steps of their own type
    do = (min(Tk, 4096) / (1 + max(lams)) * randn(g, 1, Tq, H, dv)).to(T).cuda()
    weight = na.DiffWeight(torch.tensor(lams, device="cuda"))
    f = na.diff_attention_train(q, k, v, weight)
    got = na.diff_attention_backward(do, f, q, k, v, weight).dv[0, :, 0]
    scale = float(torch.tensor(d ** -0.5, dtype=torch.float32))
    want = room = 0.0
    for h, lam in enumerate(weight.value.tolist()):
        at = slice(2 * h, 2 * h + 2)
        p, S = maps(q[0, :, at].double().cpu(), k[0].double().cpu(), scale, au.seen(Tq, Tk, -1, -1))
        kap = (2 * (d + 8) * S + 16) * E + (Tq * H / 16 + 32) * E
        x, y = p[0] - lam * p[1], do[0, :, h].double().cpu()
        want = want + x.t() @ y
        room = room + (U + kap) * ((p[0] + lam * p[1]).t() @ y.abs()) + 2.0 ** -39 * (1 + max(lams)) * y.abs().sum(0)
    au.within(got, want, room + U * want.abs() + 2.0 ** -25, "dv")


# a key that takes nearly all of a row and has no value itself: the row is what the others add, 2^-25.5 of it each (values
# of hundreds; few rows, and many rows in tiles that are shared)
@pytest.mark.parametrize("d,dv", WIDTHS)
@pytest.mark.parametrize("B,Tq,Tk,sink", [(1, 1, 4000, 0), (1, 1, 300, 299), (2, 3, 9001, 4500), (100, 130, 70, 3), (1, 40, 2100, 7)])
def test_keys_of_little_weight_count(d, dv, B, Tq, Tk, sink):
    g = gen(Tk + d)
    q, k, v = randn(g, 1, Tq, 2, d) * 0.05, randn(g, 1, Tk, 2, d) * 0.05, 200 + 100 * randn(g, 1, Tk, 1, dv)
    q[..., 0] = 1.0
    k[..., 0], v[0, sink] = 0.0, 0.0
    scale = float(torch.tensor(d ** -0.5, dtype=torch.float32))
    k[0, sink, 0, 0] = 25.5 * math.log(2) / scale                       # of the first map alone
    q, k, v = (t.to(T).expand(B, *t.shape[1:]).contiguous().cuda() for t in (q, k, v))
    for lam in (0.0, 2.0 ** -20):
        weight = na.DiffWeight(torch.tensor([lam], device="cuda"))
        f = na.diff_attention_train(q, k, v, weight)
        assert torch.equal(na.diff_attention(q, k, v, weight), f.o)
        v64 = v[0, :, 0].double().cpu()
        p, S = maps(q[0].double().cpu(), k[0].double().cpu(), scale, au.seen(Tq, Tk, -1, -1))
        kappa = (2 * (d + 8) * S + 16) * E + (Tk / 16 + 32) * E
        o = p @ v64
        room = (U + kappa) * (p @ v64.abs()) + 2.0 ** -32 * v64.abs().sum(0)
        for b in (0, B - 1):
            au.within(f.o[b, :, 0], o[0] - lam * o[1], room[0] + lam * room[1] + U * (o[0] - lam * o[1]).abs() + 2.0 ** -25)
            for i in (0, 1):
                scales = f.stats[i, 1:, b * Tq:(b + 1) * Tq].repeat_interleave(128, 0)[:dv].t()
                kept = f.kept[b * Tq:(b + 1) * Tq, 0, i].double() * scales.double()
                au.within(kept, o[i], room[i] + o[i].abs().amax(1, keepdim=True) * (2.0 ** -16 * 1.01 + 4 * E), ("kept", i))
