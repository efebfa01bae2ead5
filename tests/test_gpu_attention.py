"""Differential attention, forward and backward, against its 64-bit form (bounds: attention_util)."""
import math

import pytest
import torch

import attention_util as au
from paper_2607_12505_amd import nmattention as na
from paper_2607_12505_amd import nmblock as nb

pytestmark = pytest.mark.gpu
TYPES = [torch.float16, torch.bfloat16]


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(g, T, *shape):
    return torch.randn(*shape, generator=g).to(T).cuda()


def compare(res, name, got, shape=None):
    """Rows of sequences against the 64-bit form; the others (NaN there) are not looked at."""
    want, room = res[name]
    got = got.detach().cpu().reshape(want.shape)
    live = ~torch.isnan(want)
    fine = torch.isfinite(want) | torch.isnan(want)
    assert torch.equal(got.double()[~fine], want[~fine]), name         # logarithms of empty rows
    live &= fine
    au.within(got[live], want[live], room.expand_as(want)[live], name)


def products(f):
    """p_i v of the codes that a forward pass kept."""
    dv = f.kept.shape[-1]
    scale = f.stats[:, 1:].repeat_interleave(128, 1)[:, :dv]            # [2 H, dv, rows]
    return f.kept.double() * scale.unflatten(0, (-1, 2)).permute(3, 0, 1, 2).double()


def check(q, k, v, weight, lam, spans, window, grad=None, scale=None, **extent):
    """All outputs of one call; with grad also the gradients."""
    T, dims = q.dtype, q.dim()
    flat = lambda t: t.reshape(-1, *t.shape[-2:])  # noqa: E731
    s = q.shape[-1] ** -0.5 if scale is None else scale
    s = float(torch.tensor(s, dtype=torch.float32))
    res = au.attention(flat(q), flat(k), flat(v), lam.tolist(), s, spans, *window, T,
                       None if grad is None else flat(grad))
    o = na.diff_attention(q, k, v, weight, scale=scale, window=window, **extent)
    compare(res, "o", o)
    if grad is None:
        return o
    f = na.diff_attention_train(q, k, v, weight, scale=scale, window=window, **extent)
    compare(res, "o", f.o)
    compare(res, "lse", f.stats[:, 0])
    compare(res, "kept", products(f))
    got = na.diff_attention_backward(grad, f, q, k, v, weight, scale=scale, window=window, **extent)
    for name in ("dq", "dk", "dv", "dlam"):
        compare(res, name, getattr(got, name))
    again = na.diff_attention_backward(grad, f, q, k, v, weight, scale=scale, window=window, **extent)
    for a, b, name in zip(got, again, got._fields):
        if a is not None:
            live = ~torch.isnan(res[name][0]).reshape(a.shape) if name in res else torch.ones(a.shape, dtype=torch.bool)
            assert torch.equal(a.cpu()[live], b.cpu()[live])           # the same bits every time
    return o


def dense(g, T, B, Tq, Tk, H, Hk, d, dv):
    q, k, v = randn(g, T, B, Tq, 2 * H, d), randn(g, T, B, Tk, 2 * Hk, d), randn(g, T, B, Tk, Hk, dv)
    spans = [(slice(b * Tq, (b + 1) * Tq), slice(b * Tk, (b + 1) * Tk)) for b in range(B)]
    lam = torch.rand(H, generator=g) * 0.8
    return q, k, v, lam.cuda(), spans


# one row, one key, tiles' ends and one past them, every width class, odd widths, shared keys, few rows over long keys
SHAPES = [(1, 1, 1, 1, 1, 64, 128), (2, 1, 33, 2, 1, 64, 128), (1, 31, 1, 1, 1, 32, 64), (1, 32, 64, 2, 2, 16, 16),
          (2, 33, 65, 3, 3, 64, 128), (1, 128, 128, 1, 1, 64, 64), (1, 129, 127, 2, 1, 24, 40), (1, 200, 300, 1, 1, 128, 256),
          (1, 70, 90, 2, 2, 128, 200), (2, 37, 41, 2, 1, 13, 29), (1, 150, 33, 4, 1, 65, 129), (1, 5, 700, 8, 2, 64, 128),
          (1, 577, 577, 1, 1, 64, 128), (3, 2, 130, 6, 1, 96, 100), (1, 260, 64, 1, 1, 1, 1), (1, 66, 140, 3, 1, 128, 256)]


@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("window", [(-1, -1), (-1, 0), (40, 3)])
@pytest.mark.parametrize("B,Tq,Tk,H,Hk,d,dv", SHAPES)
def test_against_the_definition(T, window, B, Tq, Tk, H, Hk, d, dv):
    g = gen(B + Tq * 3 + Tk * 5 + d)
    q, k, v, lam, spans = dense(g, T, B, Tq, Tk, H, Hk, d, dv)
    check(q, k, v, na.DiffWeight(lam), lam, spans, window, grad=randn(g, T, B, Tq, H, dv))


def test_single_tokens_over_a_long_cache_agree_with_rows_of_a_prompt():
    # the keys are split over workgroups: every split, the last ones without keys, and lengths from none on
    T, g, H, Hk, d, dv, n = torch.bfloat16, gen(9), 8, 2, 64, 128, 5000
    cache_k, cache_v = randn(g, T, 6, n, 2 * Hk, d), randn(g, T, 6, n, Hk, dv)
    q = randn(g, T, 6, 1, 2 * H, d)
    lam = (torch.rand(H, generator=g) * 0.8).cuda()
    lens = [0, 1, 31, 33, 4097, n]
    k_lens = torch.tensor(lens, dtype=torch.int32).cuda()
    for b, m in enumerate(lens):                          # what lies behind a sequence does not matter
        cache_k[b, m:], cache_v[b, m:] = math.nan, math.inf
    spans = [(slice(b, b + 1), slice(b * n, b * n + m)) for b, m in enumerate(lens)]
    o = check(q, cache_k, cache_v, na.DiffWeight(lam), lam, spans, (-1, 0), k_lens=k_lens)
    assert (o[0] == 0).all()                              # no keys
    f = na.diff_attention_train(q, cache_k, cache_v, na.DiffWeight(lam), causal=True, k_lens=k_lens)
    assert torch.equal(f.o, o) and torch.isinf(f.stats[:, 0, 0]).all()


@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("window", [(-1, -1), (-1, 0)])
def test_padded_sequences_leave_the_padding_alone(T, window):
    g, B, n, H, Hk, d, dv = gen(10), 5, 150, 4, 2, 64, 128
    q, k, v, lam, _ = dense(g, T, B, n, n, H, Hk, d, dv)
    do = randn(g, T, B, n, H, dv)
    lens = [150, 0, 1, 64, 131]
    dev = torch.tensor(lens, dtype=torch.int32).cuda()
    for b, m in enumerate(lens):
        q[b, m:], k[b, m:], v[b, m:], do[b, m:] = math.nan, math.inf, math.nan, -math.inf
    spans = [(slice(b * n, b * n + m), slice(b * n, b * n + m)) for b, m in enumerate(lens)]
    weight = na.DiffWeight(lam)
    check(q, k, v, weight, lam, spans, window, grad=do, q_lens=dev, k_lens=dev)
    out = torch.full((B, n, H, dv), 5.0, dtype=T, device="cuda")
    f = na.diff_attention_train(q, k, v, weight, window=window, q_lens=dev, k_lens=dev, out=out)
    into = [torch.full_like(t, 5.0) for t in (q, k, v)]
    na.diff_attention_backward(do, f, q, k, v, weight, window=window, q_lens=dev, k_lens=dev, dq=into[0], dk=into[1],
                               dv=into[2])
    for t in (out, *into):
        for b, m in enumerate(lens):
            assert (t[b, m:] == 5.0).all() and not (t[b, :m] == 5.0).all(dim=-1).any()


@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("window", [(-1, -1), (-1, 0), (20, 20)])
def test_packed_sequences(T, window):
    g, H, Hk, d, dv = gen(11), 3, 1, 48, 64
    ql, kl = [70, 0, 1, 129, 33], [70, 5, 0, 140, 20]
    q, k, v = randn(g, T, sum(ql) + 9, 2 * H, d), randn(g, T, sum(kl) + 4, 2 * Hk, d), randn(g, T, sum(kl) + 4, Hk, dv)
    do = randn(g, T, sum(ql) + 9, H, dv)
    ends = [torch.tensor([0] + x).cumsum(0) for x in (ql, kl)]
    qo, ko = (e.to(torch.int32).cuda() for e in ends)
    spans = [(slice(int(ends[0][b]), int(ends[0][b + 1])), slice(int(ends[1][b]), int(ends[1][b + 1])))
             for b in range(len(ql))]
    lam = (torch.rand(H, generator=g) * 0.8).cuda()
    extent = dict(q_offsets=qo, k_offsets=ko, max_q=max(ql), max_k=max(kl) + 3)
    check(q, k, v, na.DiffWeight(lam), lam, spans, window, grad=do, **extent)
    # rows behind the last sequence stay as they were
    out = torch.full((q.shape[0], H, dv), 5.0, dtype=T, device="cuda")
    na.diff_attention(q, k, v, na.DiffWeight(lam), window=window, out=out, **extent)
    assert (out[sum(ql):] == 5.0).all()


def test_offsets_and_lengths_outside_the_tensors_are_held_inside():
    T, g = torch.float16, gen(12)
    q, k, v = randn(g, T, 40, 2, 32), randn(g, T, 40, 2, 32), randn(g, T, 40, 1, 64)
    weight = na.DiffWeight(torch.tensor([0.3], device="cuda"))
    wild = torch.tensor([-7, 10, 4, 1 << 30], dtype=torch.int32).cuda()
    held = torch.tensor([0, 10, 10, 40], dtype=torch.int32).cuda()
    # the third sequence starts at 4 by the wild ones: 4 .. 40
    a = na.diff_attention(q, k, v, weight, q_offsets=wild, max_q=40)
    b = na.diff_attention(q, k, v, weight, q_offsets=torch.tensor([4, 40], dtype=torch.int32).cuda(), max_q=40)
    assert torch.equal(a[10:], b[10:])
    assert na.diff_attention(q, k, v, weight, q_offsets=held, max_q=40).isfinite().all()
    lens = torch.tensor([99, -4], dtype=torch.int32).cuda()
    q4, k4, v4 = (t.view(2, 20, *t.shape[1:]) for t in (q, k, v))
    a = na.diff_attention(q4, k4, v4, weight, k_lens=lens)
    assert torch.equal(a[0], na.diff_attention(q4[:1], k4[:1], v4[:1], weight)[0]) and (a[1] == 0).all()


@pytest.mark.parametrize("T", TYPES)
def test_learned_vectors_and_their_gradients(T):
    g, B, n, H, Hk, d, dv = gen(13), 2, 90, 4, 2, 64, 128
    q, k, v, _, spans = dense(g, T, B, n, n, H, Hk, d, dv)
    do = randn(g, T, B, n, H, dv) + 0.25
    for shape in ((d,), (H, d), (H, 3), (200,)):
        vec = [(0.2 * torch.randn(*shape, generator=g)).cuda() for _ in range(4)]
        q1, k1, q2, k2 = (t.double().cpu().expand(H, shape[-1]) for t in vec)
        e1, e2 = torch.exp((q1 * k1).sum(-1)), torch.exp((q2 * k2).sum(-1))
        lam = e1 - e2 + float(torch.tensor(0.35))
        weight = na.DiffWeight.of_vectors(*vec, init=0.35)
        res = au.attention(q.flatten(0, 1), k.flatten(0, 1), v.flatten(0, 1), lam.tolist(), d ** -0.5, spans, -1, 0, T,
                           do.flatten(0, 1))
        f = na.diff_attention_train(q, k, v, weight, causal=True)
        got = na.diff_attention_backward(do, f, q, k, v, weight, causal=True)
        # lam itself is within (n + 16) e of its terms: far inside the bounds of a map's rounding
        for name in ("o", "dq", "dk", "dv", "dlam"):
            compare(res, name, getattr(f, name) if name == "o" else getattr(got, name))
        dl, room = res["dlam"]
        wide = (shape[-1] + 80) * au.E * (1 + (q1 * k1).abs().sum(-1) + (q2 * k2).abs().sum(-1))
        for name, other, f1 in (("dq1", k1, e1), ("dk1", q1, e1), ("dq2", k2, -e2), ("dk2", q2, -e2)):
            want = (dl * f1)[:, None] * other
            off = ((room + wide * dl.abs()) * f1.abs())[:, None] * other.abs()
            if len(shape) == 1:
                want, off = want.sum(0), off.sum(0) + 16 * au.E * want.abs().sum(0)
            au.within(getattr(got, name), want, off + 1e-30, name)


def test_gradients_against_differences():
    # along one direction of all inputs at once; the 64-bit form stands for the function (its difference quotient
    # has an error of h^2), its gradient for the kernels', within the kernels' own bounds
    T, g, B, n, H, Hk, d, dv = torch.bfloat16, gen(14), 1, 40, 2, 1, 32, 64
    q, k, v, lam, spans = dense(g, T, B, n, n, H, Hk, d, dv)
    do = randn(g, T, B, n, H, dv)
    weight = na.DiffWeight(lam)
    f = na.diff_attention_train(q, k, v, weight, causal=True)
    got = na.diff_attention_backward(do, f, q, k, v, weight, causal=True)
    flat = [t.double().cpu().flatten(0, 1) for t in (q, k, v)]
    way = [torch.randn(t.shape, generator=g, dtype=torch.float64) for t in flat]
    wl, l64 = torch.randn(H, generator=g, dtype=torch.float64), lam.double().cpu()
    h = 1e-4

    def value(s):
        o = au.attention(*(t + s * w for t, w in zip(flat, way)), (l64 + s * wl).tolist(), d ** -0.5, spans, -1, 0, T)
        return float((o["o"][0] * do.double().cpu().flatten(0, 1)).sum())
    slope = (value(h) - value(-h)) / (2 * h)
    res = au.attention(*flat, l64.tolist(), d ** -0.5, spans, -1, 0, T, do.flatten(0, 1))
    mine = sum(float((t.double().cpu().reshape(w.shape) * w).sum()) for t, w in zip(got[:3], way))
    mine += float((got.dlam.double().cpu() * wl).sum())
    room = sum(float((res[x][1].expand_as(w) * w.abs()).sum()) for x, w in zip(("dq", "dk", "dv"), way))
    room += float((res["dlam"][1] * wl.abs()).sum()) + 1e-3 * abs(slope)
    assert abs(slope - mine) <= room


@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("pad", [0, 1, 4])
def test_inside_the_rows_of_one_product(T, pad):
    # q, k and v are columns of wider rows; gradients go to the columns of another buffer
    g, B, n, H, Hk, d, dv = gen(15), 2, 75, 4, 2, 64, 128
    w = 2 * H * d + 2 * Hk * d + Hk * dv
    qkv = randn(g, T, B, n, w + pad)
    def cut(t):  # noqa: E306
        return (t[..., :2 * H * d].unflatten(-1, (2 * H, d)),
                t[..., 2 * H * d:2 * H * d + 2 * Hk * d].unflatten(-1, (2 * Hk, d)), t[..., w - Hk * dv:w].unflatten(-1, (Hk, dv)))
    q, k, v = cut(qkv)
    lam = (torch.rand(H, generator=g) * 0.8).cuda()
    weight, do = na.DiffWeight(lam), randn(g, T, B, n, H, dv)
    near = [t.contiguous() for t in (q, k, v)]
    f, f2 = na.diff_attention_train(q, k, v, weight, causal=True), na.diff_attention_train(*near, weight, causal=True)
    for a, b in zip(f, f2):
        assert torch.equal(a, b)
    grads = torch.full_like(qkv, 5.0)
    into = cut(grads)
    out = na.diff_attention_backward(do, f, q, k, v, weight, causal=True, dq=into[0], dk=into[1], dv=into[2])
    want = na.diff_attention_backward(do, f2, *near, weight, causal=True)
    for a, b in zip(out[:4], want[:4]):
        assert torch.equal(a, b)
    assert (grads[..., w:] == 5.0).all()
    # heads before tokens, and rows of o inside wider ones
    heads_first = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in near]
    wide = torch.full((B, n, H, dv + 12), 5.0, dtype=T, device="cuda")
    assert torch.equal(na.diff_attention(*heads_first, weight, causal=True, out=wide[..., :dv]), f.o)
    assert (wide[..., dv:] == 5.0).all()
    for a, b in zip(na.diff_attention_backward(do, f, *heads_first, weight, causal=True)[:4], want[:4]):
        assert torch.equal(a, b)


# parts of few and of many rows over long keys, their number and widths odd, alone and by several row tiles
@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("B,Tq,Tk,H,Hk,d,dv", [(1, 1, 3000, 1, 1, 64, 33), (1, 100, 3001, 2, 1, 64, 128), (1, 3, 2050, 3, 1, 31, 63),
                                               (1, 70, 1500, 1, 1, 128, 256), (1, 1, 2000, 3, 3, 127, 255)])
def test_parts_of_the_keys(T, B, Tq, Tk, H, Hk, d, dv):
    g = gen(Tk)
    q, k, v, lam, spans = dense(g, T, B, Tq, Tk, H, Hk, d, dv)
    check(q, k, v, na.DiffWeight(lam), lam, spans, (-1, 0), grad=randn(g, T, B, Tq, H, dv))


@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("window", [(-1, 0), (40, 3)])
@pytest.mark.parametrize("B,Tq,Tk,H,Hk,d,dv", [(1, 200, 300, 1, 1, 128, 128), (2, 70, 90, 4, 2, 100, 90), (1, 129, 128, 2, 1, 72, 16),
                                               (1, 90, 1500, 2, 1, 128, 120), (1, 1, 3000, 1, 1, 97, 127), (1, 2, 7, 2, 2, 65, 1)])
def test_keys_as_wide_as_values(T, window, B, Tq, Tk, H, Hk, d, dv):
    g = gen(B + Tq * 3 + Tk * 5 + d)
    q, k, v, lam, spans = dense(g, T, B, Tq, Tk, H, Hk, d, dv)
    check(q, k, v, na.DiffWeight(lam), lam, spans, window, grad=randn(g, T, B, Tq, H, dv))


@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("d,dv", [(32, 64), (64, 128), (61, 107), (128, 128), (128, 256), (100, 200)])
def test_rows_that_see_one_key_have_no_gradient_of_scores(T, d, dv):
    # p is 1 whatever the score: q and k get zeros, not the roundings of dp - D
    g, H, Hk = gen(18), 4, 2
    for B, Tq, Tk, window in ((57, 1, 1, (-1, 0)), (2, 3, 1, (-1, -1)), (1, 200, 200, (0, 0)), (1, 9, 40, (0, 0)), (2, 40, 40, (-1, 0))):
        q, k, v, lam, spans = dense(g, T, B, Tq, Tk, H, Hk, d, dv)
        do, weight = randn(g, T, B, Tq, H, dv), na.DiffWeight(lam)
        check(q, k, v, weight, lam, spans, window, grad=do)
        got = na.diff_attention_backward(do, na.diff_attention_train(q, k, v, weight, window=window), q, k, v, weight,
                                         window=window)
        if window == (-1, 0) and Tk > 1:                  # the first row alone, whose key others see
            assert (got.dq[:, 0] == 0).all() and not (got.dq[:, 1:] == 0).any(dim=-1).all()
        else:
            assert (got.dq == 0).all() and (got.dk == 0).all()


@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("n", [1, 75, 130])
def test_expanded_inputs(T, n):
    # rows that are all one place in memory: those behind the last are not
    g, B, H, Hk, d, dv = gen(16), 2, 4, 2, 64, 128
    q, k, v, lam, _ = dense(g, T, B, n, n, H, Hk, d, dv)
    do, weight = randn(g, T, B, n, H, dv), na.DiffWeight(lam)
    for places in ((B, 1), (1, n), (1, 1)):
        cut = [t[:places[0], :places[1]].expand_as(t) for t in (q, k, v, do)]
        for which in range(4):
            some = [c if i == which else t for i, (c, t) in enumerate(zip(cut, (q, k, v, do)))]
            near = [t.contiguous() for t in some]
            f = na.diff_attention_train(*some[:3], weight, causal=True)
            want = na.diff_attention_train(*near[:3], weight, causal=True)
            for a, b in zip(f, want):
                assert torch.equal(a, b)
            for a, b in zip(na.diff_attention_backward(some[3], f, *some[:3], weight, causal=True)[:4],
                            na.diff_attention_backward(near[3], want, *near[:3], weight, causal=True)[:4]):
                assert torch.equal(a, b)
    for out in (torch.empty(B, 1, H, dv, dtype=T, device="cuda").expand(B, 9, H, dv),
                torch.empty(1, 9, H, dv, dtype=T, device="cuda").expand(B, 9, H, dv)):
        with pytest.raises(ValueError):
            na.diff_attention(q[:, :1].expand(B, 9, 2 * H, d), k, v, weight, out=out)


def test_strides_of_dimensions_of_one():
    T, g = torch.float16, gen(17)
    q, k, v, lam, _ = dense(g, T, 1, 1, 40, 1, 1, 64, 128)
    do, weight = randn(g, T, 1, 1, 1, 128), na.DiffWeight(lam)
    far = 1 << 40
    some = [q.as_strided(q.shape, (far + 1, far + 3, 64, 1)), k.as_strided(k.shape, (3, 128, 64, 1)),
            v.as_strided(v.shape, (5, 128, far + 7, 1)), do.as_strided(do.shape, (far, far, far, 1))]
    f, want = na.diff_attention_train(*some[:3], weight), na.diff_attention_train(q, k, v, weight)
    for a, b in zip(f, want):
        assert torch.equal(a, b)
    for a, b in zip(na.diff_attention_backward(some[3], f, *some[:3], weight)[:4],
                    na.diff_attention_backward(do, want, q, k, v, weight)[:4]):
        assert torch.equal(a, b)


@pytest.mark.parametrize("T", TYPES)
def test_rows_that_see_nothing(T):
    # more rows than keys under the causal mask: the first rows see none
    g, H, d, dv = gen(16), 2, 64, 128
    q, k, v, lam, spans = dense(g, T, 1, 200, 70, H, H, d, dv)
    do = randn(g, T, 1, 200, H, dv)
    f = na.diff_attention_train(q, k, v, na.DiffWeight(lam), causal=True)
    assert (f.o[0, :130] == 0).all() and (f.kept[:130] == 0).all() and (f.stats[:, 0, :130] == math.inf).all()
    assert (f.stats[:, 1:, :130] == 0).all()
    got = na.diff_attention_backward(do, f, q, k, v, na.DiffWeight(lam), causal=True)
    assert (got.dq[0, :130] == 0).all()
    check(q, k, v, na.DiffWeight(lam), lam, spans, (-1, 0), grad=do)
    check(q, k, v, na.DiffWeight(lam), lam, spans, (0, 0), grad=do)     # one key a row
    # no keys at all
    f = na.diff_attention_train(q, k[:, :0], v[:, :0], na.DiffWeight(lam))
    assert (f.o == 0).all() and (f.stats[:, 0] == math.inf).all()
    got = na.diff_attention_backward(do, f, q, k[:, :0], v[:, :0], na.DiffWeight(lam))
    assert (got.dq == 0).all() and got.dk.shape[1] == 0 and (got.dlam == 0).all()
    # no rows: gradients of the keys and of the weight are zero
    f = na.diff_attention_train(q[:, :0], k, v, na.DiffWeight(lam))
    got = na.diff_attention_backward(do[:, :0], f, q[:, :0], k, v, na.DiffWeight(lam))
    assert (got.dk == 0).all() and (got.dv == 0).all() and (got.dlam == 0).all()
    f = na.diff_attention_train(q[:0], k[:0], v[:0], na.DiffWeight(lam))
    assert (na.diff_attention_backward(do[:0], f, q[:0], k[:0], v[:0], na.DiffWeight(lam)).dlam == 0).all()


@pytest.mark.parametrize("T", TYPES)
def test_scores_of_every_size(T):
    # maxima that grow from key to key (each tile's sums are rescaled), scores near zero, and one key above all
    g, H, d, dv, n = gen(17), 1, 64, 128, 300
    q, k, v, lam, spans = dense(g, T, 1, n, n, H, H, d, dv)
    rise = torch.linspace(0.05, 4, n)[None, :, None, None].to(T).cuda()
    check(q.abs(), (k.abs() * rise), v, na.DiffWeight(lam), lam, spans, (-1, -1), scale=0.05)
    check(q.abs(), (k.abs() * rise.flip(1)), v, na.DiffWeight(lam), lam, spans, (-1, -1), scale=0.05)
    check(q, k, v, na.DiffWeight(lam), lam, spans, (-1, -1), scale=1e-4)
    k2 = k.clone()
    k2[0, 137] *= 30
    check(q, k2, v, na.DiffWeight(lam), lam, spans, (-1, -1))


def test_values_that_are_not_finite_stay_in_their_rows():
    T, g, H = torch.float16, gen(18), 2
    q, k, v, lam, _ = dense(g, T, 1, 96, 96, H, H, 32, 64)
    weight = na.DiffWeight(lam)
    want = na.diff_attention(q, k, v, weight, causal=True)
    q2 = q.clone()
    q2[0, 17, 1, 3] = math.nan
    o = na.diff_attention(q2, k, v, weight, causal=True)
    assert o[0, 17, 0].isnan().all()
    o[0, 17, 0] = want[0, 17, 0]
    assert torch.equal(o, want)
    k2 = k.clone()
    k2[0, 70, 0, 3] = math.inf                             # rows before it do not see it
    o = na.diff_attention(q, k2, v, weight, causal=True)
    assert torch.equal(o[0, :70], want[0, :70]) and torch.equal(o[0, :, 1], want[0, :, 1])
    lam2 = lam.clone()
    lam2[1] = math.nan
    o = na.diff_attention(q, k, v, na.DiffWeight(lam2), causal=True)
    assert torch.equal(o[:, :, 0], want[:, :, 0]) and o[:, :, 1].isnan().all()


def test_keys_past_32_bits_of_offset():
    # a cache of 9 GB whose sequences lie 2^31 values apart, read at its end
    T, g, n, H = torch.bfloat16, gen(19), 2048, 1
    far = (1 << 31) + 4096
    room = torch.empty(2 * far, dtype=T, device="cuda")
    k = room[:far + n * 64].as_strided((2, n, 2, 32), (far, 64, 32, 1))
    v = randn(g, T, 2, n, 1, 64)
    k.copy_(randn(g, T, 2, n, 2, 32))
    q = randn(g, T, 2, 3, 2, 32)
    weight = na.DiffWeight(torch.tensor([0.4], device="cuda"))
    assert torch.equal(na.diff_attention(q, k, v, weight, causal=True), na.diff_attention(q, k.contiguous(), v, weight,
                                                                                         causal=True))
    # tokens far apart: one sequence across more than 2^32 bytes
    k = room.as_strided((1, 1024, 2, 32), (0, (1 << 22) - 64, 32, 1))
    k.copy_(randn(g, T, 1, 1024, 2, 32))
    assert torch.equal(na.diff_attention(q[:1], k, v[:1, :1024], weight),
                       na.diff_attention(q[:1], k.contiguous(), v[:1, :1024], weight))
    do, f = randn(g, T, 1, 3, 1, 64), na.diff_attention_train(q[:1], k, v[:1, :1024], weight)
    a = na.diff_attention_backward(do, f, q[:1], k, v[:1, :1024], weight)
    b = na.diff_attention_backward(do, f, q[:1], k.contiguous(), v[:1, :1024], weight)
    for x, y in zip(a[:4], b[:4]):
        assert torch.equal(x, y)


def chain(qkv, pos, axes, weight, do, H, Hk, d, dv):
    """Rotary, attention and the gradients back to the projections."""
    heads = 2 * H + 2 * Hk
    turned = na.rotary(qkv[..., :heads * d].unflatten(-1, (heads, d)), pos, axes)
    q, k, v = turned[..., :2 * H, :], turned[..., 2 * H:, :], qkv[..., heads * d:].unflatten(-1, (Hk, dv))
    f = na.diff_attention_train(q, k, v, weight, causal=True)
    both = torch.empty_like(turned)
    got = na.diff_attention_backward(do, f, q, k, v, weight, causal=True, dq=both[..., :2 * H, :], dk=both[..., 2 * H:, :])
    na.rotary_backward(both, pos, axes, out=both)
    return (f.o, both, got.dv, *got[4:])


def test_the_attention_half_of_a_block():
    # int8 projections, rotary, attention, the norm of each head and the int8 product back, and all gradients of the middle
    T, g, B, n, H, Hk, d, dv = torch.float16, gen(20), 2, 197, 6, 3, 64, 128
    width, heads = 768, 2 * H + 2 * Hk
    axes = na.RotaryAxes.of_sections((16, 16), own_ladders=True)
    at = torch.arange(n)
    pos = torch.stack((at // 14, at % 14)).to(torch.int32).repeat(1, B).cuda()
    wq = nb.ScaledWeight.from_float((torch.randn(heads * d + Hk * dv, width, generator=g) * width ** -0.5).cuda())
    wo = nb.ScaledWeight.from_float((torch.randn(width, H * dv, generator=g) * 0.03).cuda())
    vec = [(0.2 * torch.randn(d, generator=g)).cuda() for _ in range(4)]
    weight = na.DiffWeight.of_vectors(*vec, init=0.3)
    norm = nb.Norm("rms", torch.full((dv,), 0.7, device="cuda"))
    x = randn(g, T, B, n, width)
    qkv = nb.linear_i8(x, wq)
    do = randn(g, T, B, n, H, dv)
    o, both, dvv, *vectors = chain(qkv, pos, axes, weight, do, H, Hk, d, dv)
    _, z = nb.norm_residual(None, o, pre=norm)
    assert nb.linear_i8(z.flatten(-2), wo).shape == x.shape
    # the parts against their own forms
    want, room = au.rotary(qkv[..., :heads * d].reshape(-1, heads, d), pos, axes.freqs.tolist(), axes.axis.tolist(), "halves")
    turned = na.rotary(qkv[..., :heads * d].unflatten(-1, (heads, d)), pos, axes)
    au.within(turned.reshape(want.shape), want, room + au.UNIT[T] * want.abs() + au.TINY[T])
    lam = torch.exp((vec[0] * vec[1]).double().sum()) - torch.exp((vec[2] * vec[3]).double().sum()) + 0.3
    spans = [(slice(b * n, (b + 1) * n),) * 2 for b in range(B)]
    flat = turned.reshape(-1, heads, d)
    res = au.attention(flat[:, :2 * H], flat[:, 2 * H:], qkv[..., heads * d:].reshape(-1, Hk, dv), [float(lam)] * H,
                       d ** -0.5, spans, -1, 0, T, do.flatten(0, 1))
    compare(res, "o", o)
    compare(res, "dv", dvv)
    both_room = torch.cat([res[x][1].expand_as(res[x][0]) for x in ("dq", "dk")], 1)
    both_want = torch.cat([res[x][0] for x in ("dq", "dk")], 1)
    back, rest = au.rotary(both_want, pos, axes.freqs.tolist(), axes.axis.tolist(), "halves", back=True)
    # a rotated pair's error is at most the sum of both channels'
    half = both_room.view(-1, heads, 2, d // 2).sum(2, keepdim=True).expand(-1, -1, 2, -1).reshape(both_room.shape)
    au.within(both.reshape(back.shape), back, half + rest + 2 * au.UNIT[T] * back.abs() + au.UNIT[T] * half + au.TINY[T])


def test_captured_graphs_replay_what_eager_calls_give():
    T, g, B, n, H, Hk, d, dv = torch.bfloat16, gen(21), 2, 100, 4, 2, 64, 128
    heads = 2 * H + 2 * Hk
    axes = na.RotaryAxes.of_sections((16, 16))
    pos = torch.randint(0, 24, (2, B * n), generator=g, dtype=torch.int32).cuda()
    weight = na.DiffWeight.of_vectors(*((0.2 * torch.randn(d, generator=g)).cuda() for _ in range(4)), init=0.3)
    qkv, do = randn(g, T, B, n, heads * d + Hk * dv), randn(g, T, B, n, H, dv)
    q1, cache_k, cache_v = randn(g, T, 3, 1, 2 * H, d), randn(g, T, 3, 900, 2 * Hk, d), randn(g, T, 3, 900, Hk, dv)
    lens = torch.tensor([900, 5, 431], dtype=torch.int32).cuda()
    for _ in range(2):                                     # loaded before capture
        chain(qkv, pos, axes, weight, do, H, Hk, d, dv)
        na.diff_attention(q1, cache_k, cache_v, weight, k_lens=lens)
    graphs, outs = [], []
    for _ in range(2):                                     # two graphs, each with workspaces of its own
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append((*chain(qkv, pos, axes, weight, do, H, Hk, d, dv),
                         na.diff_attention(q1, cache_k, cache_v, weight, k_lens=lens)))
        graphs.append(graph)
    for turn in range(3):
        qkv.copy_(randn(gen(30 + turn), T, *qkv.shape))
        q1.copy_(randn(gen(40 + turn), T, *q1.shape))
        lens.copy_(torch.tensor([900 - 300 * turn, 5 + turn, 431], dtype=torch.int32))
        eager = (*chain(qkv, pos, axes, weight, do, H, Hk, d, dv),
                 na.diff_attention(q1, cache_k, cache_v, weight, k_lens=lens))
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for got in outs:
            for a, b in zip(got, eager):
                assert torch.equal(a, b)


def test_other_streams():
    T, g = torch.float16, gen(22)
    q, k, v, lam, _ = dense(g, T, 2, 300, 300, 4, 2, 64, 128)
    do, weight = randn(g, T, 2, 300, 4, 128), na.DiffWeight(lam)
    f = na.diff_attention_train(q, k, v, weight)
    want = na.diff_attention_backward(do, f, q, k, v, weight)
    sides = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for side in sides:                                     # two calls at once
        side.wait_stream(torch.cuda.current_stream())
        f2 = na.diff_attention_train(q, k, v, weight, stream=side)
        got.append((f2, na.diff_attention_backward(do, f2, q, k, v, weight, stream=side)))
    for side, (f2, grads) in zip(sides, got):
        side.synchronize()
        assert torch.equal(f2.o, f.o) and torch.equal(f2.stats, f.stats)
        for a, b in zip(grads[:4], want[:4]):
            assert torch.equal(a, b)


def test_refusals():
    T, g = torch.float16, gen(23)
    q, k, v, lam, _ = dense(g, T, 2, 20, 30, 4, 2, 32, 64)
    w = na.DiffWeight(lam)
    call = na.diff_attention
    lens = torch.tensor([3, 4], dtype=torch.int32).cuda()
    bad = [(q.float(), k.float(), v.float(), w), (q, k.bfloat16(), v, w), (q[:, :, :7], k, v, w), (q[:, :, :6], k, v, w),
           (q, k[:, :, :3], v, w), (q, k[:1], v[:1], w), (q, k, v[:, :10], w), (q, k[..., :31], v, w), (q[0], k, v, w),
           (q.transpose(2, 3), k, v, w), (q.cpu(), k, v, w), (q, k.cpu(), v, w), (q, k, v, na.DiffWeight(lam[:3].contiguous()))]
    for args in bad:
        with pytest.raises(ValueError):
            call(*args)
    for more in (dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(causal=True, window=(3, 0)),
                 dict(q_lens=lens.long()), dict(k_lens=lens[:1]), dict(q_lens=lens.cpu()), dict(max_q=3),
                 dict(k_offsets=lens), dict(out=torch.empty(2, 20, 4, 63, dtype=T, device="cuda")),
                 dict(out=torch.empty(2, 20, 4, 64, device="cuda"))):
        with pytest.raises(ValueError):
            call(q, k, v, w, **more)
    p = [t[0] for t in (q, k, v)]
    off = torch.tensor([0, 10, 20], dtype=torch.int32).cuda()
    for more in (dict(q_offsets=off), dict(q_offsets=off, max_q=20, q_lens=lens), dict(q_offsets=off, max_q=20, k_offsets=off),
                 dict(q_offsets=off.float(), max_q=20), dict(q_offsets=off, max_q=20, k_offsets=off[:2], max_k=9)):
        with pytest.raises(ValueError):
            call(*p, w, **more)
    with pytest.raises(Exception):
        call(torch.zeros(1, 4, 2, 129, dtype=T, device="cuda"), torch.zeros(1, 4, 2, 129, dtype=T, device="cuda"),
             torch.zeros(1, 4, 1, 8, dtype=T, device="cuda"), na.DiffWeight(lam[:1].contiguous()))
    f = na.diff_attention_train(q, k, v, w)
    do = torch.zeros_like(f.o)
    for args in ((do[:, :19], f), (do.float(), f), (do, na.DiffForward(f.o, None, f.stats)),
                 (do, na.DiffForward(f.o, f.kept, f.stats[:, :1])), (do, na.DiffForward(f.o, f.kept.half(), f.stats))):
        with pytest.raises(ValueError):
            na.diff_attention_backward(*args, q, k, v, w)
    with pytest.raises(ValueError):
        na.diff_attention_backward(do, f, q, k, v, w, dq=torch.empty_like(k))
    for vec in ([lam] * 3 + [lam[:2].contiguous()], [lam.double()] * 4, [lam.cpu()] * 4):
        with pytest.raises(ValueError):
            na.DiffWeight.of_vectors(*vec, init=0.1)
    with pytest.raises(ValueError):
        na.DiffWeight(lam.half())
