"""Every variant of differential attention against its 64-bit form (bounds: attention_util; shapes: attention_cases, of which
test_attention_variants checks what they reach)."""
import math

import pytest
import torch

import attention_cases as cases
from paper_2607_12505_amd import nmattention as na
from test_gpu_attention import check, compare, dense, gen, products, randn
import attention_util as au

pytestmark = pytest.mark.gpu
TYPES = [torch.float16, torch.bfloat16]
WINDOWS = [(-1, -1), (-1, 0), (40, 3), (-1, 9), (25, -1)]


@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("n,shape", list(enumerate(cases.MANY_ROWS + cases.MANY_ROWS_WIDE)))
def test_many_rows(T, n, shape):
    B, Tq, Tk, H, Hk, d, dv = shape
    g = gen(n)
    q, k, v, lam, spans = dense(g, T, *shape)
    do = randn(g, T, B, Tq, H, dv)
    for window in (WINDOWS[n % 5], WINDOWS[(n + 1) % 5]):
        check(q, k, v, na.DiffWeight(lam), lam, spans, window, grad=do)


@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("window", [(-1, -1), (-1, 0), (30, 2)])
@pytest.mark.parametrize("B,n,keys,H,Hk,d,dv", cases.PADDED)
def test_many_rows_of_padded_sequences(T, window, B, n, keys, H, Hk, d, dv):
    # lengths from none to all; what lies behind them is not read, and not written
    g = gen(B + n)
    q, k, v, lam, _ = dense(g, T, B, n, n, H, Hk, d, dv)
    do = randn(g, T, B, n, H, dv)
    lens = [n, 0, 1, 64, 129] + [b * 37 % (n + 1) for b in range(5, B)]
    kl = [max(0, m - 3) if b % 3 else m for b, m in enumerate(lens)]
    for b, (m, j) in enumerate(zip(lens, kl)):
        q[b, m:], do[b, m:], k[b, j:], v[b, j:] = math.nan, math.inf, -math.inf, math.nan
    spans = [(slice(b * n, b * n + m), slice(b * n, b * n + j)) for b, (m, j) in enumerate(zip(lens, kl))]
    how = dict(zip(("q_lens", "k_lens"), (torch.tensor(x, dtype=torch.int32).cuda() for x in (lens, kl))))
    weight = na.DiffWeight(lam)
    check(q, k, v, weight, lam, spans, window, grad=do, **how)
    out, into = torch.full((B, n, H, dv), 5.0, dtype=T, device="cuda"), [torch.full_like(t, 5.0) for t in (q, k, v)]
    f = na.diff_attention_train(q, k, v, weight, window=window, out=out, **how)
    na.diff_attention_backward(do, f, q, k, v, weight, window=window, dq=into[0], dk=into[1], dv=into[2], **how)
    for t, ends in ((out, lens), (into[0], lens), (into[1], kl), (into[2], kl)):
        for b, m in enumerate(ends):
            assert (t[b, m:] == 5.0).all() and not (t[b, :m] == 5.0).all(dim=-1).any()


@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("window", [(-1, -1), (-1, 0), (30, 2)])
@pytest.mark.parametrize("B,rows,keys,H,Hk,d,dv", cases.PACKED)
def test_many_rows_of_packed_sequences(T, window, B, rows, keys, H, Hk, d, dv):
    g = gen(H + d)
    ql = [260, 0, 1, 64, 129, rows] + [b * 53 % 190 for b in range(6, B)]
    kl = [200, 9, 0, 64, 129, keys] + [b * 71 % 190 for b in range(6, B)]
    ends = [torch.tensor([0] + x).cumsum(0) for x in (ql, kl)]
    nq, nk = int(ends[0][-1]), int(ends[1][-1])
    q, k, v = randn(g, T, nq + 5, 2 * H, d), randn(g, T, nk + 2, 2 * Hk, d), randn(g, T, nk + 2, Hk, dv)
    do, lam = randn(g, T, nq + 5, H, dv), (torch.rand(H, generator=g) * 0.8).cuda()
    q[nq:], do[nq:], k[nk:], v[nk:] = math.nan, math.nan, math.inf, math.nan
    spans = [(slice(int(ends[0][b]), int(ends[0][b + 1])), slice(int(ends[1][b]), int(ends[1][b + 1]))) for b in range(len(ql))]
    qo, ko = (e.to(torch.int32).cuda() for e in ends)
    how = dict(q_offsets=qo, k_offsets=ko, max_q=max(ql), max_k=max(kl))
    check(q, k, v, na.DiffWeight(lam), lam, spans, window, grad=do, **how)
    out = torch.full((q.shape[0], H, dv), 5.0, dtype=T, device="cuda")
    na.diff_attention(q, k, v, na.DiffWeight(lam), window=window, out=out, **how)
    assert (out[nq:] == 5.0).all()


@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("n,case", list(enumerate(cases.PARTS)))
def test_parts_of_the_keys(T, n, case):
    shape, given, _ = case
    B, Tq, Tk, H, Hk, d, dv = shape
    g = gen(n + 70)
    q, k, v, lam, spans = dense(g, T, *shape)
    how = {}
    if given:
        lens = [Tk] + [Tq + (Tk - Tq) * (b * 7919 % B) // B for b in range(1, B)]
        lens[-1] = 0
        for b, m in enumerate(lens):
            k[b, m:], v[b, m:] = math.inf, math.nan
        spans = [(slice(b * Tq, (b + 1) * Tq), slice(b * Tk, b * Tk + m)) for b, m in enumerate(lens)]
        how = dict(k_lens=torch.tensor(lens, dtype=torch.int32).cuda())
    weight = na.DiffWeight(lam)
    for window in ((-1, 0), (Tk // 3, 0)):
        check(q, k, v, weight, lam, spans, window, grad=randn(g, T, B, Tq, H, dv), **how)


@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("window", [(-1, -1), (-1, 0), (300, 3)])
@pytest.mark.parametrize("n,case", list(enumerate(cases.ROW_PARTS)))
def test_parts_of_the_rows(T, n, case, window):
    shape, _ = case
    g = gen(n + 90)
    q, k, v, lam, spans = dense(g, T, *shape)
    check(q, k, v, na.DiffWeight(lam), lam, spans, window, grad=randn(g, T, shape[0], shape[1], shape[3], shape[6]))


@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("n,shape", list(enumerate(cases.SHARED)))
def test_keys_that_very_many_heads_share(T, n, shape):
    g = gen(n + 110)
    q, k, v, lam, spans = dense(g, T, *shape)
    check(q, k, v, na.DiffWeight(lam), lam, spans, (-1, 0), grad=randn(g, T, shape[0], shape[1], shape[3], shape[6]))


@pytest.mark.parametrize("T", TYPES)
def test_many_rows_inside_one_product_with_learned_vectors_and_a_graph(T):
    # as a step of training has them: columns of wider rows, a weight of each head's own, captured and replayed
    g, (B, n, _, H, Hk, d, dv) = gen(77), cases.STEP
    w = 2 * H * d + 2 * Hk * d + Hk * dv
    qkv = randn(g, T, B, n, w + 8)
    q, k = qkv[..., :2 * H * d].unflatten(-1, (2 * H, d)), qkv[..., 2 * H * d:2 * H * d + 2 * Hk * d].unflatten(-1, (2 * Hk, d))
    v = qkv[..., w - Hk * dv:w].unflatten(-1, (Hk, dv))
    vec = [(0.2 * torch.randn(H, d, generator=g)).cuda() for _ in range(4)]
    a, b, c, e = (t.double().cpu() for t in vec)
    lam = torch.exp((a * b).sum(-1)) - torch.exp((c * e).sum(-1)) + float(torch.tensor(0.3))
    weight, do = na.DiffWeight.of_vectors(*vec, init=0.3), randn(g, T, B, n, H, dv)

    def step():
        f = na.diff_attention_train(q, k, v, weight, causal=True)
        return f, na.diff_attention_backward(do, f, q, k, v, weight, causal=True)
    f, got = step()
    spans = [(slice(s * n, (s + 1) * n),) * 2 for s in range(B)]
    res = au.attention(q.flatten(0, 1), k.flatten(0, 1), v.flatten(0, 1), lam.tolist(), d ** -0.5, spans, -1, 0, T,
                       do.flatten(0, 1))
    compare(res, "o", f.o)
    compare(res, "kept", products(f))
    for name in ("dq", "dk", "dv", "dlam"):
        compare(res, name, getattr(got, name))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f2, got2 = step()
    for turn in range(3):
        qkv.copy_(randn(gen(80 + turn), T, *qkv.shape))
        f, got = step()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip((*f, *got), (*f2, *got2)):
            assert torch.equal(x, y)
