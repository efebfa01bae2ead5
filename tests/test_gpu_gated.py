"""The gated feed-forward block and its gradients, against the plain form in 64 bits (bounds: block_util)."""
import pytest
import torch

import block_util as bu
from paper_2607_12505_amd import nmblock as nb

pytestmark = pytest.mark.gpu
ACTS = ["silu", "gelu", "gelu_tanh", "relu", "sigmoid"]


def gen(seed):
    return torch.Generator().manual_seed(seed)


def case(m, k, n, T, bias, N=8, M=8, act="silu", seed=0):
    g = gen(seed + m + 3 * k + n)
    x = (torch.randn(m, k, generator=g) * torch.exp(0.5 * torch.randn(m, 1, generator=g))).to(T).cuda()
    (wg, cg), (wu, cu) = bu.weight(g, n, k, N, M), bu.weight(g, n, k, N, M)
    size = 1.0 / (40 * k ** 0.5)                        # so that g is of order one
    cg, cu = cg / 1e-3 * size * (M / N) ** 0.5, cu / 1e-3 * size
    bg, bu_ = (0.3 * torch.randn(n, generator=g), 0.3 * torch.randn(n, generator=g)) if bias else (None, None)
    w = nb.GatedWeight.from_int8(wg, cg, wu, cu, bias_gate=bg, bias_up=bu_, act=act, N=N, M=M)
    return x, w, (wg, cg, bg, wu, cu, bu_, act), g


@pytest.mark.parametrize("T", bu.TYPES)
@pytest.mark.parametrize("m,k,n", [(1, 64, 32), (1, 1024, 1000), (3, 17, 5), (16, 256, 16), (17, 130, 33),
                                   (33, 1, 1), (64, 2048, 48), (65, 771, 129), (200, 384, 100), (700, 96, 515)])
def test_forward(T, m, k, n):
    x, w, plain, _ = case(m, k, n, T, bias=n % 2 == 1)
    want, mag = bu.gated(*bu.codes(x), *plain)
    bu.close(nb.gated_ffn(x, w), want, T, mag, 4)


@pytest.mark.parametrize("act", ACTS)
def test_activations(act):
    x, w, plain, _ = case(50, 160, 70, torch.float32, True, act=act, seed=5)
    x = 8 * x                                           # far into the tails
    want, mag = bu.gated(*bu.codes(x), *plain)
    bu.close(nb.gated_ffn(x, w), want, torch.float32, mag, 4)


@pytest.mark.parametrize("N,M", [(2, 4), (1, 4), (1, 8), (2, 8), (3, 8), (4, 8), (5, 8), (6, 8)])
@pytest.mark.parametrize("m", [1, 20, 300])
def test_patterns(N, M, m):
    x, w, plain, _ = case(m, 272, 72, torch.bfloat16, True, N, M)
    want, mag = bu.gated(*bu.codes(x), *plain)
    bu.close(nb.gated_ffn(x, w, out_dtype=torch.float32), want, torch.float32, mag, 4)


# the 8-wave tiles, the tile of which two share a compute unit (with and without a short last k-step), sparse weights
@pytest.mark.parametrize("N,M,m,k,n", [(8, 8, 18464, 1024, 320), (8, 8, 8011, 1040, 1603), (8, 8, 20000, 64, 900),
                                       (8, 8, 30000, 17, 700), (2, 4, 9000, 256, 1024), (2, 8, 20000, 512, 512)])
def test_large_shapes_by_sampled_rows(N, M, m, k, n):
    x, w, plain, g = case(m, k, n, torch.half, False, N, M)
    h = nb.gated_ffn(x, w)
    rows = torch.cat([torch.arange(0, 4), torch.arange(m - 4, m), torch.randint(0, m, (100,), generator=g)])
    want, mag = bu.gated(*bu.codes(x[rows]), *plain)
    bu.close(h[rows], want, torch.half, mag, 4)


GRAD_SHAPES = [(1, 64, 32), (2, 1, 1), (5, 17, 3), (63, 100, 40), (64, 128, 64), (65, 200, 33), (130, 771, 129),
               (300, 64, 257), (1000, 48, 70), (4100, 32, 20)]


def check_grads(got, want, T):
    for name, (ref, room) in want.items():
        t = getattr(got, name)
        dtype = torch.float32 if name.startswith("dbias") else T
        bu.close(t, ref, dtype, room / bu.E, 1)


@pytest.mark.parametrize("T", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("m,k,n", GRAD_SHAPES)
def test_backward(T, m, k, n):
    act = ACTS[(m + k + n) % 5]
    x, w, plain, g = case(m, k, n, T, bias=n % 2 == 1, act=act)
    q, s = nb.quantize_rows(x)
    dh = torch.randn(m, n, generator=g).to(T).cuda()
    got = nb.gated_ffn_backward(q, s, w, dh)
    check_grads(got, bu.gated_grads(q[:, :k], s, *plain, dh, T), T)
    again = nb.gated_ffn_backward(q, s, w, dh)
    assert all(torch.equal(a, b) for a, b in zip(got, again) if a is not None)


@pytest.mark.parametrize("T", [torch.float16, torch.bfloat16])
def test_backward_with_split_reductions(T):
    # a long batch and a small weight: the weights' gradient is summed in parts
    m, k, n = 9000, 96, 64
    x, w, plain, g = case(m, k, n, T, True, act="gelu")
    q, s = nb.quantize_rows(x)
    dh = torch.randn(m, n + 3, generator=g).to(T).cuda()[:, 1:n + 1]
    got = nb.gated_ffn_backward(q, s, w, dh)
    check_grads(got, bu.gated_grads(q[:, :k], s, *plain, dh, T), T)


def test_backward_of_zero_scales_and_empty_rows():
    x, w, plain, g = case(70, 80, 40, torch.float16, True)
    x[3], x[69] = 0, 0
    q, s = nb.quantize_rows(x)
    dh = torch.randn(70, 40, generator=g).half().cuda()
    got = nb.gated_ffn_backward(q, s, w, dh)
    check_grads(got, bu.gated_grads(q[:, :80], s, *plain, dh, torch.float16), torch.float16)
    empty = nb.gated_ffn_backward(q[:0], s[:0], w, dh[:0])
    assert empty.dx.shape == (0, 80) and (empty.dw_gate == 0).all() and (empty.dbias_up == 0).all()


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "sigmoid"])
def test_backward_against_differences(act):
    # the derivative along random directions of dequantised weights, inputs and biases, by central differences of
    # the 64-bit forward (step 1e-4: its own error is 1e-8).  The kernel's operands are rounded to binary16: each
    # term is within 2^-11 + 2^-11 (its own rounding and the output's) of exact.
    m, k, n, h = 40, 64, 48, 1e-4
    x, w, (wg, cg, bg, wu, cu, bu_, _), g = case(m, k, n, torch.float16, True, act=act, seed=9)
    q, s = nb.quantize_rows(x)
    dh = torch.randn(m, n, generator=g).half().cuda()
    got = nb.gated_ffn_backward(q, s, w, dh)
    at = {"x": q[:, :k].double().cpu() * s.double().cpu()[:, None], "wg": wg.double() * cg.double()[:, None],
          "wu": wu.double() * cu.double()[:, None], "bg": bg.double(), "bu": bu_.double()}
    grads = {"x": got.dx, "wg": got.dw_gate, "wu": got.dw_up, "bg": got.dbias_gate, "bu": got.dbias_up}

    def value(v):
        f, _ = bu.act(v["x"] @ v["wg"].t() + v["bg"], act)
        return float((f * (v["x"] @ v["wu"].t() + v["bu"]) * dh.double().cpu()).sum())

    for name, grad in grads.items():
        way = torch.randn(at[name].shape, generator=g, dtype=torch.float64)
        slope = (value(dict(at, **{name: at[name] + h * way})) - value(dict(at, **{name: at[name] - h * way}))) / (2 * h)
        # the gradient's entries are sums of many terms: allow 2^-10 of the root of their squares, four times over
        terms = way * grad.double().cpu()
        assert abs(float(terms.sum()) - slope) <= 4 * 2.0 ** -10 * float(terms.norm()) * 4 + 1e-5, name


def test_graphs_and_streams():
    x, w, _, g = case(150, 128, 96, torch.bfloat16, True)
    q, s = nb.quantize_rows(x)
    dh = torch.randn(150, 96, generator=g).bfloat16().cuda()
    h, grads = nb.gated_ffn(x, w), nb.gated_ffn_backward(q, s, w, dh)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = nb.gated_ffn_backward(q, s, w, dh, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(grads, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h2, back = nb.gated_ffn(x, w), nb.gated_ffn_backward(q, s, w, dh)
    for _ in range(3):
        for t in (h2, *back):
            t.fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(h, h2) and all(torch.equal(a, b) for a, b in zip(grads, back))


def test_refusals():
    x, w, (wg, cg, bg, wu, cu, bu_, _), _ = case(8, 64, 32, torch.float16, True)
    q, s = nb.quantize_rows(x)
    dh = torch.zeros(8, 32, device="cuda").half()
    sparse = case(8, 64, 32, torch.float16, False, 2, 4)[1]
    bad = [
        lambda: nb.gated_ffn_backward(q, s, w, dh.float()),
        lambda: nb.gated_ffn_backward(q, s, w, dh[:7]),
        lambda: nb.gated_ffn_backward(q, s, w, dh[:, :31]),
        lambda: nb.gated_ffn_backward(q, s, w, dh.cpu()),
        lambda: nb.gated_ffn_backward(q, s, sparse, dh),
        lambda: nb.gated_ffn_backward(q[:, :48], s, w, dh),
        lambda: nb.gated_ffn(x[:, :60], w),
        lambda: nb.GatedWeight.from_int8(wg, cg, wu[:16], cu),
        lambda: nb.GatedWeight.from_int8(wg, cg, wu, cu, bias_gate=bg),
        lambda: nb.GatedWeight.from_int8(wg, cg, wu, cu, act="swish"),
        lambda: nb.GatedWeight.from_int8(wg * 0, cg, wu * 0, cu, N=2, M=4, trainable=True),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was accepted")


@pytest.mark.parametrize("T", bu.TYPES)
def test_a_token_has_the_same_bits_in_every_batch(T):
    # one token, a few, and a batch of tiles run different kernels on the same sums
    for N, M in ((8, 8), (2, 4), (4, 8)):
        x, w, (wg, cg, bg, *_), _ = case(700, 256, 100, T, True, N, M)
        lin = nb.ScaledWeight.from_int8(wg, cg, bias=bg, N=N, M=M)
        for call, weight in ((nb.gated_ffn, w), (nb.linear_i8, lin)):
            all_ = call(x, weight)
            for part in (1, 3, 20, 50):
                assert torch.equal(call(x[:part], weight), all_[:part])


@pytest.mark.parametrize("m,k,n", [(5, 17, 3), (387, 131, 70)])
def test_codes_without_padding(m, k, n):
    x, w, plain, g = case(m, k, n, torch.bfloat16, True, act="gelu")
    q, s = nb.quantize_rows(x)
    dh = torch.randn(m, n, generator=g).bfloat16().cuda()
    assert torch.equal(nb.gated_ffn_i8(q[:, :k], s, w), nb.gated_ffn_i8(q, s, w))
    for got, want in zip(nb.gated_ffn_backward(q[:, :k].contiguous(), s, w, dh), nb.gated_ffn_backward(q, s, w, dh)):
        assert torch.equal(got, want)


@pytest.mark.parametrize("T", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("m,k,n", [(5, 17, 3), (130, 96, 40), (1000, 48, 70)])
def test_scales_of_either_sign(T, m, k, n):
    # a channel (or token) with a negative scale is the negated codes with the positive one
    act = ACTS[(m + k) % 5]
    x, _, (wg, cg, bg, wu, cu, bu_, _), g = case(m, k, n, T, True, act=act)
    q, s = nb.quantize_rows(x)
    dh = torch.randn(m, n, generator=g).to(T).cuda()
    sg, su, ss = (torch.where(torch.rand(c, generator=g) < 0.5, -1, 1) for c in (n, n, m))

    def weight(a, b, c, d):
        return nb.GatedWeight.from_int8(a, b, c, d, bias_gate=bg, bias_up=bu_, act=act, trainable=True)

    def flip(w, sign):
        return (w * sign[:, None]).to(torch.int8)

    signed, codes = weight(wg, cg * sg, wu, cu * su), weight(flip(wg, sg), cg, flip(wu, su), cu)
    neg = flip(q, ss.cuda())
    assert torch.equal(nb.gated_ffn_i8(q, s * ss.cuda(), signed), nb.gated_ffn_i8(neg, s, codes))
    got = nb.gated_ffn_backward(q, s * ss.cuda(), signed, dh)
    want = bu.gated_grads(neg[:, :k], s, flip(wg, sg), cg, bg, flip(wu, su), cu, bu_, act, dh, T)
    check_grads(got, want, T)
    for a, b in zip(got, nb.gated_ffn_backward(neg, s, codes, dh)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("T", bu.TYPES)
def test_gelu_keeps_its_relative_accuracy_in_the_tail(T):
    # g is given exactly (one code of 1 a row, its scale |g|), u is 1.  In units of 2^-24 of the result: the fitted
    # tail 2.6; its argument, a rounded product and sum and a reciprocal within an ulp, 2.5 times up to 2.6; eight steps of
    # Horner's rule at 1.75 times their result 14; the exponential and its correction 4; three products 3: 31.
    g = torch.cat([torch.linspace(-12, 12, 4001), torch.tensor([0.0, 100.0, 3e38, -100.0, -1e30])])
    q = torch.zeros(len(g), 16, dtype=torch.int8)
    q[:, 0] = torch.sign(g)
    one, zero = torch.ones(3, 1, dtype=torch.int8), torch.zeros(3)
    w = nb.GatedWeight.from_int8(one, zero + 1, 0 * one, zero + 1, bias_gate=zero, bias_up=zero + 1, act="gelu")
    h = nb.gated_ffn_i8(q.cuda(), g.abs().cuda(), w, out_dtype=T)
    v = g.double()
    want = (v * 0.5 * torch.special.erfc(-v / 2 ** 0.5))[:, None].expand(-1, 3)
    if T == torch.float16:
        want = torch.where(want > 65519.0, torch.inf, want)
    bu.close(h, want, T, want.abs(), 32)


# the tile of which two workgroups share a compute unit: every type of its staging, biases, activations and a last k-step
# of 16, 48 and 64 bytes
@pytest.mark.parametrize("T", bu.TYPES)
@pytest.mark.parametrize("m,k,n,act", [(20011, 208, 701, "gelu"), (18464, 1000, 830, "relu"), (33000, 64, 515, "gelu_tanh"),
                                       (20000, 72, 700, "sigmoid")])
def test_two_workgroups_a_unit_by_sampled_rows(T, m, k, n, act):
    x, w, plain, g = case(m, k, n, T, True, act=act)
    out = torch.full((m + 1, n + 5), 7.0, dtype=T, device="cuda")
    h = nb.gated_ffn(x, w, out=out[:m, 2:n + 2])
    rows = torch.cat([torch.arange(0, 4), torch.arange(m - 4, m), torch.randint(0, m, (100,), generator=g)])
    want, mag = bu.gated(*bu.codes(x[rows]), *plain)
    bu.close(h[rows], want, T, mag, 4)
    assert (out[m:] == 7).all() and (out[:, :2] == 7).all() and (out[:, n + 2:] == 7).all()
