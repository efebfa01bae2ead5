"""Rotary positions with several axes, forward and backward, against their 64-bit form (bounds: attention_util)."""
import math

import pytest
import torch

import attention_util as au
from paper_2607_12505_amd import nmattention as na

pytestmark = pytest.mark.gpu
TYPES = [torch.float16, torch.bfloat16, torch.float32]


def gen(seed):
    return torch.Generator().manual_seed(seed)


def check(got, x, pos, axes, freqs, axis, back=False):
    want, room = au.rotary(x.reshape(-1, *x.shape[-2:]), pos, freqs, axis, axes.style, back)
    u = au.UNIT[x.dtype]
    au.within(got.reshape(want.shape), want, room + u * want.abs() + au.TINY[x.dtype])


# one pair, whole pieces, odd widths, pairs that end inside a piece, the widest heads; tokens from one on
@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("style", ["halves", "pairs"])
@pytest.mark.parametrize("tokens,heads,d,sections", [
    (1, 1, 2, (1,)), (1, 32, 64, (16, 16)), (7, 3, 64, (32,)), (33, 5, 91, (13, 12, 12)), (200, 2, 64, (8, 8, 8)),
    (65, 4, 48, (4, 2, 1, 1)), (3, 2, 1024, (512,)), (50, 3, 130, (33, 32)), (1000, 1, 16, (8,)), (19, 6, 80, (20, 20))])
def test_forward_and_back(T, style, tokens, heads, d, sections):
    g = gen(tokens + d)
    axes = na.RotaryAxes.of_sections(sections, own_ladders=d % 4 == 0, style=style)
    freqs, axis = axes.freqs.tolist(), axes.axis.tolist()
    x = torch.randn(tokens, heads, d, generator=g).to(T).cuda()
    pos = torch.randint(-300, 5000, (len(sections), tokens), generator=g, dtype=torch.int32).cuda()
    check(na.rotary(x, pos, axes), x, pos, axes, freqs, axis)
    check(na.rotary_backward(x, pos, axes), x, pos, axes, freqs, axis, back=True)
    kept = x[..., 2 * sum(sections):]
    assert torch.equal(na.rotary(x, pos, axes)[..., 2 * sum(sections):], kept)


def test_gradient_against_differences():
    # (rotary(x + h v) - rotary(x - h v)) . dy / 2 h = v . rotary_backward(dy): linear, so exact but for rounding
    g = gen(3)
    axes = na.RotaryAxes.of_sections((5, 4, 3))
    x, v, dy = (torch.randn(20, 3, 30, generator=g).cuda() for _ in range(3))
    pos = torch.randint(0, 100, (3, 20), generator=g, dtype=torch.int32).cuda()
    slope = ((na.rotary(x + v, pos, axes).double() - na.rotary(x - v, pos, axes).double()) / 2 * dy.double()).sum()
    back = (na.rotary_backward(dy, pos, axes).double() * v.double()).sum()
    size = (dy.double().abs() * (x.abs() + v.abs()).double()).sum()
    assert abs(float(slope - back)) <= 64 * au.E * float(size)


@pytest.mark.parametrize("T", [torch.float32, torch.bfloat16])
def test_far_positions_keep_their_angles(T):
    g = gen(4)
    axes = na.RotaryAxes([1.0, 0.37, 1e-4], [0, 1, 0])
    x = torch.randn(64, 2, 6, generator=g).to(T).cuda()
    pos = torch.randint(-2 ** 31 + 1, 2 ** 31 - 1, (2, 64), generator=g, dtype=torch.int64).to(torch.int32).cuda()
    check(na.rotary(x, pos, axes), x, pos, axes, [1.0, 0.37, 1e-4], [0, 1, 0])


def test_float_positions_and_shared_rows_of_them():
    g = gen(5)
    axes = na.RotaryAxes.of_sections((4, 4), theta=100.0)
    x = torch.randn(30, 2, 16, generator=g).half().cuda()
    pos = (torch.rand(2, 30, generator=g) * 2 - 1).cuda()
    check(na.rotary(x, pos, axes), x, pos, axes, axes.freqs.tolist(), axes.axis.tolist())
    one = pos[:1].expand(2, 30)                          # a row for both axes
    check(na.rotary(x, one, axes), x, one, axes, axes.freqs.tolist(), axes.axis.tolist())
    wide = torch.cat((pos, pos), 1)[:, 7:37]             # rows further apart than their length
    check(na.rotary(x, wide, axes), x, wide, axes, axes.freqs.tolist(), axes.axis.tolist())


@pytest.mark.parametrize("pad", [0, 3, 8])
def test_inside_wider_rows_in_place_and_into_a_cache(pad):
    g = gen(6)
    axes = na.RotaryAxes.of_sections((8, 8))
    row = torch.randn(2, 9, 6 * 32 + pad, generator=g).half().cuda()
    x = row[..., :6 * 32].unflatten(-1, (6, 32))         # [sequences, tokens, heads, d]
    pos = torch.randint(0, 50, (2, 18), generator=g, dtype=torch.int32).cuda()
    want = na.rotary(x.reshape(18, 6, 32).contiguous(), pos, axes)
    assert torch.equal(na.rotary(x, pos, axes).reshape(18, 6, 32), want)
    q, k = na.rotary_qk(x[..., :4, :], x[..., 4:, :], pos, axes)
    assert torch.equal(torch.cat((q, k), -2).reshape(18, 6, 32), want)
    cache = torch.full((2, 40, 6, 32), 7.0, dtype=torch.float16, device="cuda")
    first = pos.view(2, 2, 9)[..., 0].contiguous()       # one new token of each sequence
    na.rotary(x[:, 0], first, axes, out=cache[:, 11])
    assert torch.equal(cache[:, 11], want.view(2, 9, 6, 32)[:, 0])
    cache[:, 11] = 7.0
    assert (cache == 7.0).all()
    tail = row[..., 6 * 32:].clone()
    assert na.rotary(x, pos, axes, out=x) is x
    assert torch.equal(x.reshape(18, 6, 32), want) and torch.equal(row[..., 6 * 32:], tail)


def test_heads_before_tokens_and_values_that_are_not_finite():
    g = gen(7)
    axes = na.RotaryAxes.of_sections((8,))
    x = torch.randn(5, 13, 16, generator=g).cuda()       # [heads, tokens, d]
    pos = torch.arange(13, dtype=torch.int32).cuda()
    assert torch.equal(na.rotary(x.transpose(0, 1), pos, axes), na.rotary(x.transpose(0, 1).contiguous(), pos, axes))
    x[2, 3, 1], x[2, 3, 15] = math.inf, math.nan
    y = na.rotary(x.transpose(0, 1), pos, axes)
    bad = ~torch.isfinite(y)
    assert bad[3, 2, 1] and bad[3, 2, 9] and bad[3, 2, 15] and bad[3, 2, 7] and int(bad.sum()) == 4


def test_no_tokens_and_no_heads():
    axes = na.RotaryAxes.of_sections((4,))
    pos = torch.zeros(1, 0, dtype=torch.int32, device="cuda")
    assert na.rotary(torch.zeros(0, 2, 8, device="cuda"), pos, axes).shape == (0, 2, 8)
    assert na.rotary(torch.zeros(3, 0, 8, device="cuda"), torch.zeros(1, 3, dtype=torch.int32, device="cuda"),
                     axes).shape == (3, 0, 8)


def test_refusals():
    axes = na.RotaryAxes.of_sections((4, 4))
    x = torch.zeros(3, 2, 16, device="cuda", dtype=torch.float16)
    pos = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    for bad in (x.double(), x[..., :15], x[0, 0], x.transpose(1, 2), x.cpu()):
        with pytest.raises(ValueError):
            na.rotary(bad, pos, axes)
    for bad in (pos[:1], pos[:, :2], pos.long(), pos.cpu(), torch.zeros(3, 2, dtype=torch.int32, device="cuda").t()):
        with pytest.raises(ValueError):
            na.rotary(x, bad, axes)
    with pytest.raises(ValueError):
        na.rotary(x, pos, axes, out=x[:2])
    with pytest.raises(ValueError):
        na.rotary_qk(x, x[:2], pos, axes)
    with pytest.raises(ValueError):
        na.rotary(torch.zeros(2, 5, 2, 16, device="cuda")[:, :3], torch.zeros(2, 6, dtype=torch.int32, device="cuda"), axes)
    for args in (([], []), ([1.0], [0, 1]), ([1.0], [-1]), ([math.inf], [0])):
        with pytest.raises(ValueError):
            na.RotaryAxes(*args)
    with pytest.raises(ValueError):
        na.RotaryAxes([1.0], [0], style="thirds")


def test_expanded_inputs():
    axes, T = na.RotaryAxes.of_sections((4, 4)), torch.bfloat16
    x = torch.randn(1, 3, 16, generator=torch.Generator().manual_seed(8)).to(T).cuda()
    pos = torch.arange(14, dtype=torch.int32).view(2, 7).cuda()
    for some in (x.expand(7, 3, 16), x[:, :1].expand(7, 5, 16)):
        assert torch.equal(na.rotary(some, pos, axes), na.rotary(some.contiguous(), pos, axes))
        with pytest.raises(ValueError):
            na.rotary(some, pos, axes, out=some)


def test_given_stream_and_captured_graph():
    g = gen(8)
    axes = na.RotaryAxes.of_sections((16, 16))
    x = torch.randn(40, 4, 64, generator=g).half().cuda()
    pos = torch.randint(0, 24, (2, 40), generator=g, dtype=torch.int32).cuda()
    want = na.rotary(x, pos, axes)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = na.rotary(x, pos, axes, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    out = torch.empty_like(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        na.rotary(x, pos, axes, out=out)
        na.rotary_backward(out, pos, axes, out=out)
    for seed in (1, 2, 3):
        x.copy_(torch.randn(40, 4, 64, generator=gen(seed)).half())
        eager = na.rotary_backward(na.rotary(x, pos, axes), pos, axes)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
