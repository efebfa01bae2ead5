"""Measured cases of the transformer-block operators: the product in 8-bit integers with scales for each token and
channel, the norms around a block with its gate and residual scale, and the gated feed-forward block.

Formulas (T: the type of the activations; sums and norms in 32 bits or more, one rounding to T at each operator's end):

* row codes: s[i] = max_t |x[i,t]| / 127, q[i,t] = rint(x[i,t] * (127 / max_t |x[i,t]|)), both quotients and the product
  in binary32; a row whose largest magnitude is below 2^-100 has s = 0 and zero codes.
* linear: y[i,j] = s[i] c[j] sum_t q[i,t] w[j,t] + b[j]; w int8 with scales c.
* norm: u = post(y); res = alpha r + gate u; z = pre(res).  A norm is RMS or layer norm with weight and (layer norm) bias;
  post may be absent; gate rows are shared by m / groups consecutive tokens.
* norm backward: from dz and dres, at the given y and res: dy, dr, and the sums over tokens for gate, weights and biases.
* gated: h = act(g) u with g = linear(x; w_gate), u = linear(x; w_up).
* gated backward: from dh, at the given codes: dx, dw_gate, dw_up (of the dequantised operands) and the bias sums.
* block: norm with row codes of z, gated block, row codes of h, linear back to the residual's width, norm.
"""
import math

import torch

own = False

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
ACTS = ("silu", "gelu", "gelu_tanh", "relu", "sigmoid")


# ---------------------------------------------------------------- cases

def listed():
    return [
        # ViT-L fc1 for one token: latency of the smallest serving call
        dict(name="linear_token", op="linear", m=1, k=1024, n=4096, dtype="fp16", N=8, M=8, bias=True, strided=False),
        # a classifier head on a ragged batch: every size odd, 32-bit activations
        dict(name="linear_odd_fp32", op="linear", m=97, k=1021, n=1001, dtype="fp32", N=8, M=8, bias=True, strided=True),
        # ViT-L fc2 of one 384 x 384 image, 2:4 sparse
        dict(name="linear_sparse_image", op="linear", m=577, k=4096, n=1024, dtype="bf16", N=2, M=4, bias=True,
             strided=False),
        # ViT-L fc1 at batch 32: the largest product
        dict(name="linear_vit_l", op="linear", m=18464, k=1024, n=4096, dtype="fp16", N=8, M=8, bias=True, strided=False),
        # the norms around a block for one token
        dict(name="norm_token", op="norm", m=1, d=1024, dtype="bf16", pre="rms", post="none", groups=1, alpha=1.0),
        # ViT-L at batch 32: layer norms with a learned gate per channel
        dict(name="norm_vit_l", op="norm", m=18464, d=1024, dtype="bf16", pre="layer", post="none", groups=1, alpha=1.0),
        # DeiT-S at batch 64, a gate per image, both norms and a residual scale: training step
        dict(name="norm_bwd_deit_s", op="norm_bwd", m=12608, d=384, dtype="fp16", pre="layer", post="rms", groups=64,
             alpha=0.75),
        # ViT-L at batch 32, layer norms before and after: training step
        dict(name="norm_bwd_vit_l", op="norm_bwd", m=18464, d=1024, dtype="bf16", pre="layer", post="layer", groups=1,
             alpha=1.0),
        # gated block of ViT-L width (two thirds of 4096 hidden channels) for one token
        dict(name="gated_token", op="gated", m=1, k=1024, n=2736, dtype="fp16", act="silu", bias=False, N=8, M=8),
        # the same at batch 32
        dict(name="gated_vit_l", op="gated", m=18464, k=1024, n=2736, dtype="bf16", act="silu", bias=False, N=8, M=8),
        # gated block of DeiT-B width at batch 32: training step
        dict(name="gated_bwd_deit_b", op="gated_bwd", m=6304, k=768, n=2048, dtype="bf16", act="gelu", bias=True),
        # a whole feed-forward half of DeiT-B at batch 8, the product back 2:4 sparse
        dict(name="block_deit_b", op="block", m=1576, d=768, n=2048, dtype="fp16", act="silu", N=2, M=4),
    ]


LARGEST = 18464 * 1024 * 4096   # multiply-adds of the largest listed case


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("linear", "linear", "norm", "norm_bwd", "gated", "gated_bwd", "block"))
    dtype = rng.choice(("fp16", "bf16"))
    if op in ("norm", "norm_bwd"):
        d = _log_int(rng, 64, 2048)
        m = _log_int(rng, 1, min(18464, 18464 * 1024 // d))
        groups = rng.choice((1, 1, rng.randint(1, 64)))
        m = max(1, m // groups) * groups
        return dict(op=op, m=m, d=d if rng.random() < 0.4 else max(64, d // 8 * 8),
                    dtype=rng.choice((dtype, dtype, "fp32")), pre=rng.choice(("rms", "layer")),
                    post=rng.choice(("none", "rms", "layer")), groups=groups, alpha=round(rng.uniform(0.5, 1.5), 3))
    k, n = _log_int(rng, 64, 4096), _log_int(rng, 64, 4096)
    if rng.random() < 0.6:
        k, n = max(64, k // 16 * 16), max(64, n // 16 * 16)
    N, M = 8, 8
    if op != "gated_bwd" and rng.random() < 0.4:
        N, M = rng.choice(((2, 4), (1, 4), (2, 8), (4, 8)))
        k = max(64, k // 16 * 16)
    # multiply-adds of one token, those of 16-bit operands twice
    one = {"linear": k * n, "gated": 2 * k * n, "gated_bwd": 10 * k * n, "block": 3 * k * n}[op]
    m = _log_int(rng, 1, max(1, min(18464, LARGEST // one)))
    if op == "linear":
        return dict(op=op, m=m, k=k, n=n, dtype=rng.choice((dtype, dtype, "fp32")), N=N, M=M, bias=rng.random() < 0.5,
                    strided=rng.random() < 0.3)
    act = rng.choice(ACTS)
    if op == "gated":
        return dict(op=op, m=m, k=k, n=n, dtype=rng.choice((dtype, dtype, "fp32")), act=act, bias=rng.random() < 0.5,
                    N=N, M=M)
    if op == "gated_bwd":
        return dict(op=op, m=m, k=k, n=n, dtype=dtype, act=act, bias=rng.random() < 0.5)
    return dict(op=op, m=m, d=max(64, k // 16 * 16), n=max(64, n // 16 * 16), dtype=dtype, act=act, N=N, M=M)


def _stored(n, k, N, M):
    """Bytes of an N:M weight: its values and two or three position bits for each."""
    return n * k if N * 8 > 5 * M else int(n * k * N / M * (1 + (2 if M == 4 else 3) / 8))


def work(case):
    op, m = case["op"], case["m"]
    eb = 4 if case["dtype"] == "fp32" else 2
    if op in ("norm", "norm_bwd"):
        d, post = case["d"], case["post"] != "none"
        params = d * 4 * (case["groups"] + 1 + (case["pre"] == "layer") + post + (case["post"] == "layer"))
        if op == "norm":
            return {"bytes": 4 * m * d * eb + params, "flops": 12 * m * d}
        return {"bytes": 6 * m * d * eb + 2 * params, "flops": 30 * m * d}
    n = case["n"]
    if op == "linear":
        k = case["k"]
        return {"bytes": m * k * eb + _stored(n, k, case["N"], case["M"]) + m * n * eb + 8 * n, "flops": 2 * m * n * k}
    if op == "gated":
        k = case["k"]
        return {"bytes": m * k * eb + 2 * _stored(n, k, case["N"], case["M"]) + m * n * eb + 16 * n,
                "flops": 4 * m * n * k}
    if op == "gated_bwd":
        k = case["k"]
        return {"bytes": m * k + 2 * n * k + m * n * eb + m * k * eb + 2 * n * k * eb + 24 * n, "flops": 12 * m * n * k}
    d = case["d"]
    return {"bytes": 4 * m * d * eb + 2 * n * d + _stored(d, n, case["N"], case["M"]), "flops": 6 * m * n * d}


# ---------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _acts(g, m, k, T, strided=False):
    """Activations as they leave a norm: tokens of unequal size, a few channels that stand out."""
    x = _randn(g, m, k) * torch.exp(0.3 * _randn(g, m, 1)) * torch.exp(0.4 * _randn(g, 1, k))
    if strided:   # a column slice of a wider buffer
        wide = torch.empty(m, k + 24, device="cuda", dtype=T)
        wide[:, :k] = x
        return wide[:, :k]
    return x.to(T)


def _weight(g, n, k, N, M):
    """Normal weights, the N largest of each M consecutive ones kept, in int8 with a scale for each channel."""
    w = _randn(g, n, k) * 0.02
    if N < M:
        groups = w.view(n, k // M, M)
        drop = groups.abs().topk(M - N, dim=2, largest=False).indices
        w = groups.scatter(2, drop, 0.0).view(n, k)
    c = torch.clamp(w.abs().amax(1) / 127, min=1e-8)
    return torch.clamp(torch.round(w / c[:, None]), -127, 127).to(torch.int8), c


def _bias(g, n, wanted):
    return _randn(g, n) * 0.1 if wanted else None


def _norm_params(g, d, kind):
    if kind == "none":
        return None
    return {"kind": kind, "w": 1 + 0.1 * _randn(g, d), "b": 0.1 * _randn(g, d) if kind == "layer" else None, "eps": 1e-6}


def _codes(x):
    """Codes and scales of rows, for the cases whose path starts from them."""
    x = x.float()
    top = x.abs().amax(1)
    live = top >= 2.0 ** -100
    c = torch.full_like(top, 127.0)
    s, inv = torch.where(live, top.div(c), 0.0), torch.where(live, c.div(top), 0.0)
    return torch.clamp(torch.round(x * inv[:, None]), -127, 127), s


def prepare(case, seed):
    g, op, T, m = _gen(seed), case["op"], DTYPES[case["dtype"]], case["m"]
    s = dict(case, T=T)
    if op == "linear":
        s["x"] = _acts(g, m, case["k"], T, case["strided"])
        s["w"], s["c"] = _weight(g, case["n"], case["k"], case["N"], case["M"])
        s["b"] = _bias(g, case["n"], case["bias"])
    elif op in ("norm", "norm_bwd"):
        d = case["d"]
        s["y"], s["r"] = (0.7 * _randn(g, m, d) + 0.1).to(T), (2 * _randn(g, m, d) + 0.3).to(T)
        s["gate"] = (0.3 + 0.2 * _randn(g, case["groups"], d))
        s["pre_p"], s["post_p"] = _norm_params(g, d, case["pre"]), _norm_params(g, d, case["post"])
        if op == "norm_bwd":   # r stands for the residual that the forward pass left
            s["dz"], s["dres"] = (0.5 * _randn(g, m, d)).to(T), _randn(g, m, d).to(T)
    elif op in ("gated", "gated_bwd"):
        n, k, N, M = case["n"], case["k"], case.get("N", 8), case.get("M", 8)
        (s["wg"], s["cg"]), (s["wu"], s["cu"]) = _weight(g, n, k, N, M), _weight(g, n, k, N, M)
        s["bg"], s["bu"] = _bias(g, n, case["bias"]), _bias(g, n, case["bias"])
        s["x"] = _acts(g, m, k, T)
        if op == "gated_bwd":
            q, s["sx"] = _codes(s.pop("x"))
            s["xq"] = q.to(torch.int8)
            s["dh"] = _randn(g, m, n).to(T)
    else:
        d, n = case["d"], case["n"]
        s["y"], s["r"] = (0.7 * _randn(g, m, d)).to(T), (2 * _randn(g, m, d)).to(T)
        s["gate"], s["gate2"] = 0.3 + 0.2 * _randn(g, 1, d), 0.3 + 0.2 * _randn(g, 1, d)
        s["pre_p"], s["next_p"] = _norm_params(g, d, "layer"), _norm_params(g, d, "layer")
        (s["wg"], s["cg"]), (s["wu"], s["cu"]) = _weight(g, n, d, 8, 8), _weight(g, n, d, 8, 8)
        s["w"], s["c"] = _weight(g, d, n, case["N"], case["M"])
        s["b"], s["bg"], s["bu"] = _bias(g, d, True), None, None
    if own:   # what a user's program lays out once: the weights
        from paper_2607_12505_amd import nmblock as nb
        if "w" in s:
            s["lin"] = nb.ScaledWeight.from_int8(s["w"], s["c"], bias=s["b"], N=case["N"], M=case["M"])
        if "wg" in s:
            N, M = (case.get("N", 8), case.get("M", 8)) if op == "gated" else (8, 8)
            s["gw"] = nb.GatedWeight.from_int8(s["wg"], s["cg"], s["wu"], s["cu"], bias_gate=s["bg"], bias_up=s["bu"],
                                               act=case["act"], N=N, M=M, trainable=op == "gated_bwd")
        for name in ("pre", "post", "next"):
            p = s.get(name + "_p")
            s[name + "_n"] = None if p is None else nb.Norm(p["kind"], p["w"], p["b"], p["eps"])
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2607_12505_amd import nmblock as nb
    op = s["op"]
    if op == "linear":
        return nb.linear_i8(s["x"], s["lin"])
    if op == "norm":
        return nb.norm_residual(s["y"], s["r"], pre=s["pre_n"], post=s["post_n"], gate=s["gate"], alpha=s["alpha"])
    if op == "norm_bwd":
        return nb.norm_residual_backward(s["dz"], s["dres"], s["y"], s["r"], pre=s["pre_n"], post=s["post_n"],
                                         gate=s["gate"], alpha=s["alpha"])._asdict()
    if op == "gated":
        return nb.gated_ffn(s["x"], s["gw"])
    if op == "gated_bwd":
        return nb.gated_ffn_backward(s["xq"], s["sx"], s["gw"], s["dh"])._asdict()
    res, zq, sz = nb.norm_residual_i8(s["y"], s["r"], pre=s["pre_n"], gate=s["gate"])
    h = nb.gated_ffn_i8(zq, sz, s["gw"], out_dtype=s["T"])
    return nb.norm_residual(nb.linear_i8(h, s["lin"]), res, pre=s["next_n"], gate=s["gate2"])


def _plain_linear(q, s, w, c, b):
    y = (q @ w.float().t()) * s[:, None] * c
    return y if b is None else y + b


def _plain_norm(v, p):
    if p is None:
        return v
    if p["kind"] == "layer":
        v = v - v.mean(1, keepdim=True)
    v = v * torch.rsqrt((v * v).mean(1, keepdim=True) + p["eps"]) * p["w"]
    return v if p["b"] is None else v + p["b"]


def _rows(gate, m):
    return gate if gate.shape[0] in (1, m) else gate.repeat_interleave(m // gate.shape[0], 0)


def _plain_norm_residual(y, r, pre, post, gate, alpha):
    res = alpha * r.float() + _rows(gate, r.shape[0]) * _plain_norm(y.float(), post)
    return res, _plain_norm(res, pre)


def _plain_norm_grad(v, dy, p):
    """Gradients of a norm at v: of v, of the weight, of the bias, and the normalised v times weight plus bias."""
    if p is None:
        return dy, None, None, v
    layer = p["kind"] == "layer"
    if layer:
        v = v - v.mean(1, keepdim=True)
    scale = torch.rsqrt((v * v).mean(1, keepdim=True) + p["eps"])
    hat = v * scale
    g = dy * p["w"]
    back = g - hat * (g * hat).mean(1, keepdim=True)
    if layer:
        back = back - g.mean(1, keepdim=True)
    out = hat * p["w"] + p["b"] if layer else hat * p["w"]
    return back * scale, (dy * hat).sum(0), dy.sum(0) if layer else None, out


def _plain_act(g, act):
    """act(g) and its derivative."""
    if act == "silu":
        e = 1 / (1 + torch.exp(-g))
        return g * e, e * (1 + g * (1 - e))
    if act == "sigmoid":
        e = 1 / (1 + torch.exp(-g))
        return e, e * (1 - e)
    if act == "relu":
        return torch.where(g > 0, g, 0.0), torch.where(g > 0, 1.0, 0.0)
    if act == "gelu":
        p = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * p, p + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    a, b = math.sqrt(2 / math.pi), 0.044715
    t = torch.tanh(a * (g + b * g * g * g))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * a * (1 + 3 * b * g * g)


def _plain_gated(q, sx, s):
    g, u = _plain_linear(q, sx, s["wg"], s["cg"], s["bg"]), _plain_linear(q, sx, s["wu"], s["cu"], s["bu"])
    return _plain_act(g, s["act"])[0] * u


def _run_plain(s):
    op, T = s["op"], s["T"]
    if op == "linear":
        return _plain_linear(*_codes(s["x"]), s["w"], s["c"], s["b"]).to(T)
    if op == "norm":
        res, z = _plain_norm_residual(s["y"], s["r"], s["pre_p"], s["post_p"], s["gate"], s["alpha"])
        return res.to(T), z.to(T)
    if op == "norm_bwd":
        dres, dw, db, _ = _plain_norm_grad(s["r"].float(), s["dz"].float(), s["pre_p"])
        dres = dres + s["dres"].float()
        m, gate = dres.shape[0], s["gate"]
        rows = _rows(gate, m)
        dy, dwp, dbp, u = _plain_norm_grad(s["y"].float(), dres * rows, s["post_p"])
        dgate = (dres * u).view(gate.shape[0], -1, gate.shape[1]).sum(1)
        return dict(dy=dy.to(T), dr=(s["alpha"] * dres).to(T), dgate=dgate, dpre_weight=dw, dpre_bias=db,
                    dpost_weight=dwp, dpost_bias=dbp)
    if op == "gated":
        return _plain_gated(*_codes(s["x"]), s).to(T)
    if op == "gated_bwd":
        q, sx, dh = s["xq"].float(), s["sx"], s["dh"].float()
        g, u = _plain_linear(q, sx, s["wg"], s["cg"], s["bg"]), _plain_linear(q, sx, s["wu"], s["cu"], s["bu"])
        a, da = _plain_act(g, s["act"])
        dg, du = dh * u * da, dh * a
        x = q * sx[:, None]
        dx = dg @ (s["wg"].float() * s["cg"][:, None]) + du @ (s["wu"].float() * s["cu"][:, None])
        bias = s["bg"] is not None
        return dict(dx=dx.to(T), dw_gate=(dg.t() @ x).to(T), dw_up=(du.t() @ x).to(T),
                    dbias_gate=dg.sum(0) if bias else None, dbias_up=du.sum(0) if bias else None)
    res, z = _plain_norm_residual(s["y"], s["r"], s["pre_p"], None, s["gate"], 1.0)
    res, h = res.to(T), _plain_gated(*_codes(z), s).to(T)
    y = _plain_linear(*_codes(h), s["w"], s["c"], s["b"]).to(T)
    out, z = _plain_norm_residual(y, res, s["next_p"], None, s["gate2"], 1.0)
    return out.to(T), z.to(T)


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_codes(x):
    """Codes are decided in binary32, as defined; they and their scales are then exact."""
    x = x.to(torch.float32)
    top = torch.max(torch.abs(x), dim=1).values
    num = torch.full_like(top, 127.0)
    tiny = top < 2.0 ** -100
    inv = torch.where(tiny, torch.zeros_like(top), torch.div(num, top))
    q = torch.round(torch.mul(x, inv.unsqueeze(1))).clamp(-127, 127).double()
    return q, torch.where(tiny, torch.zeros_like(top), torch.div(top, num)).double()


def _exact_product(q, s, w, c, b):
    y = s.unsqueeze(1) * torch.matmul(q, w.double().t().contiguous()) * c.double().unsqueeze(0)
    return y + b.double() if b is not None else y


def _exact_hat(v, p):
    mu = v.mean(1, keepdim=True) if p["kind"] == "layer" else torch.zeros_like(v[:, :1])
    var = ((v - mu) ** 2).mean(1, keepdim=True)
    return (v - mu) / torch.sqrt(var + p["eps"]), 1 / torch.sqrt(var + p["eps"])


def _exact_affine(hat, p):
    return hat * p["w"].double() + (p["b"].double() if p["b"] is not None else 0.0)


def _exact_gate(gate, m):
    return gate.double()[torch.arange(m, device=gate.device) // (m // gate.shape[0])]


def _exact_around(y, r, pre, post, gate, alpha):
    u = y.double() if post is None else _exact_affine(_exact_hat(y.double(), post)[0], post)
    res = alpha * r.double() + _exact_gate(gate, r.shape[0]) * u
    return res, _exact_affine(_exact_hat(res, pre)[0], pre)


def _exact_act(g, act):
    sig = torch.sigmoid(g)
    if act == "silu":
        return g * sig, sig + g * sig * (1 - sig)
    if act == "sigmoid":
        return sig, sig * (1 - sig)
    if act == "relu":
        return torch.clamp(g, min=0), (g > 0).double()
    if act == "gelu":
        cdf = 0.5 * torch.erfc(-g / math.sqrt(2))
        return g * cdf, cdf + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    inner = math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)
    t = torch.tanh(inner)
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t ** 2) * math.sqrt(2 / math.pi) * (1 + 0.134145 * g ** 2)


def exact(case, seed):
    s = prepare(case, seed)
    op, T = case["op"], s["T"]
    if op == "linear":
        return _exact_product(*_exact_codes(s["x"]), s["w"], s["c"], s["b"])
    if op == "norm":
        return _exact_around(s["y"], s["r"], s["pre_p"], s["post_p"], s["gate"], s["alpha"])
    if op == "norm_bwd":
        pre, post, m = s["pre_p"], s["post_p"], case["m"]
        dz, gate = s["dz"].double(), _exact_gate(s["gate"], m)

        def through(v, dv, p):   # (hat-gradient projected) / deviation
            hat, inv = _exact_hat(v, p)
            t = dv * p["w"].double()
            mean = t.mean(1, keepdim=True) if p["kind"] == "layer" else 0.0
            return inv * (t - mean - hat * (t * hat).mean(1, keepdim=True)), hat

        d, hat = through(s["r"].double(), dz, pre)
        d = d + s["dres"].double()
        out = dict(dr=case["alpha"] * d, dpre_weight=(dz * hat).sum(0),
                   dpre_bias=dz.sum(0) if pre["kind"] == "layer" else None, dpost_weight=None, dpost_bias=None)
        y = s["y"].double()
        if post is None:
            out["dy"], u = d * gate, y
        else:
            out["dy"], yhat = through(y, d * gate, post)
            u = _exact_affine(yhat, post)
            out["dpost_weight"] = (d * gate * yhat).sum(0)
            out["dpost_bias"] = (d * gate).sum(0) if post["kind"] == "layer" else None
        out["dgate"] = (d * u).reshape(case["groups"], m // case["groups"], case["d"]).sum(1)
        return out
    if op == "gated":
        q, sx = _exact_codes(s["x"])
        g, u = _exact_product(q, sx, s["wg"], s["cg"], s["bg"]), _exact_product(q, sx, s["wu"], s["cu"], s["bu"])
        return _exact_act(g, case["act"])[0] * u
    if op == "gated_bwd":
        q, sx, dh = s["xq"].double(), s["sx"].double(), s["dh"].double()
        g, u = _exact_product(q, sx, s["wg"], s["cg"], s["bg"]), _exact_product(q, sx, s["wu"], s["cu"], s["bu"])
        a, slope = _exact_act(g, case["act"])
        dg, du = dh * u * slope, dh * a
        wg, wu = s["cg"].double().unsqueeze(1) * s["wg"].double(), s["cu"].double().unsqueeze(1) * s["wu"].double()
        x = sx.unsqueeze(1) * q
        return dict(dx=dg @ wg + du @ wu, dw_gate=dg.t().contiguous() @ x, dw_up=du.t().contiguous() @ x,
                    dbias_gate=dg.sum(0) if case["bias"] else None, dbias_up=du.sum(0) if case["bias"] else None)
    # each operator of the chain ends in its own rounding to T
    res, z = _exact_around(s["y"], s["r"], s["pre_p"], None, s["gate"], 1.0)
    q, sz = _exact_codes(z)
    g, u = _exact_product(q, sz, s["wg"], s["cg"], None), _exact_product(q, sz, s["wu"], s["cu"], None)
    h = (_exact_act(g, case["act"])[0] * u).to(T)
    y = _exact_product(*_exact_codes(h), s["w"], s["c"], s["b"]).to(T)
    return _exact_around(y, res.to(T), s["next_p"], None, s["gate2"], 1.0)
