"""Measured cases of the operators of a decoder block's training step: the norm and position rotation of queries and keys with
its gradient, the matrix product with bias, activation and residual with its gradients, and the orthogonalised update.

`listed()` names the cases, `draw()` gives further ones of the same ranges, `prepare()` makes what a training program
holds before the call, `run()` is one pass: with `own` set through the library's entry points, otherwise in plain torch
operations in 32 bits, rounded once at the end.  `exact()` states the same results in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda:0"
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
COEFFICIENTS = [(3.4445, -4.7750, 2.0315)] * 5
EPS_NORM, EPS_UPDATE = 1e-6, 1e-7


# --------------------------------------------------------------------------------------------------------------
# Cases.  Widths, heads and lengths are those of the GPT-2-XL-shaped (1600 wide, 25 heads of 64, 1024 tokens, 6400 in the
# feed-forward layer) and BERT-large-shaped (1024 wide, 16 heads of 64, 512 tokens, 4096) workloads, or generic.
# --------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one new token in each of 8 sequences, at far positions: latency alone
        {"name": "norm_rotate_one", "op": "norm_rotate", "B": 8, "T": 1, "Hq": 25, "Hk": 25, "D": 64, "R": 64, "act": "bf16",
         "weight": "f32", "inter": False, "packed": True, "far": True},
        # a decoder's training forward, q and k inside what one projection wrote
        {"name": "norm_rotate_batch", "op": "norm_rotate", "B": 8, "T": 1024, "Hq": 25, "Hk": 25, "D": 64, "R": 64,
         "act": "bf16", "weight": "f32", "inter": False, "packed": True, "far": False},
        # its backward pass
        {"name": "norm_rotate_grad_batch", "op": "norm_rotate_grad", "B": 8, "T": 1024, "Hq": 25, "Hk": 25, "D": 64, "R": 64,
         "act": "bf16", "weight": "f32", "inter": False, "packed": True, "far": False},
        # an odd length with shared key heads, half of each head rotated, in fp32
        {"name": "norm_rotate_grad_shared", "op": "norm_rotate_grad", "B": 3, "T": 1037, "Hq": 16, "Hk": 4, "D": 128, "R": 64,
         "act": "f32", "weight": "f32", "inter": True, "packed": False, "far": False},
        # one token through the up-projection: the weights are read once
        {"name": "linear_one", "op": "linear", "n": 1, "i": 1600, "o": 6400, "act": "bf16", "out": "bf16", "w_t": False,
         "bias": True, "f": "gelu", "residual": False, "pre": False},
        # a ragged batch through a layer of odd widths, weights held as [out, in]
        {"name": "linear_odd", "op": "linear", "n": 777, "i": 1601, "o": 1999, "act": "f16", "out": "f16", "w_t": True,
         "bias": True, "f": "silu", "residual": True, "pre": False},
        # the up-projection of 8 x 1024 tokens, its pre-activation kept for the backward pass
        {"name": "linear_up", "op": "linear", "n": 8192, "i": 1600, "o": 6400, "act": "bf16", "out": "bf16", "w_t": False,
         "bias": True, "f": "gelu", "residual": False, "pre": True},
        # the backward pass of the down-projection behind it, through the activation; fp32 gradients for the transport
        {"name": "linear_grad_down", "op": "linear_grad", "n": 8192, "i": 6400, "o": 1600, "act": "bf16", "dw": "f32",
         "w_t": False, "f": "gelu", "residual": False},
        # an attention projection of 16 x 512 tokens, whose input also feeds a residual
        {"name": "linear_grad_square", "op": "linear_grad", "n": 8192, "i": 1024, "o": 1024, "act": "f16", "dw": "f16",
         "w_t": True, "f": None, "residual": True},
        # a small matrix: latency of a chain of dependent products
        {"name": "orthogonalize_small", "op": "orthogonalize", "b": 1, "m": 129, "n": 200, "x": "f32", "out": "bf16"},
        # one feed-forward matrix, taller than wide, result in fp32
        {"name": "orthogonalize_tall", "op": "orthogonalize", "b": 1, "m": 6400, "n": 1600, "x": "f32", "out": "f32"},
        # the attention projections of eight layers
        {"name": "orthogonalize_layers", "op": "orthogonalize", "b": 8, "m": 1600, "n": 4800, "x": "bf16", "out": "bf16"},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm_rotate", "norm_rotate_grad", "linear", "linear_grad", "orthogonalize"])
    act = rng.choice(["bf16", "bf16", "f16"])
    if op in ("norm_rotate", "norm_rotate_grad"):
        act = rng.choice([act, act, "f32"])
        D = rng.choice([64, 64, 128, 128, 80, 96, 40, 256])
        inter = rng.random() < 0.4 or D == 40
        R = rng.choice([D, D, D // 2, 16]) // 16 * 16 or 16
        Hk = rng.choice([1, 2, 4, 8, 12, 16, 25])
        Hq = Hk * rng.choice([1, 1, 2, 4])
        most = 8192 * 50 * 64 // (2 if act == "f32" else 1)
        T = _log(rng, 1, max(1, min(8192, most // ((Hq + Hk) * D))))
        B = _log(rng, 1, max(1, min(32, most // ((Hq + Hk) * D * T))))
        return {"op": op, "B": B, "T": T, "Hq": Hq, "Hk": Hk, "D": D, "R": R, "act": act, "weight": rng.choice(["f32", act]),
                "inter": inter, "packed": Hq == Hk and rng.random() < 0.5, "far": rng.random() < 0.3}
    f = rng.choice([None, "relu", "gelu", "gelu_tanh", "silu"])
    if op in ("linear", "linear_grad"):
        i, o = (rng.choice([64, 1024, 1600, 4096, 4800, 6400, _log(rng, 1, 6400), _log(rng, 33, 2500)]) for _ in range(2))
        while i * o > 1600 * 6400:
            i, o = (i + 1) // 2, (o + 1) // 2
        n = _log(rng, 1, min(32768, 8192 * 1600 * 6400 // (i * o)))
        c = {"op": op, "n": n, "i": i, "o": o, "act": act, "w_t": rng.random() < 0.5, "f": f, "residual": rng.random() < 0.5}
        if op == "linear":
            return {**c, "out": rng.choice([act, act, "f32"]), "bias": rng.random() < 0.7, "pre": rng.random() < 0.4}
        return {**c, "dw": rng.choice([act, "f32"])}
    m, n = (rng.choice([64, 768, 1024, 1600, _log(rng, 8, 4096), _log(rng, 8, 4096)]) for _ in range(2))
    low, high = sorted((m, n))
    most = 8 * 1600 * 1600 * (2 * 4800 + 1600)                                 # products of the largest listed case
    b = _log(rng, 1, max(1, min(64, most // (low * low * (2 * high + low)))))
    return {"op": op, "b": b, "m": m, "n": n, "x": rng.choice(["f32", "bf16", "f16"]), "out": rng.choice(["bf16", "bf16", "f32"])}


# --------------------------------------------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 6007 + 29)
    return g


def _randn(g, shape, dtype, sigma=1.0):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).mul_(sigma).to(dtype)


def _rotate_inputs(case, seed):
    """q, k, their weights, positions [B, T], frequencies [R / 2] in radians a position, and the gradients of both outputs."""
    g = _gen(seed)
    B, T, Hq, Hk, D, R, dt = (case[x] for x in ("B", "T", "Hq", "Hk", "D", "R", "act"))
    if case["packed"]:
        q, k, _ = _randn(g, (B, T, 3, Hq, D), TORCH[dt], 1.5).unbind(2)
    else:
        q, k = _randn(g, (B, T, Hq, D), TORCH[dt], 1.5), _randn(g, (B, T, Hk, D), TORCH[dt], 1.5)
    qw, kw = ((1.0 + 0.2 * torch.randn(D, generator=g, device=DEV)).to(TORCH[case["weight"]]) for _ in range(2))
    first = torch.randint(0, 500000 if case["far"] else 1, (B, 1), generator=g, device=DEV, dtype=torch.int32)
    positions = first + torch.arange(T, device=DEV, dtype=torch.int32)
    freqs = 10000.0 ** (-torch.arange(R // 2, device=DEV, dtype=torch.float64) * 2 / R)
    dqo = dko = None
    if case["op"] == "norm_rotate_grad":
        dqo, dko = _randn(g, (B, T, Hq, D), TORCH[dt], 0.1), _randn(g, (B, T, Hk, D), TORCH[dt], 0.1)
    return q, k, qw, kw, positions, freqs, dqo, dko


def _weights(g, case):
    i, o, dt = case["i"], case["o"], TORCH[case["act"]]
    sigma = 1.0 / math.sqrt(i)
    return _randn(g, (o, i), dt, sigma).t() if case["w_t"] else _randn(g, (i, o), dt, sigma)


def _linear_inputs(case, seed):
    """x, w, bias, residual of the forward pass."""
    g = _gen(seed)
    n, i, o = case["n"], case["i"], case["o"]
    x, w = _randn(g, (n, i), TORCH[case["act"]]), _weights(g, case)
    bias = _randn(g, (o,), torch.float32, 0.3) if case["bias"] else None
    res = _randn(g, (n, o), TORCH[case["out"]]) if case["residual"] else None
    return x, w, bias, res


def _linear_grad_inputs(case, seed):
    """dy, x, w, the pre-activation behind x, and the gradient that reaches x another way."""
    g = _gen(seed)
    n, i, o, dt = case["n"], case["i"], case["o"], TORCH[case["act"]]
    dy, w = _randn(g, (n, o), dt, 0.05), _weights(g, case)
    pre = _randn(g, (n, i), dt)
    x = ACT[case["f"]](pre.float()).to(dt) if case["f"] else pre
    res = _randn(g, (n, i), dt, 0.05) if case["residual"] else None
    return dy, x, w, (pre if case["f"] else None), res


def _update_input(case, seed):
    """A momentum of a gradient: a few strong directions over noise."""
    g = _gen(seed)
    b, m, n = case["b"], case["m"], case["n"]
    strong = torch.randn((b, m, 8), generator=g, device=DEV) @ torch.randn((b, 8, n), generator=g, device=DEV)
    x = (strong.mul_(0.5).add_(torch.randn((b, m, n), generator=g, device=DEV)) * 1e-2).to(TORCH[case["x"]])
    return x


def prepare(case, seed):
    s = dict(case)
    if own:
        from paper_2605_01989_b200 import binding
        s["dblp"] = d = binding
    empty = dict(device=DEV)
    if case["op"] in ("norm_rotate", "norm_rotate_grad"):
        s["q"], s["k"], s["qw"], s["kw"], s["positions"], s["freqs"], s["dqo"], s["dko"] = _rotate_inputs(case, seed)
        shapes = [(case["B"], case["T"], case[h], case["D"]) for h in ("Hq", "Hk")]
        s["q_out"], s["k_out"] = (torch.empty(x, dtype=TORCH[case["act"]], **empty) for x in shapes)
        s["dqw"], s["dkw"] = torch.empty_like(s["qw"]), torch.empty_like(s["kw"])
        if own and case["op"] == "norm_rotate_grad":
            s["ws"] = torch.empty(d.dblp_norm_rotate_grad_workspace_bytes(s["q"], s["k"]), dtype=torch.uint8, **empty)
    elif case["op"] == "linear":
        s["x"], s["w"], s["b"], s["res"] = _linear_inputs(case, seed)
        s["y"] = torch.empty((case["n"], case["o"]), dtype=TORCH[case["out"]], **empty)
        s["p"] = torch.empty((case["n"], case["o"]), dtype=TORCH[case["act"]], **empty) if case["pre"] else None
        if own:
            s["ws"] = torch.empty(d.dblp_linear_workspace_bytes(s["x"], s["w"])[0], dtype=torch.uint8, **empty)
    elif case["op"] == "linear_grad":
        s["dy"], s["x"], s["w"], s["p"], s["res"] = _linear_grad_inputs(case, seed)
        s["dx"] = torch.empty((case["n"], case["i"]), dtype=TORCH[case["act"]], **empty)
        shape = (case["o"], case["i"]) if case["w_t"] else (case["i"], case["o"])
        s["dwt"] = torch.empty(shape, dtype=TORCH[case["dw"]], **empty)
        s["db"] = torch.empty(case["o"], dtype=TORCH[case["dw"]], **empty)
        if own:
            s["ws"] = torch.empty(d.dblp_linear_workspace_bytes(s["x"], s["w"], s["dy"])[1], dtype=torch.uint8, **empty)
    else:
        s["g"] = _update_input(case, seed)
        s["u"] = torch.empty(s["g"].shape, dtype=TORCH[case["out"]], **empty)
        s["scale"] = math.sqrt(max(1.0, case["m"] / case["n"]))
        if own:
            s["ws"] = torch.empty(d.dblp_orthogonalize_workspace_bytes(s["g"], s["u"]), dtype=torch.uint8, **empty)
    return s


# --------------------------------------------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else PLAIN[s["op"]](s)


def _run_own(s):
    d = s["dblp"]
    if s["op"] == "norm_rotate":
        d.dblp_norm_rotate(s["q"], s["k"], s["qw"], s["kw"], s["positions"], s["freqs"], s["q_out"], s["k_out"], eps=EPS_NORM,
                           interleaved=s["inter"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if s["op"] == "norm_rotate_grad":
        d.dblp_norm_rotate_grad(s["q"], s["k"], s["qw"], s["kw"], s["positions"], s["freqs"], s["dqo"], s["dko"], s["q_out"],
                                s["k_out"], s["dqw"], s["dkw"], s["ws"], eps=EPS_NORM, interleaved=s["inter"])
        return {"dq": s["q_out"], "dk": s["k_out"], "dqw": s["dqw"], "dkw": s["dkw"]}
    if s["op"] == "linear":
        d.dblp_linear(s["x"], s["w"], s["y"], ws=s["ws"], bias=s["b"], residual=s["res"], pre=s["p"], activation=s["f"])
        return {"out": s["y"], "pre": s["p"]} if s["pre"] else {"out": s["y"]}
    if s["op"] == "linear_grad":
        dw = s["dwt"].t() if s["w_t"] else s["dwt"]
        d.dblp_linear_grad(s["dy"], s["x"], s["w"], dx=s["dx"], dw=dw, dbias=s["db"], ws=s["ws"], residual=s["res"], pre=s["p"],
                           activation=s["f"])
        return {"dx": s["dx"], "dw": dw, "dbias": s["db"]}
    d.dblp_orthogonalize(s["g"], s["u"], s["ws"], coefficients=COEFFICIENTS, eps=EPS_UPDATE, scale=s["scale"])
    return s["u"]


def _halves(x, R, inter):
    """The first and second members of the rotated pairs of x's first R columns."""
    return (x[..., 0:R:2], x[..., 1:R:2]) if inter else (x[..., :R // 2], x[..., R // 2:R])


def _rotated(x, cos, sin, R, inter):
    a, b = _halves(x, R, inter)
    ra, rb = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack((ra, rb), dim=-1).flatten(-2) if inter else torch.cat((ra, rb), dim=-1)
    return torch.cat((turned, x[..., R:]), dim=-1)


def _cos_sin(s):
    """fp32 cosine and sine of the angles, [B, T, 1, R / 2]; the angles of far positions need 64 bits."""
    angle = (s["positions"].double()[..., None] * s["freqs"]).unsqueeze(2)
    return angle.cos().float(), angle.sin().float()


def _plain_norm_rotate(s):
    cos, sin = _cos_sin(s)
    out = {}
    for n, w in (("q", "qw"), ("k", "kw")):
        x = s[n].float()
        y = x * torch.rsqrt((x * x).mean(dim=3, keepdim=True) + EPS_NORM) * s[w].float()
        out[n] = _rotated(y, cos, sin, s["R"], s["inter"]).to(s[n].dtype)
    return out


def _plain_norm_rotate_grad(s):
    cos, sin = _cos_sin(s)
    out = {}
    for n, w, do in (("q", "qw", "dqo"), ("k", "kw", "dko")):
        x = s[n].float()
        d = _rotated(s[do].float(), cos, -sin, s["R"], s["inter"])
        r = torch.rsqrt((x * x).mean(dim=3, keepdim=True) + EPS_NORM)
        wd = d * s[w].float()
        dx = r * wd - x * (r ** 3 * (wd * x).mean(dim=3, keepdim=True))
        out["d" + n] = dx.to(s[n].dtype)
        out["d" + w] = (d * x * r).sum(dim=(0, 1, 2)).to(s[w].dtype)
    return out


def _gelu(z):
    return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))


def _gelu_grad(z):
    return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)


def _tanh_arg(z):
    return math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)


def _gelu_tanh(z):
    return 0.5 * z * (1.0 + torch.tanh(_tanh_arg(z)))


def _gelu_tanh_grad(z):
    t = torch.tanh(_tanh_arg(z))
    return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * math.sqrt(2.0 / math.pi) * (1.0 + 3 * 0.044715 * z * z)


def _silu(z):
    return z / (1.0 + torch.exp(-z))


def _silu_grad(z):
    g = 1.0 / (1.0 + torch.exp(-z))
    return g * (1.0 + z * (1.0 - g))


ACT = {None: lambda z: z, "relu": lambda z: z.clamp_min(0.0), "gelu": _gelu, "gelu_tanh": _gelu_tanh, "silu": _silu}
ACT_GRAD = {"relu": lambda z: (z > 0).to(z.dtype), "gelu": _gelu_grad, "gelu_tanh": _gelu_tanh_grad, "silu": _silu_grad}


def _plain_linear(s):
    z = s["x"].float() @ s["w"].float()
    if s["b"] is not None:
        z = z + s["b"]
    y = ACT[s["f"]](z)
    if s["res"] is not None:
        y = y + s["res"].float()
    out = {"out": y.to(s["y"].dtype)}
    if s["pre"]:
        out["pre"] = z.to(s["x"].dtype)
    return out


def _plain_linear_grad(s):
    dy, x, w = s["dy"].float(), s["x"].float(), s["w"].float()
    dx = dy @ w.t()
    if s["res"] is not None:
        dx = dx + s["res"].float()
    if s["f"]:
        dx = dx * ACT_GRAD[s["f"]](s["p"].float())
    return {"dx": dx.to(s["x"].dtype), "dw": (x.t() @ dy).to(s["dwt"].dtype), "dbias": dy.sum(dim=0).to(s["db"].dtype)}


def _newton_schulz(x):
    """The iteration on the shorter side of x [batch, m, n], in x's type."""
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2)
    for a, b, c in COEFFICIENTS:
        A = x @ x.transpose(1, 2)
        x = a * x + (b * A + c * (A @ A)) @ x
    return x.transpose(1, 2) if tall else x


def _plain_orthogonalize(s):
    x = s["g"].float()
    x = x / (x.square().sum(dim=(1, 2), keepdim=True).sqrt() + EPS_UPDATE)
    return (_newton_schulz(x) * s["scale"]).to(s["u"].dtype)


PLAIN = {"norm_rotate": _plain_norm_rotate, "norm_rotate_grad": _plain_norm_rotate_grad, "linear": _plain_linear,
         "linear_grad": _plain_linear_grad, "orthogonalize": _plain_orthogonalize}


# --------------------------------------------------------------------------------------------------------------
# What a pass cannot do without
# --------------------------------------------------------------------------------------------------------------
def work(case):
    if case["op"] in ("norm_rotate", "norm_rotate_grad"):
        tokens = case["B"] * case["T"]
        n = tokens * (case["Hq"] + case["Hk"]) * case["D"]
        small = 4 * tokens + 4 * case["R"] + 2 * case["D"] * BYTES[case["weight"]]
        if case["op"] == "norm_rotate":
            return {"bytes": 2 * n * BYTES[case["act"]] + small, "flops": 7 * n}
        return {"bytes": 3 * n * BYTES[case["act"]] + small + 2 * case["D"] * BYTES[case["weight"]], "flops": 14 * n}
    if case["op"] == "linear":
        n, i, o, a = case["n"], case["i"], case["o"], BYTES[case["act"]]
        out = n * o * BYTES[case["out"]] * (2 if case["residual"] else 1) + (n * o * a if case["pre"] else 0)
        return {"bytes": (n * i + i * o) * a + out + (4 * o if case["bias"] else 0), "flops": 2 * n * i * o}
    if case["op"] == "linear_grad":
        n, i, o, a, dw = case["n"], case["i"], case["o"], BYTES[case["act"]], BYTES[case["dw"]]
        read = (n * o + n * i + i * o) * a + (n * i * a if case["f"] else 0) + (n * i * a if case["residual"] else 0)
        return {"bytes": read + n * i * a + (i * o + o) * dw, "flops": 4 * n * i * o}
    m, n = sorted((case["m"], case["n"]))
    per = (m * m * n + m * m * m + 2 * m * m * n) * len(COEFFICIENTS)          # two of the products are symmetric
    return {"bytes": case["b"] * m * n * (BYTES[case["x"]] + BYTES[case["out"]]), "flops": case["b"] * per}


# --------------------------------------------------------------------------------------------------------------
# The results in 64 bits, from the definitions
# --------------------------------------------------------------------------------------------------------------
def _turn(x, positions, freqs, inter, back):
    """Pairs of x [B, T, H, D] as complex numbers times exp(i angle), or times its conjugate."""
    R = 2 * freqs.numel()
    phase = torch.polar(torch.ones_like(freqs).expand(*positions.shape, -1), positions.double()[..., None] * freqs)[:, :, None]
    if inter:
        z = torch.view_as_complex(x[..., :R].reshape(*x.shape[:3], R // 2, 2).contiguous())
    else:
        z = torch.complex(x[..., :R // 2].contiguous(), x[..., R // 2:R].contiguous())
    z = z * (phase.conj() if back else phase)
    y = x.clone()
    y[..., :R] = torch.view_as_real(z).flatten(3) if inter else torch.cat((z.real, z.imag), dim=3)
    return y


def _exact_norm_rotate(case, seed):
    q, k, qw, kw, positions, freqs, dqo, dko = _rotate_inputs(case, seed)
    res = {}
    for name, x, w, do in (("q", q, qw, dqo), ("k", k, kw, dko)):
        x, w = x.double(), w.double()
        norm = torch.sqrt(x.pow(2).sum(3, keepdim=True) / case["D"] + EPS_NORM)
        unit = x / norm
        if case["op"] == "norm_rotate":
            res[name] = _turn(unit * w, positions, freqs, case["inter"], False)
            continue
        d = _turn(do.double(), positions, freqs, case["inter"], True)
        res["d%sw" % name] = torch.einsum("bthd,bthd->d", d, unit)
        along = torch.einsum("bthd,bthd->bth", d * w, unit) / case["D"]
        res["d" + name] = (d * w - unit * along[..., None]) / norm
    return res


def _normal_cdf(z):
    return 0.5 * torch.special.erfc(-z / math.sqrt(2.0))


def _exact_activation(f, z, slope):
    """f(z), or with `slope` its derivative, in 64 bits."""
    if f is None:
        return z
    if f == "relu":
        return (z > 0).double() if slope else torch.where(z > 0, z, 0.0)
    if f == "silu":
        g = torch.sigmoid(z)
        return g + z * g * torch.sigmoid(-z) if slope else z * g
    if f == "gelu":
        return _normal_cdf(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi) if slope else z * _normal_cdf(z)
    c = math.sqrt(8.0 / math.pi)                       # (1 + tanh u) / 2 = sigmoid(2 u)
    g = torch.sigmoid(c * (z + 0.044715 * z * z * z))
    return g + z * g * (1 - g) * c * (1 + 0.134145 * z * z) if slope else z * g


def _exact_linear(case, seed):
    x, w, bias, res = _linear_inputs(case, seed)
    z = torch.mm(x.double(), w.double())
    if bias is not None:
        z += bias.double()
    y = _exact_activation(case["f"], z, False)
    out = {"out": y if res is None else y + res.double()}
    if case["pre"]:
        out["pre"] = z
    return out


def _exact_linear_grad(case, seed):
    dy, x, w, pre, res = _linear_grad_inputs(case, seed)
    dy, x, w = dy.double(), x.double(), w.double()
    dx = torch.mm(dy, w.T)
    if res is not None:
        dx += res.double()
    if pre is not None:
        dx *= _exact_activation(case["f"], pre.double(), True)
    return {"dx": dx, "dw": torch.mm(x.T, dy), "dbias": torch.mv(dy.T, torch.ones(dy.shape[0], dtype=torch.float64, device=DEV))}


def _exact_orthogonalize(case, seed):
    """Matrix by matrix, by powers of the smaller Gram matrix: x (a + b G + c G^2), G = x^T x, or from the left."""
    g = _update_input(case, seed)
    out = torch.empty(g.shape, dtype=torch.float64, device=DEV)
    for j in range(case["b"]):
        x = g[j].double()
        x = x / (torch.linalg.vector_norm(x) + EPS_UPDATE)
        eye = torch.eye(min(case["m"], case["n"]), dtype=torch.float64, device=DEV)
        for a, b, c in COEFFICIENTS:
            if case["m"] > case["n"]:
                G = torch.mm(x.T, x)
                x = torch.mm(x, a * eye + b * G + c * torch.mm(G, G))
            else:
                G = torch.mm(x, x.T)
                x = torch.mm(a * eye + b * G + c * torch.mm(G, G), x)
        out[j] = x * math.sqrt(max(1.0, case["m"] / case["n"]))
    return out


def exact(case, seed):
    if case["op"] in ("norm_rotate", "norm_rotate_grad"):
        return _exact_norm_rotate(case, seed)
    return {"linear": _exact_linear, "linear_grad": _exact_linear_grad, "orthogonalize": _exact_orthogonalize}[case["op"]](case, seed)
