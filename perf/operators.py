"""The operators of a training step beside the contractions: layer norm in both directions, orthogonalised updates.

A case is a dict of plain values; its "op" says which operator it is:

  norm_fwd       rows of C values -> their normalisation, and the mean and 1/deviation that the backward pass needs
  norm_bwd       the gradients of the input, gamma and beta from the output's
  orthogonalize  update matrices -> five Newton-Schulz steps towards their orthogonal factors

Rows are tokens or pixels, C their channels.  Sizes are those of the networks in `nets`, of bench.py's GEMM sweep, and
generic ones of language models.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
STEPS, NS_EPS = 5, 1e-7
NS = (3.4445, -4.7750, 2.0315)
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}

# the weight matrices of ResNet-18, filters as rows
RESNET18 = ("64x147," + "64x576," * 4 + "128x576,128x64," + "128x1152," * 3 + "256x1152,256x128," + "256x2304," * 3
            + "512x2304,512x256," + "512x4608," * 3 + "1000x512")


def listed():
    return [
        # one token of a served model: latency counts
        {"name": "norm_fwd_1x1024", "op": "norm_fwd", "M": 1, "C": 1024, "pitch": 1024, "x": "bf16", "y": "bf16"},
        # fp32 activations, odd channels in a padded buffer
        {"name": "norm_fwd_777x1001_f32", "op": "norm_fwd", "M": 777, "C": 1001, "pitch": 1008, "x": "f32", "y": "f32"},
        # the rows of the GEMM sweep's largest product: a training batch of 16384 tokens
        {"name": "norm_fwd_16384x4096", "op": "norm_fwd", "M": 16384, "C": 4096, "pitch": 4096, "x": "bf16", "y": "bf16"},
        # long rows of an fp32 residual stream, normalised for the tensor cores
        {"name": "norm_fwd_4096x16384", "op": "norm_fwd", "M": 4096, "C": 16384, "pitch": 16384, "x": "f32", "y": "bf16"},
        # a small batch before the last layer of VGG-7: a launch or two of microseconds
        {"name": "norm_bwd_128x1024", "op": "norm_bwd", "M": 128, "C": 1024, "pitch": 1024, "x": "bf16", "y": "bf16"},
        # odd rows and channels, gradients and activations of different types
        {"name": "norm_bwd_2999x1001", "op": "norm_bwd", "M": 2999, "C": 1001, "pitch": 1001, "x": "f32", "y": "bf16"},
        # the pixels of a first-stage layer of ResNet-18 at 64 images: many short rows
        {"name": "norm_bwd_200704x64", "op": "norm_bwd", "M": 200704, "C": 64, "pitch": 64, "x": "bf16", "y": "bf16"},
        # a training batch of 16384 tokens
        {"name": "norm_bwd_16384x4096", "op": "norm_bwd", "M": 16384, "C": 4096, "pitch": 4096, "x": "bf16", "y": "bf16"},
        # one 3x3 layer of 64 channels: sixteen launches of almost nothing
        {"name": "orthogonalize_64x576", "op": "orthogonalize", "shapes": "64x576", "g": "f32"},
        # all weights of ResNet-18 in one call
        {"name": "orthogonalize_resnet18", "op": "orthogonalize", "shapes": RESNET18, "g": "f32"},
        # an odd tall matrix: more outputs than inputs
        {"name": "orthogonalize_5001x2047", "op": "orthogonalize", "shapes": "5001x2047", "g": "f32"},
        # the weights of the GEMM sweep's largest product and a wider layer beside it
        {"name": "orthogonalize_4096_and_8192", "op": "orthogonalize", "shapes": "4096x4096,4096x8192", "g": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["norm_fwd", "norm_bwd", "orthogonalize"])
    if op == "orthogonalize":
        shapes, left = [], 4096 * 4096 + 4096 * 8192
        for _ in range(rng.choice([1, 1, 2, 3, 8])):
            r, c = _log_int(rng, 1, 8192), _log_int(rng, 1, 8192)
            while r * c > left or min(r, c) > 4096:
                r, c = (r + 1) // 2, (c + 1) // 2
            left = max(1, left - r * c)
            shapes.append("%dx%d" % (r, c))
        return {"op": op, "shapes": ",".join(shapes), "g": rng.choice(["bf16", "f32"])}
    C = _log_int(rng, 16, 32768)
    if rng.random() < 0.5:
        C = -(-C // 8) * 8
    M = _log_int(rng, 1, max(1, min(262144, 16384 * 4096 // C)))
    pitch = C + rng.choice([0, 0, 1, 8, 24])
    return {"op": op, "M": M, "C": C, "pitch": pitch, "x": rng.choice(["bf16", "f32"]), "y": rng.choice(["bf16", "f32"])}


def _shapes(case):
    return [tuple(int(v) for v in s.split("x")) for s in case["shapes"].split(",")]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    s = {"case": case}
    if case["op"] == "orthogonalize":
        # a momentum: a few directions that the batches agree on, above the noise of the samples
        s["G"] = [_momentum(normal, r, c).to(DTYPE[case["g"]]) for r, c in _shapes(case)]
        s["O"] = [torch.empty(r, c, dtype=torch.bfloat16, device="cuda") for r, c in _shapes(case)]
        return s
    M, C, pitch = case["M"], case["C"], case["pitch"]
    # activations: rows of different size and offset, channels of different size
    x = normal(M, pitch) * (0.5 + normal(C if pitch == C else pitch).abs())
    x = x * (0.25 + 1.5 * normal(M, 1).abs()) + 0.5 * normal(M, 1)
    s["X"] = x.to(DTYPE[case["x"]])
    s["gamma"] = 1.0 + 0.3 * normal(C)
    if case["op"] == "norm_fwd":
        s["beta"] = 0.3 * normal(C)
        s["Y"] = torch.empty(M, C, dtype=DTYPE[case["y"]], device="cuda")
        s["mean"], s["rstd"] = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
        return s
    v = s["X"][:, :C].double()
    mean = v.mean(1)
    s["mean"], s["rstd"] = mean.float(), ((v - mean[:, None]).square().mean(1) + EPS).rsqrt().float()
    s["dY"] = (normal(M, pitch) * (0.1 + normal(M, 1).abs())).to(DTYPE[case["y"]])
    s["dX"] = torch.empty(M, C, dtype=DTYPE[case["y"]], device="cuda")
    s["dgamma"], s["dbeta"] = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    return s


def _momentum(normal, r, c):
    k = max(1, min(r, c) // 16)
    return 0.01 * (normal(r, k) @ normal(k, c) / math.sqrt(k) + 0.5 * normal(r, c))


# ---- plain forms: 32 bits, one rounding at the end
def _norm_fwd(s):
    C = s["case"]["C"]
    x = s["X"][:, :C].float()
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = 1.0 / (d.square().mean(1, keepdim=True) + EPS).sqrt()
    y = d * rstd * s["gamma"] + s["beta"]
    return y.to(s["Y"].dtype), mean[:, 0], rstd[:, 0]


def _norm_bwd(s):
    C = s["case"]["C"]
    xh = (s["X"][:, :C].float() - s["mean"][:, None]) * s["rstd"][:, None]
    dy = s["dY"][:, :C].float()
    g = dy * s["gamma"]
    dx = (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)) * s["rstd"][:, None]
    return dx.to(s["dX"].dtype), (dy * xh).sum(0), dy.sum(0)


def _orthogonalize(G):
    a, b, c = NS
    x = G.float() if G.shape[0] <= G.shape[1] else G.float().T
    # the norm in 64 bits: a long sum of squares
    x = x / x.double().square().sum().sqrt().clamp(min=NS_EPS).float()
    for _ in range(STEPS):
        s = x @ x.T
        x = a * x + (b * s + c * (s @ s)) @ x
    return (x if G.shape[0] <= G.shape[1] else x.T).to(torch.bfloat16)


# ---- the framework's calls
def _own_norm_fwd(s):
    from paper_1605_04711_b200 import twn
    c = s["case"]
    twn.layer_norm_fwd(s["X"], c["pitch"], c["M"], c["C"], s["gamma"], s["beta"], EPS, s["Y"], c["C"], s["mean"], s["rstd"])
    return s["Y"], s["mean"], s["rstd"]


def _own_norm_bwd(s):
    from paper_1605_04711_b200 import twn
    c = s["case"]
    if "ws" not in s:
        s["ws"] = torch.empty(twn.layer_norm_bwd_workspace_bytes(c["M"], c["C"]), dtype=torch.uint8, device="cuda")
    twn.layer_norm_bwd(s["dY"], c["pitch"], s["X"], c["pitch"], c["M"], c["C"], s["gamma"], s["mean"], s["rstd"],
                       s["dX"], c["C"], s["dgamma"], s["dbeta"], s["ws"])
    return s["dX"], s["dgamma"], s["dbeta"]


def _own_orthogonalize(s):
    from paper_1605_04711_b200 import twn
    items = [(G, G.shape[0], G.shape[1], O) for G, O in zip(s["G"], s["O"])]
    if "ws" not in s:
        s["ws"] = torch.empty(twn.orthogonalize_workspace_bytes([i[1:3] for i in items]), dtype=torch.uint8, device="cuda")
    twn.orthogonalize_batch(items, STEPS, NS_EPS, s["ws"])
    return s["O"]


def run(s):
    op = s["case"]["op"]
    if own:
        return {"norm_fwd": _own_norm_fwd, "norm_bwd": _own_norm_bwd, "orthogonalize": _own_orthogonalize}[op](s)
    if op == "orthogonalize":
        return [_orthogonalize(G) for G in s["G"]]
    return _norm_fwd(s) if op == "norm_fwd" else _norm_bwd(s)


def work(case):
    if case["op"] == "orthogonalize":
        size = 2 if case["g"] == "bf16" else 4
        flops = nbytes = 0
        for r, c in _shapes(case):
            m, n = min(r, c), max(r, c)
            # a symmetric product needs one triangle
            flops += STEPS * (m * (m + 1) * n + m * (m + 1) * m + 2 * m * m * n)
            nbytes += r * c * (size + 2)
        return {"bytes": nbytes, "flops": flops}
    M, C = case["M"], case["C"]
    x, y = (2 if case[k] == "bf16" else 4 for k in ("x", "y"))
    if case["op"] == "norm_fwd":
        return {"bytes": M * C * (x + y) + 8 * C + 8 * M, "flops": 8 * M * C}
    return {"bytes": M * C * (x + 2 * y) + 12 * C + 8 * M, "flops": 14 * M * C}


# ---- the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "orthogonalize":
        return [_polar_steps(G.double()) for G in s["G"]]
    C = case["C"]
    x = s["X"][:, :C].double()
    if case["op"] == "norm_fwd":
        mean = x.sum(1) / C
        var = torch.einsum("ij,ij->i", x - mean[:, None], x - mean[:, None]) / C
        rstd = (var + EPS).pow(-0.5)
        return (x - mean[:, None]).mul_(rstd[:, None]).mul_(s["gamma"].double()).add_(s["beta"].double()), mean, rstd
    mean, rstd = s["mean"].double(), s["rstd"].double()
    n = (x - mean[:, None]) * rstd[:, None]
    dy = s["dY"][:, :C].double()
    dgamma = torch.einsum("ij,ij->j", dy, n)
    dbeta = torch.einsum("ij->j", dy)
    p = dy * s["gamma"].double()
    p0, p1 = p.sum(1) / C, torch.einsum("ij,ij->i", p, n) / C
    return (p - p0[:, None] - n * p1[:, None]) * rstd[:, None], dgamma, dbeta


def _polar_steps(G):
    """As the odd polynomial p(t) = a t + b t^3 + c t^5, iterated, applied to the singular values through G's smaller Gram
    matrix kept factored: every step multiplies the iterate by a + b S + c S^2 from the shorter side."""
    a, b, c = NS
    tall = G.shape[0] > G.shape[1]
    X = G / max(float(torch.linalg.vector_norm(G)), NS_EPS)
    eye = torch.eye(min(G.shape), dtype=torch.float64, device=G.device)
    for _ in range(STEPS):
        S = X.mT @ X if tall else X @ X.mT
        Q = torch.addmm(b * S, S, S, alpha=c) + a * eye
        X = X @ Q if tall else Q @ X
    return X
