"""The feed-forward operators as cases that can be timed and compared: microscaled 4-bit storage
(quantisation and back), the product of two matrices held that way, the gated feed-forward block and its
training step.

A case is a dict of plain values.  ``listed()`` gives the standing cases, ``draw(rng)`` one more of the
same ranges, ``prepare(case, seed)`` what a program holds before the call (device tensors, workspaces,
output buffers), ``run(state)`` one pass, ``work(case)`` the bytes and operations that a pass cannot do
without, ``exact(case, seed)`` the outputs from the definition in 64 bits.

With ``own`` false a pass is made of elementary torch operations in 32 bits (the plain form); with
``own`` true it makes the calls that a program makes of ``paper_2109_00170_amd``.

Microscaled 4-bit storage: a row is cut into blocks of 32 columns (padded with zeros to whole groups of
four blocks).  A block has one scale 2^e, e = floor(log2 max|x|) - 2, stored as e + 127 in a byte, and
each element the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (with a sign) to x * 2^-e in four bits, ties to
the even code; the even column of a pair has the low four bits of the byte.  A block that holds an
infinity or a NaN has scale byte 255 and stands for NaN.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)

# ------------------------------------------------------------------------------- the cases


def listed():
    return [
        # one token's activations on their way into a 4-bit layer: latency alone counts
        {"name": "quantize_token", "op": "quantize", "rows": 1, "cols": 2048, "dtype": "bf16"},
        # a feature matrix of odd sizes in half precision: rows that start at any even address
        {"name": "quantize_odd", "op": "quantize", "rows": 777, "cols": 1111, "dtype": "f16"},
        # the weights of a large layer as training leaves them, on their way into storage
        {"name": "quantize_weights", "op": "quantize", "rows": 16384, "cols": 8192, "dtype": "f32"},
        # a classifier's fully connected layer (2048 -> 1000, as in the ResNet-50 shapes) on one image
        {"name": "linear_token", "op": "linear", "M": 1, "N": 1000, "K": 2048, "dtype": "bf16", "act": "none"},
        # one decoding step of a few requests through a wide layer: the weights' bytes count
        {"name": "linear_decode", "op": "linear", "M": 12, "N": 16384, "K": 8192, "dtype": "bf16", "act": "none"},
        # a pointwise layer of MobileNetV1 (512 -> 512 on 14x14, 31 images) as a product, odd in every direction
        {"name": "linear_odd", "op": "linear", "M": 6076, "N": 511, "K": 500, "dtype": "f32", "act": "relu6"},
        # a long prompt through a large square layer: the matrix instructions count
        {"name": "linear_prompt", "op": "linear", "M": 8192, "N": 8192, "K": 8192, "dtype": "bf16", "act": "relu"},
        # one token through the gated block: the two projections' bytes count
        {"name": "gated_token", "op": "gated", "T": 1, "D": 2048, "F": 8192, "dtype": "bf16", "gate": "silu",
         "bias": False},
        # a ragged batch of tokens in half precision
        {"name": "gated_odd", "op": "gated", "T": 333, "D": 1000, "F": 2730, "dtype": "f16", "gate": "gelu_tanh",
         "bias": True},
        # a long prompt through a large block
        {"name": "gated_prompt", "op": "gated", "T": 8192, "D": 4096, "F": 16384, "dtype": "bf16", "gate": "silu",
         "bias": False},
        # a small block trained in full precision, as the framework's other layers are
        {"name": "step_small", "op": "step", "T": 500, "D": 512, "F": 1365, "dtype": "f32", "gate": "gelu",
         "bias": True},
        # a training step over a batch of long sequences
        {"name": "step_large", "op": "step", "T": 8192, "D": 4096, "F": 8192, "dtype": "bf16", "gate": "silu",
         "bias": True},
    ]


def _log(rng, lo, hi):
    """A size between lo and hi, its logarithm evenly spread; every second one a multiple of 64 where
    that is possible, as sizes of layers mostly are."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    v = min(max(v, lo), hi)
    if rng.random() < 0.5 and v >= 64:
        v -= v % 64
    return v


def draw(rng):
    op = rng.choice(["quantize", "linear", "gated", "step"])
    while True:
        if op == "quantize":
            c = {"op": op, "rows": _log(rng, 1, 16384), "cols": _log(rng, 32, 16384),
                 "dtype": rng.choice(["f32", "bf16", "f16"])}
            if c["rows"] * c["cols"] <= 16384 * 8192:
                return c
        elif op == "linear":
            c = {"op": op, "M": _log(rng, 1, 8192), "N": _log(rng, 32, 16384), "K": _log(rng, 32, 16384),
                 "dtype": rng.choice(["f32", "bf16", "f16"]), "act": rng.choice(["none", "relu", "relu6"])}
            if c["M"] * c["N"] * c["K"] <= 8192 ** 3:
                return c
        else:
            c = {"op": op, "T": _log(rng, 1, 8192), "D": _log(rng, 64, 8192), "F": _log(rng, 64, 16384),
                 "dtype": rng.choice(["bf16", "bf16", "f16", "f32"]),
                 "gate": rng.choice(["silu", "gelu", "gelu_tanh", "relu", "sigmoid"]),
                 "bias": rng.random() < 0.5}
            work_limit = 8192 * 4096 * (16384 if op == "gated" else 8192)
            if c["dtype"] == "f32":
                work_limit //= 8
            if c["T"] * c["D"] * c["F"] <= work_limit:
                return c


def work(case):
    op, s = case["op"], SIZE[case["dtype"]]
    if op == "quantize":  # to storage and back
        n = case["rows"] * case["cols"]
        stored = case["rows"] * _padded(case["cols"]) * 17 / 32
        return {"bytes": 2 * n * s + 2 * stored, "flops": 2.0 * n}
    if op == "linear":  # the rows come in the wider type, the weights in storage
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": M * K * s + N * _padded(K) * 17 / 32 + 4 * N + M * N * s, "flops": 2.0 * M * N * K}
    T, D, F = case["T"], case["D"], case["F"]
    bias = 8 * F if case["bias"] else 0
    slopes = 2 * F * s if case["bias"] else 0
    if op == "gated":
        return {"bytes": (T * D + 2 * F * D + T * F) * s + bias, "flops": 4.0 * T * D * F}
    # inputs X, Wg, Wu, dH and the biases; outputs H and the gradients, those of the biases in X's type
    return {"bytes": (2 * T * D + 4 * F * D + 2 * T * F) * s + bias + slopes, "flops": 12.0 * T * D * F}


# ------------------------------------------------------------------------------- storage, plainly


def _padded(cols):
    return (cols + 127) // 128 * 128


def _quantize_plain(x):
    rows, cols = x.shape
    b = torch.nn.functional.pad(x.float(), (0, _padded(cols) - cols)).view(rows, -1, 32)
    top = b.abs().amax(-1)
    bad = ~torch.isfinite(top)
    top = torch.where(bad, torch.ones_like(top), top)
    _, e = torch.frexp(top.double())  # top = m * 2^e with m in [0.5, 1)
    e = torch.where(top == 0, torch.full_like(e, -127), (e - 3).clamp(min=-127))
    v = b * torch.exp2(-e.double()).float().unsqueeze(-1)
    a = v.abs()
    code = torch.zeros_like(a, dtype=torch.uint8)
    for border, up in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (a >= border) if up else (a > border)
    code += torch.signbit(v).to(torch.uint8) * 8
    code = torch.where(bad.unsqueeze(-1), torch.zeros_like(code), code).view(rows, -1, 2)
    scales = torch.where(bad, torch.full_like(e, 255), e + 127).to(torch.uint8)
    return code[..., 0] + code[..., 1] * 16, scales


def _values_plain(codes, scales):
    """What codes and scales stand for, padding included, in float32."""
    grid = torch.tensor(GRID + tuple(-g for g in GRID), device=codes.device)
    v = torch.stack((grid[(codes & 15).long()], grid[(codes >> 4).long()]), -1).view(codes.shape[0], -1, 32)
    s = torch.exp2(scales.double() - 127).float()
    s = torch.where(scales == 255, torch.full_like(s, float("nan")), s)
    return (v * s.unsqueeze(-1)).view(codes.shape[0], -1)


# ------------------------------------------------------------------------------- inputs


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=g, device="cuda") * std

    op = case["op"]
    if op == "quantize":
        # activations and weights alike: columns of different size, as features have them
        x = normal(case["rows"], case["cols"]) * torch.exp(normal(case["cols"]))
        return {"X": x.clamp(-3e4, 3e4).to(dt)}
    if op == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        return {"X": normal(M, K).to(dt), "W": normal(N, K, std=K ** -0.5), "b": normal(N, std=0.5)}
    T, D, F = case["T"], case["D"], case["F"]
    d = {"X": normal(T, D).to(dt), "Wg": normal(F, D, std=D ** -0.5).to(dt), "Wu": normal(F, D, std=D ** -0.5).to(dt),
         "bg": normal(F, std=0.5) if case["bias"] else None, "bu": normal(F, std=0.5) if case["bias"] else None}
    if op == "step":
        d["dH"] = normal(T, F).to(dt)
    return d


def prepare(case, seed):
    s = {"case": case, **_inputs(case, seed)}
    dt = DTYPES[case["dtype"]]
    op = case["op"]
    if op == "linear":  # a layer's weights are stored once
        s["Wc"], s["Ws"] = _quantize_plain(s.pop("W"))
    if not own:
        return s
    import paper_2109_00170_amd as alcs

    s["alcs"] = alcs

    def buffer(*shape, dtype=dt):
        return torch.empty(shape, dtype=dtype, device="cuda")

    def scratch(n):
        return buffer(max(int(n), 1), dtype=torch.uint8)

    if op == "quantize":
        rows, cols = case["rows"], case["cols"]
        s["codes"], s["scales"] = buffer(rows, _padded(cols) // 2, dtype=torch.uint8), buffer(rows, _padded(cols) // 32, dtype=torch.uint8)
        s["Y"] = buffer(rows, cols)
    elif op == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        s["Xc"], s["Xs"] = buffer(M, _padded(K) // 2, dtype=torch.uint8), buffer(M, _padded(K) // 32, dtype=torch.uint8)
        s["Y"] = buffer(M, N)
        s["ws"] = scratch(alcs.alcs_mx4_linear_workspace_bytes(M, N, _padded(K)))
    else:
        T, D, F = case["T"], case["D"], case["F"]
        s["H"] = buffer(T, F)
        s["ws"] = scratch(alcs.alcs_gated_ff_workspace_bytes(T, D, F, dt))
        if op == "step":
            s["G"], s["U"] = buffer(T, F), buffer(T, F)
            s["dX"], s["dWg"], s["dWu"] = buffer(T, D), buffer(F, D), buffer(F, D)
            s["dbg"] = s["dbu"] = None
            if case["bias"]:
                s["dbg"], s["dbu"] = buffer(F), buffer(F)
            s["wsb"] = scratch(alcs.alcs_gated_ff_backward_workspace_bytes(T, D, F, dt))
    return s


# ------------------------------------------------------------------------------- one pass


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    case, alcs = s["case"], s["alcs"]
    op = case["op"]
    if op == "quantize":
        alcs.alcs_mx4_quantize(s["X"], s["codes"], s["scales"])
        alcs.alcs_mx4_dequantize(s["codes"], s["scales"], s["Y"])
        return s["Y"]
    if op == "linear":
        alcs.alcs_mx4_quantize(s["X"], s["Xc"], s["Xs"])
        alcs.alcs_mx4_linear(s["Xc"], s["Xs"], s["Wc"], s["Ws"], s["b"], s["Y"], activation=case["act"], workspace=s["ws"])
        return s["Y"]
    if op == "gated":
        alcs.alcs_gated_ff(s["X"], s["Wg"], s["Wu"], s["bg"], s["bu"], s["H"], gate=case["gate"], workspace=s["ws"])
        return s["H"]
    alcs.alcs_gated_ff(s["X"], s["Wg"], s["Wu"], s["bg"], s["bu"], s["H"], gate=case["gate"], G=s["G"], U=s["U"],
                       workspace=s["ws"])
    alcs.alcs_gated_ff_backward(s["X"], s["Wg"], s["Wu"], s["G"], s["U"], s["dH"], s["dX"], s["dWg"], s["dWu"], s["dbg"],
                                s["dbu"], gate=case["gate"], workspace=s["wsb"])
    out = [s["H"], s["dX"], s["dWg"], s["dWu"]]
    return out + [s["dbg"], s["dbu"]] if case["bias"] else out


def _gate(kind, g, slope):
    """The gate's value at g and, where asked for, its derivative."""
    if kind == "relu":
        return torch.relu(g), (g > 0).to(g.dtype) if slope else None
    if kind == "silu":
        p = torch.sigmoid(g)
        return g * p, p * (1 + g * (1 - p)) if slope else None
    if kind == "sigmoid":
        p = torch.sigmoid(g)
        return p, p * (1 - p) if slope else None
    if kind == "gelu":
        c = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * c, c + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi)) if slope else None
    a = math.sqrt(2 / math.pi)
    t = torch.tanh(a * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * a * (1 + 3 * 0.044715 * g * g) if slope else None


def _run_plain(s):
    case = s["case"]
    op, dt = case["op"], DTYPES[case["dtype"]]
    if op == "quantize":
        codes, scales = _quantize_plain(s["X"])
        return _values_plain(codes, scales)[:, : case["cols"]].to(dt)
    if op == "linear":
        y = _values_plain(*_quantize_plain(s["X"])) @ _values_plain(s["Wc"], s["Ws"]).t() + s["b"]
        if case["act"] != "none":
            y = y.clamp(0, 6) if case["act"] == "relu6" else y.clamp(min=0)
        return y.to(dt)
    X, Wg, Wu = s["X"].float(), s["Wg"].float(), s["Wu"].float()
    G, U = X @ Wg.t(), X @ Wu.t()
    if case["bias"]:
        G, U = G + s["bg"], U + s["bu"]
    a, slope = _gate(case["gate"], G, op == "step")
    H = (a * U).to(dt)
    if op == "gated":
        return H
    dH = s["dH"].float()
    dU, dG = dH * a, dH * U * slope
    out = [H, (dG @ Wg + dU @ Wu).to(dt), (dG.t() @ X).to(dt), (dU.t() @ X).to(dt)]
    return out + [dG.sum(0).to(dt), dU.sum(0).to(dt)] if case["bias"] else out


# ------------------------------------------------------------------------------- the definition in 64 bits


def _stored64(x):
    """The values that the 4-bit storage of x [rows, cols] stands for, in float64, by distance to the grid."""
    rows, cols = x.shape
    out = torch.empty(rows, cols, dtype=torch.float64, device=x.device)
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    step = max(1, (1 << 21) // cols)
    for r in range(0, rows, step):
        part = x[r:r + step].double()
        n = part.shape[0]
        p = torch.zeros(n, _padded(cols), dtype=torch.float64, device=x.device)
        p[:, :cols] = part
        p = p.view(n, -1, 32)
        top = p.abs().amax(-1, keepdim=True)
        e = torch.floor(torch.log2(top))
        e = torch.where(torch.exp2(e) > top, e - 1, e)  # a logarithm rounded up to the next whole number
        e = torch.where(torch.exp2(e + 1) <= top, e + 1, e)
        unit = torch.exp2((e - 2).clamp(min=-127))
        far = (p.abs() / unit).unsqueeze(-1).sub(grid).abs()
        # the nearest, and of two equally near ones that of even position
        order = far * 2 + (torch.arange(8, device=x.device) % 2) * 1e-12
        v = grid[order.argmin(-1)] * unit * torch.sign(p)
        v = torch.where(torch.isfinite(top), v, torch.full_like(v, float("nan")))
        out[r:r + step] = v.view(n, -1)[:, :cols]
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "quantize":
        return _stored64(s["X"])
    if op == "linear":
        y = torch.matmul(_stored64(s["X"]), _stored64(s["W"]).t().contiguous()).add_(s["b"].double())
        if case["act"] == "none":
            return y
        y = torch.where(y < 0, torch.zeros_like(y), y)
        return torch.where(y > 6, torch.full_like(y, 6.0), y) if case["act"] == "relu6" else y
    X, Wg, Wu = s["X"].double(), s["Wg"].double(), s["Wu"].double()
    G = torch.matmul(X, Wg.t().contiguous())
    U = torch.matmul(X, Wu.t().contiguous())
    if case["bias"]:
        G, U = G.add_(s["bg"].double()), U.add_(s["bu"].double())
    kind = case["gate"]
    if op == "step":
        G.requires_grad_(True)
    if kind == "silu":
        a = G / (1 + torch.exp(-G))
    elif kind == "sigmoid":
        a = 1 / (1 + torch.exp(-G))
    elif kind == "relu":
        a = torch.where(G > 0, G, torch.zeros_like(G))
    elif kind == "gelu":
        a = G * torch.special.ndtr(G)
    else:  # 0.5 (1 + tanh z) = 1 / (1 + exp(-2z))
        a = G / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (G + 0.044715 * G ** 3)))
    H = (a * U).detach()
    if op == "gated":
        return H
    dH = s["dH"].double()
    dU = dH * a.detach()
    (dG,) = torch.autograd.grad(a, G, dH * U)
    out = [H, torch.matmul(dG, Wg).add_(torch.matmul(dU, Wu)), torch.matmul(dG.t().contiguous(), X),
           torch.matmul(dU.t().contiguous(), X)]
    return out + [dG.sum(0), dU.sum(0)] if case["bias"] else out
