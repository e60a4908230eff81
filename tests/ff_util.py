"""Plain forms of the feed-forward operators in float64, and how far a result in fewer bits may lie away.

Half a step of a type is finfo.eps / 2 relative to the value; a float32 sum of n products of absolute value
at most S in total is off by at most n * 2^-23 * S (each addition by half a step of a partial sum, doubled for
matrix instructions that cut rather than round)."""
import math

import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
GATES = ["none", "relu", "silu", "gelu", "gelu_tanh", "sigmoid"]


def gate64(kind, g):
    if kind == "none":
        return g.clone()
    if kind == "relu":
        return g.clamp(min=0)
    if kind == "silu":
        return g * torch.sigmoid(g)
    if kind == "sigmoid":
        return torch.sigmoid(g)
    if kind == "gelu":
        return 0.5 * g * (1 + torch.erf(g * math.sqrt(0.5)))
    return 0.5 * g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))


def slope64(kind, g):
    g = g.detach().clone().requires_grad_(True)
    (d,) = torch.autograd.grad(gate64(kind, g).sum(), g)
    return d


def product(a, b):
    """a b^T in float64 of contiguous operands."""
    return torch.matmul(a, b.t().contiguous())


def gated_ref(X, Wg, Wu, bg, bu, kind):
    """(H, G, U) and their tolerances before rounding to the outputs' type."""
    X, Wg, Wu = X.double(), Wg.double(), Wu.double()
    D = X.shape[1]
    out = []
    for W, b in ((Wg, bg), (Wu, bu)):
        v, s = product(X, W), product(X.abs(), W.abs())
        if b is not None:
            v, s = v + b.double(), s + b.double().abs()
        out.append((v, (D + 2) * 2.0 ** -23 * s))
    (G, eg), (U, eu) = out
    a = gate64(kind, G)
    # no gate is steeper than 1.13; exponential, reciprocal and erf: 2^-20 of the argument, or of a unit result
    ea = 1.13 * eg + 2.0 ** -20 * (G.abs() + a.abs())
    return (a * U, G, U), (ea * U.abs() + (a.abs() + ea) * eu, eg, eu)


def backward_ref(X, Wg, Wu, G, U, dH, kind):
    """(dX, dWg, dWu, dbg, dbu) from stored G and U, and their tolerances before rounding to the outputs' type."""
    half = HALF[X.dtype]
    X, Wg, Wu, G, U, dH = (t.double() for t in (X, Wg, Wu, G, U, dH))
    T, F = G.shape
    a, d = gate64(kind, G), slope64(kind, G)
    dU, dG = dH * a, dH * U * d
    # the functions as above (a derivative is a sum of terms up to |G| / 2), three float32 products, then rounding
    # to the operands' type
    eu = dH.abs() * 2.0 ** -20 * (G.abs() + a.abs()) + (half + 2.0 ** -22) * dU.abs()
    eg = (dH * U).abs() * 2.0 ** -20 * (1 + G.abs() + d.abs()) + (half + 2.0 ** -22) * dG.abs()

    def mm(p, q):
        return torch.matmul(p.contiguous(), q.contiguous())

    dX = mm(dG, Wg) + mm(dU, Wu)
    sX = mm(dG.abs() + eg, Wg.abs()) + mm(dU.abs() + eu, Wu.abs())
    tX = mm(eg, Wg.abs()) + mm(eu, Wu.abs()) + (2 * F + 2) * 2.0 ** -23 * sX
    res, tol = [dX], [tX]
    for v, e in ((dG, eg), (dU, eu)):
        res.append(mm(v.t(), X))
        tol.append(mm(e.t(), X.abs()) + (T + 2) * 2.0 ** -23 * mm(v.abs().t() + e.t(), X.abs()))
    for v, e in ((dG, eg), (dU, eu)):
        res.append(v.sum(0))
        tol.append(e.sum(0) + (T + 2) * 2.0 ** -23 * (v.abs() + e).sum(0))
    return res, tol


def check(got, ref, tol, what):
    """Every element within tol of ref, plus the rounding to got's type (half a step, of the smallest normal
    number at least)."""
    half = HALF[got.dtype]
    tiny = torch.finfo(got.dtype).tiny
    bound = tol + half * (ref.abs() + tol).clamp(min=tiny)
    err = (got.double() - ref).abs()
    bad = ~(err <= bound)
    assert not bad.any(), "%s: %d of %d outside, worst ratio %.3g, at %s" % (
        what, int(bad.sum()), bad.numel(), float((err / bound).nan_to_num(nan=1e30).max()), bad.nonzero()[0].tolist())


# ------------------------------------------------------------------------------- 4-bit storage


def padded(cols):
    return (cols + 127) // 128 * 128


def quantize_ref(x):
    """(codes, scales) of x [rows, cols] on the CPU, from the definition: distances to the grid in float64."""
    rows, cols = x.shape
    p = torch.zeros(rows, padded(cols), dtype=torch.float64)
    p[:, :cols] = x.double().cpu()
    p = p.view(rows, padded(cols) // 32, 32)
    top = p.abs().amax(-1)
    bad = ~torch.isfinite(top)
    e = torch.tensor([[math.frexp(v)[1] - 1 if 0 < v < math.inf else -1000 for v in row] for row in top.tolist()],
                     dtype=torch.float64).view(top.shape)
    e = (e - 2).clamp(min=-127)
    unit = torch.exp2(e).unsqueeze(-1)
    far = (p.abs() / unit).unsqueeze(-1).sub(GRID).abs()
    code = (far * 2 + (torch.arange(8) % 2) * 1e-12).argmin(-1)
    code = code + 8 * torch.signbit(p)
    code = torch.where(bad.unsqueeze(-1), torch.zeros_like(code), code).view(rows, padded(cols) // 2, 2)
    scales = torch.where(bad, torch.full_like(e, 255.0), e + 127)
    return (code[..., 0] + 16 * code[..., 1]).to(torch.uint8), scales.to(torch.uint8)


def stored64(codes, scales):
    """What codes and scales stand for, padding included, in float64."""
    grid = torch.cat([GRID, -GRID]).to(codes.device)
    v = torch.stack([grid[(codes & 15).long()], grid[(codes >> 4).long()]], -1).view(codes.shape[0], -1, 32)
    s = torch.exp2(scales.double() - 127)
    s = torch.where(scales == 255, torch.full_like(s, math.nan), s)
    return (v * s.unsqueeze(-1)).view(codes.shape[0], -1)


def linear_ref(xc, xs, wc, ws, bias, act):
    """(Y, tolerance) of the product of two stored matrices."""
    X, W = stored64(xc, xs), stored64(wc, ws)
    y, s = product(X, W), product(X.abs(), W.abs())
    if bias is not None:
        y, s = y + bias.double(), s + bias.double().abs()
    tol = (X.shape[1] + 2) * 2.0 ** -23 * s
    if act in ("relu", "relu6"):
        y = torch.where(y > 0, y, torch.zeros_like(y))   # NaN gives 0
        tol = tol.nan_to_num(nan=0.0)
    return (y.clamp(max=6) if act == "relu6" else y), tol


def guarded(*shape, dtype):
    """An output tensor inside a larger one whose other elements are checked by .intact()."""
    n = math.prod(shape)
    whole = torch.full((n + 512,), -77.0 if dtype.is_floating_point else 77, dtype=dtype, device="cuda")
    t = whole[256:256 + n].view(shape)
    return t, lambda: bool((whole[:256] == whole[0]).all() and (whole[256 + n:] == whole[0]).all() and abs(float(whole[0])) == 77)
