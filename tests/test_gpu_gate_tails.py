"""Gates and their slopes where they are small: relative to their own size, since what they are multiplied with may be large.

Bounds, in relative terms.  An argument x that is off by a share d moves exp(x) by |x| d, and erfc(x) by at most
(2 x^2 + 1) d (its logarithm's derivative is at most x + sqrt(x^2 + 2) in size).  Steps of float32 are 2^-24 of the value;
functions of the library are off by at most 4 units in the last place (2^-21), the hardware's exp2 and reciprocal by 1."""
import math

import pytest
import torch

import paper_2109_00170_amd as alcs
from ff_util import check
from test_gpu_gated_ff import scratch

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
STEP = 2.0 ** -24


def sigmoid64(g):
    return torch.sigmoid(g)      # 1 / (1 + exp(-g)): no cancellation


def value64(kind, g):
    """(value, bound)"""
    if kind == "gelu":           # x = g / sqrt 2, its constant and its product rounded; erfc; two products
        v = 0.5 * g * torch.special.erfc(-g * math.sqrt(0.5))
        return v, v.abs() * ((g * g + 1) * 2 * STEP + 2.0 ** -20)
    if kind == "gelu_tanh":      # the argument: at most eight roundings
        z = 2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)
        v = g * sigmoid64(z)
        return v, v.abs() * (z.abs() * 10 * STEP + 2.0 ** -20)
    s = sigmoid64(g)
    v = g * s if kind == "silu" else s
    return v, v.abs() * (g.abs() * 3 * STEP + 2.0 ** -20)


def slope64(kind, g):
    if kind == "sigmoid":        # s (1 - s), both as above
        d = sigmoid64(g) * sigmoid64(-g)
        return d, d * (g.abs() * 6 * STEP + 2.0 ** -19)
    c = 0.5 * torch.special.erfc(-g * math.sqrt(0.5))
    p = g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    return c + p, c * ((g * g + 1) * 2 * STEP + 2.0 ** -20) + p.abs() * ((g * g + 1) * 2 * STEP + 2.0 ** -20)


@pytest.mark.parametrize("T", [33, 900])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh", "sigmoid"])
def test_values(kind, dtype, T):
    # G = g and U = a power of two, both exactly
    far = {"gelu": -12.0, "gelu_tanh": -9.0}.get(kind, -80.0)
    g = torch.linspace(far, 1.0, T).to(dtype).cuda()
    top = 2.0 ** (10 if dtype == torch.float16 else 40)
    X = torch.stack([g, torch.ones_like(g)], 1).contiguous()
    Wg = torch.tensor([[1.0, 0.0]] * 3, dtype=dtype, device="cuda")
    Wu = torch.tensor([[0.0, top]] * 3, dtype=dtype, device="cuda")
    H = torch.empty(T, 3, dtype=dtype, device="cuda")
    alcs.alcs_gated_ff(X, Wg, Wu, None, None, H, gate=kind)
    v, tol = value64(kind, g.double())
    for k in range(3):
        check(H[:, k], v * top, tol * top, "%s of %s" % (kind, dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["gelu", "sigmoid"])
def test_slopes(kind, dtype):
    # one row and one column, so that dWg is dG = dH U gate'(G) and dWu is dU = dH gate(G)
    F = 501
    far = 12.0 if kind == "gelu" else 80.0
    g = torch.linspace(-far, 1.0 if kind == "gelu" else far, F).to(dtype).cuda()
    top = 2.0 ** (10 if dtype == torch.float16 else 40)
    one = torch.ones(F, 1, dtype=dtype, device="cuda")
    U, dH = torch.ones(1, F, dtype=dtype, device="cuda"), torch.full((1, F), top, dtype=dtype, device="cuda")
    dWg, dWu = torch.empty_like(one), torch.empty_like(one)
    dbg, dbu = (torch.empty(F, dtype=dtype, device="cuda") for _ in range(2))
    alcs.alcs_gated_ff_backward(one[:1], one, one, g.view(1, F), U, dH, None, dWg, dWu, dbg, dbu, gate=kind,
                                workspace=scratch(alcs.alcs_gated_ff_backward_workspace_bytes(1, 1, F, dtype)))
    (v, tv), (d, td) = value64(kind, g.double()), slope64(kind, g.double())
    for got, ref, tol, what in ((dWg, d, td, "dWg"), (dbg, d, td, "dbg"), (dWu, v, tv, "dWu"), (dbu, v, tv, "dbu")):
        check(got.view(-1), ref * top, (tol + 2 * STEP * ref.abs()) * top, "%s %s of %s" % (what, kind, dtype))
