"""Feed-forward layers where offsets pass 32 bits, workspaces hold anything, and numbers are subnormal."""
import pytest
import torch

import paper_2109_00170_amd as alcs
from test_gpu_gated_ff import scratch
from test_gpu_large_tiles import HALVES, TYPES, equal, small

pytestmark = pytest.mark.gpu


def matmul32(a, b):
    """Of small whole numbers: exact in float32 too."""
    return torch.matmul(a.float(), b.float())


def test_results_of_more_than_2_to_32_elements():
    T, D, F = 70000, 8, 65544
    dtype = torch.bfloat16
    X, Wg, Wu = small(T, D, 1, dtype), small(F, D, 2, dtype), small(F, D, 3, dtype)
    H = torch.empty(T, F, dtype=dtype, device="cuda")
    alcs.alcs_gated_ff(X, Wg, Wu, None, None, H, gate="none")
    wg, wu = Wg.t().contiguous(), Wu.t().contiguous()
    for r in range(0, T, 5000):
        equal(H[r:r + 5000], matmul32(X[r:r + 5000], wg) * matmul32(X[r:r + 5000], wu), "rows from %d on" % r)
    # the same tensor through storage and back: blocks of whole numbers up to 6 in size lose nothing
    H.clamp_(-2, 2)
    c, s = alcs.alcs_mx4_quantize(H)
    Y = torch.empty_like(H)
    alcs.alcs_mx4_dequantize(c, s, Y)
    assert all(torch.equal(Y[r:r + 5000], H[r:r + 5000]) for r in range(0, T, 5000))


def test_product_of_more_than_2_to_32_elements():
    M, N = 70000, 65541
    x, w = small(M, 100, 1, torch.bfloat16), small(N, 100, 2, torch.bfloat16)
    (xc, xs), (wc, ws) = alcs.alcs_mx4_quantize(x), alcs.alcs_mx4_quantize(w)
    Y = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    alcs.alcs_mx4_linear(xc, xs, wc, ws, None, Y)
    w = w.t().contiguous()
    for r in range(0, M, 5000):
        equal(Y[r:r + 5000], matmul32(x[r:r + 5000], w), "rows from %d on" % r)


def test_gradients_over_more_than_2_to_32_elements():
    T, D, F = 70000, 8, 65541
    dtype = torch.bfloat16
    X, Wg, Wu = small(T, D, 1, dtype), small(F, D, 2, dtype), small(F, D, 3, dtype)
    gen = torch.Generator(device="cuda").manual_seed(4)
    G, U, dH = (torch.randint(-1, 2, (T, F), generator=gen, device="cuda", dtype=torch.int8).to(dtype) for _ in range(3))
    dX, dWg, dWu = torch.empty_like(X), torch.empty_like(Wg), torch.empty_like(Wu)
    dbg, dbu = (torch.empty(F, dtype=dtype, device="cuda") for _ in range(2))
    alcs.alcs_gated_ff_backward(X, Wg, Wu, G, U, dH, dX, dWg, dWu, dbg, dbu, gate="none",
                                workspace=scratch(alcs.alcs_gated_ff_backward_workspace_bytes(T, D, F, dtype)))
    sums = [torch.zeros(F, D, device="cuda"), torch.zeros(F, D, device="cuda"), torch.zeros(F, device="cuda"), torch.zeros(F, device="cuda")]
    for r in range(0, T, 5000):
        at = slice(r, r + 5000)
        dG, dU, x = (dH[at] * U[at]).float(), (dH[at] * G[at]).float(), X[at].float()
        equal(dX[at], matmul32(dG, Wg) + matmul32(dU, Wu), "dX, rows from %d on" % r)
        for s, v in zip(sums, (torch.matmul(dG.t().contiguous(), x), torch.matmul(dU.t().contiguous(), x), dG.sum(0), dU.sum(0))):
            s += v
    for got, want, what in zip((dWg, dWu, dbg, dbu), sums, ("dWg", "dWu", "dbg", "dbu")):
        equal(got, want, what)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,D,F", [(40, 33, 21), (100, 2051, 43), (300, 520, 136), (500, 1000, 70)])
def test_workspaces_that_hold_anything(T, D, F, dtype):
    # (255: NaN in every type)
    X, Wg, Wu = small(T, D, 1, dtype), small(F, D, 2, dtype), small(F, D, 3, dtype)
    G, U, dH = (small(T, F, i, dtype) for i in (4, 5, 6))
    res = []
    for fill in (0, 255):
        H = torch.empty(T, F, dtype=dtype, device="cuda")
        grads = [torch.empty(*s, dtype=dtype, device="cuda") for s in ((T, D), (F, D), (F, D), (F,), (F,))]
        ws = scratch(alcs.alcs_gated_ff_workspace_bytes(T, D, F, dtype)).fill_(fill)
        alcs.alcs_gated_ff(X, Wg, Wu, None, None, H, gate="none", workspace=ws)
        ws = scratch(alcs.alcs_gated_ff_backward_workspace_bytes(T, D, F, dtype)).fill_(fill)
        alcs.alcs_gated_ff_backward(X, Wg, Wu, G, U, dH, *grads, gate="none", workspace=ws)
        (xc, xs), (wc, wsc) = alcs.alcs_mx4_quantize(X), alcs.alcs_mx4_quantize(Wg)
        Y = torch.empty(T, F, dtype=dtype, device="cuda")
        ws = scratch(alcs.alcs_mx4_linear_workspace_bytes(T, F, 2 * xc.shape[1])).fill_(fill)
        alcs.alcs_mx4_linear(xc, xs, wc, wsc, None, Y, workspace=ws)
        res.append([H, *grads, Y])
    equal(res[0][0], matmul32(X, Wg.t().contiguous()) * matmul32(X, Wu.t().contiguous()), "H")
    equal(res[0][6], matmul32(X, Wg.t().contiguous()), "Y")
    assert all(torch.equal(a, b) for a, b in zip(*res))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [5, 100, 3000])
def test_subnormal_numbers(T, dtype):
    # one factor's smallest numbers, times 1: the sums and the results keep them
    D, F = 640, 4096 if T == 3000 else 24
    tiny = torch.finfo(dtype).tiny
    step = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}[dtype]
    X = torch.zeros(T, D, dtype=torch.float64)
    X[:, 3] = torch.arange(T) % 100 * step
    X[0, 3], X[1, 3] = tiny, -tiny / 2
    X = X.to(dtype).cuda()
    Wg = torch.zeros(F, D, dtype=dtype, device="cuda")
    Wg[:, 3] = 1
    Wu = Wg.clone()
    H, G, U = (torch.empty(T, F, dtype=dtype, device="cuda") for _ in range(3))
    alcs.alcs_gated_ff(X, Wg, Wu, None, torch.ones(F, device="cuda"), H, gate="none", G=G, U=U)
    assert torch.equal(G, X[:, 3:4].expand(T, F).contiguous())
    assert torch.equal(H, G)     # times 1 + a number far below half a step of 1
