"""The 256 x 256 tiles of the feed-forward products (k_big), in all their forms: each case asks the library's rule whether
they are what it runs.  Ragged rows, columns and ends of K, odd and even numbers of K tiles, one tile a workgroup and
two, dX's second segment.  Operands are small whole numbers, so that float32 sums are exact in any order and a result has one
right value; the functions behind the sums are compared at random values."""
import pytest
import torch

import paper_2109_00170_amd as alcs
from ff_util import GATES, guarded, product, stored64
from test_gpu_gated_ff import operands, run_backward, run_forward, scratch
from tile_plan import backward_plan, forward_plan, linear_plan

pytestmark = pytest.mark.gpu
HALVES = [torch.bfloat16, torch.float16]
TYPES = [torch.float32] + HALVES

# rows, columns of the result (of each projection), K
FORWARD = [(2041, 4090, 584), (2041, 4090, 645), (4093, 4090, 581), (3100, 4090, 1240)]
LINEAR = [(4093, 4091, 1100), (4096, 4090, 1500), (5900, 5110, 1408)]
DX = [(4093, 4083, 270), (4090, 4088, 330), (8190, 4083, 270)]       # T, D, F
DW = [(701, 2035, 4090), (760, 2040, 4085), (700, 4083, 4090)]


def units():
    return torch.cuda.get_device_properties(torch.cuda.current_device()).multi_processor_count


def small(rows, cols, seed, dtype):
    """-1, 0 and 1 (half of them 0)."""
    v = torch.randint(0, 4, (rows, cols), generator=torch.Generator().manual_seed(seed))
    return ((v == 1).float() - (v == 2).float()).to(dtype).cuda()


def equal(got, ref, what):
    want = ref.float().to(got.dtype)
    bad = got != want
    assert not bool(bad.any()), "%s: %d of %d, first at %s" % (what, int(bad.sum()), bad.numel(), bad.nonzero()[0].tolist())


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("T,F,D", FORWARD)
def test_forward(T, F, D, dtype):
    assert forward_plan(T, D, F, dtype, cus=units()).kind == "256"
    X, Wg, Wu = small(T, D, 1, dtype), small(F, D, 2, dtype), small(F, D, 3, dtype)
    (H, i1), (G, i2), (U, i3) = (guarded(T, F, dtype=dtype) for _ in range(3))
    ws = scratch(alcs.alcs_gated_ff_workspace_bytes(T, D, F, dtype))
    alcs.alcs_gated_ff(X, Wg, Wu, None, None, H, gate="none", G=G, U=U, workspace=ws)
    g, u = product(X.double(), Wg.double()), product(X.double(), Wu.double())
    assert float(g.abs().max()) ** 2 < 2 ** 24
    equal(G, g, "G")
    equal(U, u, "U")
    equal(H, g * u, "H")
    assert i1() and i2() and i3()


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("kind", GATES)
def test_forward_gates(kind, dtype):
    T, F, D = FORWARD[0]
    X, Wg, Wu, bg, bu = operands(T, D, F, dtype, 4)
    run_forward(X, Wg, Wu, bg, bu, kind, kind in ("silu", "gelu"), None, kind)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,cols", LINEAR)
def test_product(M, N, cols, dtype):
    K = (cols + 127) // 128 * 128
    assert linear_plan(M, N, K, cus=units()).kind == "256"
    gen = torch.Generator().manual_seed(M)

    def stored(rows):  # any code, units of 1/2, 1 and 2; padding as alcs_mx4_quantize leaves it
        c = torch.randint(0, 256, (rows, K // 2), generator=gen).to(torch.uint8)
        c[:, cols // 2:] = 0
        return c.cuda(), torch.randint(126, 129, (rows, K // 32), generator=gen).to(torch.uint8).cuda()

    (xc, xs), (wc, ws) = stored(M), stored(N)
    bias = torch.randint(-40, 41, (N,), generator=gen).float().cuda()
    ref = product(stored64(xc, xs), stored64(wc, ws)) + bias.double()
    for act in ("none", "relu6"):
        Y, intact = guarded(M, N, dtype=dtype)
        alcs.alcs_mx4_linear(xc, xs, wc, ws, bias, Y, activation=act)
        equal(Y, ref if act == "none" else ref.clamp(0, 6), act)
        assert intact()


def gradients(T, D, F, dtype, dX, dW):
    """What alcs_gated_ff_backward gives for the gate "none" (dU = dH G, dG = dH U, again -1, 0 and 1)."""
    X, Wg, Wu = small(T, D, 1, dtype), small(F, D, 2, dtype), small(F, D, 3, dtype)
    G, U, dH = (small(T, F, i, dtype) for i in (4, 5, 6))
    outs = [guarded(*s, dtype=dtype) if want else (None, None) for s, want in (((T, D), dX), ((F, D), dW), ((F, D), dW), ((F,), True), ((F,), True))]
    alcs.alcs_gated_ff_backward(X, Wg, Wu, G, U, dH, *(o for o, _ in outs), gate="none",
                                workspace=scratch(alcs.alcs_gated_ff_backward_workspace_bytes(T, D, F, dtype)))
    X, Wg, Wu, G, U, dH = (t.double() for t in (X, Wg, Wu, G, U, dH))
    dG, dU = dH * U, dH * G
    if dX:
        equal(outs[0][0], torch.matmul(dG, Wg) + torch.matmul(dU, Wu), "dX")
    if dW:
        equal(outs[1][0], torch.matmul(dG.t().contiguous(), X), "dWg")
        equal(outs[2][0], torch.matmul(dU.t().contiguous(), X), "dWu")
    equal(outs[3][0], dG.sum(0), "dbg")
    equal(outs[4][0], dU.sum(0), "dbu")
    assert all(o is None or intact() for o, intact in outs)


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("T,D,F", DX)
def test_gradient_of_the_input(T, D, F, dtype):
    assert backward_plan(T, D, F, dtype, cus=units()).dX_alone.kind == "256"
    gradients(T, D, F, dtype, True, False)


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("T,D,F", DW)
def test_gradients_of_the_weights(T, D, F, dtype):
    assert backward_plan(T, D, F, dtype, cus=units()).dW_alone.kind == "256"
    gradients(T, D, F, dtype, False, True)


@pytest.mark.parametrize("T,D,F", [(3070, 4083, 4091)])
def test_all_gradients(T, D, F):
    plan = backward_plan(T, D, F, torch.bfloat16, cus=units())
    assert not plan.together and plan.dX.kind == plan.dW.kind == "256"
    gradients(T, D, F, torch.bfloat16, True, True)
    run_backward(T, D, F, torch.bfloat16, "silu", 3, "random values")
