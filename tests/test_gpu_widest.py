"""The feed-forward operators at their widest, on whole numbers: float32 sums of a million terms are exact in any order, so that
every result has one right value and a K tile that is left out, or read from elsewhere, shows."""
import pytest
import torch

import paper_2109_00170_amd as alcs
from ff_util import guarded, product, stored64
from test_gpu_gated_ff import scratch
from test_gpu_large_tiles import TYPES, equal, gradients, small

pytestmark = pytest.mark.gpu
WIDE = [(70, 2 ** 20, 3), (70, 2 ** 20 - 1, 3), (5, 2 ** 20, 8), (70, 3, 2 ** 20), (70, 8, 2 ** 20 - 3), (3, 5, 2 ** 20)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,D,F", WIDE)
def test_forward(T, D, F, dtype):
    X, Wg, Wu = small(T, D, 1, dtype), small(F, D, 2, dtype), small(F, D, 3, dtype)
    g, u = product(X.double(), Wg.double()), product(X.double(), Wu.double())
    assert float(g.abs().max()) ** 2 < 2 ** 24 and float(u.abs().max()) ** 2 < 2 ** 24
    if D > 64:  # the last 64 columns can be seen in the result
        less = product(X[:, :-64].double(), Wg[:, :-64].double())
        assert not torch.equal(less.to(dtype), g.to(dtype))
    for room in (0, alcs.alcs_gated_ff_workspace_bytes(T, D, F, dtype)):
        (H, i1), (G, i2), (U, i3) = (guarded(T, F, dtype=dtype) for _ in range(3))
        alcs.alcs_gated_ff(X, Wg, Wu, None, None, H, gate="none", G=G, U=U, workspace=scratch(room) if room else None)
        equal(G, g, "G")
        equal(U, u, "U")
        equal(H, g * u, "H")
        assert i1() and i2() and i3()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,D,F", WIDE)
def test_gradients(T, D, F, dtype):
    gradients(T, D, F, dtype, True, True)


@pytest.mark.parametrize("M,N", [(3, 5), (70, 130)])
def test_product(M, N):
    K = 2 ** 23
    gen = torch.Generator().manual_seed(M)

    def stored(rows):  # -1, 0 and 1
        c = torch.tensor([0, 0, 2, 10], dtype=torch.uint8)[torch.randint(0, 4, (rows, K), generator=gen)].view(rows, K // 2, 2)
        return (c[..., 0] + 16 * c[..., 1]).cuda(), torch.full((rows, K // 32), 127, dtype=torch.uint8, device="cuda")

    (xc, xs), (wc, ws) = stored(M), stored(N)
    ref = torch.zeros(M, N, dtype=torch.float64, device="cuda")
    step = 2 ** 19
    for k in range(0, K, step):
        part = [t[:, k // n:(k + step) // n].contiguous() for t, n in ((xc, 2), (xs, 32), (wc, 2), (ws, 32))]
        last = product(stored64(*part[:2]), stored64(*part[2:]))
        ref += last
    assert not torch.equal((ref - last).float(), ref.float())
    for room in (0, alcs.alcs_mx4_linear_workspace_bytes(M, N, K)):
        Y, intact = guarded(M, N, dtype=torch.float32)
        alcs.alcs_mx4_linear(xc, xs, wc, ws, None, Y, workspace=scratch(room) if room else None)
        equal(Y, ref, "product")
        assert intact()


@pytest.mark.parametrize("dtype", TYPES)
def test_storage(dtype):
    # one row of 2^26 columns, and the same blocks as rows of 1024
    x = torch.randn(1, 2 ** 26, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)).to(dtype)
    c, s = alcs.alcs_mx4_quantize(x)
    c2, s2 = alcs.alcs_mx4_quantize(x.view(2 ** 16, 1024))
    assert torch.equal(c.view(-1), c2.view(-1)) and torch.equal(s.view(-1), s2.view(-1))
    y, y2 = torch.empty_like(x), torch.empty_like(x).view(2 ** 16, 1024)
    alcs.alcs_mx4_dequantize(c, s, y)
    alcs.alcs_mx4_dequantize(c2, s2, y2)
    assert torch.equal(y.view(-1), y2.view(-1)) and float(y.abs().max()) > 4
