"""The gated feed-forward block and its gradients against float64, element by element with derived bounds."""
import pytest
import torch

import paper_2109_00170_amd as alcs
from ff_util import GATES, backward_ref, check, gate64, gated_ref, guarded

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def normal(*shape, seed, std=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype).cuda()


def scratch(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def operands(T, D, F, dtype, seed, bias=True):
    X = normal(T, D, seed=seed, dtype=dtype)
    Wg, Wu = (normal(F, D, seed=seed + i, std=D ** -0.5, dtype=dtype) for i in (1, 2))
    bg, bu = (normal(F, seed=seed + i, std=0.5) if bias else None for i in (3, 4))
    return X, Wg, Wu, bg, bu


def run_forward(X, Wg, Wu, bg, bu, kind, keep, ws, what):
    T, F = X.shape[0], Wg.shape[0]
    (H, i1), (G, i2), (U, i3) = (guarded(T, F, dtype=X.dtype) for _ in range(3))
    alcs.alcs_gated_ff(X, Wg, Wu, bg, bu, H, gate=kind, G=G if keep else None, U=U if keep else None, workspace=ws)
    ref, tol = gated_ref(X, Wg, Wu, bg, bu, kind)
    check(H, ref[0], tol[0], what + " H")
    if keep:
        check(G, ref[1], tol[1], what + " G")
        check(U, ref[2], tol[2], what + " U")
    assert i1() and i2() and i3()
    return H


# the forms for few rows and their borders, tiles of 64 and 128 rows (K shared out where a workspace is given; several tiles to a
# compute unit); sizes that are whole 16-byte pieces and sizes that are not
FORWARD = [(1, 1, 1), (1, 64, 64), (1, 8200, 24), (2, 9, 17), (16, 128, 40), (17, 131, 33), (33, 64, 66), (64, 520, 48),
           (65, 96, 70), (70, 31, 9), (100, 4104, 24), (100, 4101, 23), (129, 200, 257), (300, 1000, 520), (2048, 72, 2048),
           (2100, 136, 2052), (4097, 72, 4100)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("i", range(len(FORWARD)))
def test_forward(i, dtype):
    T, D, F = FORWARD[i]
    kind = GATES[(i + TYPES.index(dtype)) % 6]
    X, Wg, Wu, bg, bu = operands(T, D, F, dtype, 10 * i, bias=i % 3 != 1)
    for keep, ws in ((False, None), (True, scratch(alcs.alcs_gated_ff_workspace_bytes(T, D, F, dtype)))):
        run_forward(X, Wg, Wu, bg, bu, kind, keep, ws, "%s %s %s" % (FORWARD[i], dtype, kind))


@pytest.mark.parametrize("T,D,F", [(100, 2056, 16380), (128, 2111, 16300), (256, 4096, 8192)])
def test_forward_deep(T, D, F):
    # one workgroup to a compute unit, many K tiles
    X, Wg, Wu, bg, bu = operands(T, D, F, torch.bfloat16, 4)
    run_forward(X, Wg, Wu, bg, bu, "silu", True, scratch(alcs.alcs_gated_ff_workspace_bytes(T, D, F, torch.bfloat16)), "deep")


@pytest.mark.parametrize("kind", GATES)
@pytest.mark.parametrize("dtype", TYPES)
def test_gates_over_their_range(kind, dtype):
    # D = 1: G runs from -40 to 40
    X = torch.linspace(-40, 40, 801).view(801, 1).to(dtype).cuda()
    one = torch.ones(3, 1, dtype=dtype, device="cuda")
    run_forward(X, one, one * 2, None, None, kind, True, None, kind)


def same(a, b):
    return torch.equal(a, b)


@pytest.mark.parametrize("T", [3, 90])
@pytest.mark.parametrize("dtype", TYPES)
def test_operands_as_views(T, dtype):
    X, Wg, Wu, bg, bu = operands(T, 64, 40, dtype, 77)
    want = run_forward(X, Wg, Wu, bg, bu, "silu", True, None, "packed")
    both, mixed, wide = torch.cat([Wg, Wu]), torch.stack([Wg, Wu], 1).view(80, 64), torch.zeros(T, 200, dtype=dtype, device="cuda")
    wide[:, 3:67] = X
    for x, a, b in ((X, both[:40], both[40:]), (X, mixed[0::2], mixed[1::2]), (wide[:, 3:67], Wg, Wu)):
        run_forward(x, a, b, bg, bu, "silu", True, None, "views")
    H = torch.empty_like(want)
    alcs.alcs_gated_ff(X[:1].expand(T, 64), Wg, Wu, bg, bu, H)
    assert bool((H == H[:1]).all())


def test_rows_that_lie_far_apart():
    # offsets of more than 2^32 bytes
    D, F, step = 64, 32, 2 ** 30 + 64
    flat = torch.empty(step * 4 + D, dtype=torch.bfloat16, device="cuda")
    X = torch.as_strided(flat, (5, D), (step, 1))
    X.copy_(normal(5, D, seed=1, dtype=torch.bfloat16))
    _, Wg, Wu, bg, bu = operands(5, D, F, torch.bfloat16, 2)
    run_forward(X, Wg, Wu, bg, bu, "silu", False, None, "far")
    W = torch.as_strided(flat, (3, D), (2 * step, 1))
    run_forward(normal(80, D, seed=3, dtype=torch.bfloat16), W, Wu[:3], None, None, "silu", False, None, "far weights")


BACKWARD = [(1, 1, 1), (1, 64, 64), (3, 17, 9), (16, 128, 40), (65, 96, 70), (100, 33, 260), (129, 200, 257), (300, 520, 136),
            (2000, 24, 40), (70, 24, 4100), (520, 256, 256)]


def run_backward(T, D, F, dtype, kind, seed, what):
    X, Wg, Wu, _, _ = operands(T, D, F, dtype, seed)
    G, U, dH = (normal(T, F, seed=seed + i, dtype=dtype) for i in (5, 6, 7))
    outs = [guarded(*s, dtype=dtype) for s in ((T, D), (F, D), (F, D), (F,), (F,))]
    ws = scratch(alcs.alcs_gated_ff_backward_workspace_bytes(T, D, F, dtype))
    alcs.alcs_gated_ff_backward(X, Wg, Wu, G, U, dH, *(o for o, _ in outs), gate=kind, workspace=ws)
    ref, tol = backward_ref(X, Wg, Wu, G, U, dH, kind)
    for (o, intact), r, t, n in zip(outs, ref, tol, ("dX", "dWg", "dWu", "dbg", "dbu")):
        check(o, r, t, what + " " + n)
        assert intact(), n
    return X, Wg, Wu, G, U, dH, [o for o, _ in outs], ws


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("i", range(len(BACKWARD)))
def test_backward(i, dtype):
    kind = GATES[(i + 2 * TYPES.index(dtype)) % 6]
    run_backward(*BACKWARD[i], dtype, kind, 1000 + 10 * i, "%s %s %s" % (BACKWARD[i], dtype, kind))


@pytest.mark.parametrize("T,D,F", [(4096, 2048, 72), (72, 2048, 2048), (4000, 2056, 100), (72, 4104, 2056), (4100, 4104, 200)])
def test_backward_large_tiles(T, D, F):
    run_backward(T, D, F, torch.bfloat16, "silu", 3, "%s" % ((T, D, F),))


@pytest.mark.parametrize("kind", GATES)
def test_gradients_against_differences(kind):
    T, D, F = 5, 12, 8
    X, Wg, Wu, bg, bu = operands(T, D, F, torch.float32, 31)
    H, G, U = (torch.empty(T, F, device="cuda") for _ in range(3))
    alcs.alcs_gated_ff(X, Wg, Wu, bg, bu, H, gate=kind, G=G, U=U)
    dH = normal(T, F, seed=40)
    grads = [torch.empty(*s, device="cuda") for s in ((T, D), (F, D), (F, D), (F,), (F,))]
    alcs.alcs_gated_ff_backward(X, Wg, Wu, G, U, dH, *grads, gate=kind,
                                workspace=scratch(alcs.alcs_gated_ff_backward_workspace_bytes(T, D, F, torch.float32)))

    def value(x, wg, wu, b1, b2):
        g, u = x @ wg.t() + b1, x @ wu.t() + b2
        return float((gate64(kind, g) * u * dH.double()).sum())

    at = [t.double() for t in (X, Wg, Wu, bg, bu)]
    h = 1e-5
    for k in range(5):
        way = torch.randn(at[k].shape, generator=torch.Generator().manual_seed(50 + k), dtype=torch.float64).cuda()
        up, down = ([t + s * h * way if i == k else t for i, t in enumerate(at)] for s in (1, -1))
        slope = (value(*up) - value(*down)) / (2 * h)
        mine = float((grads[k].double() * way).sum())
        # central differences: h^2 of a third derivative, cancellation 1e-16 / h; float32 gradients of up to 60 terms
        scale = float((grads[k].double().abs() * way.abs()).sum())
        assert abs(mine - slope) <= 2e-5 * scale + 1e-6, (kind, k, mine, slope)


def test_backward_parts_of_the_gradients():
    X, Wg, Wu, G, U, dH, outs, ws = run_backward(90, 64, 48, torch.bfloat16, "silu", 5, "all")
    again = [torch.empty_like(o) for o in outs]
    alcs.alcs_gated_ff_backward(X, Wg, Wu, G, U, dH, again[0], None, None, None, None, workspace=ws)
    alcs.alcs_gated_ff_backward(X, Wg, Wu, G, U, dH, None, again[1], again[2], None, None, workspace=ws)
    alcs.alcs_gated_ff_backward(X, Wg, Wu, G, U, dH, None, None, None, again[3], again[4], workspace=ws)
    for a, b in zip(outs, again):
        assert same(a, b)
    both = torch.cat([Wg, Wu])
    alcs.alcs_gated_ff_backward(X, both[:48], both[48:], G, U, dH, *again[:3], None, None, workspace=ws)
    assert same(again[0], outs[0])


@pytest.mark.parametrize("kind", GATES)
@pytest.mark.parametrize("dtype", TYPES)
def test_slopes_far_out(kind, dtype):
    # one row and one column, so that dWg is dG and dWu is dU: far from 0 every gate is flat or the line g
    top = 6e4 if dtype == torch.float16 else 3e38
    far = torch.tensor([200.0, 1e4, top], dtype=dtype)
    G = torch.cat([far, -far]).view(1, 6).cuda()
    one = torch.ones(6, 1, dtype=dtype, device="cuda")
    big = 2.0 ** 10 if dtype == torch.float16 else 2.0 ** 100
    for u, h in ((0.5, 2.0), (big, 1 / big), (1 / big, 1.0)):
        U, dH = torch.full_like(G, u), torch.full_like(G, h)
        dWg, dWu = torch.empty_like(one), torch.empty_like(one)
        alcs.alcs_gated_ff_backward(one[:1], one, one, G, U, dH, None, dWg, dWu, None, None, gate=kind,
                                    workspace=scratch(alcs.alcs_gated_ff_backward_workspace_bytes(1, 1, 6, dtype)))
        up, down = {"none": (1, 1), "sigmoid": (0, 0)}.get(kind, (1, 0))
        assert dWg.view(-1).tolist() == [u * h * up] * 3 + [u * h * down] * 3, (kind, u, h)
    # and where both factors' product would overflow, but the slope is 0
    if kind not in ("none", "sigmoid") and dtype != torch.float16:
        alcs.alcs_gated_ff_backward(one[:1], one, one, G, torch.full_like(G, big), torch.full_like(G, big), None, dWg, dWu, None, None,
                                    gate=kind, workspace=scratch(alcs.alcs_gated_ff_backward_workspace_bytes(1, 1, 6, dtype)))
        assert dWg.view(-1)[3:].tolist() == [0.0] * 3


def apart(t, pitch, offset):
    """t's values as rows `pitch` elements apart that start `offset` elements into a tensor."""
    whole = torch.zeros(offset + (t.shape[0] - 1) * pitch + t.shape[1], dtype=t.dtype, device="cuda")
    v = torch.as_strided(whole, t.shape, (pitch, 1), offset)
    v.copy_(t)
    return v


@pytest.mark.parametrize("pitch,offset", [(72, 0), (72, 1), (65, 0), (2 ** 21 + 8, 0), (2 ** 21 + 9, 3)])
@pytest.mark.parametrize("dtype", TYPES)
def test_rows_that_have_to_be_copied(dtype, pitch, offset):
    # rows of whole pieces that start elsewhere or lie far apart: with room for copies, without, and without a workspace
    T, D, F = 150, 64, 100
    X, Wg, Wu, bg, bu = operands(T, D, F, dtype, 55)
    n = alcs.alcs_gated_ff_workspace_bytes(T, D, F, dtype)
    x, a, b = (apart(t, pitch, offset) for t in (X, Wg, Wu))
    for xs, ws in (((x, Wg, Wu), n), ((X, a, Wu), n), ((x, a, b), n), ((x, a, b), n + 8 * (T + 2 * F) * (D + 8)), ((X, Wg, b), 0)):
        run_forward(*xs, bg, bu, "silu", True, scratch(ws) if ws else None, "%d %d" % (pitch, offset))
    G, U, dH = (normal(T, F, seed=i, dtype=dtype) for i in (5, 6, 7))
    ws = scratch(alcs.alcs_gated_ff_backward_workspace_bytes(T, D, F, dtype))
    want, got = ([torch.empty(*s, dtype=dtype, device="cuda") for s in ((T, D), (F, D), (F, D), (F,), (F,))] for _ in range(2))
    alcs.alcs_gated_ff_backward(X, Wg, Wu, G, U, dH, *want, workspace=ws)
    for ops in ((x, Wg, b), (x, a, b)):
        alcs.alcs_gated_ff_backward(*ops, G, U, dH, *got, workspace=ws)
        assert all(same(p, q) for p, q in zip(want, got))


@pytest.mark.parametrize("dtype", TYPES[:2])
@pytest.mark.parametrize("T,D,F", [(70, 2 ** 20, 3), (70, 2 ** 20 - 1, 3), (70, 3, 2 ** 20), (70, 8, 2 ** 20 - 3)])
def test_widest(T, D, F, dtype):
    X, Wg, Wu, bg, bu = operands(T, D, F, dtype, 9)
    run_forward(X, Wg, Wu, bg, bu, "silu", False, scratch(alcs.alcs_gated_ff_workspace_bytes(T, D, F, dtype)), "widest")
    del X, Wg, Wu
    run_backward(T, D, F, dtype, "silu", 19, "widest")


def test_no_rows():
    X, Wg, Wu, bg, bu = operands(4, 32, 16, torch.bfloat16, 1)
    empty = torch.empty(0, 16, dtype=torch.bfloat16, device="cuda")
    alcs.alcs_gated_ff(X[:0], Wg, Wu, bg, bu, empty)
    outs = [torch.full(s, 7.0, dtype=torch.bfloat16, device="cuda") for s in ((16, 32), (16, 32), (16,), (16,))]
    alcs.alcs_gated_ff_backward(X[:0], Wg, Wu, empty, empty, empty, X[:0].clone(), *outs)
    assert all(bool((o == 0).all()) for o in outs)


def test_a_row_that_is_not_finite_stays_alone():
    for T in (10, 100):
        X, Wg, Wu, bg, bu = operands(T, 40, 24, torch.bfloat16, 1)
        X[3, 5] = float("nan")
        H = torch.empty(T, 24, dtype=torch.bfloat16, device="cuda")
        alcs.alcs_gated_ff(X, Wg, Wu, bg, bu, H)
        bad = torch.isnan(H)
        assert bool(bad[3].all()) and int(bad.sum()) == 24


def test_a_gradient_that_is_not_finite_stays_alone():
    # a NaN in one row of dH: that row of dX, that column's gradients, and nothing beside them
    T, D, F = 100, 40, 24
    X, Wg, Wu, _, _ = operands(T, D, F, torch.bfloat16, 1)
    G, U, dH = (normal(T, F, seed=i, dtype=torch.bfloat16) for i in (5, 6, 7))
    dH[3, 5] = float("nan")
    outs = [torch.empty(*s, dtype=torch.bfloat16, device="cuda") for s in ((T, D), (F, D), (F, D), (F,), (F,))]
    alcs.alcs_gated_ff_backward(X, Wg, Wu, G, U, dH, *outs, workspace=scratch(alcs.alcs_gated_ff_backward_workspace_bytes(T, D, F, torch.bfloat16)))
    for o, row, n in zip(outs, (3, 5, 5, 5, 5), (D, D, D, 1, 1)):
        bad = torch.isnan(o)
        assert bool(bad[row].all()) and int(bad.sum()) == n


def test_two_calls_at_once():
    # on two streams, each with a workspace of its own
    T, D, F = 700, 1000, 520
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    sets = [operands(T, D, F, torch.bfloat16, seed) for seed in (1, 21)]
    wants = [run_forward(*o, "silu", True, None, "alone") for o in sets]
    n = alcs.alcs_gated_ff_workspace_bytes(T, D, F, torch.bfloat16)
    spaces, outs = [scratch(n) for _ in sets], [torch.empty_like(w) for w in wants]
    singles = []
    for o, ws in zip(sets, spaces):
        h = torch.empty_like(wants[0])
        alcs.alcs_gated_ff(*o, h, workspace=ws)
        singles.append(h)
    torch.cuda.synchronize()
    for _ in range(20):
        for o, ws, h, st in zip(sets, spaces, outs, (s1, s2)):
            alcs.alcs_gated_ff(*o, h, workspace=ws, stream=st)
    torch.cuda.synchronize()
    assert all(same(a, b) for a, b in zip(outs, singles))


def test_equal_calls_and_another_stream():
    X, Wg, Wu, bg, bu = operands(200, 2000, 64, torch.bfloat16, 1)
    ws = scratch(alcs.alcs_gated_ff_workspace_bytes(200, 2000, 64, torch.bfloat16))
    a, b = (torch.empty(200, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    alcs.alcs_gated_ff(X, Wg, Wu, bg, bu, a, workspace=ws)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    alcs.alcs_gated_ff(X, Wg, Wu, bg, bu, b, workspace=ws, stream=s)
    s.synchronize()
    assert same(a, b)


def test_block_of_gated_layer_and_four_bit_projection():
    """The operators as a feed-forward part uses them: trained in 16 bits, its down projection stored in 4 bits;
    captured and replayed on new tokens."""
    T, D, F = 96, 128, 336
    X, Wg, Wu, bg, bu = operands(T, D, F, torch.bfloat16, 1)
    Wd = normal(D, F, seed=9, std=F ** -0.5)
    wc, ws = alcs.alcs_mx4_quantize(Wd)
    H, G, U = (torch.empty(T, F, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    hc, hs = alcs.alcs_mx4_quantize(H)
    Y = torch.empty(T, D, dtype=torch.bfloat16, device="cuda")
    dH = normal(T, F, seed=10, dtype=torch.bfloat16)
    grads = [torch.empty(*s, dtype=torch.bfloat16, device="cuda") for s in ((T, D), (F, D), (F, D), (F,), (F,))]
    w1 = scratch(alcs.alcs_gated_ff_workspace_bytes(T, D, F, torch.bfloat16))
    w2 = scratch(alcs.alcs_mx4_linear_workspace_bytes(T, D, 2 * hc.shape[1]))
    w3 = scratch(alcs.alcs_gated_ff_backward_workspace_bytes(T, D, F, torch.bfloat16))

    def step():
        alcs.alcs_gated_ff(X, Wg, Wu, bg, bu, H, G=G, U=U, workspace=w1)
        alcs.alcs_mx4_quantize(H, hc, hs)
        alcs.alcs_mx4_linear(hc, hs, wc, ws, None, Y, workspace=w2)
        alcs.alcs_gated_ff_backward(X, Wg, Wu, G, U, dH, *grads, workspace=w3)

    from ff_util import linear_ref
    step()
    torch.cuda.synchronize()
    check(H, *(t[0] for t in gated_ref(X, Wg, Wu, bg, bu, "silu")), "H")
    check(Y, *linear_ref(hc, hs, wc, ws, None, "none"), "Y")
    for g, r, t in zip(grads, *backward_ref(X, Wg, Wu, G, U, dH, "silu")):
        check(g, r, t, "gradient")
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        step()
    torch.cuda.synchronize()
    outs = [H, Y, *grads]
    for rep in range(4):
        X.copy_(normal(T, D, seed=100 + rep, dtype=torch.bfloat16))
        for o in outs:
            o.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        for o in outs:
            o.fill_(float("nan"))
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, outs):
            assert same(a, b) and not bool(torch.isnan(a).any())


def test_refusals():
    X, Wg, Wu, bg, bu = operands(8, 32, 16, torch.bfloat16, 1)
    H = torch.empty(8, 16, dtype=torch.bfloat16, device="cuda")
    V, E = pytest.raises(ValueError), pytest.raises(alcs.AlcsError)
    f = alcs.alcs_gated_ff
    with V: f(X.t(), Wg, Wu, bg, bu, H)
    with V: f(X.double(), Wg, Wu, bg, bu, H)
    with V: f(X.cpu(), Wg, Wu, bg, bu, H)
    with V: f(X, Wg.float(), Wu, bg, bu, H)
    with V: f(X, Wg[:, :16], Wu, bg, bu, H)
    with V: f(X, Wg, Wu[:8], bg, bu, H)
    with V: f(X, Wg, Wu, bg.to(torch.bfloat16), bu, H)
    with V: f(X, Wg, Wu, bg[:15], bu, H)
    with V: f(X, Wg, Wu, bg, bu, H.float())
    with V: f(X, Wg, Wu, bg, bu, torch.empty(8, 32, dtype=torch.bfloat16, device="cuda")[:, ::2])
    with V: f(X, Wg, Wu, bg, bu, H, G=H[:4], U=H[:4])
    with V: f(X, Wg, Wu, bg, bu, H, workspace=torch.zeros(4, device="cuda"))
    with pytest.raises(KeyError): f(X, Wg, Wu, bg, bu, H, gate="tanh")
    with E: f(X, Wg, Wu, bg, bu, H, gate=6)
    with E: f(X, Wg, Wu, bg, bu, H, G=torch.empty_like(H))           # G without U
    with E: f(X, Wg, Wu, bg, bu, H, workspace=scratch(100)[1:])
    with E: f(X[:, :0], Wg[:, :0], Wu[:, :0], bg, bu, H)
    with V: alcs.alcs_gated_ff_workspace_bytes(4, 4, 4, torch.float64)
    with E: alcs.alcs_gated_ff_workspace_bytes(-1, 4, 4, torch.float32)
    b = alcs.alcs_gated_ff_backward
    dX, dW, db = torch.empty_like(X), torch.empty_like(Wg), torch.empty(16, dtype=torch.bfloat16, device="cuda")
    ws = scratch(alcs.alcs_gated_ff_backward_workspace_bytes(8, 32, 16, torch.bfloat16))
    with E: b(X, Wg, Wu, H, H, H, dX, dW, dW.clone(), None, None)                          # no workspace
    with E: b(X, Wg, Wu, H, H, H, dX, dW, dW.clone(), None, None, workspace=ws[:-16])      # a smaller one
    with E: b(X, Wg, Wu, H, H, H, dX, dW, None, None, None, workspace=ws)
    with E: b(X, Wg, Wu, H, H, H, dX, None, None, db, None, workspace=ws)
    with V: b(X, Wg, Wu, H, H, H, dX[:4], None, None, None, None, workspace=ws)
    with V: b(X, Wg, Wu, H, H, H, dX, dW, dW.clone(), db.float(), db.float(), workspace=ws)
    with V: b(X, Wg, Wu, H, H, H.float(), dX, None, None, None, None, workspace=ws)
