"""Refusals of the feed-forward operators that need no GPU: by the C entries before a device is asked for,
and by the native entry of the launches."""
import ctypes

import pytest
import torch

import paper_2109_00170_amd as alcs

INVALID, UNSUPPORTED = -1, -2
P = ctypes.c_void_p(4096)      # never followed: every call here is refused before
L = ctypes.c_longlong


def lib():
    return alcs.load_library()


def test_storage_entries_refuse():
    q, d = lib().alcs_mx4_quantize, lib().alcs_mx4_dequantize
    for rows, cols, dtype, rc in ((-1, 4, 0, INVALID), (1, 0, 0, INVALID), (1, 4, 3, INVALID), (1, 4, -1, INVALID), (1, 2 ** 28 + 1, 0, UNSUPPORTED)):
        assert q(P, L(cols), L(rows), cols, dtype, P, P, None) == rc
        assert d(P, P, L(rows), cols, dtype, P, None) == rc
    assert q(P, L(-1), L(1), 4, 0, P, P, None) == INVALID
    for x, c, s in ((None, P, P), (P, None, P), (P, P, None), (P, ctypes.c_void_p(4104), P), (P, P, ctypes.c_void_p(4098))):
        assert q(x, L(4), L(1), 4, 0, c, s, None) == INVALID
        assert d(c, s, L(1), 4, 0, x, None) == INVALID
    assert q(P, L(2 ** 28), L(2 ** 40), 2 ** 28, 0, P, P, None) == UNSUPPORTED
    assert q(None, L(4), L(0), 4, 0, None, None, None) == 0 and d(None, None, L(0), 4, 0, None, None) == 0


def test_product_entry_refuses():
    f = lib().alcs_mx4_linear

    def call(M=4, N=4, K=128, dtype=0, act=0, xc=P, xs=P, wc=P, ws=P, y=P, space=None):
        return f(xc, xs, wc, ws, None, y, M, N, K, dtype, act, space, L(0), None)

    for kw in (dict(M=-1), dict(N=0), dict(K=0), dict(K=100), dict(dtype=3), dict(act=3), dict(act=-1), dict(y=None), dict(xc=None),
               dict(ws=None), dict(wc=ctypes.c_void_p(4104)), dict(xs=ctypes.c_void_p(4097)), dict(space=ctypes.c_void_p(4100))):
        assert call(**kw) == INVALID, kw
    assert call(N=2 ** 28 + 1) == UNSUPPORTED
    assert call(M=0, xc=None) == 0


def test_gated_entries_refuse():
    f, b = lib().alcs_gated_ff, lib().alcs_gated_ff_backward

    def forward(T=4, D=8, F=8, ld=8, dtype=0, gate=2, X=P, Wg=P, H=P, G=None, U=None, space=None):
        return f(X, L(ld), Wg, L(8), P, L(8), None, None, H, G, U, T, D, F, dtype, gate, space, L(0), None)

    def backward(T=4, D=8, F=8, ld=8, dtype=0, gate=2, X=P, dH=P, dW=(P, P), db=(P, P)):
        return b(X, L(ld), P, L(8), P, L(8), P, P, dH, P, *dW, *db, T, D, F, dtype, gate, None, L(0), None)

    for call in (forward, backward):
        for kw in (dict(T=-1), dict(D=0), dict(F=0), dict(dtype=3), dict(gate=6), dict(gate=-1), dict(ld=-1), dict(X=None)):
            assert call(**kw) == INVALID, kw
        assert call(T=2 ** 28 + 1) == UNSUPPORTED
    for kw in (dict(G=P), dict(U=P), dict(H=None), dict(Wg=None), dict(space=ctypes.c_void_p(8))):
        assert forward(**kw) == INVALID, kw
    for kw in (dict(dH=None), dict(dW=(P, None)), dict(dW=(None, P)), dict(db=(P, None))):
        assert backward(**kw) == INVALID, kw
    assert forward(T=0, X=None, H=None) == 0


def test_workspace_sizes_refuse():
    with pytest.raises(ValueError):
        alcs.alcs_gated_ff_workspace_bytes(4, 4, 4, torch.float64)
    with pytest.raises(ValueError):
        alcs.alcs_mx4_linear_workspace_bytes(2 ** 31, 4, 128)
    for call in (lambda: alcs.alcs_mx4_linear_workspace_bytes(4, 4, 127), lambda: alcs.alcs_gated_ff_workspace_bytes(-1, 4, 4, torch.float32),
                 lambda: alcs.alcs_gated_ff_backward_workspace_bytes(4, 0, 4, torch.bfloat16)):
        with pytest.raises(alcs.AlcsError) as e:
            call()
        assert e.value.status == INVALID


def test_tensors_that_are_not_on_a_gpu_are_refused():
    x, u = torch.zeros(4, 128), torch.zeros(4, 64, dtype=torch.uint8)
    s, h = torch.zeros(4, 4, dtype=torch.uint8), torch.zeros(4, 4)
    for call in (lambda: alcs.alcs_mx4_quantize(x, u, s), lambda: alcs.alcs_mx4_dequantize(u, s, x),
                 lambda: alcs.alcs_mx4_linear(u, s, u, s, None, h), lambda: alcs.alcs_gated_ff(x, x, x, None, None, h),
                 lambda: alcs.alcs_gated_ff_backward(x, x, x, h, h, h, x, x, x, None, None)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_sizes_beyond_the_limits():
    f, b = lib().alcs_gated_ff, lib().alcs_gated_ff_backward
    for T, D, F in ((2 ** 26 + 1, 8, 8), (100, 2 ** 20 + 1, 8), (100, 8, 2 ** 20 + 8)):
        for dtype in (0, 1, 2):
            assert f(P, L(D), P, L(D), P, L(D), None, None, P, None, None, T, D, F, dtype, 2, None, L(0), None) == UNSUPPORTED
            assert b(P, L(D), P, L(D), P, L(D), P, P, P, P, P, P, P, P, T, D, F, dtype, 2, P, L(2 ** 60), None) == UNSUPPORTED
            assert lib().alcs_gated_ff_workspace_bytes(T, D, F, dtype) == UNSUPPORTED
            assert lib().alcs_gated_ff_backward_workspace_bytes(T, D, F, dtype) == UNSUPPORTED
    for M, N, K in ((2 ** 26 + 1, 8, 128), (8, 2 ** 26 + 1, 128), (8, 8, 2 ** 23 + 128)):
        assert lib().alcs_mx4_linear(P, P, P, P, None, P, M, N, K, 0, 0, None, L(0), None) == UNSUPPORTED
        assert lib().alcs_mx4_linear_workspace_bytes(M, N, K) == UNSUPPORTED
