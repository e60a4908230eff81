"""The feed-forward products' choice of kernels (csrc/alcs_tile_plan.h), asked for the 256 compute units of an MI355X."""
import torch

from test_gpu_large_tiles import DW, DX, FORWARD, LINEAR
from tile_plan import backward_plan, forward_plan, linear_plan

BF = torch.bfloat16


def test_large_tiles_are_what_their_tests_run():
    forms = {"forward": [forward_plan(T, D, F, BF) for T, F, D in FORWARD],
             "product": [linear_plan(M, N, (cols + 127) // 128 * 128) for M, N, cols in LINEAR],
             "dX": [backward_plan(T, D, F, BF).dX_alone for T, D, F in DX], "dW": [backward_plan(T, D, F, BF).dW_alone for T, D, F in DW]}
    for form, plans in forms.items():
        assert all(p.kind == "256" and p.splits == 1 for p in plans), (form, plans)
        assert any(p.tiles <= 256 for p in plans) and any(p.tiles > 256 for p in plans), form   # one tile a workgroup, and two
        segments = 2 if form == "dX" else 1
        assert {p.ktiles // segments % 2 for p in plans} == {0, 1}, form                         # odd and even numbers
        assert all(p.ktiles // segments >= 5 for p in plans), form


def test_sizes_of_the_middle_and_few_rows():
    assert forward_plan(1, 2048, 8192, BF).kind == forward_plan(64, 1000, 2728, BF).kind == "few"
    assert forward_plan(64, 2048, 4096, BF).kind == "64"
    assert forward_plan(256, 4096, 8192, BF).deep and not forward_plan(512, 1024, 4096, BF).deep
    # without room for the sums K is not shared out
    assert forward_plan(100, 4104, 24, BF).splits > 1 and forward_plan(100, 4104, 24, BF, workspace=0).splits == 1
    assert linear_plan(65, 129, 640).splits == 1 and linear_plan(100, 200, 4096).splits > 1
