"""The feed-forward products' choice of kernels (csrc/alcs_tile_plan.h), asked for the 256 compute units of an MI355X."""
import pytest
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


F32 = torch.float32
MEASURED = [  # T, D, F, type: the fastest of the kernels that were timed for a product of these sizes, operands in the last cache
    (333, 1000, 2730, BF, "64"), (333, 1000, 2730, torch.float16, "64"), (333, 1024, 2730, BF, "64"), (333, 1000, 3400, BF, "64"),
    (333, 1000, 4096, BF, "64"), (333, 1000, 5440, BF, "64"), (250, 1024, 4100, BF, "64"), (500, 1000, 2200, BF, "64"),
    (500, 2000, 2200, BF, "128"), (333, 488, 2730, BF, "64"), (333, 512, 2730, BF, "64"), (700, 1000, 4096, BF, "128"),
    (700, 1024, 4096, BF, "128"), (1000, 1000, 4096, BF, "128"), (1000, 1024, 4096, BF, "128"), (600, 1024, 4096, BF, "128"),
    (520, 2048, 4096, BF, "128"), (400, 512, 6000, BF, "128"), (512, 1000, 4224, BF, "128"), (300, 1000, 7000, BF, "128"),
    (1500, 512, 3000, BF, "128"), (100, 1000, 17000, BF, "128"), (700, 2048, 4096, BF, "128"), (900, 1000, 3000, BF, "128"),
    (520, 512, 4096, BF, "128"),
    # one set of operands over and over
    (500, 512, 1365, F32, "64"), (65, 4096, 16384, BF, "128"), (2048, 4096, 4096, BF, "256"),
    (64, 1000, 2728, BF, "few"), (32, 2048, 4096, BF, "few"), (64, 2048, 4096, BF, "64"), (16, 4096, 8192, BF, "64"),
    (16, 8192, 2048, BF, "64"), (16, 512, 16384, BF, "64"), (16, 4096, 8192, F32, "few"), (32, 4096, 8192, F32, "64"),
    (64, 2047, 4096, F32, "few"), (64, 4095, 8191, F32, "few"), (1, 4095, 8191, BF, "few")]


@pytest.mark.parametrize("T,D,F,dtype,kind", MEASURED)
def test_choices_that_were_measured(T, D, F, dtype, kind):
    assert forward_plan(T, D, F, dtype, workspace=0).kind == kind


def test_gradients_together_where_that_was_faster():
    for T, D, F, dtype, together in ((500, 512, 1365, F32, True), (333, 1000, 2730, BF, True), (256, 512, 2048, BF, True),
                                     (2048, 1024, 4096, BF, True), (2048, 4096, 4096, BF, False)):
        assert backward_plan(T, D, F, dtype).together == together
    assert backward_plan(512, 1024, 4096, BF).dX_alone[:2] in (("64", 4), ("64", 8))


@pytest.mark.parametrize("M,N,K,kind", [(1, 8192, 8192, "few"), (1, 16384, 8192, "64"), (16, 11008, 4096, "few"), (32, 8192, 8192, "64")])
def test_four_bit_choices_that_were_measured(M, N, K, kind):
    assert linear_plan(M, N, K).kind == kind
