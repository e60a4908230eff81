"""Which kernels a feed-forward product takes, asked of the library's own rules without a GPU."""
import collections
import ctypes
import functools
import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
KINDS = ("256", "128", "64", "few")      # rows of a tile: k_big, k_mid, k_mid; k_few
BIG = 1 << 62

Plan = collections.namedtuple("Plan", "kind splits tiles ktiles deep")
Backward = collections.namedtuple("Backward", "together dX dW dX_alone dW_alone")


@functools.lru_cache(None)
def _library():
    with tempfile.TemporaryDirectory() as d:
        so = os.path.join(d, "tile_plan.so")
        subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", os.path.join(ROOT, "include"),
                               "-I", os.path.join(ROOT, "paper_2109_00170_amd", "csrc"),
                               os.path.join(HERE, "native", "tile_plan.cpp"), "-o", so])
        lib = ctypes.CDLL(so)
    lib.forward_time.restype = ctypes.c_double
    return lib


def _plan(out):
    return Plan(KINDS[out[0]], out[1], out[2], out[3], bool(out[4]))


def _code(dtype):
    return ("torch.float32", "torch.bfloat16", "torch.float16").index(str(dtype))


def linear_plan(M, N, K, workspace=BIG, cus=256):
    """Of alcs_mx4_linear; K: stored columns."""
    out = (ctypes.c_int * 5)()
    _library().linear_plan(M, N, K, ctypes.c_longlong(workspace), cus, out)
    return _plan(out)


def forward_plan(T, D, F, dtype, workspace=BIG, cus=256):
    """Of alcs_gated_ff."""
    out = (ctypes.c_int * 5)()
    _library().forward_plan(_code(dtype), T, D, F, ctypes.c_longlong(workspace), cus, out)
    return _plan(out)


def backward_plan(T, D, F, dtype, cus=256):
    """Of alcs_gated_ff_backward: of a call for all gradients, and of one for dX or both dW alone."""
    out = (ctypes.c_int * 21)()
    _library().backward_plan(_code(dtype), T, D, F, cus, out)
    return Backward(bool(out[0]), *(_plan(out[i:i + 5]) for i in (1, 6, 11, 16)))


def forward_time(T, D, F, dtype, kind, splits=1, cus=256):
    return _library().forward_time(_code(dtype), T, D, F, KINDS.index(kind), splits, cus)
