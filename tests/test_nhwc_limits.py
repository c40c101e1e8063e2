"""Sizes and numbers at the limits of the channels-last entry points (no GPU needed)."""
import ctypes
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p(0x1000)
NULL = ctypes.c_void_p(0)
SZ = ctypes.c_size_t
HIP = -5        # what a call that is not refused returns where there is no GPU

without_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="accepted calls would run on addresses that do not exist")


@pytest.fixture(scope="module")
def lib():
    l = ctypes.CDLL(os.path.join(ROOT, "paper_1611_07151_amd", "libsq.so"))
    i, vp = ctypes.c_int, ctypes.c_void_p
    l.sq_nhwc_pack.argtypes = [vp, i] * 2 + [i] * 5
    l.sq_nhwc_unpack.argtypes = [vp, i] * 2 + [i] * 7
    l.sq_nhwc_group_norm.argtypes = [vp, vp, i, vp, vp] + [i] * 5 + [ctypes.c_float] + [i] * 3 + [vp, SZ]
    l.sq_nhwc_group_norm_workspace_bytes.restype = SZ
    l.sq_linear_forward.argtypes = [vp] * 5 + [i] * 9 + [vp, SZ]
    l.sq_linear_workspace_bytes.restype = SZ
    return l


def linear(lib, rows, cin, cout, ti):
    need = lib.sq_linear_workspace_bytes(rows, cin, cout, ti, cin, 1)
    return lib.sq_linear_forward(P, P, NULL, NULL, P, ti, ti, rows, cin, cout, 0, cin, 0, cout, P, need)


@without_gpu
@pytest.mark.parametrize("ti", (0, 1))
def test_products_that_fit_a_launch_are_not_refused(lib, ti):
    """2^29 rows, 2^29 layers and 2^35 results, of sums of any length: what sq.h promises."""
    sizes = sorted({2 ** e + d for e in range(30) for d in (-1, 0, 1)} | {3, 100, 1000, 3 * 2 ** 20})
    for rows in sizes:
        for cout in sizes[::2] if rows % 2 else sizes[1::2]:
            if min(rows, cout) > 0 and max(rows, cout) <= 2 ** 29 and rows * cout <= 2 ** 35:
                for cin in (1, 3, 8, 16, 32, 33, 40, 64, 65, 257, 1000, 4096):
                    assert linear(lib, rows, cin, cout, ti) == HIP, (rows, cin, cout)
