"""How the products of 4-bit rows and the attention to an encoder's states are shared out (no GPU needed)."""
import ctypes
import os
import random

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16 = 0, 1


@pytest.fixture(scope="module")
def lib():
    l = ctypes.CDLL(os.path.join(ROOT, "paper_1611_07151_amd", "libsq.so"))
    l.sq_cross_attention_workspace_bytes.restype = ctypes.c_size_t
    return l


def shares_of(lib, n, lq, lk, heads, kv, d, dt):
    """How many workgroups share a row's states, by the workspace for their sums."""
    need = lib.sq_cross_attention_workspace_bytes(n, lq, lk, heads, kv, d, dt)
    rows, width = n * lq * heads, (d + 3) // 4 * 16
    for shares in range(2, 65):
        if need == (rows * shares * width + 255) // 256 * 256 + rows * shares * 16:
            return shares
    assert need == 0
    return 1


def test_joining_fits_one_launch(lib):
    """The launch that joins the shares has 2^32 threads at most, as every launch: one for four values of a row up to eight shares,
    256 a row beyond."""
    cases = [(2, 660685, 9861, 8, 8, 1, F32), (2, 9340183, 12332, 1, 1, 1, F32), (1, 2 ** 24 + 1, 2 ** 20, 1, 1, 64, BF16)]
    rng = random.Random(1)
    for _ in range(20000):
        kv = rng.choice((1, 2, 8))
        cases.append((rng.choice((1, 2, 4)), int(2 ** rng.uniform(16, 29)), int(2 ** rng.uniform(8, 30)), kv, kv, rng.choice((1, 4, 16, 64, 256)), rng.choice((F32, BF16))))
    for c in cases:
        rows, shares = c[0] * c[1] * c[3], shares_of(lib, *c)
        threads = 0 if shares == 1 else (rows * ((c[5] + 3) // 4) + 255) // 256 * 256 if shares <= 8 else rows * 256
        assert threads < 2 ** 32, (c, shares)
