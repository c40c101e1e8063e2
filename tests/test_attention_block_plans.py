"""How the products of 4-bit rows and the attention to an encoder's states are shared out (no GPU needed)."""
import ctypes
import os
import random

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16 = 0, 1

# Attention: dtype, n, lq, lk, heads, kv_heads, d -> queries to a workgroup, whether several share a query's states, with more than one
# tile of states (64, fp32 32) each.  Every width the kernels are made for, whole and odd.
TILES = {
    (BF16, 2, 2000, 130, 32, 8, 64): (256, False, True), (BF16, 4, 1000, 130, 32, 32, 48): (256, False, True), (BF16, 2, 2000, 200, 32, 8, 59): (256, False, True),
    (BF16, 2, 2000, 130, 32, 32, 32): (256, False, True), (BF16, 4, 1000, 150, 32, 8, 30): (256, False, True),
    (BF16, 8, 700, 300, 8, 8, 32): (128, False, True), (BF16, 8, 700, 300, 8, 8, 25): (128, False, True),
    (BF16, 8, 700, 300, 8, 8, 64): (128, False, True), (BF16, 8, 700, 300, 8, 4, 59): (128, False, True), (BF16, 4, 700, 300, 8, 8, 96): (128, False, True),
    (BF16, 4, 700, 300, 8, 8, 91): (128, False, True), (BF16, 4, 700, 300, 8, 8, 128): (128, False, True), (BF16, 4, 700, 200, 8, 2, 100): (128, False, True),
    (BF16, 4, 700, 200, 8, 8, 160): (128, False, True), (BF16, 4, 700, 200, 8, 8, 130): (128, False, True), (BF16, 4, 700, 200, 8, 8, 256): (128, False, True),
    (BF16, 4, 700, 200, 8, 4, 203): (128, False, True), (BF16, 1, 1030, 1000, 4, 2, 40): (128, True, True), (BF16, 1, 1030, 1000, 4, 2, 200): (128, True, True),
    (F32, 4, 700, 200, 8, 8, 32): (128, False, True), (F32, 4, 700, 200, 8, 2, 25): (128, False, True), (F32, 4, 700, 200, 8, 8, 64): (128, False, True),
    (F32, 4, 700, 200, 8, 8, 33): (128, False, True), (F32, 4, 700, 200, 8, 4, 96): (128, False, True), (F32, 4, 700, 200, 8, 8, 90): (128, False, True),
    (F32, 4, 700, 200, 8, 8, 128): (128, False, True), (F32, 4, 700, 200, 8, 8, 127): (128, False, True), (F32, 4, 700, 200, 8, 8, 160): (128, False, True),
    (F32, 4, 700, 200, 8, 8, 130): (128, False, True), (F32, 4, 700, 200, 8, 8, 256): (128, False, True), (F32, 4, 700, 200, 8, 4, 203): (128, False, True),
    (F32, 1, 1030, 300, 4, 2, 33): (128, True, True), (F32, 1, 1030, 1000, 2, 2, 96): (128, True, True), (F32, 1, 1030, 333, 8, 8, 200): (128, True, True),
}
FEW = {
    (F32, 1, 5, 200, 2, 1, 64): (16, False, False), (F32, 1, 1, 300, 1, 1, 100): (16, True, False), (F32, 3, 1, 1000, 8, 8, 25): (16, True, False),
    (BF16, 1, 5, 300, 2, 1, 64): (16, False, False), (BF16, 1, 1, 1000, 1, 1, 100): (16, True, False), (BF16, 1, 1, 5000, 2, 2, 256): (16, True, False),
}

# Products of 4-bit rows: rows, Cin, Cout -> results to a workgroup.  Every tiling with one chunk of 256 values, two and more, with edges in
# rows, in layers and in both.
TILINGS = {
    (515, 40, 2000): (64, 64), (300, 250, 3100): (64, 64), (700, 500, 700): (64, 64), (128, 700, 4100): (64, 64), (515, 1000, 515): (64, 64), (257, 1300, 704): (64, 64),
    (1030, 40, 2000): (128, 64), (2000, 250, 1030): (128, 64), (515, 500, 4100): (128, 64), (1024, 500, 2050): (128, 64), (2050, 500, 1024): (128, 64),
    (2000, 40, 2050): (128, 128), (1030, 250, 4100): (128, 128), (2050, 500, 2000): (128, 128), (515, 700, 4100): (128, 128), (1030, 1300, 2000): (128, 128),
    (2048, 1000, 1030): (128, 128), (2000, 40, 4100): (256, 256), (4100, 250, 2000): (256, 256), (2050, 500, 4100): (256, 256), (2048, 700, 4100): (256, 256),
    (2050, 1300, 4096): (256, 256),
}


def attention_form(lib, case, mask_by_queries=False):
    dt, *sizes = case
    plan = (ctypes.c_int * 3)()
    assert lib.sq_tune_cross_attention_plan(*sizes, dt, int(mask_by_queries), plan) == 0
    return plan[0], plan[1] > 1, plan[0] > 16 and plan[2] > (32 if dt == F32 else 64)


def product_form(lib, case):
    plan = (ctypes.c_int * 3)()
    assert lib.sq_tune_mxfp4_linear_plan(*case, plan) == 0
    return plan[0], plan[1]


@pytest.fixture(scope="module")
def lib():
    l = ctypes.CDLL(os.path.join(ROOT, "paper_1611_07151_amd", "libsq.so"))
    l.sq_cross_attention_workspace_bytes.restype = ctypes.c_size_t
    return l


def test_the_cases_take_the_forms_they_are_for(lib):
    """The GPU tests of the forms take their sizes from the tables above: where the choice changes, so have they to."""
    for case, form in {**TILES, **FEW}.items():
        assert attention_form(lib, case) == form, case
        # a mask by queries takes the wide blocks' place by half as wide ones
        assert attention_form(lib, case, True) == ((128,) + form[1:] if form[0] == 256 else form), case
    for case, form in TILINGS.items():
        assert product_form(lib, case) == form, case


def test_plans_of_sizes_that_are_refused(lib):
    plan = (ctypes.c_int * 3)()
    assert lib.sq_tune_mxfp4_linear_plan(0, 5, 5, plan) == -2 and lib.sq_tune_cross_attention_plan(1, 1, 9, 4, 3, 8, 0, 0, plan) == -2
    assert lib.sq_tune_mxfp4_linear_plan(2**31 - 1, 5, 2**31 - 1, plan) == -3 and lib.sq_tune_cross_attention_plan(1, 2**30, 9, 4, 2, 8, 0, 0, plan) == -3


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
