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


@without_gpu
def test_maps_that_fit_the_memory_are_not_refused(lib):
    for ti in (0, 1):
        for n in (1, 3, 2 ** 16 + 1, 2 ** 24 - 1, 2 ** 24, 2 ** 26, 2 ** 28 + 1, 2 ** 31 - 1):
            for c in (1, 3, 8, 30, 64, 512):
                for h, w in ((1, 1), (1, 2), (7, 7), (111, 111), (1024, 1024)):
                    if n * c * h * w * 4 > 2 ** 37:
                        continue
                    assert lib.sq_nhwc_pack(P, ti, P, 0, n, c, h, w, c) == HIP, (n, c, h, w)
                    assert lib.sq_nhwc_unpack(P, 0, P, ti, n, c, h, w, c, c + 2, 1) == HIP, (n, c, h, w)
                    for g in {1, 2 - c % 2, c}:
                        need = lib.sq_nhwc_group_norm_workspace_bytes(n, c, h, w, g)
                        assert lib.sq_nhwc_group_norm(P, P, ti, NULL, NULL, n, c, h, w, g, 1e-5, 0, c, c, P, need) == HIP, (n, c, h, w, g)


@without_gpu
@pytest.mark.parametrize("ti", (0, 1))
def test_images_that_fit_a_launch_are_not_refused(lib, ti):
    """Up to 2^29 pixels, 2^29 layers and 2^34 values of an image in the conversions, and 2^21 groups in the group norm."""
    sizes = sorted({2 ** e + d for e in range(30) for d in (-1, 0, 1)})
    for c in sizes:
        for w in sizes:
            if 0 < min(c, w) and max(c, w) <= 2 ** 29 and c * w <= 2 ** 34:
                assert lib.sq_nhwc_pack(P, ti, P, 0, 2, c, 1, w, c) == HIP, (c, w)
                assert lib.sq_nhwc_unpack(P, ti, P, 1, 2, c, 1, w, c, c, 0) == HIP, (c, w)
                for g in {g for g in (1, 2, 3, c, c // 2, c // 3, c // 64) if 0 < g <= 2 ** 21 and c % g == 0}:
                    need = lib.sq_nhwc_group_norm_workspace_bytes(2, c, 1, w, g)
                    assert lib.sq_nhwc_group_norm(P, P, ti, NULL, NULL, 2, c, 1, w, g, 1e-5, 0, c, c, P, need) == HIP, (c, w, g)


class _OnGpu(torch.Tensor):
    """A tensor without memory that says it lives on GPU 0."""
    @staticmethod
    def of(*shape, dtype=torch.float32):
        return torch.empty(shape, device="meta", dtype=dtype).as_subclass(_OnGpu)

    def get_device(self):
        return 0

    def data_ptr(self):
        return 0        # the library itself would say "null"


@without_gpu
def test_numbers_past_32_bits_are_refused_and_not_cut(monkeypatch):
    import paper_1611_07151_amd as sq
    monkeypatch.setattr(sq.binding, "_current_gpu", lambda: 0)
    monkeypatch.setattr(sq.binding, "_raw_stream", lambda index: 0)
    big = 2 ** 32 + 8
    m, w = _OnGpu.of(2, 3, 3, 16), _OnGpu.of(4, 16)

    def refused(status, f, *args, **kw):
        with pytest.raises(sq.SqError) as e:
            f(*args, **kw)
        assert e.value.status == status

    refused(-3, sq.sq_nhwc_pack, _OnGpu.of(1, 1, 1, big))
    refused(-3, sq.sq_nhwc_pack, _OnGpu.of(big, 1, 1, 1))
    refused(-3, sq.sq_nhwc_pack, _OnGpu.of(1, big, 1, 1))
    refused(-3, sq.sq_nhwc_unpack, m, out=_OnGpu.of(2, big + 8, 3, 3))
    refused(-2, sq.sq_nhwc_unpack, m, out=_OnGpu.of(2, 16, 3, 3), c_offset=2 ** 32)
    for groups in (2 ** 32 + 4, 4 - 2 ** 32):
        refused(-2, sq.sq_nhwc_group_norm, m, groups)
        refused(-2, sq.sq_nhwc_group_norm, m, groups, workspace=m)
    for act in (2 ** 32 + 1, 1 - 2 ** 32):
        refused(-3, sq.sq_nhwc_group_norm, m, 4, act=act)
        refused(-3, sq.sq_linear_forward, m, w, act=act)
    assert sq.sq_nhwc_group_norm_workspace_bytes(big, 64, 80, 80, 4) == 0
    assert sq.sq_nhwc_group_norm_workspace_bytes(2, 64, 80, 80, 2 ** 32 + 4) == 0
    assert sq.sq_linear_workspace_bytes(2 ** 32 + 300, 2048, 300) == 0
    assert sq.sq_linear_workspace_bytes(300, 2048, 300, ld_in=2 ** 32 + 2048) == 0
