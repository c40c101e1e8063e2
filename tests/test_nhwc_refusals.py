"""What the channels-last entry points refuse, and that they refuse it before any GPU work (no GPU needed)."""
import ctypes
import math
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p(0x1000)      # never dereferenced: validation fails first
ODD = ctypes.c_void_p(0x1001)
NULL = ctypes.c_void_p(0)
SZ = ctypes.c_size_t


@pytest.fixture(scope="module")
def lib():
    l = ctypes.CDLL(os.path.join(ROOT, "paper_1611_07151_amd", "libsq.so"))
    i, vp = ctypes.c_int, ctypes.c_void_p
    l.sq_nhwc_group_norm.argtypes = [vp, vp, i, vp, vp] + [i] * 5 + [ctypes.c_float] + [i] * 3 + [vp, SZ]
    l.sq_nhwc_group_norm_workspace_bytes.restype = SZ
    l.sq_linear_forward.argtypes = [vp] * 5 + [i] * 9 + [vp, SZ]
    l.sq_linear_workspace_bytes.restype = SZ
    return l


def test_pack(lib):
    f = lambda inp=P, ti=0, out=P, to=0, n=2, c=16, h=5, w=5, ld=16: lib.sq_nhwc_pack(inp, ti, out, to, n, c, h, w, ld)
    assert f(inp=NULL) == -1 and f(out=NULL) == -1
    for k in ("n", "c", "h", "w"):
        assert f(**{k: 0}) == -2 and f(**{k: -3}) == -2
    assert f(ld=15) == -2
    assert f(ti=2) == -3 and f(to=-1) == -3
    assert f(inp=ODD) == -3 and f(out=ODD, to=1) == -3
    assert f(inp=ctypes.c_void_p(0x1002)) == -3


def test_unpack(lib):
    f = lambda inp=P, ti=0, out=P, to=0, n=2, c=16, h=5, w=5, ld=16, oc=16, off=0: lib.sq_nhwc_unpack(inp, ti, out, to, n, c, h, w, ld, oc, off)
    assert f(inp=NULL) == -1 and f(out=NULL) == -1
    for k in ("n", "c", "h", "w"):
        assert f(**{k: 0}) == -2
    assert f(ld=15) == -2 and f(off=1) == -2 and f(off=-1) == -2 and f(oc=15) == -2 and f(oc=-2**31) == -2 and f(off=2**31 - 1) == -2
    assert f(ti=7) == -3 and f(to=2) == -3 and f(out=ODD) == -3


def test_group_norm(lib):
    def f(inp=P, out=P, dt=0, gamma=P, beta=P, n=2, c=16, h=5, w=5, g=4, eps=1e-5, act=0, ldi=16, ldo=16, ws=NULL, nb=0):
        return lib.sq_nhwc_group_norm(inp, out, dt, gamma, beta, n, c, h, w, g, eps, act, ldi, ldo, ws, nb)
    assert f(inp=NULL) == -1 and f(out=NULL) == -1
    for k in ("n", "c", "h", "w", "g"):
        assert f(**{k: 0}) == -2 and f(**{k: -1}) == -2
    assert f(g=3) == -2 and f(g=32) == -2 and f(ldi=15) == -2 and f(ldo=15) == -2
    assert f(eps=-1e-9) == -2 and f(eps=math.nan) == -2
    assert f(dt=2) == -3 and f(act=4) == -3 and f(act=-1) == -3
    assert f(inp=ODD) == -3 and f(out=ODD, dt=1) == -3 and f(gamma=ODD) == -3 and f(beta=ctypes.c_void_p(0x1002)) == -3
    assert lib.sq_nhwc_group_norm_workspace_bytes(2, 16, 5, 5, 3) == 0
    assert lib.sq_nhwc_group_norm_workspace_bytes(0, 16, 5, 5, 4) == 0
    big = dict(n=1, c=320, h=512, w=512, g=32, ldi=320, ldo=320)
    need = lib.sq_nhwc_group_norm_workspace_bytes(1, 320, 512, 512, 32)
    if need:
        assert f(**big) == -4 and f(**big, ws=P, nb=need - 1) == -4 and f(**big, ws=ctypes.c_void_p(0x1010), nb=need) == -4


def test_linear(lib):
    def f(inp=P, w=P, b=P, res=P, out=P, ti=0, to=0, rows=8, cin=16, cout=24, act=0, ldi=16, ldr=24, ldo=24, ws=NULL, nb=0):
        return lib.sq_linear_forward(inp, w, b, res, out, ti, to, rows, cin, cout, act, ldi, ldr, ldo, ws, nb)
    assert f(inp=NULL) == -1 and f(w=NULL) == -1 and f(out=NULL) == -1
    for k in ("rows", "cin", "cout"):
        assert f(**{k: 0}) == -2 and f(**{k: -1}) == -2
    assert f(ldi=15) == -2 and f(ldr=23) == -2 and f(ldo=23) == -2
    assert f(ti=2) == -3 and f(to=2) == -3 and f(ti=0, to=1) == -3 and f(act=4) == -3 and f(act=-1) == -3
    assert f(inp=ODD) == -3 and f(w=ODD) == -3 and f(b=ODD) == -3 and f(res=ODD) == -3 and f(out=ctypes.c_void_p(0x1002)) == -3
    for bad in ((0, 16, 24, 0, 16, 1), (8, 0, 24, 0, 16, 1), (8, 16, -1, 0, 16, 1), (8, 16, 24, 2, 16, 1), (300, 2048, 300, 0, 2047, 1)):
        assert lib.sq_linear_workspace_bytes(*bad) == 0
    long = dict(rows=300, cin=2048, cout=300, ldi=2048, ldr=300, ldo=300)
    need = lib.sq_linear_workspace_bytes(300, 2048, 300, 0, 2048, 1)
    assert need > 0
    assert f(**long) == -4 and f(**long, ws=P, nb=need - 1) == -4 and f(**long, ws=ctypes.c_void_p(0x1010), nb=need) == -4
    # more threads than a launch has
    assert f(rows=2**31 - 1, cin=1, cout=2**31 - 1, ldi=1, ldr=2**31 - 1, ldo=2**31 - 1) == -3


def test_sizes_whose_products_pass_64_bits(lib):
    m = 2**31 - 1
    lib.sq_nhwc_pack.argtypes = [ctypes.c_void_p, ctypes.c_int] * 2 + [ctypes.c_int] * 5
    lib.sq_nhwc_unpack.argtypes = [ctypes.c_void_p, ctypes.c_int] * 2 + [ctypes.c_int] * 7
    for n, c, h, w in ((m, m, m, m), (1, 64, m, m), (1, 256, 2**30, 2**30), (2**16, 2**16, 2**16, 2**16), (1, 1, m, m)):
        assert lib.sq_nhwc_pack(P, 0, P, 1, n, c, h, w, c) == -3
        assert lib.sq_nhwc_unpack(P, 1, P, 0, n, c, h, w, c, c, 0) == -3
        assert lib.sq_nhwc_group_norm_workspace_bytes(n, c, h, w, 1) == 0
        assert lib.sq_nhwc_group_norm(P, P, 0, NULL, NULL, n, c, h, w, 1, 1e-5, 0, c, c, P, 2**62) == -3


def test_the_binding_checks_its_tensors():
    import paper_1611_07151_amd as sq
    x, w = torch.zeros((4, 8)), torch.zeros((6, 8))
    with pytest.raises(ValueError):
        sq.sq_linear_forward(x, w)                                    # not on the GPU
    with pytest.raises(ValueError):
        sq.sq_linear_workspace_bytes(4, 8, 6, torch.float16)
    with pytest.raises(ValueError):
        sq.sq_linear_forward(x, torch.zeros((6, 7)))                  # other row length
    with pytest.raises(ValueError):
        sq.sq_linear_forward(x, w.to(torch.bfloat16))
    with pytest.raises(ValueError):
        sq.sq_linear_forward(x, w, residual=torch.zeros((4, 5)))
    with pytest.raises(ValueError):
        sq.sq_linear_forward(x, w, residual=torch.zeros((4, 6)), out_dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        sq.sq_linear_forward(x, w, torch.zeros(5))
    with pytest.raises(ValueError):
        sq.sq_linear_forward(x, w, out=torch.zeros((5, 6)))
    m = torch.zeros((1, 2, 2, 8))
    with pytest.raises(ValueError):
        sq.sq_nhwc_group_norm(m, 2)
    with pytest.raises(ValueError):
        sq.sq_nhwc_group_norm(m, 2, torch.zeros(7))
    with pytest.raises(ValueError):
        sq.sq_nhwc_group_norm(m, 2, out=m.to(torch.bfloat16))
    with pytest.raises(ValueError):
        sq.sq_nhwc_pack(m)
    with pytest.raises(ValueError):
        sq.sq_nhwc_pack(m, out=torch.zeros((1, 2, 8, 3)))
    with pytest.raises(ValueError):
        sq.sq_nhwc_unpack(m, out=torch.zeros((1, 8, 3, 2)))


class _OnGpu:
    """Shape and strides of a tensor, as the row check sees one on the GPU."""
    def get_device(self):
        return 0

    def __init__(self, t):
        self.shape, self.stride, self.is_contiguous, self.numel = t.shape, t.stride, t.is_contiguous, t.numel


def test_which_tensors_are_rows():
    from paper_1611_07151_amd.binding import SqError, _rows_of
    ok = lambda t: _rows_of(_OnGpu(t), "t", 0)
    t = torch.zeros((2, 3, 5, 16))
    assert ok(t) == 16 and ok(t[..., 4:12]) == 16 and ok(t[:1]) == 16
    assert ok(t[0, 0, :1, :7]) == 7                       # a single row has no stride
    assert ok(t[:, :1, :1, :4]) == 240
    for bad in (t.transpose(2, 3), t[:, 1:2], t[:, ::2], t[:, :2], t[..., ::2], t[:, :, :1].expand(2, 3, 4, 16), t[:, :, :4]):
        with pytest.raises(ValueError):
            ok(bad)
    with pytest.raises(ValueError):
        ok(torch.zeros(8))
    for shape, strides in (((2, 1), (2**31, 1)), ((2**31, 2), (2, 1)), ((1, 2**31), (2**31, 1))):
        with pytest.raises(SqError):
            ok(torch.empty(1, device="meta").as_strided(shape, strides))
