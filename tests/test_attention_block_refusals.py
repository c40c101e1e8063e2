"""What the 4-bit rows and the attention to an encoder's states refuse, and that they refuse it before any GPU work (no GPU needed)."""
import ctypes
import math
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p(0x1000)      # never dereferenced: validation fails first
ODD = ctypes.c_void_p(0x1001)
OFF = ctypes.c_void_p(0x1010)    # aligned to values, not to 256 bytes
NULL = ctypes.c_void_p(0)
SZ = ctypes.c_size_t
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    l = ctypes.CDLL(os.path.join(ROOT, "paper_1611_07151_amd", "libsq.so"))
    i, vp, ll = ctypes.c_int, ctypes.c_void_p, ctypes.c_longlong
    l.sq_mxfp4_packed_bytes.restype = SZ
    l.sq_mxfp4_pack.argtypes = [vp, i, vp, SZ, i, i, i]
    l.sq_mxfp4_unpack.argtypes = [vp, SZ, vp, i, i, i, i]
    l.sq_mxfp4_linear_workspace_bytes.restype = SZ
    l.sq_mxfp4_linear_forward.argtypes = [vp] * 5 + [i] * 9 + [vp, SZ]
    l.sq_cross_attention_workspace_bytes.restype = SZ
    l.sq_cross_attention_forward.argtypes = [vp] * 4 + [i] * 7 + [ctypes.c_float] + [i] * 4 + [vp, vp, ll, ll, vp, SZ]
    return l


@pytest.mark.parametrize("rows,cin,want", [(1, 1, 256 + 128), (1, 256, 256 + 128), (33, 257, 2 * 2 * 256 + 33 * 2 * 128), (32, 4096, 16 * 256 + 32 * 16 * 128),
                                           (0, 5, 0), (5, 0, 0), (-1, 5, 0), (2**31 - 1, 2**31 - 1, 2**26 * 2**23 * 256 + (2**31 - 1) * 2**23 * 128)])
def test_packed_bytes(lib, rows, cin, want):
    assert lib.sq_mxfp4_packed_bytes(rows, cin) == want


def test_pack(lib):
    f = lambda x=P, t=0, out=P, nb=BIG, rows=5, cin=40, ld=40: lib.sq_mxfp4_pack(x, t, out, nb, rows, cin, ld)
    assert f(x=NULL) == -1 and f(out=NULL) == -1
    assert f(rows=0) == -2 and f(cin=0) == -2 and f(rows=-4) == -2 and f(ld=39) == -2
    assert f(t=2) == -3 and f(t=-1) == -3 and f(x=ODD) == -3 and f(x=ODD, t=1) == -3
    assert f(out=OFF) == -4 and f(nb=lib.sq_mxfp4_packed_bytes(5, 40) - 1) == -4 and f(nb=0) == -4
    assert f(rows=2**31 - 1, cin=2**31 - 1, ld=2**31 - 1, nb=2**63) == -3       # more threads than a launch takes


def test_unpack(lib):
    f = lambda x=P, nb=BIG, out=P, t=0, rows=5, cin=40, ld=40: lib.sq_mxfp4_unpack(x, nb, out, t, rows, cin, ld)
    assert f(x=NULL) == -1 and f(out=NULL) == -1
    assert f(rows=0) == -2 and f(cin=-1) == -2 and f(ld=39) == -2
    assert f(t=2) == -3 and f(out=ODD, t=1) == -3 and f(out=ctypes.c_void_p(0x1002)) == -3
    assert f(x=OFF) == -4 and f(nb=lib.sq_mxfp4_packed_bytes(5, 40) - 1) == -4
    assert f(rows=2**31 - 1, cin=2**31 - 1, ld=2**31 - 1, nb=2**63) == -3


def test_linear(lib):
    def f(x=P, w=P, b=P, res=NULL, out=P, ti=0, to=0, rows=5, cin=40, cout=7, act=0, ldi=40, ldr=0, ldo=7, ws=P, nb=BIG):
        return lib.sq_mxfp4_linear_forward(x, w, b, res, out, ti, to, rows, cin, cout, act, ldi, ldr, ldo, ws, nb)
    assert f(x=NULL) == -1 and f(w=NULL) == -1 and f(out=NULL) == -1
    for k in ("rows", "cin", "cout"):
        assert f(**{k: 0}) == -2 and f(**{k: -1}) == -2
    assert f(ldi=39) == -2 and f(ldo=6) == -2 and f(res=P, ldr=6) == -2
    assert f(ti=3) == -3 and f(ti=-1) == -3 and f(to=2) == -3 and f(act=4) == -3 and f(act=-1) == -3
    assert f(x=ODD) == -3 and f(out=ODD) == -3 and f(b=ODD) == -3 and f(res=ODD, ldr=7) == -3
    assert f(w=OFF) == -4 and f(x=OFF, ti=2) == -4
    need = lib.sq_mxfp4_linear_workspace_bytes(100, 4096, 4096, 0)
    wide = dict(rows=100, cin=4096, cout=4096, ldi=4096, ldo=4096)
    assert need > 0 and f(**wide, nb=need - 1) == -4 and f(**wide, ws=NULL) == -4 and f(**wide, ws=OFF) == -4
    assert lib.sq_mxfp4_linear_workspace_bytes(0, 40, 7, 0) == 0 and lib.sq_mxfp4_linear_workspace_bytes(5, 40, 7, 3) == 0
    assert f(rows=2**31 - 1, cout=2**31 - 1, ldo=2**31 - 1, nb=2**63) == -3


def test_packed_is_no_type_of_other_calls(lib):
    assert lib.sq_set_dtype(2) == -3 and lib.sq_set_dtype(0) == 0
    lib.sq_linear_forward.argtypes = [ctypes.c_void_p] * 5 + [ctypes.c_int] * 9 + [ctypes.c_void_p, SZ]
    assert lib.sq_linear_forward(P, P, NULL, NULL, P, 2, 0, 5, 40, 7, 0, 40, 0, 7, NULL, 0) == -3


def test_cross_attention(lib):
    def f(q=P, k=P, v=P, out=P, dt=0, n=2, lq=5, lk=9, heads=4, kv=2, d=8, scale=0.3, ldq=32, ldk=16, ldv=16, ldo=32, lens=NULL, mask=NULL, mi=0, mr=0, ws=P, nb=BIG):
        return lib.sq_cross_attention_forward(q, k, v, out, dt, n, lq, lk, heads, kv, d, scale, ldq, ldk, ldv, ldo, lens, mask, mi, mr, ws, nb)
    assert f(q=NULL) == -1 and f(out=NULL) == -1 and f(k=NULL) == -1 and f(v=NULL) == -1
    for name in ("n", "lq", "heads", "kv", "d"):
        assert f(**{name: 0}) == -2 and f(**{name: -2}) == -2
    assert f(lk=-1) == -2 and f(kv=3) == -2 and f(kv=8) == -2
    assert f(ldq=31) == -2 and f(ldk=15) == -2 and f(ldv=15) == -2 and f(ldo=31) == -2
    assert f(scale=math.nan) == -2 and f(scale=math.inf) == -2 and f(scale=-2.0 ** 127) == -2
    assert f(mask=P, mi=-1) == -2 and f(mask=P, mr=-1) == -2
    assert f(dt=2) == -3 and f(dt=-1) == -3 and f(d=257, ldq=2000, ldk=2000, ldv=2000, ldo=2000) == -3
    for name in ("q", "k", "v", "out", "lens"):
        assert f(**{name: ODD}) == -3
    assert f(lk=2**30 + 1) == -3 and f(lq=2**30, heads=4, kv=2) == -3 and f(n=2**20, lq=2**20) == -3
    need = lib.sq_cross_attention_workspace_bytes(1, 1, 16384, 4, 2, 8, 0)
    assert need > 0
    assert f(n=1, lq=1, lk=16384, ws=NULL, nb=0) == -4 and f(n=1, lq=1, lk=16384, ws=OFF) == -4 and f(n=1, lq=1, lk=16384, nb=need - 1) == -4
    for sizes in ((0, 1, 9, 4, 2, 8, 0), (1, 1, 0, 4, 2, 8, 0), (1, 1, 9, 4, 3, 8, 0), (1, 1, 9, 4, 2, 257, 0), (1, 1, 9, 4, 2, 8, 2)):
        assert lib.sq_cross_attention_workspace_bytes(*sizes) == 0


def test_binding():
    """Tensors on the CPU never reach the library."""
    import torch

    import paper_1611_07151_amd as sq
    x = torch.zeros(4, 8)
    for call in (lambda: sq.sq_mxfp4_pack(x), lambda: sq.sq_mxfp4_unpack(torch.zeros(384, dtype=torch.uint8), 4, 8),
                 lambda: sq.sq_mxfp4_linear_forward(x, torch.zeros(384, dtype=torch.uint8), 4),
                 lambda: sq.sq_cross_attention_forward(x[None], x[None], x[None], 2)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        sq.sq_mxfp4_linear_forward(torch.zeros(384, dtype=torch.uint8), torch.zeros(384, dtype=torch.uint8), 4)     # packed rows of what size?
    assert sq.sq_mxfp4_packed_bytes(2**31, 4) == 0 and sq.sq_cross_attention_workspace_bytes(2**31, 1, 1, 1, 1, 1) == 0
