"""Channels-last operators at the ends of the number format and of the sizes, and the accuracy that the fp32 products promise.

u = 2^-24 is half a unit of fp32's last place.
"""
import math

import pytest
import torch

from test_nhwc_gpu import BF16, F32, U, check, gen, half_step, linear_case, norm_ref

pytestmark = pytest.mark.gpu

INF = float("inf")
MAX = torch.finfo(F32).max


@pytest.fixture(scope="module")
def sq():
    import paper_1611_07151_amd as m
    m.sq_init()
    return m


# One product or two for each way an fp32 product is made: wavefronts in small and large blocks, the five tilings, and
# those of them that take shares of k.  Odd steps, part steps and ragged edges among them.
FP32_FORMS = [(17, 99, 40), (300, 96, 264), (2100, 31, 600), (1300, 136, 1301), (17, 5391, 45), (5400, 520, 1400), (2806, 1343, 71),
              (3601, 328, 3584), (5518, 1169, 129), (1000, 992, 1000), (300, 2048, 300), (2043, 85, 429), (130, 1111, 2000), (17, 1632, 2152)]


# --------------------------------------------------------------------------------- infinities beside the format's ends
@pytest.mark.parametrize("near", (False, True))
@pytest.mark.parametrize("rows,cin,cout", FP32_FORMS)
def test_infinities_beside_extreme_operands(sq, rows, cin, cout, near):
    """Results that are not finite are those of the sums in fp32: a finite operand counts as finite, one that is not zero
    as not zero, and a sum past the largest number as an infinity, whatever else lies in the tile.  Rows 0 to 4 and kernels 5
    and 6 hold two operands and zeros, the other rows and kernels stay so small that no other product overflows."""
    g = gen(rows + cin)
    x = (torch.randn((rows, cin), generator=g) * 0.1).clamp(-0.9, 0.9)
    w = (torch.randn((cout, cin), generator=g) * 0.1).clamp(-0.25, 0.25)
    a, b = (cin // 2, cin // 2 + 1) if near else (0, cin - 1)
    x[:7], w[5:7] = 0, 0
    x[0, a], x[0, b], w[0, a], w[0, b] = -MAX, -INF, -0.5, 1.0           # finite - inf
    x[1, a], x[1, b], w[1, a], w[1, b] = -MAX, -MAX, 2.0, 0.0            # an overflow + 0
    x[2, a], w[2, a] = INF, 1e-42                                        # inf * subnormal
    x[3, a], x[3, b], w[3, a], w[3, b] = 1.9060151e38, 1.4985098e38, 1.0, 1.0      # just past the largest number
    x[4, a], x[4, b], w[4, a], w[4, b] = INF, MAX, 1.0, 0.0              # inf + finite * 0
    w[5, a], x[5, a] = INF, 1e-42
    w[6, a], w[6, b], x[6, a], x[6, b] = -MAX, -INF, -0.5, 1.0
    got = sq.sq_linear_forward(x.cuda(), w.cuda()).cpu()
    assert got[0, 0] == -INF and got[1, 1] == -INF and got[2, 2] == INF and got[3, 3] == INF and got[4, 4] == INF
    assert got[5, 5] == INF and got[6, 6] == -INF
    want = (x.double().cuda() @ w.double().cuda().t()).float().cpu()
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got.isinf(), want.isinf()) and torch.equal(got[got.isinf()], want[want.isinf()])
    # and what is finite keeps its accuracy: as the sums have it, and as the smallest of three bfloat16 values leaves an operand,
    # half of 2^-133 off, times the other operand; the result itself and the reference are rounded to multiples of 2^-149
    fin = want.isfinite()
    clamp = lambda t: t.double().clamp(-1e300, 1e300).abs()
    small = 2.0 ** -134 * (clamp(x).sum(1)[:, None] + clamp(w).sum(1)) + 2.0 ** -149
    terms = (clamp(x).cuda() @ clamp(w).cuda().t()).cpu()
    err, bound = (got.double() - want.double()).abs()[fin], ((cin + 16) * 2 * U * terms + small)[fin]
    assert (err <= bound).all(), float((err / bound).max())


@pytest.mark.parametrize("rows,cin,cout", [(300, 96, 264), (1000, 992, 1000), (1300, 136, 1301)])
def test_few_and_many_rows_agree_on_what_is_not_finite(sq, rows, cin, cout):
    """The first rows by themselves go to the wavefronts, all of them to tiles.  Left out are the sums of which a finite product
    passes the largest number by itself: with an infinity of the other sign behind it such a sum is inf - inf, with the infinity
    before it, where product and addition are one rounding, it is that infinity, and the order of a sum is not promised."""
    x, w = torch.randn((rows, cin), generator=gen(1)), torch.randn((cout, cin), generator=gen(2))
    x[::3, 7], x[1::5, cin - 1], w[::7, 3] = MAX, -INF, 1e-41
    w[1::7, 7], x[2::9, 3] = 0.0, INF
    x, w = x.cuda(), w.cuda()
    many = sq.sq_linear_forward(x, w, act=1)[:64]
    few = torch.cat([sq.sq_linear_forward(x[i:i + 8], w, act=1) for i in range(0, 64, 8)])
    within = (x[:64, 7].double()[:, None] * w[:, 7].double()).abs() <= MAX
    assert within.sum() > within.numel() // 2
    assert torch.equal(few.isnan()[within], many.isnan()[within]) and torch.equal(few.isinf()[within], many.isinf()[within])


# --------------------------------------------------------------------------------------- every bit of an fp32 operand
@pytest.mark.parametrize("rows,cin,cout", FP32_FORMS)
def test_fp32_products_are_exact_where_fp32_is(sq, rows, cin, cout):
    """One operand a row that is not zero, so that a result is one product, of as many bits as fp32 holds: any 24 bits times a
    power of two from either side, and (1 + i 2^-11)(1 + j 2^-11) with i, j < 16, which has 23.  Every value is found at every
    step of k; a lost or rounded part of an operand, or a product of two parts left out, shows."""
    g = gen(cin)
    k = torch.linspace(0, cin - 1, rows).round().long()
    at = torch.arange(rows)
    bits = lambda *s: (torch.randint(0, 2 ** 23, s, generator=g).double() / 2 ** 23 + 1) * (torch.randint(0, 2, s, generator=g) * 2 - 1)
    powers = lambda *s: torch.exp2(torch.randint(-20, 21, s, generator=g).double()) * (torch.randint(0, 2, s, generator=g) * 2 - 1)
    short = lambda *s: 1 + torch.randint(1, 16, s, generator=g).double() / 2 ** 11
    for left, right in ((bits, powers), (powers, bits), (short, short)):
        x = torch.zeros((rows, cin), dtype=torch.float64)
        x[at, k] = left(rows)
        w = right(cout, cin)
        want = x[at, k][:, None] * w[:, k].t()
        assert torch.equal(want.float().double(), want)
        got = sq.sq_linear_forward(x.float().cuda(), w.float().cuda()).cpu()
        assert torch.equal(got, want.float())


@pytest.mark.parametrize("rows,cin,cout", FP32_FORMS + [(200, 4096, 520), (1000, 8200, 64)])
def test_fp32_products_lose_no_more_than_fp32_sums(sq, rows, cin, cout):
    """Normally distributed operands: partial sums grow like a random walk, so n additions that are each off by at most 2u of
    the partial sum, independently, leave 2u sqrt(n / 2) of the result (root mean square), and n <= 6/16 of Cin instructions
    add to a sum; the terms' own products, and what a product leaves out, are below 4u.  1.5 sqrt(Cin) u + 4u covers these
    (operands of 16 bits would give 200 u, of 8 bits 40000 u)."""
    x, w = torch.randn((rows, cin), generator=gen(3)).cuda(), torch.randn((cout, cin), generator=gen(4)).cuda()
    got = sq.sq_linear_forward(x, w).double()
    ref = x.double() @ w.double().t()
    off = float(((got - ref).norm() / ref.norm()).cpu())
    assert off <= (1.5 * math.sqrt(cin) + 4) * U, off / U


# ----------------------------------------------------------------------- tilings and shares that other shapes do not reach
@pytest.mark.parametrize("ti,to,rows,cin,cout", [
    # bf16 rows of whole 16-byte pieces: 128 x 128 tiles with two images in LDS, and k in shares with each large tile
    (BF16, BF16, 3099, 1664, 2400), (BF16, F32, 9481, 32, 395), (BF16, BF16, 2500, 624, 1500), (BF16, BF16, 322, 8128, 5807),
    (BF16, BF16, 3418, 3808, 69), (BF16, F32, 599, 5208, 1336), (BF16, BF16, 3973, 7408, 1033), (BF16, F32, 8268, 7384, 199),
    (BF16, BF16, 889, 5816, 399), (BF16, F32, 5581, 5664, 19),
    # bf16 rows at any address, 128 x 128 in shares
    (BF16, BF16, 68, 2365, 3480), (BF16, F32, 243, 2971, 4634),
    # fp32: one team of 64 x 64, and 128 x 128 and 256 x 128, in shares; 32 x 128 without
    (F32, F32, 17, 5391, 45), (F32, F32, 2806, 1343, 71), (F32, F32, 5518, 1169, 129), (F32, F32, 8223, 1562, 68), (F32, F32, 2043, 85, 429)])
def test_linear_in_every_tiling(sq, ti, to, rows, cin, cout):
    linear_case(sq, rows, cin, cout, 0, ti, to, rows, bias=False, residual=False)
    linear_case(sq, rows, cin, cout, 3, ti, to, rows + 1, pads=(8 if cin % 8 == 0 else 3, 3, 5))


# --------------------------------------------------------------------------------------------------------- large sizes
@pytest.mark.parametrize("rows,cin,cout", [(16777216, 3, 64), (67108864, 3, 8), (2 ** 29, 1, 8)])
def test_linear_of_many_rows_with_a_short_sum(sq, rows, cin, cout):
    """fp32, more blocks of 16 x 16 than a launch of 1024 threads each has, and (the last) than one of 128 has."""
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn((rows, cin), generator=g, device="cuda")
    w = torch.randn((cout, cin), generator=g, device="cuda")
    b = torch.randn(cout, generator=g, device="cuda")
    got = sq.sq_linear_forward(x, w, b, act=1)
    for r in list(range(0, rows, rows // 5)) + [rows - (1 << 20)]:
        part = x[r:r + (1 << 20)].double()
        ref = (part @ w.double().t() + b.double()).clamp(min=0)
        bound = (cin + 16) * 2 * U * (part.abs() @ w.double().abs().t() + b.double().abs())
        assert ((got[r:r + (1 << 20)].double() - ref).abs() <= bound).all(), r


def test_conversions_of_many_small_maps(sq):
    """More maps than a launch has workgroups."""
    n, c = 2 ** 24 + 37, 3
    x = torch.arange(n * c, dtype=torch.int32, device="cuda").remainder(65521).float().reshape(n, c, 1, 1)
    assert torch.equal(sq.sq_nhwc_pack(x).reshape(n, c), x.reshape(n, c))
    wide = torch.full((n, 1, 1, 5), float("nan"), device="cuda")
    m = wide[..., 1:4]
    sq.sq_nhwc_pack(x, out=m)
    assert torch.equal(m.reshape(n, c), x.reshape(n, c)) and wide[..., 0].isnan().all() and wide[..., 4].isnan().all()
    out = torch.full((n, 5, 1, 1), float("nan"), device="cuda")
    sq.sq_nhwc_unpack(m, out=out, c_offset=2)
    assert torch.equal(out[:, 2:].reshape(n, c), x.reshape(n, c)) and out[:, :2].isnan().all()


@pytest.mark.parametrize("dt", (F32, BF16))
@pytest.mark.parametrize("n,c,groups", [(2 ** 24 + 37, 8, 1), (2 ** 24 + 37, 8, 8), (2 ** 26 + 37, 4, 1)])
def test_group_norm_of_many_small_maps(sq, n, c, groups, dt):
    """More maps than a launch has workgroups; and the same bits as the maps by themselves."""
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn((n, 1, 1, c), generator=g, device="cuda").to(dt)
    gamma, beta = torch.randn(c, generator=g, device="cuda"), torch.randn(c, generator=g, device="cuda")
    got = sq.sq_nhwc_group_norm(x, groups, gamma, beta, act=1)
    for i in list(range(0, n, n // 7)) + [n - 4096]:
        part = x[i:i + 4096].cpu().double()
        ref, bound = norm_ref(part, groups, gamma.cpu().double(), beta.cpu().double(), 1e-5, 1)
        check(got[i:i + 4096], ref, bound + half_step(ref, dt), i)


# ------------------------------------------------------------------------------------------------------------ conversion
@pytest.mark.parametrize("dst", (F32, BF16))
def test_unpack_behind_layers_that_nothing_has_written(sq, dst):
    """Without a map to write into, the layers before c_offset are zeros."""
    torch.full((1 << 20,), float("nan"), device="cuda")      # what the allocator hands out next is not zero
    m = torch.randn((2, 9, 7, 5), generator=gen(1)).cuda()
    for off in (0, 1, 3):
        got = sq.sq_nhwc_unpack(m, dtype=dst, c_offset=off)
        assert got.shape == (2, 5 + off, 9, 7) and not got[:, :off].any()
        assert torch.equal(got[:, off:], m.permute(0, 3, 1, 2).to(dst))


# ------------------------------------------------------------------------------------------------------------ group norm
@pytest.mark.parametrize("n,h,w,c,groups", [(2, 13, 13, 64, 8), (2, 80, 80, 64, 4), (1, 200, 130, 8, 1), (1, 9, 9, 5000, 2), (1, 20, 20, 9999, 1),
                                            (2, 61, 60, 200, 4), (1, 111, 111, 96, 8), (3, 64, 64, 999, 3)])
@pytest.mark.parametrize("far", (1e19, 4e19, -4e19, 1e22))
def test_group_norm_of_means_whose_squares_overflow(sq, n, h, w, c, groups, far):
    """The deviations' squares stay within fp32, the mean's does not."""
    x = (far * (1 + torch.randn((n, h, w, c), generator=gen(8)).double() * 1e-4 * min(1.0, 1e19 / abs(far)))).float()
    ref, bound = norm_ref(x.double(), groups, torch.ones(c).double(), torch.zeros(c).double(), 1e-5, 0)
    got = sq.sq_nhwc_group_norm(x.cuda(), groups)
    assert not got.isnan().any()
    check(got, ref, bound + half_step(ref, F32), (n, h, w, c, groups, far))


@pytest.mark.parametrize("n,h,w,c,groups", [(1, 13, 13, 512, 32), (4, 27, 27, 96, 8), (2, 80, 80, 64, 4), (1, 40, 40, 4096, 1), (1, 20, 20, 9999, 1),
                                            (5, 53, 57, 150, 6), (2, 111, 111, 96, 8), (1, 130, 130, 320, 32), (300, 7, 7, 64, 64)])
@pytest.mark.parametrize("mean", (0.5, 30.0))
def test_group_norm_errs_by_few_roundings(sq, n, h, w, c, groups, mean):
    """The mean error (root mean square) instead of the largest possible: a chain of at most 256 additions, each off by u of a
    partial sum, independently, leaves 16 u of a sum, hence 16 u (1 + |mean| / spread) of a normalised value through the mean and
    8 u through the variance; sqrt, quotient and product of the scale 4 u; difference, product and sum 3 u: 15 u + 16 u (1 + |mean|)
    for a spread of one."""
    x = (torch.randn((n, h, w, c), generator=gen(12)) + mean).cuda()
    got = sq.sq_nhwc_group_norm(x, groups).double()
    v = x.double().reshape(n, h * w, groups, c // groups)
    var, mu = torch.var_mean(v, (1, 3), unbiased=False, keepdim=True)
    ref = ((v - mu) / torch.sqrt(var + 1e-5)).reshape(n, h, w, c)
    off = float(((got - ref).norm() / ref.norm()).cpu())
    assert off <= (15 + 16 * (1 + mean)) * U, off / U
