"""Channels-last operators (layout conversion, group norm with activation, matrix product with bias, activation and
residual) against their definitions in 64 bits.

u = 2^-24 is half a unit of fp32's last place.  Bounds used below, for every element:
  group norm   With z = (x - mean)/s, s = sqrt(var + eps): a sum of partial sums, none longer than 256 additions in a row with
               the tree behind it, is off by at most 256 u times the sum of magnitudes, so mean by 256 u X (X = largest |x| of
               the group), the deviations by 258 u X, the variance (again summed) by (256 + 4) u var + 2*258 u X s, and z by
               at most 258 u X/s + |z| (130 + 258 X/s + 8) u  <=  K u (1 + |z|)(1 + X/s) with K = 400.
               The affine form and the activation (slope at most 1.13, its own value good to 8 u) add 12 u of what they add up.
  product      Cin products and their sum, the matrix unit's additions off by at most a whole unit (2u): (Cin + 16) * 2u *
               (sum |x||w| + |b|); activation and residual as above.
  The result's rounding: finfo(type).eps / 2 of the value.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24
ACTS = (0, 1, 2, 3)


@pytest.fixture(scope="module")
def sq():
    import paper_1611_07151_amd as m
    m.sq_init()
    return m


def gen(seed):
    return torch.Generator().manual_seed(seed)


def act64(y, act):
    if act == 1:
        return torch.where(y < 0, torch.zeros_like(y), y)
    if act == 2:
        return y / (1 + torch.exp(-y))
    if act == 3:
        return 0.5 * y * torch.special.erfc(-y / math.sqrt(2))
    return y


def wide(values, left, right, dtype, fill=float("nan")):
    """`values` [..., C] on the GPU as a slice of rows with `left` and `right` further values around them."""
    c = values.shape[-1]
    buf = torch.full(values.shape[:-1] + (left + c + right,), fill, dtype=dtype, device="cuda")
    buf[..., left:left + c] = values.to(dtype).cuda()
    return buf, buf[..., left:left + c]


def check(got, ref, bound, what):
    got = got.detach().cpu().double()
    err = (got - ref).abs()
    bad = ~(err <= bound)
    assert not bad.any(), (what, int(bad.sum()), float(err.max()), float((err / bound).nan_to_num(0).max()))


def half_step(ref, dtype):
    return torch.finfo(dtype).eps / 2 * ref.abs() * (1 + 1e-6) + torch.finfo(dtype).smallest_normal


# ------------------------------------------------------------------------------------------------------ conversions
@pytest.mark.parametrize("src", (F32, BF16))
@pytest.mark.parametrize("dst", (F32, BF16))
@pytest.mark.parametrize("n,c,h,w", [(1, 1, 1, 1), (1, 3, 7, 5), (2, 64, 8, 8), (3, 65, 9, 13), (1, 200, 1, 1), (2, 1, 13, 13),
                                     (1, 128, 55, 55), (5, 31, 1, 67), (2, 136, 27, 27), (1, 40, 12, 12)])
def test_conversions_are_exact(sq, src, dst, n, c, h, w):
    print(src, dst, n, c, h, w, flush=True)
    x = torch.randn((n, c, h, w), generator=gen(n * c + h)).to(src)
    got = sq.sq_nhwc_pack(x.cuda(), dtype=dst)
    assert got.shape == (n, h, w, c) and got.dtype == dst
    assert torch.equal(got.cpu(), x.permute(0, 2, 3, 1).to(dst))
    m = torch.randn((n, h, w, c), generator=gen(n + c + h)).to(src)
    assert torch.equal(sq.sq_nhwc_unpack(m.cuda(), dtype=dst).cpu(), m.permute(0, 3, 1, 2).to(dst))


@pytest.mark.parametrize("c,left,right", [(16, 8, 8), (17, 3, 2), (64, 0, 64), (8, 1, 0)])
@pytest.mark.parametrize("dt", (F32, BF16))
def test_conversions_of_slices_leave_the_rest_alone(sq, c, left, right, dt):
    n, h, w = 2, 9, 7
    x = torch.randn((n, c, h, w), generator=gen(5)).to(dt)
    buf, view = wide(torch.zeros((n, h, w, c)), left, right, dt)
    sq.sq_nhwc_pack(x.cuda(), out=view)
    torch.cuda.synchronize()
    assert torch.equal(view.cpu(), x.permute(0, 2, 3, 1))
    assert buf[..., :left].isnan().all() and buf[..., left + c:].isnan().all()
    out = torch.full((n, left + c + right, h, w), float("nan"), dtype=dt, device="cuda")
    sq.sq_nhwc_unpack(view, out=out, c_offset=left)
    assert torch.equal(out[:, left:left + c].cpu(), x)
    assert out[:, :left].isnan().all() and out[:, left + c:].isnan().all()


def test_conversions_round_as_the_format_says(sq):
    """Ties go to even, what lies past the largest bfloat16 to infinity, infinities and NaN stay."""
    v = torch.tensor([1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8, 3.4e38, -3.4e38, float("inf"), -float("inf"), float("nan"), -0.0,
                      2.0 ** -133, 1e-45, 65504.0, 1 + 2.0 ** -8 + 2.0 ** -20]).reshape(1, 12, 1, 1)
    want = v.to(BF16).reshape(-1)
    for got in (sq.sq_nhwc_pack(v.cuda(), dtype=BF16), sq.sq_nhwc_unpack(v.reshape(1, 1, 1, 12).cuda(), dtype=BF16)):
        got = got.cpu().reshape(-1)
        assert torch.equal(got.isnan(), want.isnan())
        assert torch.equal(got.view(torch.int16)[~want.isnan()], want.view(torch.int16)[~want.isnan()])


# ------------------------------------------------------------------------------------------------------- group norm
def norm_ref(x, groups, gamma, beta, eps, act):
    """x: channels-last, float64.  Result and the bound of the fp32 arithmetic (before the result's rounding)."""
    n, h, w, c = x.shape
    v = x.reshape(n, h * w, groups, c // groups)
    mean = v.mean((1, 3), keepdim=True)
    s = torch.sqrt(((v - mean) ** 2).mean((1, 3), keepdim=True) + eps)
    z = (v - mean) / s
    big = v.abs().amax((1, 3), keepdim=True)
    bound = 400 * U * (1 + z.abs()) * (1 + big / s)
    z, bound = z.reshape(n, h, w, c), bound.reshape(n, h, w, c)
    a = z * gamma + beta
    bound = 1.13 * (bound * gamma.abs() + 12 * U * ((z * gamma).abs() + beta.abs()))
    y = act64(a, act)
    return y, bound + 12 * U * y.abs()


def norm_case(sq, n, h, w, c, groups, act, dt, seed, left=0, right=0, affine=True, eps=1e-5, spread=1.0, shift=0.5):
    g = gen(seed)
    x = (torch.randn((n, h, w, c), generator=g) * (0.5 + torch.rand(c, generator=g)) * spread + shift * torch.randn(c, generator=g))
    buf, view = wide(x, left, right, dt)
    gamma = 1 + 0.3 * torch.randn(c, generator=g)
    beta = 0.5 * torch.randn(c, generator=g)
    ref, bound = norm_ref(view.cpu().double(), groups, gamma.double() if affine else torch.ones(c).double(),
                          beta.double() if affine else torch.zeros(c).double(), eps, act)
    obuf, out = wide(torch.zeros_like(x), left, right, dt)
    args = (gamma.cuda(), beta.cuda()) if affine else (None, None)
    print(f"norm n={n} h={h} w={w} c={c} groups={groups} act={act} {dt} left={left} right={right}", flush=True)
    got = sq.sq_nhwc_group_norm(view, groups, *args, eps=eps, act=act, out=out)
    torch.cuda.synchronize()
    check(got, ref, bound + half_step(ref, dt), (n, h, w, c, groups, act, dt))
    assert obuf[..., :left].isnan().all() and obuf[..., left + c:].isnan().all()
    if not (left or right):
        assert torch.equal(sq.sq_nhwc_group_norm(view, groups, *args, eps=eps, act=act), got)


NORM_SHAPES = [(1, 1, 1, 8, 2), (2, 1, 1, 1, 1), (1, 1, 3, 6, 3), (3, 5, 7, 12, 4), (1, 13, 13, 512, 32), (2, 13, 13, 96, 8),
               (2, 27, 27, 64, 16), (1, 27, 27, 96, 1), (4, 9, 11, 40, 40), (1, 55, 55, 32, 2), (2, 31, 33, 150, 6), (1, 111, 111, 16, 8),
               (3, 7, 7, 1000, 8), (1, 64, 64, 320, 32), (65, 3, 3, 24, 3), (1, 1, 1, 4096, 1), (1, 200, 130, 8, 1), (2, 16, 16, 7, 7),
               # more than a workgroup keeps: chunks; groups wider than a workgroup; widths that leave vectors of every size
               (1, 40, 40, 4096, 1), (2, 300, 300, 24, 2), (1, 500, 501, 8, 2), (1, 150, 150, 6, 2), (3, 64, 64, 999, 3), (1, 9, 9, 5000, 2),
               (1, 260, 260, 12, 1), (2, 170, 170, 30, 1), (1, 130, 130, 320, 32), (5, 53, 57, 150, 6), (2, 111, 111, 96, 8), (1, 20, 20, 9999, 1)]


@pytest.mark.parametrize("dt", (F32, BF16))
@pytest.mark.parametrize("n,h,w,c,groups", NORM_SHAPES)
def test_group_norm_shapes(sq, n, h, w, c, groups, dt):
    norm_case(sq, n, h, w, c, groups, (n + c) % 4, dt, n + h + c)


@pytest.mark.parametrize("dt", (F32, BF16))
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("n,h,w,c,groups", [(2, 13, 13, 64, 8), (1, 27, 29, 30, 5), (1, 80, 80, 64, 4)])
def test_group_norm_activations(sq, n, h, w, c, groups, act, dt):
    norm_case(sq, n, h, w, c, groups, act, dt, 100 + act)
    norm_case(sq, n, h, w, c, groups, act, dt, 200 + act, affine=False)


@pytest.mark.parametrize("dt", (F32, BF16))
@pytest.mark.parametrize("left,right", [(8, 8), (1, 0), (0, 3), (4, 12), (64, 64)])
@pytest.mark.parametrize("n,h,w,c,groups", [(2, 13, 13, 64, 8), (1, 55, 55, 96, 8), (3, 9, 9, 21, 3), (2, 60, 60, 200, 4)])
def test_group_norm_of_slices(sq, n, h, w, c, groups, left, right, dt):
    norm_case(sq, n, h, w, c, groups, 2, dt, 7 + left, left, right)


@pytest.mark.parametrize("n,h,w,c,groups", [(2, 13, 13, 64, 8), (1, 80, 80, 64, 4), (1, 1, 1, 16, 4)])
def test_group_norm_of_far_and_constant_values(sq, n, h, w, c, groups):
    """A mean a thousand spreads away (the bound's X/s), and equal values: the result is act(beta)."""
    norm_case(sq, n, h, w, c, groups, 0, F32, 3, spread=1e-3, shift=1.0)
    beta = torch.randn(c, generator=gen(1)).cuda()
    x = torch.full((n, h, w, c), 2.5, device="cuda")
    got = sq.sq_nhwc_group_norm(x, groups, None, beta, act=1)
    assert torch.equal(got, torch.relu(beta).expand(n, h, w, c))


@pytest.mark.parametrize("dt", (F32, BF16))
@pytest.mark.parametrize("n,h,w,c,groups", [(2, 13, 13, 64, 8), (2, 80, 80, 64, 4), (2, 30, 30, 21, 3)])
@pytest.mark.parametrize("bad", (float("inf"), float("-inf"), float("nan")))
def test_group_norm_keeps_infinities_and_nan_in_their_group(sq, n, h, w, c, groups, bad, dt):
    x = torch.randn((n, h, w, c), generator=gen(9)).to(dt)
    clean = sq.sq_nhwc_group_norm(x.cuda(), groups, act=2).cpu()
    x[1, h // 2, w - 1, c - 1] = bad
    got = sq.sq_nhwc_group_norm(x.cuda(), groups, act=2).cpu()
    cg = c // groups
    assert got[1, :, :, c - cg:].isnan().all()
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1, :, :, :c - cg], clean[1, :, :, :c - cg])


@pytest.mark.parametrize("dt", (F32, BF16))
@pytest.mark.parametrize("n,h,w,c,groups", [(2, 13, 13, 64, 8), (2, 80, 80, 64, 4), (1, 111, 111, 96, 8), (2, 30, 30, 21, 3)])
def test_group_norm_in_place(sq, n, h, w, c, groups, dt):
    x = torch.randn((n, h, w, c), generator=gen(11)).to(dt).cuda()
    want = sq.sq_nhwc_group_norm(x, groups, act=3)
    assert torch.equal(sq.sq_nhwc_group_norm(x, groups, act=3, out=x), want) and torch.equal(x, want)


# -------------------------------------------------------------------------------------------------- matrix product
def linear_case(sq, rows, cin, cout, act, ti, to, seed, bias=True, residual=True, pads=(0, 0, 0), spread=1.0):
    g = gen(seed)
    _, x = wide(torch.randn((rows, cin), generator=g) * spread, pads[0], pads[0], ti)
    w = (torch.randn((cout, cin), generator=g) * math.sqrt(2.0 / cin)).to(ti).cuda()
    b = torch.randn(cout, generator=g).cuda() if bias else None
    rbuf, res = wide(torch.randn((rows, cout), generator=g), pads[1], pads[1], to) if residual else (None, None)
    obuf, out = wide(torch.zeros((rows, cout)), pads[2], pads[2], to)
    print(f"linear rows={rows} cin={cin} cout={cout} act={act} {ti}->{to} bias={bias} residual={residual} pads={pads}", flush=True)
    got = sq.sq_linear_forward(x, w, b, act=act, residual=res, out=out)
    torch.cuda.synchronize()
    x64, w64 = x.double(), w.double()
    b64 = b.double() if bias else torch.zeros(cout, device="cuda", dtype=torch.float64)
    sums = x64 @ w64.t() + b64
    y = act64(sums, act)
    bound = 1.13 * (cin + 16) * 2 * U * (x64.abs() @ w64.abs().t() + b64.abs()) + 12 * U * y.abs()
    if residual:
        y = y + res.double()
        bound = bound + U * y.abs()
    y, bound = y.cpu(), bound.cpu()
    check(got, y, bound + half_step(y, to) + bound * torch.finfo(to).eps, (rows, cin, cout, act, ti, to))
    p = pads[2]
    assert obuf[..., :p].isnan().all() and obuf[..., p + cout:].isnan().all()
    return got


TYPES = [(F32, F32), (BF16, BF16), (BF16, F32)]
LINEAR_SHAPES = [(1, 1, 1), (1, 512, 1000), (2, 17, 5), (3, 1000, 7), (5, 64, 64), (8, 512, 512), (15, 33, 129), (16, 64, 16), (17, 96, 40),
                 (31, 8, 250), (33, 40, 64), (64, 256, 64), (65, 257, 65), (100, 72, 130), (127, 512, 129), (128, 128, 128), (129, 24, 257),
                 (200, 1536, 100), (255, 31, 255), (256, 256, 256), (300, 64, 520), (513, 99, 333), (729, 384, 192), (1000, 16, 10),
                 (1, 4096, 64), (4, 4000, 24), (40, 2048, 48)]


@pytest.mark.parametrize("ti,to", TYPES)
@pytest.mark.parametrize("rows,cin,cout", LINEAR_SHAPES)
def test_linear_shapes(sq, rows, cin, cout, ti, to):
    linear_case(sq, rows, cin, cout, (rows + cin) % 4, ti, to, rows + cin, residual=(rows + cout) % 2 == 0)


# enough work for the tiles through LDS: whole and part steps of k, ragged edges both ways, one tile row or column
LINEAR_LARGE = [(1024, 2048, 1024), (2100, 1032, 1000), (3601, 328, 3584), (13000, 200, 1000), (129, 4096, 4104), (9000, 2056, 130),
                (2187, 1000, 1001), (4100, 777, 1030), (5400, 520, 2048), (6100, 72, 1801), (905, 193, 704), (1100, 33, 520), (905, 200, 704),
                (700, 72, 600), (300, 1536, 200), (150, 2048, 500), (257, 1000, 333), (600, 40, 520), (600, 8, 520), (2100, 31, 600),
                (1500, 64, 700), (1500, 128, 700), (1500, 96, 1032), (1200, 256, 1024),
                # bf16: two teams that share k, with and without a part step, ragged edges
                (64, 1024, 1024), (70, 1032, 1000), (129, 264, 520), (33, 4096, 2050), (300, 2048, 300), (500, 4096, 4096), (490, 2056, 4001),
                (20000, 256, 8), (200, 320, 400),
                # fp32: two teams, with an odd step and a part step left over
                (729, 1536, 384), (1024, 1024, 1024), (1000, 992, 1000), (900, 1000, 999), (2146, 1057, 288)]


@pytest.mark.parametrize("ti,to", TYPES)
@pytest.mark.parametrize("rows,cin,cout", LINEAR_LARGE)
def test_linear_large(sq, rows, cin, cout, ti, to):
    linear_case(sq, rows, cin, cout, (rows + cin) % 4, ti, to, rows + cin, residual=(rows + cout) % 2 == 0)
    linear_case(sq, rows, cin, cout, 0, ti, to, rows + cin, residual=(rows + cout) % 2 == 1, pads=(8, 3, 8))


# k in shares and a second launch that adds them up: even shares, a short or long last one, part steps, rows at any address
LINEAR_SHARES = [(17, 2056, 4000), (24, 3691, 3000), (33, 4095, 130), (300, 2048, 300), (130, 1111, 2000), (500, 2500, 150), (129, 4160, 999),
                 (1000, 8200, 64), (17, 4099, 77), (729, 1536, 384), (200, 1992, 640), (257, 4000, 1000), (64, 5000, 2001)]


@pytest.mark.parametrize("ti,to", TYPES)
@pytest.mark.parametrize("rows,cin,cout", LINEAR_SHARES)
def test_linear_in_shares_of_k(sq, rows, cin, cout, ti, to):
    need = sq.sq_linear_workspace_bytes(rows, cin, cout, ti, cin, True)
    assert any(sq.sq_linear_workspace_bytes(rows, cin, cout, t) for t in (F32, BF16))
    for act in (0, 3):
        linear_case(sq, rows, cin, cout, act, ti, to, rows + cin, residual=act == 3, pads=(0, 3, 5) if act else (0, 0, 0))
    linear_case(sq, rows, cin, cout, 1, ti, to, rows, pads=(8, 0, 8))
    linear_case(sq, rows, cin, cout, 2, ti, to, rows, bias=False, pads=(1, 0, 0))
    # a workspace of the caller's, full of NaN, with a guard behind it; and the same bits as with one of the binding's
    x, w = torch.randn((rows, cin), generator=gen(1)).to(ti).cuda(), torch.randn((cout, cin), generator=gen(2)).to(ti).cuda()
    space = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")
    got = sq.sq_linear_forward(x, w, out_dtype=to, workspace=space)
    assert torch.equal(got, sq.sq_linear_forward(x, w, out_dtype=to)) and not got.isnan().any()
    assert (space[need:] == 255).all()
    if need:
        with pytest.raises(RuntimeError):
            sq.sq_linear_forward(x, w, out_dtype=to, workspace=space[:need - 1])
        with pytest.raises(RuntimeError):
            sq.sq_linear_forward(x, w, out_dtype=to, workspace=space[16:])
    # in place, captured and replayed
    out = torch.randn((rows, cout), generator=gen(3)).to(to).cuda()
    first = out.clone()
    want = sq.sq_linear_forward(x, w, act=3, residual=first)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        sq.sq_linear_forward(x, w, act=3, residual=out, out=out, workspace=space)
    stream.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sq.sq_linear_forward(x, w, act=3, residual=out, out=out, workspace=space)
    for _ in range(3):
        out.copy_(first)
        space.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("rows,cin,cout", LINEAR_SHAPES[::4] + LINEAR_LARGE[::4] + LINEAR_SHARES[::3])
@pytest.mark.parametrize("ti", (F32, BF16))
def test_linear_stays_inside_its_workspace(sq, rows, cin, cout, ti):
    """Whatever the addresses: rows of whole 16 bytes, and rows that begin at odd ones."""
    w = torch.randn((cout, cin), generator=gen(2)).to(ti).cuda()
    for pad in (0, 1):
        _, x = wide(torch.randn((rows, cin), generator=gen(1)), pad, pad, ti)
        need = sq.sq_linear_workspace_bytes(rows, cin, cout, ti, cin + 2 * pad, pad == 0)
        assert need <= sq.sq_linear_workspace_bytes(rows, cin, cout, ti)
        space = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")
        sq.sq_linear_forward(x, w, workspace=space)
        assert (space[need:] == 255).all()


@pytest.mark.parametrize("ti,to", TYPES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("rows,cin,cout", [(3, 64, 40), (70, 128, 72), (600, 64, 264)])
def test_linear_epilogues(sq, rows, cin, cout, act, ti, to):
    for bias in (False, True):
        for residual in (False, True):
            linear_case(sq, rows, cin, cout, act, ti, to, 40 + act, bias, residual)


@pytest.mark.parametrize("ti,to", TYPES)
@pytest.mark.parametrize("pads", [(8, 0, 0), (0, 8, 8), (1, 3, 5), (16, 16, 16), (4, 2, 1)])
@pytest.mark.parametrize("rows,cin,cout", [(3, 64, 40), (70, 128, 72), (300, 96, 264), (20, 45, 33)])
def test_linear_of_slices(sq, rows, cin, cout, pads, ti, to):
    linear_case(sq, rows, cin, cout, 2, ti, to, 50, pads=pads)


@pytest.mark.parametrize("rows,cin,cout", [(3, 64, 40), (300, 96, 264), (1, 512, 1000)])
@pytest.mark.parametrize("spread", (1e-20, 1e15, 1e25))
def test_linear_far_magnitudes(sq, rows, cin, cout, spread):
    linear_case(sq, rows, cin, cout, 0, F32, F32, 60, bias=False, residual=False, spread=spread)
    linear_case(sq, rows, cin, cout, 0, BF16, F32, 60, bias=False, residual=False, spread=spread)


@pytest.mark.parametrize("ti,to", TYPES)
@pytest.mark.parametrize("rows,cin,cout", [(3, 64, 40), (70, 128, 72), (300, 96, 264), (20, 45, 33), (300, 2048, 70), (1000, 992, 1000), (1100, 257, 1300),
                                           (70, 4000, 1000), (130, 1111, 2000), (24, 3691, 700)])
def test_linear_infinities_and_nan(sq, rows, cin, cout, ti, to):
    """An infinity or NaN in a row or a kernel reaches what its products reach, and nothing else."""
    g = gen(70)
    x, w = torch.randn((rows, cin), generator=g).to(ti), torch.randn((cout, cin), generator=g).to(ti)
    clean = sq.sq_linear_forward(x.cuda(), w.cuda(), out_dtype=to).cpu()
    x[1, cin - 1], x[2, 0] = float("inf"), float("nan")
    w[3, 1] = -float("inf")
    w[5, cin - 1] = 0.0
    x[0, 1] = 2.0
    got = sq.sq_linear_forward(x.cuda(), w.cuda(), out_dtype=to).cpu()
    want = (x.double() @ w.double().t())
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got.isinf(), want.isinf()) and torch.equal(got[got.isinf()].double(), want[want.isinf()])
    keep = torch.ones((rows, cout), dtype=torch.bool)
    keep[:3], keep[:, 3], keep[:, 5] = False, False, False
    assert torch.equal(got[keep], clean[keep])


@pytest.mark.parametrize("ti,to", TYPES)
@pytest.mark.parametrize("rows,cin,cout", [(3, 64, 40), (300, 2048, 72), (600, 96, 264)])
def test_linear_adds_to_its_own_output(sq, rows, cin, cout, ti, to):
    g = gen(80)
    x, w = torch.randn((rows, cin), generator=g).to(ti).cuda(), torch.randn((cout, cin), generator=g).to(ti).cuda()
    out = torch.randn((rows, cout), generator=g).to(to).cuda()
    want = sq.sq_linear_forward(x, w, act=3, residual=out.clone())
    got = sq.sq_linear_forward(x, w, act=3, residual=out, out=out)
    assert got is out and torch.equal(out, want)


@pytest.mark.parametrize("dt", (F32, BF16))
@pytest.mark.parametrize("rows,cin,cout", [(1, 4096, 512), (9, 2048, 100), (169, 2048, 128), (729, 1536, 384), (1500, 512, 900)])
def test_linear_gives_the_same_bits_again(sq, rows, cin, cout, dt):
    g = gen(90)
    x, w = torch.randn((rows, cin), generator=g).to(dt).cuda(), torch.randn((cout, cin), generator=g).to(dt).cuda()
    first = sq.sq_linear_forward(x, w, act=2)
    for _ in range(3):
        assert torch.equal(sq.sq_linear_forward(x, w, act=2), first)


@pytest.mark.parametrize("act", (1, 2, 3))
def test_activations_by_themselves(sq, act):
    """One layer with kernel 1: the result is the activation of the input.
    SiLU: the exponent's argument is rounded (|x| u), exponential, sum and reciprocal add 3u, all through x s(1 - s), and two
    products.  GELU: the tail's fit is good to 1.5e-7 of at most 1/2, its exponent t^2/2 has three roundings (t^2 Q < 0.22), some
    twenty more operations of u each on at most 1/2, and two on the result: 7.5e-8 + 13 u of |x|."""
    x = torch.cat((torch.linspace(-20, 20, 40001), torch.logspace(-30, 30, 121), -torch.logspace(-30, 2, 65), torch.tensor([0.0, -0.0])))
    got = sq.sq_linear_forward(x.reshape(-1, 1).cuda(), torch.ones((1, 1), device="cuda"), act=act).cpu().double().reshape(-1)
    x = x.double()
    ref, sig = act64(x, act), 1 / (1 + torch.exp(-x))
    bound = {1: torch.zeros_like(x), 2: x.abs() * sig * (1 - sig) * (x.abs() + 3) * U + 4 * U * ref.abs(),
             3: (7.5e-8 + 13 * U) * x.abs()}[act]
    check(got, ref, bound + torch.finfo(F32).smallest_normal, act)
    odd = torch.tensor([float("inf"), -float("inf"), float("nan")])
    got = sq.sq_linear_forward(odd.reshape(-1, 1).cuda(), torch.ones((1, 1), device="cuda"), act=act).cpu().reshape(-1)
    want = act64(odd.double(), act)
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got[~want.isnan()].double(), want[~want.isnan()])


def test_kernels_of_a_1x1_convolution_as_they_lie(sq):
    """The same layer as sq_conv2d_forward on the NCHW map: both within the products' bound of the definition."""
    g = gen(91)
    x, w, b = torch.randn((2, 48, 9, 11), generator=g).cuda(), torch.randn((40, 48, 1, 1), generator=g).cuda(), torch.randn(40, generator=g).cuda()
    conv = sq.sq_conv2d_forward(x, w, b, relu=True)
    rows = sq.sq_linear_forward(sq.sq_nhwc_pack(x), w, b, act=sq.SQ_ACT_RELU)
    sums = torch.nn.functional.conv2d(x.abs().double().cpu(), w.abs().double().cpu(), b.abs().double().cpu())
    check(sq.sq_nhwc_unpack(rows), conv.cpu().double(), 2 * (48 + 16) * 2 * U * sums, "conv")


# ------------------------------------------------------------------------------------------------------- together
def block(sq, x, p, ws=None):
    """conv -> channels last -> normalise -> widen -> back, added -> NCHW."""
    y = sq.sq_conv2d_forward(x, p["k"], p["kb"], pad=1)
    m = sq.sq_nhwc_pack(y, dtype=p["dt"])
    v = sq.sq_nhwc_group_norm(m, 8, p["gamma"], p["beta"], act=sq.SQ_ACT_SILU)
    v = sq.sq_linear_forward(v, p["w1"], p["b1"], act=sq.SQ_ACT_GELU)
    m = sq.sq_linear_forward(v, p["w2"], p["b2"], residual=m, out=m)
    return sq.sq_nhwc_unpack(m)


def block_ref(x, p):
    t = {k: v.double().cpu() for k, v in p.items() if k != "dt"}
    y = torch.nn.functional.conv2d(x.double().cpu(), t["k"], t["kb"], padding=1).permute(0, 2, 3, 1)
    v = torch.nn.functional.group_norm(y.permute(0, 3, 1, 2), 8, t["gamma"], t["beta"]).permute(0, 2, 3, 1)
    v = act64(v, 2) @ t["w1"].t() + t["b1"]
    return (y + act64(v, 3) @ t["w2"].t() + t["b2"]).permute(0, 3, 1, 2)


def block_params(dt, seed, cin=16, c=64, e=136):
    g = gen(seed)
    r = lambda *s: torch.randn(s, generator=g)
    p = dict(k=r(c, cin, 3, 3) / math.sqrt(9 * cin), kb=r(c), gamma=1 + 0.1 * r(c), beta=0.1 * r(c), b1=r(e), b2=r(c))
    p = {k: v.cuda() for k, v in p.items()}
    p.update(w1=(r(e, c) / math.sqrt(c)).to(dt).cuda(), w2=(r(c, e) / math.sqrt(e)).to(dt).cuda(), dt=dt)
    return p


@pytest.mark.parametrize("dt,tol", [(F32, 1e-4), (BF16, 5e-2)])
@pytest.mark.parametrize("n,h,w", [(1, 13, 13), (3, 27, 25)])
def test_a_block_of_them_together(sq, dt, tol, n, h, w):
    """fp32: the library's tolerance 1e-4 (1 + |ref|).  bfloat16: three maps are rounded on the way (2^-8 of values up to
    about 5, through projections of gain about 1, in quadrature below 3 * 5 * 2^-8 = 0.06 at the extremes): 5e-2 (1 + |ref|)."""
    p = block_params(dt, 3)
    x = torch.randn((n, 16, h, w), generator=gen(4)).cuda()
    got, ref = block(sq, x, p).cpu().double(), block_ref(x, p)
    assert got.shape == ref.shape
    assert ((got - ref).abs() <= tol * (1 + ref.abs())).all(), float(((got - ref).abs() / (1 + ref.abs())).max())


@pytest.mark.parametrize("dt", (F32, BF16))
def test_a_captured_block_replays_with_new_inputs(sq, dt):
    p = block_params(dt, 5)
    x = torch.empty((2, 16, 27, 27), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    x.normal_()
    with torch.cuda.stream(side):
        block(sq, x, p)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = block(sq, x, p)
    for seed in range(4):
        x.copy_(torch.randn(x.shape, generator=gen(seed)))
        want = block(sq, x, p)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), seed


def test_two_streams_at_once(sq):
    """Calls on two streams, each with its own operands and scratch, do not disturb each other."""
    ps = [block_params(F32, 6), block_params(BF16, 7)]
    xs = [torch.randn((4, 16, 27, 27), generator=gen(s)).cuda() for s in (1, 2)]
    want = [block(sq, x, p) for x, p in zip(xs, ps)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(block(sq, xs[i], ps[i]))
    torch.cuda.synchronize()
    for i in (0, 1):
        assert all(torch.equal(g, want[i]) for g in got[i])


def test_two_host_threads_at_once(sq):
    """Each with a stream of its own; the library's stream belongs to the calling thread."""
    import threading
    ps = [block_params(F32, 16), block_params(BF16, 17)]
    xs = [torch.randn((3, 16, 27, 27), generator=gen(s)).cuda() for s in (11, 12)]
    want = [block(sq, x, p) for x, p in zip(xs, ps)]
    torch.cuda.synchronize()
    got, errors = [[], []], []

    def worker(i):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(10):
                    got[i].append(block(sq, xs[i], ps[i]))
            stream.synchronize()
        except Exception as e:       # noqa: BLE001 - reported by the main thread
            errors.append(e)

    threads = [threading.Thread(target=worker, args=(i,)) for i in (0, 1)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    for i in (0, 1):
        assert all(torch.equal(g, want[i]) for g in got[i])


@pytest.mark.parametrize("dt,ld", [(BF16, 600000), (F32, 540000)])
@pytest.mark.parametrize("cout", (32, 128, 384))
def test_offsets_past_32_bits(sq, dt, ld, cout):
    """Rows that begin more than 2^31 elements (and 2^32 bytes) into their map; few and many results."""
    rows = 4100
    big = torch.empty((rows, ld), dtype=dt, device="cuda")
    x = big[:, ld - 64:]
    x.copy_(torch.randn((rows, 64), generator=gen(1)))
    w = torch.randn((cout, 64), generator=gen(2)).to(dt).cuda()
    dense = x.contiguous()
    want = sq.sq_linear_forward(dense, w, act=1)
    assert torch.equal(sq.sq_linear_forward(x, w, act=1, out=big[:, :cout]), want)
    again = sq.sq_linear_forward(dense, w, act=1, residual=want)
    assert torch.equal(sq.sq_linear_forward(x, w, act=1, residual=big[:, :cout], out=big[:, :cout]), again)
    m = x.unflatten(0, (1, 41, 100))
    want = sq.sq_nhwc_group_norm(dense.reshape(1, 41, 100, 64), 4, act=2)
    assert torch.equal(sq.sq_nhwc_group_norm(m, 4, act=2, out=big[:, :64].unflatten(0, (1, 41, 100))), want)
    assert torch.equal(sq.sq_nhwc_unpack(m, dtype=dt), dense.reshape(1, 41, 100, 64).permute(0, 3, 1, 2))
    back = dense.reshape(1, 41, 100, 64).permute(0, 3, 1, 2).contiguous()
    assert torch.equal(sq.sq_nhwc_pack(back, out=big[:, 128:192].unflatten(0, (1, 41, 100))), dense.reshape(1, 41, 100, 64))


def test_group_norm_of_a_map_past_32_bits(sq):
    """2.2 billion values: a map of 100 equal bands has the statistics of one, so each band is the result of the band alone up to
    the rounding of statistics summed in another order (a step of bfloat16 at most)."""
    band = torch.randn((1, 83, 8300, 32), generator=gen(21)).to(BF16).cuda()
    want = sq.sq_nhwc_group_norm(band, 4, act=2)
    x = band.repeat(1, 100, 1, 1)
    got = sq.sq_nhwc_group_norm(x, 4, act=2, out=x)
    for i in (0, 49, 99):
        part = got[:, 83 * i:83 * (i + 1)].float()
        assert ((part - want.float()).abs() <= 2.0 ** -7 * want.float().abs() + 1e-30).all(), i


def shifted(values, offset, dtype):
    """`values` as a dense tensor that begins `offset` values behind a 512-byte boundary, NaN around it."""
    flat = torch.full((values.numel() + 2 * offset + 8,), float("nan"), dtype=dtype, device="cuda")
    at = flat[offset:offset + values.numel()].view(values.shape)
    at.copy_(values)
    return flat, at


@pytest.mark.parametrize("offset", (1, 2, 3, 4, 8))
@pytest.mark.parametrize("ti,to", TYPES)
@pytest.mark.parametrize("rows,cin,cout", [(1, 512, 100), (8, 1111, 200), (17, 64, 33), (70, 96, 1000), (300, 2048, 300), (33, 4096, 130), (600, 200, 520),
                                           (1300, 136, 1301)])
def test_linear_operands_at_any_address(sq, rows, cin, cout, ti, to, offset):
    g = gen(90 + offset)
    xv, wv = torch.randn((rows, cin), generator=g).to(ti), (torch.randn((cout, cin), generator=g) / math.sqrt(cin)).to(ti)
    bv, rv = torch.randn(cout, generator=g), torch.randn((rows, cout), generator=g).to(to)
    sums = xv.double().cuda() @ wv.double().cuda().t() + bv.double().cuda()
    terms = xv.double().abs().cuda() @ wv.double().abs().cuda().t() + bv.double().abs().cuda()
    ref = (sums + rv.double().cuda()).cpu()
    bound = (1.13 * (cin + 16) * 2 * U * terms).cpu() + U * ref.abs()
    for moved in ("xw", "x", "w", "out"):
        x = shifted(xv, offset, ti)[1] if "x" in moved else xv.cuda()
        w = shifted(wv, offset, ti)[1] if "w" in moved else wv.cuda()
        b, res = shifted(bv, offset, F32)[1], shifted(rv, offset, to)[1]
        flat, out = shifted(torch.zeros((rows, cout)), offset if moved == "out" else 0, to)
        print(f"linear {rows}x{cin}x{cout} {ti}->{to} offset={offset} moved={moved}", flush=True)
        sq.sq_linear_forward(x, w, b, residual=res, out=out)
        check(out, ref, bound + half_step(ref, to) + bound * torch.finfo(to).eps, (rows, cin, cout, ti, to, offset, moved))
        edge = offset if moved == "out" else 0
        assert flat[:edge].isnan().all() and flat[edge + rows * cout:].isnan().all()


@pytest.mark.parametrize("rows,cin,cout", [(300, 2048, 300), (1000, 992, 1000), (24, 3691, 3000), (1300, 2600, 1040)])
@pytest.mark.parametrize("spread", (1e-20, 1e15, 1e25))
def test_linear_far_magnitudes_in_tiles(sq, rows, cin, cout, spread):
    linear_case(sq, rows, cin, cout, 0, F32, F32, 61, bias=False, residual=False, spread=spread)


def test_empty_operands_are_refused(sq):
    x, w = torch.zeros((0, 8), device="cuda"), torch.zeros((6, 8), device="cuda")
    with pytest.raises(RuntimeError):
        sq.sq_linear_forward(x, w)
    with pytest.raises(RuntimeError):
        sq.sq_linear_forward(torch.zeros((4, 0), device="cuda"), torch.zeros((6, 0), device="cuda"))
    with pytest.raises(RuntimeError):
        sq.sq_nhwc_group_norm(torch.zeros((0, 5, 5, 8), device="cuda"), 2)
    with pytest.raises(RuntimeError):
        sq.sq_nhwc_pack(torch.zeros((2, 3, 0, 5), device="cuda"))
    with pytest.raises(RuntimeError):
        sq.sq_nhwc_unpack(torch.zeros((2, 0, 5, 3), device="cuda"))


def test_shares_of_k_on_two_streams_at_once(sq):
    """Calls that take scratch, in flight together on streams of their own."""
    sizes = [(300, 2048, 300, F32), (300, 2048, 300, BF16), (24, 3691, 3000, F32), (729, 1536, 384, F32)]
    jobs = []
    for i, (rows, cin, cout, dt) in enumerate(sizes):
        x, w = torch.randn((rows, cin), generator=gen(i)).to(dt).cuda(), torch.randn((cout, cin), generator=gen(50 + i)).to(dt).cuda()
        assert sq.sq_linear_workspace_bytes(rows, cin, cout, dt)
        jobs.append((x, w, sq.sq_linear_forward(x, w, act=2)))
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for turn in range(20):
        for k, stream in enumerate(streams):
            x, w, want = jobs[(turn + k) % len(jobs)]
            with torch.cuda.stream(stream):
                got.append((sq.sq_linear_forward(x, w, act=2), want))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in got)


@pytest.mark.parametrize("offset", (1, 2, 3, 4))
@pytest.mark.parametrize("dt", (F32, BF16))
@pytest.mark.parametrize("n,h,w,c,groups", [(2, 13, 11, 64, 8), (3, 5, 7, 30, 3), (1, 70, 60, 48, 4), (1, 111, 111, 96, 8)])
def test_maps_at_any_address(sq, n, h, w, c, groups, dt, offset):
    """The same bits as from aligned copies: conversions move values, and a group norm's order of sums depends on sizes alone."""
    v = torch.randn((n, c, h, w), generator=gen(offset)).to(dt)
    dense = v.permute(0, 2, 3, 1).contiguous().cuda()
    flat, out = shifted(torch.zeros((n, h, w, c)), offset, dt)
    sq.sq_nhwc_pack(shifted(v, offset, dt)[1], out=out)
    assert torch.equal(out, dense) and flat[:offset].isnan().all() and flat[offset + v.numel():].isnan().all()
    flat, back = shifted(torch.zeros((n, c, h, w)), offset, dt)
    sq.sq_nhwc_unpack(out, out=back)
    assert torch.equal(back, v.cuda()) and flat[:offset].isnan().all() and flat[offset + v.numel():].isnan().all()
    gamma, beta = torch.randn(c, generator=gen(7)), torch.randn(c, generator=gen(8))
    want = sq.sq_nhwc_group_norm(dense, groups, gamma.cuda(), beta.cuda(), act=3)
    flat, got = shifted(torch.zeros((n, h, w, c)), offset, dt)
    sq.sq_nhwc_group_norm(out, groups, shifted(gamma, offset, F32)[1], shifted(beta, offset, F32)[1], act=3, out=got)
    assert torch.equal(got, want) and flat[:offset].isnan().all() and flat[offset + v.numel():].isnan().all()


def test_profiler_sees_the_launches(sq):
    x, w = torch.randn((64, 32), device="cuda"), torch.randn((16, 32), device="cuda")
    sq.sq_profile_begin(16)
    try:
        sq.sq_linear_forward(x, w)
        sq.sq_nhwc_group_norm(x.reshape(1, 8, 8, 32), 4)
        sq.sq_nhwc_unpack(x.reshape(1, 8, 8, 32))
    finally:
        got = sq.sq_profile_end()
    names = {e["name"].strip("|") for e in got}
    assert any(n.startswith("linear") for n in names) and any(n.startswith("group_norm") for n in names) and "nhwc_unpack" in names
    assert all(e["ms"] > 0 for e in got)
