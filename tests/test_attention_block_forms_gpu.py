"""Every form that the products of 4-bit rows and the attention to an encoder's states are made in, at sizes that are known to take it, against
the definitions in 64 bits on the GPU.  The bounds are those of test_cross_attention_gpu.py and test_mxfp4_gpu.py.
"""
import math

import pytest
import torch

import test_attention_block_plans as plans
from test_cross_attention_gpu import U, everything, gen, inputs, reference
from test_mxfp4_gpu import act64, spread

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
TYPES = {plans.F32: F32, plans.BF16: BF16}


@pytest.fixture(scope="module")
def sq():
    import paper_1611_07151_amd as m
    m.sq_init()
    return m


def close(got, ref, bound, what):
    got = got.double()
    assert torch.equal(got.isnan(), ref.isnan()), what
    err = torch.where(ref.isnan(), torch.zeros_like(ref), (got - ref).abs())
    bad = ~(err <= torch.where(ref.isnan(), torch.ones_like(ref), bound))
    assert not bad.any(), (what, int(bad.sum()), float(err.max()), float((err / bound).nan_to_num(0).max()))


def reference64(q, k, v, heads, kv, scale, seen, dt):
    parts = [reference(q[i:i + 1], k[i:i + 1], v[i:i + 1], heads, kv, scale, seen[i:i + 1], dt) for i in range(q.shape[0])]
    return torch.cat([r for r, _ in parts]), torch.cat([b for _, b in parts])


def attention_case(sq, case, seed):
    """Sizes, q, k, v on the GPU, and all states seen."""
    assert plans.attention_form(sq.lib, case) == {**plans.TILES, **plans.FEW}[case]
    code, n, lq, lk, heads, kv, d = case
    print(case, flush=True)
    return (n, lq, lk, heads, kv, d), TYPES[code], [t.cuda() for t in inputs(n, lq, lk, heads, kv, d, TYPES[code], seed)], everything(n, lq, lk).cuda()


ATTENTION = list(plans.TILES) + list(plans.FEW)


@pytest.mark.parametrize("kind", ("none", "lengths", "states", "pairs", "late"))
@pytest.mark.parametrize("case", ATTENTION)
def test_attention_and_what_is_hidden(sq, case, kind):
    """Masks with images and queries that see nothing, with NaN, infinities and the largest number in states that nobody sees."""
    (n, lq, lk, heads, kv, d), dt, (q, k, v), seen = attention_case(sq, case, 1)
    mask = lengths = None
    if kind == "lengths":
        lengths = torch.tensor([lk - 3, 0, 65, 1][:n] + [lk // 2 + i for i in range(max(n - 4, 0))], dtype=torch.int32)
        seen &= (torch.arange(lk) < lengths[:, None])[:, None].cuda()
    elif kind == "states":
        mask = torch.rand((n, lk), generator=gen(2)) < 0.6
        mask[:, lk - 1], mask[:, 0] = False, False
        mask[-1] = n == 1
    elif kind == "pairs":
        mask = torch.rand((n, lq, lk), generator=gen(2)) < 0.6
        mask[:, lq // 2], mask[:, :, lk // 3], mask[:, :, lk - 1] = False, False, False
    elif kind == "late":        # ever later states, the first queries all of them, the last none
        mask = (torch.arange(lk) * lq // lk)[None, None].expand(n, lq, lk) >= torch.arange(lq)[None, :, None]
        mask = mask.contiguous()
        mask[:, lq - 1] = lq == 1
        mask[:, :, lk // 3] = False
    if mask is not None:
        mask = mask.cuda()
        seen = seen & (mask if mask.dim() == 3 else mask[:, None])
    ref, bound = reference64(q, k, v, heads, kv, d ** -0.5, seen, dt)
    args = dict(lengths=None if lengths is None else lengths.cuda(), mask=mask)
    got = sq.sq_cross_attention_forward(q, k, v, heads, kv, **args)
    close(got, ref, bound, kind)
    assert (got[~seen.any(2)] == 0).all()
    assert torch.equal(got, sq.sq_cross_attention_forward(q, k, v, heads, kv, **args))
    hidden = ~seen.any(1)
    if hidden.any():
        for bad in (math.nan, math.inf, torch.finfo(dt).max):
            kb, vb = k.clone(), v.clone()
            kb[hidden], vb[hidden] = bad, bad
            close(sq.sq_cross_attention_forward(q, kb, vb, heads, kv, **args), ref, bound, (kind, bad))


@pytest.mark.parametrize("masked", (False, True))
@pytest.mark.parametrize("case", ATTENTION)
def test_scores_that_pass_the_base(sq, case, masked):
    """One state far above those before, in the second, third and last tile of states and in each half of a lane pair, by 2^10 (which sums
    bear), 2^20 and thousands (which they do not); masked: every other query does not see it."""
    (n, lq, lk, heads, kv, d), dt, (q, k, v), seen = attention_case(sq, case, 3)
    step = 32 if dt == F32 else 64
    q = q.abs() + 0.5
    for at in sorted(i for i in {step + 1, step + 4, 2 * step + 1, lk - 1} if i < lk):
        mask = None
        if masked:
            mask = seen.clone()
            mask[:, 1::2, at] = False
        for size in (7.0, 14.0, 2500.0):
            kj = k.clone()
            kj[:, at] = size / (1.3 * math.sqrt(d))
            ref, bound = reference64(q, kj, v, heads, kv, d ** -0.5, seen if mask is None else mask, dt)
            close(sq.sq_cross_attention_forward(q, kj, v, heads, kv, mask=mask), ref, bound, (at, size))


@pytest.mark.parametrize("case", ATTENTION)
def test_scores_that_rise_and_fall(sq, case):
    """By 2^18 and more from tile to tile, so that every tile raises the base or adds nothing."""
    (n, lq, lk, heads, kv, d), dt, (q, k, v), seen = attention_case(sq, case, 4)
    q = torch.ones_like(q)
    for slope in (0.25, -0.25, 0.5):
        ramp = ((torch.arange(lk, device="cuda") - lk / 2) * slope)[None, :, None]
        kr = torch.zeros((n, lk, kv, d), device="cuda")
        kr[..., 0] = ramp
        kr = kr.reshape(n, lk, -1).to(dt)
        ref, bound = reference64(q, kr, v, heads, kv, 1.0, seen, dt)
        close(sq.sq_cross_attention_forward(q, kr, v, heads, kv, scale=1.0), ref, bound, slope)


@pytest.mark.parametrize("scale", (0.0, -0.125, 3.0, 1e-30))
@pytest.mark.parametrize("case", ATTENTION)
def test_scales(sq, case, scale):
    (n, lq, lk, heads, kv, d), dt, (q, k, v), seen = attention_case(sq, case, 5)
    mask = (torch.rand((n, lk), generator=gen(6)) < 0.7).cuda()
    ref, bound = reference64(q, k, v, heads, kv, scale, seen & mask[:, None], dt)
    close(sq.sq_cross_attention_forward(q, k, v, heads, kv, scale=scale, mask=mask), ref, bound, scale)


@pytest.mark.parametrize("size", (1e30, 1e18, 1e-15))
@pytest.mark.parametrize("case", [c for c in ATTENTION if c[0] == plans.F32])
def test_fp32_magnitudes(sq, case, size):
    (n, lq, lk, heads, kv, d), dt, (q, k, v), seen = attention_case(sq, case, 7)
    q, k, v = q * size, k / size, v * size
    ref, bound = reference64(q, k, v, heads, kv, d ** -0.5, seen, dt)
    close(sq.sq_cross_attention_forward(q, k, v, heads, kv), ref, bound, size)


@pytest.mark.parametrize("pad", (1, 8))
@pytest.mark.parametrize("case", ATTENTION)
def test_slices_in_place(sq, case, pad):
    """Slices of wider rows at odd and whole addresses, the result over q; the rest of the rows is neither read nor written."""
    (n, lq, lk, heads, kv, d), dt, (q, k, v), seen = attention_case(sq, case, 8)
    ref, bound = reference64(q, k, v, heads, kv, d ** -0.5, seen, dt)
    qw = torch.full((n, lq, 2 * pad + heads * d), math.nan, dtype=dt, device="cuda")
    kvw = torch.full((n, lk, 2 * pad + 2 * kv * d), math.nan, dtype=dt, device="cuda")
    qv, kk, vv = qw[..., pad:pad + heads * d], kvw[..., pad:pad + kv * d], kvw[..., pad + kv * d:pad + 2 * kv * d]
    qv.copy_(q), kk.copy_(k), vv.copy_(v)
    sq.sq_cross_attention_forward(qv, kk, vv, heads, kv, out=qv)
    close(qv, ref, bound, pad)
    assert qw[..., :pad].isnan().all() and qw[..., pad + heads * d:].isnan().all()


# ------------------------------------------------------------------------------------------------ products of 4-bit rows
def values(sq, x):
    """What packed rows stand for (packing is compared bit by bit with its definition elsewhere)."""
    return sq.sq_mxfp4_unpack(sq.sq_mxfp4_pack(x), *x.shape).double()


def product64(sq, x, w, b, act, res, dt):
    X, W = values(sq, x), values(sq, w)
    y, size = X @ W.t(), X.abs() @ W.abs().t()
    if b is not None:
        y, size = y + b.double(), size + b.double().abs()
    bound = (x.shape[1] + 16) * 2 * U * size
    a = act64(y, act)
    if act:
        bound = 1.13 * bound + 8 * U * y.abs()
    if res is not None:
        a = a + res.double()
        bound = bound + U * a.abs()
    eps = torch.finfo(dt)
    return a, bound * (1 + eps.eps) + eps.eps / 2 * a.abs() * (1 + 1e-6) + eps.smallest_normal


@pytest.mark.parametrize("dt,odt", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("case", list(plans.TILINGS))
def test_product(sq, case, dt, odt):
    """Every tiling: activations, bias, blocks that are NaN, from rows as they are and packed before, then over its residual in a wider map."""
    assert plans.product_form(sq.lib, case) == plans.TILINGS[case]
    rows, cin, cout = case
    print(case, dt, odt, flush=True)
    act = (rows + cin + cout) % 4
    x, w = spread(rows, cin, 1).to(dt).cuda(), (torch.randn((cout, cin), generator=gen(2)) * math.sqrt(2 / cin)).to(dt).cuda()
    x[rows // 2, cin - 1], x[rows - 1, 0], w[cout // 3, 0], w[cout - 1, cin - 1] = math.nan, math.inf, math.inf, math.nan
    b = torch.randn(cout, generator=gen(3)).cuda() if dt == odt else None
    res = torch.randn((rows, cout), generator=gen(4)).to(odt).cuda()
    pw, px = sq.sq_mxfp4_pack(w), sq.sq_mxfp4_pack(x)
    ref, bound = product64(sq, x, w, b, act, None, odt)
    assert int(ref.isnan().sum()) == 2 * rows + 2 * cout - 4
    got = sq.sq_mxfp4_linear_forward(x, pw, cout, b, act=act, out_dtype=odt)
    close(got, ref, bound, "as they are")
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(sq.sq_mxfp4_linear_forward(px, pw, cout, b, act=act, out_dtype=odt, rows=rows, Cin=cin)))
    ref, bound = product64(sq, x, w, b, act, res, odt)
    wide = torch.full((rows, cout + 9), 7.0, dtype=odt, device="cuda")
    view = wide[:, 3:3 + cout]
    view.copy_(res)
    sq.sq_mxfp4_linear_forward(px, pw, cout, b, act=act, residual=view, out=view, rows=rows, Cin=cin)
    close(view, ref, bound, "over the residual")
    assert (wide[:, :3] == 7).all() and (wide[:, 3 + cout:] == 7).all()


@pytest.mark.parametrize("case", [(515, 40, 2000), (1030, 40, 2000), (2000, 40, 2050), (2000, 40, 4100)])
def test_far_magnitudes(sq, case):
    """Blocks near the ends of the powers of two in tiles: products that fp32 holds come out, larger ones are infinite."""
    assert plans.product_form(sq.lib, case) == plans.TILINGS[case]
    rows, cin, cout = case
    x = torch.full((rows, cin), 3.0, device="cuda")
    x[::2] *= 2.0 ** -120
    x[1::2] *= 2.0 ** 100
    w = torch.full((cout, cin), 2.0, device="cuda")
    w[::2] *= 2.0 ** 100
    w[1::2] *= 2.0 ** -100
    got = sq.sq_mxfp4_linear_forward(x, sq.sq_mxfp4_pack(w), cout).double()
    want = values(sq, x) @ values(sq, w).t()
    assert torch.equal(got[::2, ::2], want[::2, ::2]) and torch.equal(got[1::2, 1::2], want[1::2, 1::2])
    assert got[1::2, ::2].isinf().all() and (got[::2, 1::2].abs() <= 2.0 ** -126).all()


def test_packing_by_the_call_in_graphs_and_on_streams(sq):
    """Rows packed into a workspace: captured and replayed between eager calls that pack other rows, and on two streams at once."""
    cases = []
    for seed, (rows, cin, cout) in enumerate(((515, 1000, 515), (1030, 40, 2000), (2000, 40, 2050), (2000, 40, 4100))):
        need = sq.sq_mxfp4_linear_workspace_bytes(rows, cin, cout, BF16)
        assert need > 0
        x, w = spread(rows, cin, seed).to(BF16).cuda(), sq.sq_mxfp4_pack(torch.randn((cout, cin), generator=gen(seed)).cuda())
        cases.append((x, w, cout, torch.empty(need, dtype=torch.uint8, device="cuda"), torch.empty((rows, cout), dtype=BF16, device="cuda"),
                      sq.sq_mxfp4_linear_forward(x, w, cout, act=2), sq.sq_mxfp4_linear_forward(-2 * x, w, cout, act=2)))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for x, w, cout, ws, out, *_ in cases:
            sq.sq_mxfp4_linear_forward(x, w, cout, act=2, out=out, workspace=ws)
    for turn in range(4):
        for x, w, cout, ws, out, *_ in cases:
            out.zero_()
            ws.fill_(255)
        if turn % 2:
            for c in cases:
                c[0].mul_(-2)
        graph.replay()
        eager = [sq.sq_mxfp4_linear_forward(x, w, cout, act=2) for x, w, cout, *_ in cases]
        torch.cuda.synchronize()
        for c, e in zip(cases, eager):
            want = c[5 + turn % 2]
            assert torch.equal(c[4], want) and torch.equal(e, want)
        if turn % 2:
            for c in cases:
                c[0].mul_(-0.5)
    streams, results = [torch.cuda.Stream() for _ in cases], []
    torch.cuda.synchronize()
    for turn in range(4):
        for s, c in zip(streams, cases):
            with torch.cuda.stream(s):
                results.append((sq.sq_mxfp4_linear_forward(c[0], c[1], c[2], act=2), c[5]))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in results)
