"""Attention to an encoder's states against its definition in 64 bits.

u = 2^-24.  With S = the largest scale * sum_d |q_d||k_d| over the states that a query sees and A = sum p|v| / sum p:
  a score is off by (D + 2) 2u S (fp32 sums of exact or rounded products, the matrix unit's additions off by up to 2u), its exponent in base
  two and the maximum's by another 4u S each (the product with scale log2 e, the difference), the exponential itself by 2u: a p is off by
  a relative E = (2 D + 24) u S + 8u against its maximum's;
  a maximum that is raised, or sums of shares that are joined, cost 8u S + 8u each time, at most once every 32 states and once a share:
  R = (Lk / 32 + 65) (8u S + 8u);
  sums of up to Lk terms: (Lk + 16) 2u;
  bfloat16: p is rounded before it multiplies v, half a step, 2^-8, and the rounded ones may be what is added up: sum p' v / sum p' - out =
  sum (p' - p) (v - out) / sum p', at most 2^-8 sum p |v - out| / sum p' <= 2^-8 (1 + 2^-7) (A + |out|);
  so A 2 (E + R + (Lk + 16) 2u) + [2^-8 (1 + 2^-7) (A + |out|)] + 8u |out| for the numerator, the denominator and their quotient, and half a
  step of the type.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24


@pytest.fixture(scope="module")
def sq():
    import paper_1611_07151_amd as m
    m.sq_init()
    return m


def gen(seed):
    return torch.Generator().manual_seed(seed)


def reference(q, k, v, heads, kv_heads, scale, seen, dt):
    """Result [n][lq][heads * d] in 64 bits and its bound.  seen: bool [n][lq][lk]."""
    n, lq, _ = q.shape
    lk, d = k.shape[1], k.shape[2] // kv_heads
    group = heads // kv_heads
    q = q.double().reshape(n, lq, heads, d).permute(0, 2, 1, 3)
    k, v = (t.double().reshape(n, lk, kv_heads, d).permute(0, 2, 1, 3).repeat_interleave(group, 1) for t in (k, v))
    m = seen[:, None]
    zero = torch.zeros((), dtype=torch.float64, device=q.device)
    s = torch.where(m, scale * (q @ k.transpose(2, 3)), zero - math.inf)
    big = torch.where(m, abs(scale) * (q.abs() @ k.abs().transpose(2, 3)), zero)
    big = big.amax(3, keepdim=True) if lk else torch.zeros(n, heads, lq, 1, dtype=torch.float64, device=q.device)
    top = s.amax(3, keepdim=True) if lk else torch.full((n, heads, lq, 1), -math.inf, dtype=torch.float64, device=q.device)
    p = torch.exp(s - torch.where(top == -math.inf, zero, top))
    total = p.sum(3, keepdim=True)
    safe = torch.where(total == 0, zero + 1, total)
    out, a = p @ v / safe, p @ v.abs() / safe
    e = (2 * d + 24) * U * big + 8 * U
    r = (lk / 32 + 65) * (8 * U * big + 8 * U)
    eps = torch.finfo(dt)
    bound = a * 2 * (e + r + (lk + 16) * 2 * U) + (2.0 ** -8 * (1 + 2.0 ** -7) * (a + out.abs()) if dt == BF16 else 0) + 8 * U * out.abs()
    bound = bound * (1 + eps.eps) + eps.eps / 2 * out.abs() * (1 + 1e-6) + eps.smallest_normal
    back = lambda t: t.permute(0, 2, 1, 3).reshape(n, lq, heads * d)
    return back(out), back(bound)


def check(got, ref, bound, what):
    got = got.cpu().double()
    err = (got - ref).abs()
    bad = ~(err <= bound)
    assert not bad.any(), (what, int(bad.sum()), float(err.max()), float((err / bound).nan_to_num(0).max()))


def inputs(n, lq, lk, heads, kv_heads, d, dt, seed, spread=1.0):
    g = gen(seed)
    q = (torch.randn((n, lq, heads * d), generator=g) * spread).to(dt)
    return q, torch.randn((n, lk, kv_heads * d), generator=g).to(dt), torch.randn((n, lk, kv_heads * d), generator=g).to(dt)


def everything(n, lq, lk):
    return torch.ones((n, lq, lk), dtype=torch.bool)


SIZES = [(1, 1, 1, 1, 1, 1), (1, 1, 2, 1, 1, 3), (2, 1, 31, 2, 2, 8), (1, 3, 32, 3, 3, 25), (2, 2, 33, 4, 2, 32), (1, 31, 63, 2, 1, 33), (3, 33, 64, 2, 2, 40),
         (1, 127, 65, 1, 1, 64), (1, 128, 77, 2, 2, 64), (2, 129, 77, 8, 8, 48), (1, 300, 129, 4, 4, 80), (2, 65, 200, 6, 2, 96), (1, 40, 333, 2, 2, 100),
         (1, 17, 1000, 8, 2, 128), (1, 5, 257, 2, 1, 130), (1, 64, 96, 1, 1, 160), (1, 33, 300, 2, 2, 200), (1, 70, 130, 1, 1, 256), (2, 1, 5000, 4, 1, 64),
         (1, 1, 4097, 16, 2, 128), (3, 1, 729, 8, 8, 64), (1, 9, 3000, 2, 2, 25), (2, 1, 2048, 3, 3, 256), (1, 2, 1500, 12, 12, 72), (16, 50, 20, 16, 16, 16),
         (1, 1, 700, 40, 1, 64), (1, 16, 900, 1, 1, 31), (1, 700, 64, 1, 1, 128), (5, 260, 300, 5, 5, 64)]


@pytest.mark.parametrize("dt", (F32, BF16))
@pytest.mark.parametrize("n,lq,lk,heads,kv,d", SIZES)
def test_sizes(sq, n, lq, lk, heads, kv, d, dt):
    print(n, lq, lk, heads, kv, d, dt, flush=True)
    q, k, v = inputs(n, lq, lk, heads, kv, d, dt, lq + lk + d)
    ref, bound = reference(q, k, v, heads, kv, d ** -0.5, everything(n, lq, lk), dt)
    q, k, v = q.cuda(), k.cuda(), v.cuda()
    got = sq.sq_cross_attention_forward(q, k, v, heads, kv)
    assert got.shape == q.shape and got.dtype == dt
    check(got, ref, bound, (n, lq, lk, heads, kv, d))
    assert torch.equal(got, sq.sq_cross_attention_forward(q, k, v, heads, kv))


@pytest.mark.parametrize("dt", (F32, BF16))
@pytest.mark.parametrize("n,lq,lk,heads,kv,d", [(5, 1, 100, 4, 2, 64), (5, 40, 77, 2, 2, 48), (5, 1, 3000, 2, 2, 128), (5, 200, 300, 3, 1, 33), (5, 3, 130, 8, 8, 25)])
@pytest.mark.parametrize("kind", ("lengths", "states", "pairs", "pairs and lengths", "shared pairs"))
def test_masks(sq, n, lq, lk, heads, kv, d, dt, kind):
    """Images and queries that see nothing, one state, everything; hidden places hold NaN and infinities."""
    print(n, lq, lk, heads, kv, d, dt, kind, flush=True)
    g = gen(lq + lk)
    q, k, v = inputs(n, lq, lk, heads, kv, d, dt, lk + d)
    lengths = torch.tensor([0, 1, lk, lk // 2 + 1, -3], dtype=torch.int32) if "lengths" in kind else None
    mask, seen = None, everything(n, lq, lk)
    if lengths is not None:
        seen &= torch.arange(lk) < lengths[:, None, None]
    if kind == "states":
        mask = torch.rand((n, lk), generator=g) < 0.6
        mask[0], mask[1], mask[2], mask[3] = False, True, False, False
        mask[2, lk - 1] = mask[3, 0] = True
        seen = seen & mask[:, None]
    elif "pairs" in kind:
        mask = torch.rand((1 if kind == "shared pairs" else n, lq, lk), generator=g) < 0.6
        mask[:, lq // 2], mask[:, 0, :lk - 1] = False, False
        mask[-1, lq - 1] = True
        mask[:, :, lk // 3] = False
        mask = mask.expand(n, lq, lk)
        seen = seen & mask
    hidden = ~seen.any(1)          # states that no query of the image sees
    ref, bound = reference(q, k, v, heads, kv, d ** -0.5, seen, dt)
    args = dict(lengths=None if lengths is None else lengths.cuda(), mask=None if mask is None else mask.cuda() if mask.is_contiguous() else mask[:1].cuda().expand(n, lq, lk))
    plain = sq.sq_cross_attention_forward(q.cuda(), k.cuda(), v.cuda(), heads, kv, **args)
    check(plain, ref, bound, kind)
    assert (plain.cpu()[~seen.any(2)] == 0).all()
    for bad in (math.nan, math.inf, torch.finfo(dt).max, -math.inf):
        kb, vb = k.clone(), v.clone()
        kb[hidden], vb[hidden] = bad, bad
        check(sq.sq_cross_attention_forward(q.cuda(), kb.cuda(), vb.cuda(), heads, kv, **args), ref, bound, (kind, bad))


@pytest.mark.parametrize("dt", (F32, BF16))
@pytest.mark.parametrize("lq,lk", [(40, 150), (1, 2500), (7, 64)])
def test_a_bad_state_reaches_those_who_see_it_alone(sq, lq, lk, dt):
    n, heads, d = 2, 2, 64
    q, k, v = inputs(n, lq, lk, heads, heads, d, dt, 3)
    mask = torch.ones((n, lq, lk), dtype=torch.bool)
    at = lk // 2
    mask[0, ::2, at] = False
    ref, bound = reference(q, k, v, heads, heads, d ** -0.5, mask, dt)
    for which in "kv":
        kb, vb = k.clone(), v.clone()
        (kb if which == "k" else vb)[0, at, :d] = math.nan        # of the first head
        got = sq.sq_cross_attention_forward(q.cuda(), kb.cuda(), vb.cuda(), heads, mask=mask.cuda()).cpu()
        struck = torch.zeros_like(got, dtype=torch.bool)
        struck[0, 1::2, :d] = True
        assert got[struck].isnan().all()
        check(torch.where(struck, torch.zeros_like(got), got), torch.where(struck, torch.zeros_like(ref), ref), bound, which)


@pytest.mark.parametrize("dt", (F32, BF16))
@pytest.mark.parametrize("scale", (0.0, -0.125, 1.0, 3.0, 1e-30))
def test_scales(sq, dt, scale):
    n, lq, lk, heads, d = 2, 37, 200, 2, 64
    q, k, v = inputs(n, lq, lk, heads, heads, d, dt, 5)
    mask = torch.rand((n, lk), generator=gen(6)) < 0.7
    ref, bound = reference(q, k, v, heads, heads, scale, mask[:, None].expand(n, lq, lk), dt)
    for rows in (slice(0, lq), slice(0, 1)):
        got = sq.sq_cross_attention_forward(q[:, rows].cuda().contiguous(), k.cuda(), v.cuda(), heads, scale=scale, mask=mask.cuda())
        check(got, ref[:, rows], bound[:, rows], scale)


@pytest.mark.parametrize("dt", (F32, BF16))
def test_far_scores(sq, dt):
    """Scores of some thousands, rising, falling and equal along the states: the running maximum at every turn."""
    n, lq, lk, d = 1, 5, 500, 32
    for order in (1, -1, 0):
        q = torch.ones((n, lq, d)).to(dt)
        ramp = (torch.arange(lk) - lk / 2) * order * 0.25
        k = ramp[None, :, None].expand(n, lk, d).contiguous().to(dt)
        v = torch.randn((n, lk, d), generator=gen(8)).to(dt)
        ref, bound = reference(q, k, v, 1, 1, 1.0, everything(n, lq, lk), dt)
        check(sq.sq_cross_attention_forward(q.cuda(), k.cuda(), v.cuda(), 1, scale=1.0), ref, bound, order)
        check(sq.sq_cross_attention_forward(q[:, :1].cuda(), k.cuda(), v.cuda(), 1, scale=1.0), ref[:, :1], bound[:, :1], order)


@pytest.mark.parametrize("dt", (F32, BF16))
@pytest.mark.parametrize("lq,lk,heads,kv,d,pad", [(30, 77, 2, 2, 40, 8), (1, 600, 4, 2, 64, 5), (140, 90, 2, 1, 25, 3), (1, 2000, 2, 2, 48, 1)])
def test_slices_in_place_and_the_rest_of_the_rows(sq, lq, lk, heads, kv, d, pad, dt):
    """q, k and v as slices of wider rows at odd addresses, the result over q; the rest of the rows is neither read nor written."""
    n = 2
    q, k, v = inputs(n, lq, lk, heads, kv, d, dt, 7)
    ref, bound = reference(q, k, v, heads, kv, d ** -0.5, everything(n, lq, lk), dt)
    qw = torch.full((n, lq, pad + heads * d + pad), math.nan, dtype=dt, device="cuda")
    kvw = torch.full((n, lk, pad + 2 * kv * d + 1), math.nan, dtype=dt, device="cuda")
    qv, kk, vv = qw[..., pad:pad + heads * d], kvw[..., pad:pad + kv * d], kvw[..., pad + kv * d:pad + 2 * kv * d]
    qv.copy_(q), kk.copy_(k), vv.copy_(v)
    sq.sq_cross_attention_forward(qv, kk, vv, heads, kv, out=qv)
    check(qv, ref, bound, (lq, lk))
    assert qw[..., :pad].isnan().all() and qw[..., pad + heads * d:].isnan().all()


def test_maps_as_queries(sq):
    """A channels-last map [N][H][W][C] is its pixels."""
    q, k, v = inputs(2, 63, 50, 4, 4, 32, BF16, 9)
    flat = sq.sq_cross_attention_forward(q.cuda(), k.cuda(), v.cuda(), 4)
    m = sq.sq_cross_attention_forward(q.cuda().reshape(2, 7, 9, 128), k.cuda().reshape(2, 5, 10, 128), v.cuda().reshape(2, 5, 10, 128), 4)
    assert m.shape == (2, 7, 9, 128) and torch.equal(m.reshape(2, 63, 128), flat)


@pytest.mark.parametrize("lq", (1, 200))
def test_no_states(sq, lq):
    for dt in (F32, BF16):
        q = torch.randn((2, lq, 64), generator=gen(1)).to(dt).cuda()
        k = q.new_empty((2, 0, 64))
        assert (sq.sq_cross_attention_forward(q, k, k, 2, out=torch.full_like(q, math.nan)) == 0).all()


@pytest.mark.parametrize("lq", (1, 150))
def test_states_past_32_bits(sq, lq):
    """States whose offsets pass 2^32 bytes, and a mask behind 2^31 bytes."""
    n, lk, d, ld = 2, 700, 64, 2 ** 21 + 8
    q, k, v = inputs(n, lq, lk, 1, 1, d, BF16, 10)
    wide = torch.empty((n, lk, ld), dtype=BF16, device="cuda")
    kk, vv = wide[..., 100:100 + d], wide[..., -d:]
    kk.copy_(k), vv.copy_(v)
    mask = torch.rand((n, lq, lk), generator=gen(11)) < 0.7
    room = torch.zeros(2 ** 31 + 2 ** 20 + lq * lk, dtype=torch.uint8, device="cuda")
    far = room.as_strided((n, lq, lk), (2 ** 31 + 2 ** 20, lk, 1))
    far.copy_(mask)
    ref, bound = reference(q, k, v, 1, 1, d ** -0.5, mask, BF16)
    check(sq.sq_cross_attention_forward(q.cuda(), kk, vv, 1, mask=far), ref, bound, lq)


def test_graph_streams_and_workspaces(sq):
    """Captured with workspaces of their own and replayed between eager calls; two streams at once."""
    cases = []
    for n, lq, lk, heads, kv, d in ((2, 1, 3000, 8, 2, 128), (1, 300, 200, 4, 4, 64), (1, 20, 4000, 2, 2, 40)):
        q, k, v = (t.cuda() for t in inputs(n, lq, lk, heads, kv, d, BF16, 12))
        ws = torch.empty(max(1, sq.sq_cross_attention_workspace_bytes(n, lq, lk, heads, kv, d, BF16)), dtype=torch.uint8, device="cuda")
        cases.append((q, k, v, heads, kv, ws, torch.empty_like(q), sq.sq_cross_attention_forward(q, k, v, heads, kv)))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for q, k, v, heads, kv, ws, out, _ in cases:
            sq.sq_cross_attention_forward(q, k, v, heads, kv, out=out, workspace=ws)
    for turn in range(3):
        for c in cases:
            c[6].zero_()
            c[5].fill_(255)
        graph.replay()
        eager = [sq.sq_cross_attention_forward(*c[:5]) for c in cases]
        torch.cuda.synchronize()
        for c, e in zip(cases, eager):
            assert torch.equal(c[6], c[7]) and torch.equal(e, c[7])
    streams, results = [torch.cuda.Stream() for _ in cases], []
    for turn in range(4):
        for s, c in zip(streams, cases):
            with torch.cuda.stream(s):
                results.append((sq.sq_cross_attention_forward(*c[:5]), c[7]))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in results)


@pytest.mark.parametrize("n,lq,lk,heads,kv,d,dt,kind", [(8, 1025, 200, 8, 8, 64, BF16, "none"), (8, 1025, 200, 8, 8, 64, BF16, "states"), (8, 1025, 200, 8, 8, 64, BF16, "pairs"),
                                                       (8, 1030, 130, 8, 4, 30, BF16, "pairs"), (8, 1030, 130, 8, 4, 30, BF16, "none"), (4, 600, 300, 8, 8, 96, F32, "states"),
                                                       (4, 700, 200, 8, 8, 128, BF16, "lengths")])
def test_many_rows(sq, n, lq, lk, heads, kv, d, dt, kind):
    """Enough rows for the widest blocks; the reference in 64 bits on the GPU."""
    print(n, lq, lk, heads, kv, d, dt, kind, flush=True)
    q, k, v = inputs(n, lq, lk, heads, kv, d, dt, 21)
    seen, mask, lengths = everything(n, lq, lk), None, None
    if kind == "lengths":
        lengths = torch.tensor([lk, 0, 65, 1], dtype=torch.int32)
        seen = (torch.arange(lk) < lengths[:, None])[:, None].expand(n, lq, lk)
    elif kind == "states":
        mask = torch.rand((n, lk), generator=gen(22)) < 0.5
        mask[1] = False
        seen = mask[:, None].expand(n, lq, lk)
    elif kind == "pairs":
        mask = torch.rand((n, lq, lk), generator=gen(22)) < 0.5
        mask[:, ::7] = False
        seen = mask
    cuda = lambda t: None if t is None else t.cuda()
    ref, bound = reference_on_gpu(q, k, v, heads, kv, d ** -0.5, seen, dt)
    got = sq.sq_cross_attention_forward(q.cuda(), k.cuda(), v.cuda(), heads, kv, mask=cuda(mask), lengths=cuda(lengths))
    check(got, ref, bound, kind)
    assert torch.equal(got, sq.sq_cross_attention_forward(q.cuda(), k.cuda(), v.cuda(), heads, kv, mask=cuda(mask), lengths=cuda(lengths)))


def reference_on_gpu(q, k, v, heads, kv_heads, scale, seen, dt):
    parts = [reference(*(t[i:i + 1].cuda() for t in (q, k, v)), heads, kv_heads, scale, seen[i:i + 1].cuda(), dt) for i in range(q.shape[0])]
    return torch.cat([r.cpu() for r, _ in parts]), torch.cat([b.cpu() for _, b in parts])


@pytest.mark.parametrize("lq", (1, 300))
@pytest.mark.parametrize("size", (1e30, 1e18, 1e-15))
def test_fp32_magnitudes(sq, lq, size):
    """fp32 values as large and small as they come, with scores that stay ordinary: every value keeps its own accuracy."""
    n, lk, heads, d = 1, 170, 2, 64
    q, k, v = inputs(n, lq, lk, heads, heads, d, F32, 23)
    q, k, v = q * size, k / size, v * size
    ref, bound = reference(q, k, v, heads, heads, d ** -0.5, everything(n, lq, lk), F32)
    check(sq.sq_cross_attention_forward(q.cuda(), k.cuda(), v.cuda(), heads), ref, bound, size)


@pytest.mark.parametrize("dt", (F32, BF16))
@pytest.mark.parametrize("lq", (1, 200))
def test_scores_that_jump(sq, lq, dt):
    """A state far above all before it, in every place of a tile, and one that only some queries see."""
    n, lk, d = 1, 300, 64
    for at in (0, 1, 31, 32, 63, 64, 127, 199, 299):
        q, k, v = inputs(n, lq, lk, 1, 1, d, dt, 24)
        q[:] = q.abs() + 0.5
        k[:, at] = 40.0
        mask = torch.ones((n, lq, lk), dtype=torch.bool)
        mask[:, 1::2, at] = False
        ref, bound = reference(q, k, v, 1, 1, 1.0, mask, dt)
        check(sq.sq_cross_attention_forward(q.cuda(), k.cuda(), v.cuda(), 1, scale=1.0, mask=mask.cuda()), ref, bound, at)
        ref, bound = reference(q, k, v, 1, 1, 1.0, everything(n, lq, lk), dt)
        check(sq.sq_cross_attention_forward(q.cuda(), k.cuda(), v.cuda(), 1, scale=1.0), ref, bound, at)


@pytest.mark.parametrize("lq", (1, 90))
def test_block(sq, lq):
    """The operators as a network runs them: group norm, projections in 4 bits, attention to states of other lengths, projection back
    onto the map.  Every step against its definition on what the step before gave."""
    n, c, states, heads, lk = 2, 256, 96, 4, 77
    g = gen(13)
    m = torch.randn((n, 1, lq, c), generator=g).to(BF16).cuda()
    enc = torch.randn((n, lk, states), generator=g).to(BF16).cuda()
    w = {k: (torch.randn(s, generator=g) / math.sqrt(s[1])).to(BF16).cuda() for k, s in (("q", (c, c)), ("kv", (2 * c, states)), ("o", (c, c)))}
    lengths = torch.tensor([lk, 30], dtype=torch.int32).cuda()
    packed = {k: sq.sq_mxfp4_pack(t) for k, t in w.items()}
    norm = sq.sq_nhwc_group_norm(m, 32)
    q = sq.sq_mxfp4_linear_forward(norm, packed["q"], c)
    kv = sq.sq_mxfp4_linear_forward(enc, packed["kv"], 2 * c)
    a = sq.sq_cross_attention_forward(q, kv[..., :c], kv[..., c:], heads, lengths=lengths)
    out = sq.sq_mxfp4_linear_forward(a, packed["o"], c, residual=m)

    def project(x, name, res=None):
        flat = x.reshape(-1, x.shape[-1])
        X = sq.sq_mxfp4_unpack(sq.sq_mxfp4_pack(flat), *flat.shape).double()
        W = sq.sq_mxfp4_unpack(packed[name], *w[name].shape).double()
        y, size = X @ W.t(), X.abs() @ W.abs().t()
        y = y if res is None else y + res.reshape(-1, y.shape[1]).double()
        return y, (X.shape[1] + 16) * 2 * U * size * 1.01 + U * y.abs() + 2.0 ** -8 * y.abs() * 1.000001 + 2.0 ** -126

    for got, (ref, bound) in ((q, project(norm, "q")), (kv, project(enc, "kv")), (out, project(a, "o", m))):
        check(got.reshape(ref.shape), ref.cpu(), bound.cpu(), "projection")
    seen = (torch.arange(lk) < lengths.cpu()[:, None])[:, None].expand(n, lq, lk)
    ref, bound = reference(q.cpu().reshape(n, lq, c), kv.cpu()[..., :c], kv.cpu()[..., c:], heads, heads, (c // heads) ** -0.5, seen, BF16)
    check(a.reshape(n, lq, c), ref, bound, "attention")


def test_refusals_of_the_binding(sq):
    q = torch.zeros(2, 5, 64, device="cuda")
    k = torch.zeros(2, 9, 32, device="cuda")
    f = sq.sq_cross_attention_forward
    for call in (lambda: f(q, k, k, 4), lambda: f(q, k, k[:, :8], 4, 2), lambda: f(q, k.bfloat16(), k.bfloat16(), 4, 2), lambda: f(q.half(), k.half(), k.half(), 4, 2),
                 lambda: f(q, k[:1], k[:1], 4, 2), lambda: f(q, k.cpu(), k.cpu(), 4, 2), lambda: f(q, k, k, 4, 2, lengths=torch.zeros(3, dtype=torch.int32, device="cuda")),
                 lambda: f(q, k, k, 4, 2, lengths=torch.zeros(2, dtype=torch.int64, device="cuda")), lambda: f(q, k, k, 4, 2, mask=torch.ones(2, 5, device="cuda") > 0),
                 lambda: f(q, k, k, 4, 2, mask=torch.ones(2, 9, device="cuda")), lambda: f(q, k, k, 4, 2, mask=(torch.ones(9, 2, device="cuda") > 0).t()),
                 lambda: f(q, k, k, 4, 2, out=q[:, :4]), lambda: f(q, k.transpose(0, 1).contiguous().transpose(0, 1), k, 4, 2)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: f(q, k, k, 4, 3), lambda: f(q, k, k, 0), lambda: f(q, k, k, 4, 2, scale=math.inf), lambda: f(q[:, :0], k, k, 4, 2)):
        with pytest.raises(sq.SqError):
            call()
