"""Attention to an encoder's states where scores or sums pass the range of fp32, in every form of the kernels (few rows and tiles, one
workgroup or several for a row's states), against its definition in 64 bits.

Scores here are whole multiples of one power of two that bfloat16 and fp32 operands give exactly, so that which state is a query's largest is
certain, and with a gap of at least 200 in the exponent all others weigh exactly nothing: the result is that state's values, once weighted and
once divided.  fp32: a weight off by 4u (u = 2^-24; three pieces: products off by 2u more), the quotient by 2u, the fp32 sum with zeros by
none: 16u |v|.  bfloat16: the weight is rounded to half a step, 2^-8, and the result to half a step.
"""
import math

import pytest
import torch

from test_cross_attention_gpu import check, everything, gen, inputs, reference_on_gpu

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24


@pytest.fixture(scope="module")
def sq():
    import paper_1611_07151_amd as m
    m.sq_init()
    return m


# n, lq, lk, heads, kv_heads, d
FORMS = [(F32, 1, 5, 200, 2, 1, 64), (F32, 1, 1, 300, 1, 1, 100), (F32, 1, 1030, 130, 8, 8, 64), (F32, 1, 1030, 300, 4, 2, 33), (F32, 1, 1030, 65, 16, 16, 160),
         (F32, 3, 1, 1000, 8, 8, 25), (BF16, 1, 5, 300, 2, 1, 64), (BF16, 1, 1, 1000, 1, 1, 100), (BF16, 1, 700, 300, 8, 8, 64), (BF16, 8, 500, 130, 16, 16, 64),
         (BF16, 2, 2000, 130, 32, 8, 64), (BF16, 4, 1000, 150, 32, 8, 30),
         (BF16, 1, 1030, 1000, 4, 2, 40), (BF16, 1, 1030, 130, 8, 8, 160), (BF16, 2, 70, 200, 4, 4, 59)]


def levels(n, lq, lk, heads, kv, d, dt, unit_q, unit_k, shift, seed):
    """q, k, v, and the exact scores [n][lq][lk] of every head in units of unit_q * unit_k: whole numbers, each state's different, raised by
    `shift`, the odd queries' negated."""
    g = gen(seed)
    order = torch.stack([torch.randperm(lk, generator=g) for _ in range(n)]) - lk // 2
    high, low = order // 16 * 16, order % 16
    k = torch.zeros((n, lk, kv, d))
    k[..., 0], k[..., 1], k[..., 2] = high[:, :, None].float(), low[:, :, None].float(), float(shift)
    q = torch.zeros((n, lq, heads, d))
    q[..., :3] = 1.0
    q[:, 1::2, :, :2] = -1.0
    v = torch.randn((n, lk, kv * d), generator=g).to(dt)
    sign = torch.ones(lq, dtype=torch.float64)
    sign[1::2] = -1
    score = sign[None, :, None] * order[:, None].double() + shift
    return ((q * unit_q).reshape(n, lq, -1).to(dt), (k * unit_k).reshape(n, lk, -1).to(dt), v, score)


def largest(v, score, seen, heads, kv, scale):
    """The values of the state with the largest scaled score among the seen; zeros where none is."""
    n, lk, _ = v.shape
    s = torch.where(seen, score * math.copysign(1.0, scale), torch.full_like(score, -math.inf))
    at = s.argmax(2)
    per = v.double().reshape(n, lk, kv, -1).repeat_interleave(heads // kv, 2).reshape(n, lk, -1)
    out = per.gather(1, at[..., None].expand(-1, -1, per.shape[2]))
    return torch.where(seen.any(2, keepdim=True), out, torch.zeros_like(out))


def bound_of(ref, dt):
    return ref.abs() * (16 * U if dt == F32 else 2 * 2.0 ** -8 * 1.01) + 2.0 ** -126


@pytest.mark.parametrize("scale", (1e10, -1e10, 1e20, 8.0e37, -2.0 ** 126))
@pytest.mark.parametrize("dt,n,lq,lk,heads,kv,d", FORMS)
@pytest.mark.parametrize("shift", (0, -2048, 2048))
def test_large_scales(sq, dt, n, lq, lk, heads, kv, d, shift, scale):
    """Scores of both signs, all below and all above zero, far past 2^24 and past the largest fp32 number."""
    print(dt, n, lq, lk, heads, kv, d, shift, scale, flush=True)
    q, k, v, score = levels(n, lq, lk, heads, kv, d, dt, 1.0, 1.0, shift, lk + d)
    ref = largest(v, score, everything(n, lq, lk), heads, kv, scale)
    check(sq.sq_cross_attention_forward(q.cuda(), k.cuda(), v.cuda(), heads, kv, scale=scale), ref, bound_of(ref, dt), (shift, scale))


@pytest.mark.parametrize("dt,n,lq,lk,heads,kv,d", FORMS)
@pytest.mark.parametrize("shift", (0, -2048))
@pytest.mark.parametrize("kind", ("none", "lengths", "states", "pairs"))
def test_products_past_the_range(sq, dt, n, lq, lk, heads, kv, d, shift, kind):
    """Products of queries and keys that are infinite in fp32, above or below; queries that see nothing still get zeros."""
    print(dt, n, lq, lk, heads, kv, d, shift, kind, flush=True)
    q, k, v, score = levels(n, lq, lk, heads, kv, d, dt, 2.0 ** 80, 2.0 ** 60, shift, lk + d)
    seen, mask, lengths = everything(n, lq, lk), None, None
    if kind == "lengths":
        lengths = torch.tensor([lk // 2 + 3] + [0] * (n - 1), dtype=torch.int32)
        seen = (torch.arange(lk) < lengths[:, None])[:, None].expand(n, lq, lk)
    elif kind == "states":
        mask = torch.rand((n, lk), generator=gen(3)) < 0.5
        mask[-1] = n == 1
        seen = mask[:, None].expand(n, lq, lk)
    elif kind == "pairs":
        mask = torch.rand((n, lq, lk), generator=gen(3)) < 0.5
        mask[:, lq // 2] = False
        mask[:, 0], mask[:, 0, lk // 3] = False, lq > 1
        seen = mask
    ref = largest(v, score, seen, heads, kv, 1.0)
    cuda = lambda t: None if t is None else t.cuda()
    got = sq.sq_cross_attention_forward(q.cuda(), k.cuda(), v.cuda(), heads, kv, scale=1.0, mask=cuda(mask), lengths=cuda(lengths))
    check(got, ref, bound_of(ref, dt), (shift, kind))


@pytest.mark.parametrize("dt,n,lq,lk,heads,kv,d", FORMS)
@pytest.mark.parametrize("masked", (False, True))
def test_ordinary_scores_of_products_past_the_range(sq, dt, n, lq, lk, heads, kv, d, masked):
    """Every product passes the range, the scaled scores are ordinary: a softmax of many weights."""
    print(dt, n, lq, lk, heads, kv, d, masked, flush=True)
    q, k, v = inputs(n, lq, lk, heads, kv, d, dt, 31)
    q[..., ::d], k[..., ::d] = 16.0, 16.0       # the same in every score: 2^8 * 2^70 * 2^60 is infinite
    q, k = (q.float() * 2.0 ** 70).to(dt), (k.float() * 2.0 ** 60).to(dt)
    mask = torch.rand((n, lk), generator=gen(32)) < 0.7 if masked else None
    seen = mask[:, None].expand(n, lq, lk) if masked else everything(n, lq, lk)
    scale = 2.0 ** -126 / 64
    ref, bound = reference_on_gpu(q, k, v, heads, kv, scale, seen, dt)
    check(sq.sq_cross_attention_forward(q.cuda(), k.cuda(), v.cuda(), heads, kv, scale=scale, mask=mask.cuda() if masked else None), ref, bound, masked)


@pytest.mark.parametrize("dt,n,lq,lk,heads,kv,d", FORMS)
def test_a_key_that_is_not_finite_beside_scores_past_the_range(sq, dt, n, lq, lk, heads, kv, d):
    """Results that a NaN key leaves undefined are NaN, never zeros."""
    print(dt, n, lq, lk, heads, kv, d, flush=True)
    q, k, v, score = levels(n, lq, lk, heads, kv, d, dt, 1.0, 1.0, -2048, 5)
    k[0, lk // 2] = math.nan
    got = sq.sq_cross_attention_forward(q.cuda(), k.cuda(), v.cuda(), heads, kv, scale=2.0 ** 126).cpu()
    assert got[0].isnan().all()
    ref = largest(v, score, everything(n, lq, lk), heads, kv, 1.0)
    check(got[1:], ref[1:], bound_of(ref[1:], dt), "others")


@pytest.mark.parametrize("dt,n,lq,lk,heads,kv,d", FORMS)
@pytest.mark.parametrize("masked", (False, True))
@pytest.mark.parametrize("jump", (False, True))
def test_values_whose_sums_pass_the_range(sq, dt, n, lq, lk, heads, kv, d, masked, jump):
    """Values up to 2^127 of either sign: every weighted mean is finite, sums of them are not.  jump: scores that stand far above those before,
    which sums are not yet brought down for."""
    print(dt, n, lq, lk, heads, kv, d, masked, jump, flush=True)
    q, k, v = inputs(n, lq, lk, heads, kv, d, dt, 41)
    if jump:
        q, k = q.abs(), k / 8
        k[:, lk // 2:] = k[:, lk // 2:].abs() + 0.25 * torch.rand((n, lk - lk // 2, 1), generator=gen(42)).to(dt)
    v = torch.where(torch.rand(v.shape, generator=gen(43)) < 0.9, 1.0, -1.0) * (v.float().abs() % 1 + 0.5) * 2.0 ** 126
    v[..., ::3] *= 2.0 ** -20
    v = v.to(dt)
    mask = torch.rand((n, lk), generator=gen(44)) < 0.7 if masked else None
    seen = mask[:, None].expand(n, lq, lk) if masked else everything(n, lq, lk)
    ref, bound = reference_on_gpu(q, k, v, heads, kv, d ** -0.5, seen, dt)
    check(sq.sq_cross_attention_forward(q.cuda(), k.cuda(), v.cuda(), heads, kv, mask=mask.cuda() if masked else None), ref, bound, (masked, jump))


@pytest.mark.parametrize("dt,n,lq,lk,heads,kv,d", FORMS)
def test_values_that_are_not_finite_stay_in_their_place(sq, dt, n, lq, lk, heads, kv, d):
    """Without a mask a NaN or infinite value makes those results NaN or infinite that it is part of, and leaves the others."""
    q, k, v = inputs(n, lq, lk, heads, kv, d, dt, 45)
    ref, bound = reference_on_gpu(q, k, v, heads, kv, d ** -0.5, everything(n, lq, lk), dt)
    bad = v.clone()
    bad[0, lk // 3, 0], bad[0, lk - 1, d // 2], bad[0, 0, d - 1] = math.nan, math.inf, -math.inf
    got = sq.sq_cross_attention_forward(q.cuda(), k.cuda(), bad.cuda(), heads, kv).cpu()
    struck = torch.zeros_like(got, dtype=torch.bool).reshape(n, lq, heads, d)
    for i in (0, d // 2, d - 1):
        struck[0, :, :heads // kv, i] = True
    struck = struck.reshape(n, lq, heads * d)
    assert not got[struck].isfinite().any()
    check(torch.where(struck, torch.zeros_like(got), got), torch.where(struck, torch.zeros_like(ref), ref), bound, "others")


@pytest.mark.parametrize("dt,n,lq,lk,heads,kv,d", FORMS)
@pytest.mark.parametrize("kind", ("none", "states", "pairs"))
def test_queries_that_are_not_finite(sq, dt, n, lq, lk, heads, kv, d, kind):
    """A query with a NaN or an infinity gets NaN where it sees anything, zeros where it does not, and leaves the others alone."""
    q, k, v = inputs(n, lq, lk, heads, kv, d, dt, 51)
    mask, seen = None, everything(n, lq, lk)
    if kind == "states":
        mask = torch.rand((n, lk), generator=gen(52)) < 0.5
        mask[-1], mask[0, 0] = False, n > 1
        seen = mask[:, None].expand(n, lq, lk)
    elif kind == "pairs":
        mask = torch.rand((n, lq, lk), generator=gen(52)) < 0.5
        mask[:, ::3] = False
        seen = mask
    ref, bound = reference_on_gpu(q, k, v, heads, kv, d ** -0.5, seen, dt)
    bad = q.clone().reshape(n, lq, heads, d)
    bad[:, ::2, 0, 0], bad[:, 1::2, heads - 1, d - 1] = math.nan, math.inf
    struck = ~bad.isfinite().all(3, keepdim=True) & seen.any(2)[..., None, None]
    struck = struck.expand(n, lq, heads, d).reshape(n, lq, heads * d)
    got = sq.sq_cross_attention_forward(bad.reshape(n, lq, heads * d).cuda(), k.cuda(), v.cuda(), heads, kv, mask=None if mask is None else mask.cuda()).cpu()
    assert got[struck].isnan().all()
    check(torch.where(struck, torch.zeros_like(got), got), torch.where(struck, torch.zeros_like(ref), ref), bound, kind)


@pytest.mark.parametrize("scale", (1e-42, -1e-42, 1e-37))
@pytest.mark.parametrize("dt,n,lq,lk,heads,kv,d", FORMS)
def test_scales_below_the_normal_numbers(sq, dt, n, lq, lk, heads, kv, d, scale):
    """All scores are as good as equal."""
    q, k, v = inputs(n, lq, lk, heads, kv, d, dt, 53)
    ref, bound = reference_on_gpu(q, k, v, heads, kv, scale, everything(n, lq, lk), dt)
    check(sq.sq_cross_attention_forward(q.cuda(), k.cuda(), v.cuda(), heads, kv, scale=scale), ref, bound, scale)


@pytest.mark.parametrize("size", (1e-20, 1e-28, 1e20))
@pytest.mark.parametrize("dt,n,lq,lk,heads,kv,d", FORMS)
def test_small_and_large_values_under_large_scales(sq, dt, n, lq, lk, heads, kv, d, size):
    """Weights that are far from one because a large score's product is rounded lose nothing of small values and do not overflow large ones."""
    q, k, v, score = levels(n, lq, lk, heads, kv, d, dt, 1.0, 1.0, 0, 61)
    v = (v.float() * size).to(dt)
    for scale in (3e7, 1e8, 3.1e8, 1.1e9, 3.7e9, 7.3e9):
        ref = largest(v, score, everything(n, lq, lk), heads, kv, scale)
        check(sq.sq_cross_attention_forward(q.cuda(), k.cuda(), v.cuda(), heads, kv, scale=scale), ref, bound_of(ref, dt), (size, scale))
