"""Measured calls of the operators of a cross-attention block on channels-last maps: rows in microscaled 4-bit floating point and
their matrix product, and attention of the pixels of a map to an encoder's states.

A case is a plain dict.  Its "op" names the entry points:
  pack     sq_mxfp4_pack of rows [rows][cin], and sq_mxfp4_unpack, which gives the values that the codes stand for
  linear   sq_mxfp4_linear_forward: rows [rows][cin], given in "dtype" and brought to 4 bits by the call, by kernels [cout][cin] that are
           packed ahead of time
  cross    sq_cross_attention_forward: queries [n][lq][heads * d] to states [n][lk][kv_heads * d]
"extra" is the number of further values behind the operator's own ones in each row of its input (a slice of a wider map).  "act" is
the activation.  "mask" of a cross case: none, lengths (how many states an image has), states (which ones, by image) or pairs (which
ones, by image and query); the last three leave some images or queries without any.  "kv_in_one": keys and values are the two halves
of one projection's rows.
"""
import math

import torch

own = False     # False: the operators in plain torch operations; True: the library's entry points

ACTS = ("none", "relu", "silu", "gelu")      # in the order of the library's codes
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # a few pooled rows: the latency of a conversion
        {"name": "pack_bf16_r8", "op": "pack", "dtype": "bf16", "rows": 8, "cin": 512, "extra": 0},
        # the pixels of the middle maps at the benchmark's batch
        {"name": "pack_f32_b64", "op": "pack", "dtype": "f32", "rows": 46656, "cin": 384, "extra": 0},
        # the class scores of one image from its pooled layers
        {"name": "mx_linear_f32_r1", "op": "linear", "dtype": "f32", "rows": 1, "cin": 512, "cout": 1000, "act": "none", "residual": False, "extra": 0},
        # a wide layer on a few rows: its kernels are what is read
        {"name": "mx_linear_bf16_r8", "op": "linear", "dtype": "bf16", "rows": 8, "cin": 4096, "cout": 4096, "act": "gelu", "residual": False, "extra": 0},
        # odd layers of three ragged maps, read from a slice of a wider one: the last block of a row has three values
        {"name": "mx_linear_f32_odd", "op": "linear", "dtype": "f32", "rows": 2187, "cin": 99, "cout": 333, "act": "silu", "residual": True, "extra": 5},
        # a wide layer on the pixels of a large batch
        {"name": "mx_linear_bf16_b96", "op": "linear", "dtype": "bf16", "rows": 16224, "cin": 4096, "cout": 4096, "act": "gelu", "residual": True, "extra": 0},
        # one query to the pixels of one middle map: the smallest call
        {"name": "cross_bf16_q1", "op": "cross", "dtype": "bf16", "n": 1, "lq": 1, "lk": 729, "heads": 8, "kv_heads": 8, "d": 64, "mask": "none", "kv_in_one": True},
        # single queries of a serving batch to long encoders' states, four query heads to each head of the states
        {"name": "cross_bf16_q1_long", "op": "cross", "dtype": "bf16", "n": 8, "lq": 1, "lk": 16384, "heads": 32, "kv_heads": 8, "d": 128, "mask": "lengths", "kv_in_one": False},
        # the pixels of the middle maps to short sequences of states of different lengths
        {"name": "cross_bf16_short", "op": "cross", "dtype": "bf16", "n": 16, "lq": 729, "lk": 77, "heads": 8, "kv_heads": 8, "d": 48, "mask": "lengths", "kv_in_one": True},
        # odd sizes with a mask of its own for every query
        {"name": "cross_f32_odd", "op": "cross", "dtype": "f32", "n": 3, "lq": 169, "lk": 333, "heads": 6, "kv_heads": 3, "d": 25, "mask": "pairs", "kv_in_one": False},
        # the fp32 maps of a small batch to the pixels of smaller maps
        {"name": "cross_f32_b4", "op": "cross", "dtype": "f32", "n": 4, "lq": 3025, "lk": 729, "heads": 8, "kv_heads": 8, "d": 64, "mask": "states", "kv_in_one": True},
        # the largest: wide maps to long sequences
        {"name": "cross_bf16_b16", "op": "cross", "dtype": "bf16", "n": 16, "lq": 3025, "lk": 4096, "heads": 16, "kv_heads": 16, "d": 64, "mask": "none", "kv_in_one": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 100)


def draw(rng):
    op = rng.choice(("pack", "linear", "linear", "linear", "cross", "cross", "cross", "cross"))
    if op == "cross":
        group, kv = rng.choice((1, 1, 1, 2, 4, 8)), rng.choice((1, 2, 3, 4, 6, 8, 12, 16))
        case = {"op": op, "dtype": rng.choice(("bf16", "bf16", "f32")), "n": _log(rng, 1, 16), "lq": rng.choice((1, _log(rng, 1, 4096), _log(rng, 64, 4096))),
                "lk": _log(rng, 1, 16384), "heads": kv * group, "kv_heads": kv,
                "d": rng.choice((rng.randint(1, 128), 8 * rng.randint(2, 16), 32, 64, 64, 128)),
                "mask": rng.choice(("none", "none", "lengths", "states", "pairs")), "kv_in_one": rng.random() < 0.5}
        most, shrink = _cost(listed()[10] if case["dtype"] == "f32" else listed()[11]), ("n", "lk", "lq", "heads", "kv_heads")
    else:
        # layers as the maps of this library have them (multiples of eight), or any number
        step = rng.choice((1, 8, 32, 32))
        case = {"op": op, "dtype": rng.choice(("f32", "bf16")), "rows": _log(rng, 1, 46656 if op == "pack" else 16384),
                "cin": max(step, _log(rng, 16, 4096) // step * step), "extra": rng.choice((0, 0, 0, 8, 24, rng.randint(1, 40)))}
        if op == "linear":
            case.update(cout=max(step, _log(rng, 10, 4096) // step * step), act=rng.choice(ACTS), residual=rng.random() < 0.5)
        most, shrink = _cost(listed()[1] if op == "pack" else listed()[5]), ("rows",)
    turn = 0
    while _cost(case) > most:
        key = shrink[turn % len(shrink)]
        if key == "heads":
            # keep the number of query heads to each head of the states
            if case["kv_heads"] > 1:
                case["heads"] = case["heads"] // case["kv_heads"] * (case["kv_heads"] // 2)
                case["kv_heads"] //= 2
        elif key != "kv_heads":
            case[key] = max(1, case[key] // 2)
        turn += 1
    return case


def _size(t):
    return 4 if t == "f32" else 2


def work(case):
    if case["op"] == "cross":
        n, lq, lk, d = case["n"], case["lq"], case["lk"], case["d"]
        size, pairs = _size(case["dtype"]), case["n"] * case["heads"] * float(case["lq"]) * case["lk"]
        mask = {"none": 0.0, "lengths": 4.0 * n, "states": float(n * lk), "pairs": float(n) * lq * lk}[case["mask"]]
        # every query with every state: a mask may leave fewer, but how many is a matter of the inputs
        return {"bytes": size * (2.0 * n * lq * case["heads"] * d + 2.0 * n * lk * case["kv_heads"] * d) + mask, "flops": 4.0 * pairs * d}
    rows, cin, size = case["rows"], case["cin"], _size(case["dtype"])
    blocks = (cin + 31) // 32
    if case["op"] == "pack":
        # to codes and scales and back to values in fp32; largest magnitude, scaling and rounding counted as three
        return {"bytes": rows * (float(cin) * (size + 4) + 2 * 17.0 * blocks), "flops": 3.0 * rows * cin}
    cout = case["cout"]
    return {"bytes": rows * float(cin) * size + cout * 17.0 * blocks + size * float(rows) * cout * (2 if case["residual"] else 1) + 4.0 * cout,
            "flops": 2.0 * rows * cin * cout}


# ----------------------------------------------------------------------------------------------------- inputs and state
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, std=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * std


def _in_wider(values, extra, dtype):
    """The values as the first of rows that are `extra` values wider."""
    if not extra:
        return values.to(dtype)
    wide = torch.zeros(values.shape[:-1] + (values.shape[-1] + extra,), device="cuda", dtype=dtype)
    wide[..., :values.shape[-1]] = values
    return wide[..., :values.shape[-1]]


def _inputs(case, seed):
    g = _gen(seed)
    s = {"op": case["op"]}
    t = TYPES[case["dtype"]]
    if case["op"] == "cross":
        n, lq, lk, kv, d = case["n"], case["lq"], case["lk"], case["kv_heads"], case["d"]
        s["heads"], s["kv_heads"], s["scale"] = case["heads"], kv, d ** -0.5
        s["q"] = _normal(g, (n, lq, case["heads"] * d)).to(t)
        states = _normal(g, (n, lk, 2 * kv * d)).to(t)
        s["k"], s["v"] = states[..., :kv * d], states[..., kv * d:]
        if not case["kv_in_one"]:
            s["k"], s["v"] = s["k"].contiguous(), s["v"].contiguous()
        s["lengths"] = s["mask"] = None
        if case["mask"] == "lengths":
            s["lengths"] = torch.randint(lk // 2, lk + 1, (n,), generator=g, device="cuda", dtype=torch.int32)
            if n > 1:
                s["lengths"][-1] = 0
        elif case["mask"] == "states":
            s["mask"] = torch.rand((n, lk), generator=g, device="cuda") < 0.8
            if n > 1:
                s["mask"][-1] = False
        elif case["mask"] == "pairs":
            s["mask"] = torch.rand((n, lq, lk), generator=g, device="cuda") < 0.8
            s["mask"][:, lq // 2] = False
        return s
    # layers of different spread, a few of them far wider, as maps in front of a projection have them
    spread = 0.5 + torch.rand(case["cin"], generator=g, device="cuda")
    spread = torch.where(torch.rand(case["cin"], generator=g, device="cuda") < 0.02, 10 * spread, spread)
    s["x"] = _in_wider(_normal(g, (case["rows"], case["cin"])) * spread, case["extra"], t)
    if case["op"] == "linear":
        s["w"] = _normal(g, (case["cout"], case["cin"]), math.sqrt(2.0 / case["cin"])).to(t)
        s["b"] = torch.rand(case["cout"], generator=g, device="cuda") * 0.2 - 0.1
        s["residual"] = _normal(g, (case["rows"], case["cout"])).to(t) if case["residual"] else None
        s["act"] = ACTS.index(case["act"])
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "linear":      # the kernels in 4 bits: a program brings them there once
        s["cout"] = case["cout"]
        if own:
            import paper_1611_07151_amd as sq
            s["w"] = sq.sq_mxfp4_pack(s["w"])
        else:
            s["w"] = _four_bits(s["w"])
    return s


# --------------------------------------------------------------------------------------------------------- the operators
def _four_bits(x):
    """The values that rows of x keep in blocks of 32 with a common power of two and elements of 4 bits (0, 0.5, 1, 1.5, 2, 3, 4, 6)."""
    rows, cin = x.shape
    blocks = (cin + 31) // 32
    v = torch.zeros((rows, blocks * 32), device=x.device, dtype=torch.float32)
    v[:, :cin] = x
    v = v.reshape(rows, blocks, 32)
    most = v.abs().amax(2, keepdim=True)
    exponent = (torch.frexp(most)[1] - 3).clamp(min=-127)       # of the largest magnitude, less the 2 of the largest element
    a = torch.ldexp(v.abs(), -exponent)
    # steps of 0.5 below 2, of 1 below 4, of 2 above; halves to even
    a = torch.where(a < 2, torch.round(2 * a) * 0.5, torch.where(a < 4, torch.round(a), torch.round(0.5 * a) * 2)).clamp(max=6)
    a = torch.ldexp(a, exponent)
    return torch.where(v < 0, -a, a).reshape(rows, blocks * 32)[:, :cin].contiguous()


def _act(y, act):
    if act == 1:
        return torch.where(y < 0, torch.zeros_like(y), y)
    if act == 2:
        return y / (1 + torch.exp(-y))
    if act == 3:
        return 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    return y


def _seen(s, lk):
    """[n][1 or lq][lk]: which states a query sees, or None for all."""
    if s["lengths"] is not None:
        return (torch.arange(lk, device="cuda") < s["lengths"][:, None])[:, None]
    if s["mask"] is not None:
        return s["mask"] if s["mask"].dim() == 3 else s["mask"][:, None]
    return None


def _plain_cross(s):
    q, k, v, kv = s["q"], s["k"], s["v"], s["kv_heads"]
    n, lq, width = q.shape
    lk, d = k.shape[1], k.shape[2] // kv
    group = s["heads"] // kv
    seen = _seen(s, lk)
    out = torch.empty_like(q)
    at_once = max(1, 2 ** 28 // (s["heads"] * lq * lk))      # images whose scores are in memory at a time
    for i in range(0, n, at_once):
        j = min(n, i + at_once)
        qi = q[i:j].float().reshape(j - i, lq, kv, group, d).permute(0, 2, 1, 3, 4).reshape(j - i, kv, lq * group, d)
        ki = k[i:j].float().reshape(j - i, lk, kv, d).permute(0, 2, 3, 1).contiguous()
        vi = v[i:j].float().reshape(j - i, lk, kv, d).permute(0, 2, 1, 3).contiguous()
        p = (torch.matmul(qi, ki) * s["scale"]).reshape(j - i, kv, lq, group, lk)
        if seen is not None:
            p = torch.where(seen[i:j, None, :, None], p, torch.full_like(p, -math.inf))
        most = p.amax(4, keepdim=True)
        p = torch.exp(p - torch.where(most == -math.inf, torch.zeros_like(most), most))
        total = p.sum(4, keepdim=True)
        o = torch.matmul(p.reshape(j - i, kv, lq * group, lk), vi).reshape(j - i, kv, lq, group, d)
        o = o / torch.where(total == 0, torch.ones_like(total), total)
        out[i:j] = o.permute(0, 2, 1, 3, 4).reshape(j - i, lq, width).to(q.dtype)
    return out


def _plain(s):
    if s["op"] == "cross":
        return _plain_cross(s)
    if s["op"] == "pack":
        return _four_bits(s["x"])
    y = _act(torch.matmul(_four_bits(s["x"]), s["w"].t()) + s["b"], s["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["x"].dtype)


def run(state):
    s = state
    if not own:
        return _plain(s)
    import paper_1611_07151_amd as sq
    if s["op"] == "pack":
        return sq.sq_mxfp4_unpack(sq.sq_mxfp4_pack(s["x"]), *s["x"].shape)
    if s["op"] == "linear":
        return sq.sq_mxfp4_linear_forward(s["x"], s["w"], s["cout"], s["b"], act=s["act"], residual=s["residual"])
    return sq.sq_cross_attention_forward(s["q"], s["k"], s["v"], s["heads"], s["kv_heads"], scale=s["scale"], lengths=s["lengths"], mask=s["mask"])


def _exact_four_bits(x):
    """The same values by another way: the nearest element by the borders between them, a border itself to the even neighbour."""
    x = x.double()
    rows, cin = x.shape
    elements = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda", dtype=torch.float64)
    borders = (elements[1:] + elements[:-1]) / 2
    parts = []
    for part in torch.split(x, 32, dim=1):
        most = part.abs().max(dim=1, keepdim=True).values
        scale = torch.exp2(torch.floor(torch.log2(most.clamp(min=2.0 ** -125))) - 2)
        # log2 is rounded: put the power right where it stepped over a border
        scale = torch.where(scale * 8 <= most, scale * 2, torch.where((scale * 4 > most) & (scale > 2.0 ** -127), scale / 2, scale))
        ratio = (part.abs() / scale).contiguous()
        low, high = torch.bucketize(ratio, borders), torch.bucketize(ratio, borders, right=True)     # they differ on a border
        index = torch.where(low % 2 == 0, low, high)
        parts.append(torch.sign(part) * elements[index] * scale)
    return torch.cat(parts, dim=1)


def exact(case, seed):
    """The definitions in 64 bits."""
    s = _inputs(case, seed)
    if case["op"] == "pack":
        return _exact_four_bits(s["x"])
    if case["op"] == "linear":
        y = torch.addmm(s["b"].double(), _exact_four_bits(s["x"]), _exact_four_bits(s["w"]).t())
        act = case["act"]
        if act == "relu":
            y = y.clamp(min=0)
        elif act == "silu":
            y = y * torch.sigmoid(y)
        elif act == "gelu":
            y = 0.5 * y * torch.special.erfc(-y / math.sqrt(2))
        return y if s["residual"] is None else y + s["residual"].double()
    n, lq, heads, d, lk = case["n"], case["lq"], case["heads"], case["d"], case["lk"]
    seen = _seen(s, lk)
    out = torch.zeros((n, lq, heads * d), device="cuda", dtype=torch.float64)
    for i in range(n):
        for h in range(heads):
            own_head = h // (heads // case["kv_heads"])
            k, v = (s[name][i, :, own_head * d:(own_head + 1) * d].double() for name in ("k", "v"))
            score = torch.mm(s["q"][i, :, h * d:(h + 1) * d].double(), k.t()) * s["scale"]
            if seen is not None:
                score = score.masked_fill(~seen[i].expand(lq, lk), -math.inf)
            p = torch.nan_to_num(torch.softmax(score, dim=1), nan=0.0)      # a query that sees nothing: zeros
            out[i, :, h * d:(h + 1) * d] = torch.mm(p, v)
    return out
