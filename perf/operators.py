"""Measured calls of the channels-last operators: layout conversion, group norm with an activation, and the matrix product of
rows with bias, activation and residual.

A case is a plain dict.  Its "op" names the entry point:
  pack, unpack   sq_nhwc_pack / sq_nhwc_unpack: NCHW map to channels-last map and back, "src" and "dst" the two types
  norm           sq_nhwc_group_norm on a channels-last map
  linear         sq_linear_forward: rows [rows][cin] by kernels [cout][cin]
"extra" is the number of further layers that lie behind the operator's own ones in each row of the map it reads (it then reads
a slice of a wider map, as one behind a concatenation does).  "act" is the activation.
"""
import math

import torch

own = False     # False: the operators in plain torch operations; True: the library's entry points

ACTS = ("none", "relu", "silu", "gelu")      # in the order of the library's codes
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # a map on its way out of the NCHW layers of one image, as the classifier's stage has it: the smallest conversion
        {"name": "unpack_bf16_b1", "op": "unpack", "src": "bf16", "dst": "f32", "n": 1, "c": 512, "h": 13, "w": 13, "extra": 0},
        # the fp32 map of the first fire layers at the benchmark's batch, into the reduced-precision channels-last form
        {"name": "pack_f32_bf16_b64", "op": "pack", "src": "f32", "dst": "bf16", "n": 64, "c": 128, "h": 55, "w": 55, "extra": 0},
        # one image's last map: the latency of a normalisation
        {"name": "norm_f32_b1", "op": "norm", "dtype": "f32", "n": 1, "c": 512, "h": 13, "w": 13, "groups": 32, "act": "silu", "extra": 0},
        # an ordinary serving batch of the middle maps
        {"name": "norm_bf16_b16", "op": "norm", "dtype": "bf16", "n": 16, "c": 384, "h": 27, "w": 27, "groups": 32, "act": "relu", "extra": 0},
        # groups of odd width in a slice of a wider map with a ragged extent
        {"name": "norm_f32_odd", "op": "norm", "dtype": "f32", "n": 5, "c": 150, "h": 53, "w": 57, "groups": 6, "act": "gelu", "extra": 7},
        # the largest maps of the network, the benchmark's batch
        {"name": "norm_bf16_b64", "op": "norm", "dtype": "bf16", "n": 64, "c": 96, "h": 111, "w": 111, "groups": 8, "act": "silu", "extra": 0},
        # the class scores of one image from its pooled layers
        {"name": "linear_f32_r1", "op": "linear", "dtype": "f32", "rows": 1, "cin": 512, "cout": 1000, "act": "none", "residual": False, "extra": 0},
        # a wide layer on a few rows: its kernels are what is read
        {"name": "linear_bf16_r8", "op": "linear", "dtype": "bf16", "rows": 8, "cin": 4096, "cout": 4096, "act": "gelu", "residual": False, "extra": 0},
        # the pixels of one middle map, back from its widened form, added to the map
        {"name": "linear_bf16_b1", "op": "linear", "dtype": "bf16", "rows": 729, "cin": 1536, "cout": 384, "act": "none", "residual": True, "extra": 0},
        # odd layers of three ragged maps, read from a slice of a wider one
        {"name": "linear_f32_odd", "op": "linear", "dtype": "f32", "rows": 2187, "cin": 99, "cout": 333, "act": "silu", "residual": True, "extra": 5},
        # a wide fp32 layer on the pixels of the benchmark's batch
        {"name": "linear_f32_b64", "op": "linear", "dtype": "f32", "rows": 10816, "cin": 2048, "cout": 2048, "act": "gelu", "residual": True, "extra": 0},
        # the largest: a wide reduced-precision layer on the pixels of a large batch
        {"name": "linear_bf16_b96", "op": "linear", "dtype": "bf16", "rows": 16224, "cin": 4096, "cout": 4096, "act": "gelu", "residual": True, "extra": 0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    op = rng.choice(("pack", "unpack", "norm", "norm", "norm", "linear", "linear", "linear", "linear"))
    extra = rng.choice((0, 0, 0, 8, 24, rng.randint(1, 40)))
    if op == "linear":
        # layers as the maps of this library have them (multiples of eight), or any number
        step = rng.choice((1, 8, 8, 32))
        case = {"op": op, "dtype": rng.choice(("f32", "bf16")), "rows": _log(rng, 1, 16384),
                "cin": max(step, _log(rng, 16, 4096) // step * step), "cout": max(step, _log(rng, 10, 4096) // step * step),
                "act": rng.choice(ACTS), "residual": rng.random() < 0.5, "extra": extra}
        small, most = "rows", _cost(listed()[10] if case["dtype"] == "f32" else listed()[11])
    else:
        h = _log(rng, 7, 112)
        w = max(5, h + rng.randint(-5, 5))
        case = {"op": op, "n": _log(rng, 1, 64), "h": h, "w": w}
        if op == "norm":
            groups = rng.choice((1, 2, 4, 6, 8, 16, 32))
            width = rng.choice((rng.randint(1, 32), rng.choice((2, 4, 8, 12, 16, 32))))
            case.update(dtype=rng.choice(("f32", "bf16")), c=groups * width, groups=groups, act=rng.choice(ACTS), extra=extra)
        else:
            case.update(src=rng.choice(("f32", "f32", "bf16")), dst=rng.choice(("f32", "bf16")), c=_log(rng, 3, 512), extra=extra)
        small, most = "n", _cost(listed()[5])
    while _cost(case) > most:
        case[small] = max(1, case[small] // 2)
    return case


def _size(t):
    return 4 if t == "f32" else 2


def work(case):
    if case["op"] == "linear":
        rows, cin, cout, size = case["rows"], case["cin"], case["cout"], _size(case["dtype"])
        values = rows * cin + cout * cin + rows * cout * (2 if case["residual"] else 1)
        return {"bytes": float(size * values + 4 * cout), "flops": 2.0 * rows * cin * cout}
    values = case["n"] * case["c"] * case["h"] * case["w"]
    if case["op"] == "norm":
        # sum, squared deviation and its sum (4), the affine form (2), the activation counted as four
        return {"bytes": 2.0 * _size(case["dtype"]) * values + 8.0 * case["c"], "flops": 10.0 * values}
    return {"bytes": float((_size(case["src"]) + _size(case["dst"])) * values), "flops": 0.0}


# ----------------------------------------------------------------------------------------------------- inputs and state
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, std=1.0, mean=0.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * std + mean


def _in_wider(values, extra, dtype):
    """The values as the first layers of rows that are `extra` layers wider."""
    if not extra:
        return values.to(dtype)
    wide = torch.zeros(values.shape[:-1] + (values.shape[-1] + extra,), device="cuda", dtype=dtype)
    wide[..., :values.shape[-1]] = values
    return wide[..., :values.shape[-1]]


def _map(g, n, h, w, c):
    """A map as a convolution leaves it: layers of different spread and mean."""
    return _normal(g, (n, h, w, c)) * (0.5 + torch.rand(c, generator=g, device="cuda")) + _normal(g, (c,), 0.5)


def prepare(case, seed):
    g = _gen(seed)
    s = {"op": case["op"]}
    if case["op"] == "linear":
        t = TYPES[case["dtype"]]
        s["x"] = _in_wider(_normal(g, (case["rows"], case["cin"])), case["extra"], t)
        s["w"] = _normal(g, (case["cout"], case["cin"]), math.sqrt(2.0 / case["cin"])).to(t)
        s["b"] = torch.rand(case["cout"], generator=g, device="cuda") * 0.2 - 0.1
        s["residual"] = _normal(g, (case["rows"], case["cout"])).to(t) if case["residual"] else None
        s["act"] = ACTS.index(case["act"])
    elif case["op"] == "norm":
        c = case["c"]
        s["x"] = _in_wider(_map(g, case["n"], case["h"], case["w"], c), case["extra"], TYPES[case["dtype"]])
        s["gamma"], s["beta"] = 1.0 + _normal(g, (c,), 0.1), _normal(g, (c,), 0.1)
        s["groups"], s["eps"], s["act"] = case["groups"], 1e-5, ACTS.index(case["act"])
    else:
        values, s["dst"] = _map(g, case["n"], case["h"], case["w"], case["c"]), TYPES[case["dst"]]
        if case["op"] == "pack":
            s["x"] = values.permute(0, 3, 1, 2).contiguous().to(TYPES[case["src"]])
        else:
            s["x"] = _in_wider(values, case["extra"], TYPES[case["src"]])
    return s


# --------------------------------------------------------------------------------------------------------- the operators
def _act(y, act):
    if act == 1:
        return torch.where(y < 0, torch.zeros_like(y), y)
    if act == 2:
        return y / (1 + torch.exp(-y))
    if act == 3:
        return 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    return y


def _plain(s):
    x = s["x"]
    if s["op"] == "pack":
        return x.permute(0, 2, 3, 1).to(s["dst"]).contiguous()
    if s["op"] == "unpack":
        return x.permute(0, 3, 1, 2).to(s["dst"]).contiguous()
    if s["op"] == "norm":
        n, h, w, c = x.shape
        v = x.float().reshape(n, h * w, s["groups"], c // s["groups"])
        v = v - v.mean((1, 3), keepdim=True)
        v = v * torch.rsqrt((v * v).mean((1, 3), keepdim=True) + s["eps"])
        return _act(v.reshape(n, h, w, c) * s["gamma"] + s["beta"], s["act"]).to(x.dtype)
    y = _act(torch.matmul(x.float(), s["w"].float().t()) + s["b"], s["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(x.dtype)


def run(state):
    s = state
    if not own:
        return _plain(s)
    import paper_1611_07151_amd as sq
    if s["op"] == "pack":
        return sq.sq_nhwc_pack(s["x"], dtype=s["dst"])
    if s["op"] == "unpack":
        return sq.sq_nhwc_unpack(s["x"], dtype=s["dst"])
    if s["op"] == "norm":
        return sq.sq_nhwc_group_norm(s["x"], s["groups"], s["gamma"], s["beta"], eps=s["eps"], act=s["act"])
    return sq.sq_linear_forward(s["x"], s["w"], s["b"], act=s["act"], residual=s["residual"])


def exact(case, seed):
    """The definitions in 64 bits.  The conversions round each value once at most: their value in 64 bits is the input's own."""
    s = prepare(case, seed)
    x = s["x"].double()
    if s["op"] == "pack":
        return torch.movedim(x, 1, -1).contiguous()
    if s["op"] == "unpack":
        return torch.movedim(x, -1, 1).contiguous()
    if s["op"] == "norm":
        # per image and group, over all pixels and the group's neighbouring layers
        groups = torch.stack(torch.chunk(x, s["groups"], dim=3))                   # [group][image][h][w][layer]
        var, mean = torch.var_mean(groups, dim=(2, 3, 4), unbiased=False, keepdim=True)
        y = torch.cat(tuple((groups - mean) / torch.sqrt(var + s["eps"])), dim=3) * s["gamma"].double() + s["beta"].double()
    else:
        y = torch.addmm(s["b"].double(), x, s["w"].double().t())
    act = case["act"]
    if act == "relu":
        y = y.clamp(min=0)
    elif act == "silu":
        y = y * torch.sigmoid(y)
    elif act == "gelu":
        y = 0.5 * y * torch.special.erfc(-y / math.sqrt(2))
    if case["op"] == "linear" and s["residual"] is not None:
        y = y + s["residual"].double()
    return y
