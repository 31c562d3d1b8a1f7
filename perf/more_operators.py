"""4-bit transforms and a layer of experts, the vertex functions of a served deep network, as timed cases.

Rows in microscaled 4-bit floating point hold 32 neighbouring values as e2m1
numbers (0, 1/2, 1, 3/2, 2, 3, 4, 6 and a sign; two a byte, the first in the low
half) times one power of two, held as its exponent + 127 in a byte.  A block
whose largest magnitude is A has the exponent max(floor(log2 A) - 2, -127), its
values are rounded to the nearest number, ties to the even one, at most 6.

Kinds of case
  rows     rows of float32 or bfloat16 to 4 bits and back: what they stand for.
  product  act(rs * (x w^T) + b) on 4-bit rows of w (an output channel each) and of
           x (a vertex each), which come in 4 bits or as floats that the call
           rounds.  x: m x k, w: n x k, out: m x n.  deg: rs is the degree scaling
           deg^-1/2 of a GCN transform.
  experts  a layer of which every vertex takes the top_k of e experts: a router's
           logits x r^T + b choose them (ties to the lowest index; a bias of -inf
           closes an expert), their softmax over the chosen (renorm) or over all
           weights them.  An expert is down(act(up(x))), or, gated, down(act(gate(x))
           * up(x)), gate's rows before up's; its weights are bfloat16 or 4-bit rows.
           x: m x f, h hidden channels, out: m x f, with the chosen experts and
           their weights.
"""
import math

import torch

own = False
DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2, "mx4": 17 / 32}
MOST_ROWS = 512             # of an experts case: a batch of requests
MOST_WEIGHTS = 440 << 20    # bytes of its experts


# --------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------
def _rows_case(m, k, dtype, **kw):
    return dict(kind="rows", m=m, k=k, dtype=dtype, **kw)


def _product(m, k, n, x, out, act="none", bias=True, deg=False, **kw):
    return dict(kind="product", m=m, k=k, n=n, x=x, out=out, act=act, bias=bias, deg=deg, **kw)


def _experts(m, f, h, e, top_k, dtype, weights, act="relu", gated=False, bias=False, closed=False, renorm=True, **kw):
    return dict(kind="experts", m=m, f=f, h=h, e=e, top_k=top_k, dtype=dtype, weights=weights, act=act, gated=gated,
                bias=bias, closed=closed, renorm=renorm, **kw)


def listed():
    return [
        # the raw features of a 1M-vertex graph put away in 4 bits, 602 of them in bfloat16
        _rows_case(1 << 20, 602, "bf16", name="rows_features_1m"),
        # the weights of one wide transform, an odd number of rows, from float32
        _rows_case(4099, 4096, "f32", name="rows_weights_4k"),
        # one vertex asked for: latency, the weights are read for a single row
        _product(1, 1024, 1024, "f32", "f32", "relu", name="product_one_vertex"),
        # a batch of asked vertices, bounded by the weights' bytes
        _product(48, 4096, 4096, "bf16", "bf16", "relu", name="product_batch_48"),
        # the first transform of a 1M-vertex GCN, 602 raw features in bfloat16
        _product(1 << 20, 602, 128, "bf16", "bf16", deg=True, bias=False, name="product_gcn_1m_602"),
        # a hidden transform of rows that are in 4 bits already, a ragged vertex count
        _product(40001, 1024, 1024, "mx4", "bf16", "relu", name="product_hidden_40k"),
        # the largest product: wide vertices, all of the matrix cores
        _product(16384, 4096, 4096, "mx4", "bf16", name="product_wide_16k"),
        # one vertex of a small network with experts: latency
        _experts(1, 128, 256, 4, 1, "f32", "bf16", "relu", bias=True, name="experts_one_vertex"),
        # one vertex of a wide network, gated experts in 4 bits
        _experts(1, 1024, 4096, 8, 2, "bf16", "mx4", "sigmoid", True, name="experts_one_wide"),
        # a few vertices, odd widths, bfloat16 weights, some experts closed, no renormalisation
        _experts(19, 602, 1001, 16, 2, "f32", "bf16", "elu", bias=True, closed=True, renorm=False,
                 name="experts_odd_19"),
        # a batch of requests that takes most experts, a row or two each
        _experts(64, 1024, 4096, 64, 2, "bf16", "mx4", "sigmoid", True, name="experts_batch_64"),
        # the largest batch: every expert, dozens of rows each
        _experts(MOST_ROWS, 2048, 4096, 32, 4, "bf16", "mx4", "sigmoid", True, name="experts_batch_512"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rows", "product", "product", "experts", "experts"])
    if kind == "rows":
        k = _log_int(rng, 1, 16384)
        return _rows_case(_log_int(rng, 1, min(1 << 20, (1 << 28) // k)), k, rng.choice(["f32", "bf16"]))
    if kind == "product":
        x = rng.choice(["mx4", "mx4", "bf16", "f32"])
        k, n = _log_int(rng, 1, 4096), _log_int(rng, 1, 4096)
        most = min(1 << 20, (1 << 38) // (k * n), (1 << 28) // max(k, n))
        return _product(_log_int(rng, 1, max(1, most)), k, n, x, rng.choice(["f32", "bf16"]),
                        rng.choice(["none", "relu", "elu", "sigmoid", "tanh"]), rng.random() < 0.5,
                        rng.random() < 0.3)
    weights, gated = rng.choice(["mx4", "mx4", "bf16"]), rng.random() < 0.6
    f, h, e = _log_int(rng, 16, 4096), _log_int(rng, 16, 8192), _log_int(rng, 2, 64)
    e = max(2, min(e, int(MOST_WEIGHTS / (f * h * (2 + gated) * SIZE[weights]))))
    return _experts(_log_int(rng, 1, MOST_ROWS), f, h, e, rng.randint(1, min(4, e)), rng.choice(["f32", "bf16", "bf16"]),
                    weights, rng.choice(["relu", "elu", "sigmoid", "tanh"]), gated, rng.random() < 0.5,
                    rng.random() < 0.3, rng.random() < 0.7)


# --------------------------------------------------------------------------
# 4-bit rows in torch
# --------------------------------------------------------------------------
VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _blocks(x):
    """x as (rows, blocks, 32), zeros behind the last column"""
    m, k = x.shape
    pad = x.new_zeros((m, -(-k // 32) * 32))
    pad[:, :k] = x
    return pad.view(m, -1, 32)


def _power(e):
    """2^e in float32, e from -127 to 127"""
    return torch.where(e > -127, (e + 127) << 23, torch.full_like(e, 1 << 22)).int().view(torch.float32)


def _round(x):
    """(numbers of the blocks of float32 rows, their exponents)"""
    v = _blocks(x)
    top = v.abs().amax(2, keepdim=True)
    e = ((top.view(torch.int32) >> 23) - 127 - 2).clamp_min(-127)
    t = v * _power(-e)  # (exact but for values that come to 0)
    a = t.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return torch.copysign((torch.round(a / step) * step).clamp_max(6.0), t), e


def _stand_for(x):
    """what the 4-bit rows of float32 rows stand for"""
    v, e = _round(x)
    return (v * _power(e)).view(x.shape[0], -1)[:, :x.shape[1]]


def _pitched(t, dtype, unit=16):
    """t in a buffer whose row pitch is a multiple of `unit` bytes, as the library's matrices are"""
    es = torch.empty(0, dtype=dtype).element_size()
    ld = -(-t.shape[1] * es // unit) * unit // es
    buf = torch.zeros((t.shape[0], ld), dtype=dtype, device=t.device)
    buf[:, :t.shape[1]] = t
    return buf[:, :t.shape[1]]


def _pack(x):
    """(bytes, scale bytes) of float32 rows"""
    v, e = _round(x)
    a = v.abs()
    code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
    code |= (v < 0).to(torch.uint8) << 3
    code = code.view(x.shape[0], -1, 2)
    q = (code[:, :, 0] | code[:, :, 1] << 4)[:, :-(-x.shape[1] // 2)]
    return q, (e[:, :, 0] + 127).to(torch.uint8)


def _unpack(q, scale, k):
    """float32 rows of k columns that 4-bit rows stand for"""
    m = q.shape[0]
    table = torch.tensor(VALUES + tuple(-v for v in VALUES), device=q.device)
    v = table[torch.stack([q & 15, q >> 4], 2).view(m, -1).long()]
    return (_blocks(v) * _power(scale.int()[:, :, None] - 127)).view(m, -1)[:, :k]


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(case)
    m = case["m"]

    def vector(n, mean=0.0, dev=0.1):
        return torch.randn(n, generator=g, device=DEV) * dev + mean

    def features(rows, cols):
        """rows of different sizes, their columns too"""
        x = torch.randn((rows, cols), generator=g, device=DEV)
        x *= torch.rand((rows, 1), generator=g, device=DEV) * 2 + 0.1
        return x.mul_(torch.rand(cols, generator=g, device=DEV) + 0.5)

    def four_bits(rows, cols, dev):
        """4-bit rows of normal values, made in pieces"""
        q = torch.empty((rows, -(-cols // 32) * 16), dtype=torch.uint8, device=DEV)
        scale = torch.empty((rows, -(-cols // 128) * 4), dtype=torch.uint8, device=DEV)
        piece = max(1, (1 << 25) // cols)
        for at in range(0, rows, piece):
            a, b = _pack(torch.randn((min(piece, rows - at), cols), generator=g, device=DEV) * dev)
            q[at:at + piece, :a.shape[1]], scale[at:at + piece, :b.shape[1]] = a, b
        return q[:, :-(-cols // 2)], scale[:, :-(-cols // 32)]

    if case["kind"] == "rows":
        s["x"] = _pitched(features(m, case["k"]), DTYPES[case["dtype"]])
        return s
    if case["kind"] == "product":
        k, n = case["k"], case["n"]
        s["w"], s["w_scale"] = four_bits(n, k, 1 / math.sqrt(k))
        if case["x"] == "mx4":
            s["rows"], s["x_scale"] = four_bits(m, k, 1.0)
        else:
            x = features(m, k)
            if m > 4:
                x[m // 3] = 0  # a vertex without features
            s["rows"], s["x_scale"] = _pitched(x, DTYPES[case["x"]]), None
        s["b"] = vector(n) if case["bias"] else None
        s["degrees"] = (torch.randint(0, 200, (m,), generator=g, device=DEV, dtype=torch.int32)
                        if case["deg"] else None)
        return s
    f, h, e = case["f"], case["h"], case["e"]
    wide = e * h * (1 + case["gated"])
    s["rows"] = _pitched(torch.randn((m, f), generator=g, device=DEV), DTYPES[case["dtype"]])
    s["router"] = _pitched(torch.randn((e, f), generator=g, device=DEV) / math.sqrt(f), DTYPES[case["dtype"]])
    s["router_b"] = vector(e) if case["bias"] or case["closed"] else None
    if case["closed"]:
        s["router_b"][torch.arange(e, device=DEV) % 3 == 1] = -math.inf
    for name, rows, cols in (("up", wide, f), ("down", e * f, h)):
        s[name + "_scale"] = None
        if case["weights"] == "mx4":
            s[name], s[name + "_scale"] = four_bits(rows, cols, 1 / math.sqrt(cols))
        else:
            w = torch.randn((rows, cols), generator=g, device=DEV, dtype=torch.bfloat16)
            s[name] = _pitched(w.mul_(1 / math.sqrt(cols)), torch.bfloat16)
        s[name + "_b"] = vector(rows) if case["bias"] else None
    return s


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------
def _act(name, v):
    if name == "relu":
        return torch.where(v > 0, v, torch.zeros_like(v))
    if name == "elu":
        return torch.where(v > 0, v, torch.expm1(v))
    if name == "sigmoid":
        return 1 / (1 + torch.exp(-v))
    return torch.tanh(v) if name == "tanh" else v


def _plain_rows(s):
    return _stand_for(s["x"].float()).to(s["x"].dtype)


def _plain_product(s):
    k = s["k"]
    x = _stand_for(s["rows"].float()) if s["x_scale"] is None else _unpack(s["rows"], s["x_scale"], k)
    v = x @ _unpack(s["w"], s["w_scale"], k).T
    if s["degrees"] is not None:
        d = s["degrees"].float()
        v = v * torch.where(d > 0, 1 / torch.sqrt(d), torch.zeros_like(d))[:, None]
    if s["b"] is not None:
        v = v + s["b"]
    return _act(s["act"], v).to(DTYPES[s["out"]])


def _plain_route(s):
    """(chosen experts, -1 where none is left; their weights); logits in 64 bits: an
    expert is chosen by which of two close values is larger"""
    logits = s["rows"].double() @ s["router"].double().T
    if s["router_b"] is not None:
        logits = logits + s["router_b"].double()
    left = logits.clone()
    at, best = [], []
    for _ in range(s["top_k"]):
        top = left.amax(1, keepdim=True)
        first = (left == top).int().argmax(1, keepdim=True)  # (the lowest of equal ones)
        at.append(first)
        best.append(top)
        left = left.scatter(1, first, -math.inf)
    index, best = torch.cat(at, 1), torch.cat(best, 1)
    closed = best == -math.inf
    top = torch.where(closed[:, :1], torch.zeros_like(best[:, :1]), best[:, :1])
    p = torch.exp((best - top).float())
    total = p if s["renorm"] else torch.exp((logits - top).float())
    total = total.sum(1, keepdim=True)
    p = torch.where(closed, torch.zeros_like(p), p / total)
    return torch.where(closed, torch.full_like(index, -1), index).int(), p


def _weights(s, name, at, rows, cols):
    """rows at.. of an expert's weights in float32"""
    w = s[name][at:at + rows]
    return w.float() if s[name + "_scale"] is None else _unpack(w, s[name + "_scale"][at:at + rows], cols)


def _plain_experts(s):
    f, h = s["f"], s["h"]
    wide = h * (1 + s["gated"])
    index, p = _plain_route(s)
    x = s["rows"].float()
    y = torch.zeros_like(x)
    for e in range(s["e"]):
        v = x @ _weights(s, "up", e * wide, wide, f).T
        if s["up_b"] is not None:
            v = v + s["up_b"][e * wide:(e + 1) * wide]
        v = _act(s["act"], v[:, :h]) * v[:, h:] if s["gated"] else _act(s["act"], v)
        v = v @ _weights(s, "down", e * f, f, h).T
        if s["down_b"] is not None:
            v = v + s["down_b"][e * f:(e + 1) * f]
        y += v * torch.where(index == e, p, torch.zeros_like(p)).sum(1, keepdim=True)
    return y.to(s["rows"].dtype), index, p


def _own_rows(s):
    from paper_2009_00804_amd import layers as LY

    q, scale = LY.quantize_rows_mx4(s["x"])
    return LY.dequantize_rows_mx4(q, scale, s["k"], dtype=s["x"].dtype)


def _own_product(s):
    from paper_2009_00804_amd import layers as LY

    return LY.mx4_linear(s["rows"], s["w"], s["w_scale"], x_scale=s["x_scale"], bias=s["b"], act=s["act"],
                         row_scale_deg=s["degrees"], out_dtype=DTYPES[s["out"]])


def _own_experts(s):
    from paper_2009_00804_amd import layers as LY

    return LY.expert_layer(s["rows"], s["router"], s["up"], s["down"], up_scale=s["up_scale"],
                           down_scale=s["down_scale"], router_bias=s["router_b"], up_bias=s["up_b"],
                           down_bias=s["down_b"], top_k=s["top_k"], act=s["act"], gated=s["gated"],
                           renormalise=s["renorm"])


def run(state):
    if own:
        return {"rows": _own_rows, "product": _own_product, "experts": _own_experts}[state["kind"]](state)
    return {"rows": _plain_rows, "product": _plain_product, "experts": _plain_experts}[state["kind"]](state)


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------
def work(case):
    m = case["m"]
    if case["kind"] == "rows":
        return {"bytes": 2 * m * case["k"] * SIZE[case["dtype"]], "flops": 4 * m * case["k"]}
    if case["kind"] == "product":
        k, n = case["k"], case["n"]
        b = m * k * SIZE[case["x"]] + n * k * SIZE["mx4"] + m * n * SIZE[case["out"]]
        return {"bytes": b + 4 * m * case["deg"] + 4 * n * case["bias"], "flops": 2 * m * k * n}
    f, h, e, top_k = case["f"], case["h"], case["e"], case["top_k"]
    e_open = sum(not (case["closed"] and i % 3 == 1) for i in range(e))
    top_k = min(top_k, e_open)
    # experts that some row is expected to take
    taken = e_open * (1 - (1 - top_k / e_open) ** m)
    b = taken * f * h * (2 + case["gated"]) * SIZE[case["weights"]] + e * f * SIZE[case["dtype"]]
    b += 2 * m * f * SIZE[case["dtype"]] + 8 * m * case["top_k"]
    return {"bytes": b, "flops": 2 * m * f * (e + top_k * h * (2 + case["gated"]))}


# --------------------------------------------------------------------------
# the definition in 64 bits
# --------------------------------------------------------------------------
def _exact_values(x):
    """What 4-bit rows of float64 rows stand for: the nearest of the format's numbers, by comparison"""
    m, k = x.shape
    v = torch.nn.functional.pad(x, (0, -k % 32)).unflatten(1, (-1, 32))
    big = v.abs().max(dim=2, keepdim=True)[0]
    unit = torch.exp2((torch.frexp(big)[1] - 3).clamp(min=-127).double())  # (big in [2^(e-1), 2^e))
    unit = torch.where(big > 0, unit, 2.0 ** -127)
    size, found = v.abs() / unit, torch.zeros_like(v)
    for low, high, to_high in ((0, .5, False), (.5, 1, True), (1, 1.5, False), (1.5, 2, True), (2, 3, False),
                               (3, 4, True), (4, 6, False)):
        half = (low + high) / 2
        found = torch.where((size > half) | ((size == half) & to_high), high, found)
    return (torch.sign(v) * found * unit).flatten(1)[:, :k]


def _exact_unpack(q, scale, k):
    """float64 rows that 4-bit rows stand for, from the bits of the numbers"""
    bits = torch.stack([q.bitwise_and(15), q.div(16, rounding_mode="floor")], dim=-1).flatten(1).long()
    sign, exponent, half = bits // 8, bits // 2 % 4, bits % 2
    size = torch.where(exponent == 0, half * 0.5, (1 + half * 0.5) * torch.exp2(exponent.double() - 1))
    unit = torch.exp2(scale.double() - 127).repeat_interleave(32, dim=1)
    return ((1 - 2 * sign) * size)[:, :k] * unit[:, :k]


def _exact_act(name, v):
    return {"relu": lambda: v.clamp(min=0), "elu": lambda: torch.nn.functional.elu(v),
            "sigmoid": lambda: torch.sigmoid(v), "tanh": lambda: torch.tanh(v)}.get(name, lambda: v)()


def _exact_rows(s):
    piece = max(1, (1 << 26) // s["k"])
    return torch.cat([_exact_values(t.double()).to(s["x"].dtype) for t in s["x"].split(piece)])


def _exact_product(s):
    k = s["k"]
    w = _exact_unpack(s["w"], s["w_scale"], k)
    out = []
    piece = max(1, (1 << 26) // max(k, s["n"]))
    for at in range(0, s["m"], piece):
        x = s["rows"][at:at + piece]
        if s["x_scale"] is None:
            x = _exact_values(x.double())
        else:
            x = _exact_unpack(x, s["x_scale"][at:at + piece], k)
        v = torch.mm(x, w.t())
        if s["degrees"] is not None:
            d = s["degrees"][at:at + piece].double().unsqueeze(1)
            v = v * torch.where(d > 0, d.clamp(min=1).pow(-0.5), 0.0)
        if s["b"] is not None:
            v += s["b"].double()
        out.append(_exact_act(s["act"], v))
    return torch.cat(out)


def _exact_experts(s):
    f, h, k = s["f"], s["h"], s["top_k"]
    x = s["rows"].double()
    logits = torch.mm(x, s["router"].double().t())
    if s["router_b"] is not None:
        logits = logits + s["router_b"].double()
    order = torch.sort(logits, dim=1, descending=True, stable=True)[1][:, :k]
    mine = logits.gather(1, order)
    p = torch.softmax(mine, dim=1) if s["renorm"] else torch.softmax(logits, dim=1).gather(1, order)
    order = order.masked_fill(torch.isneginf(mine), -1)
    p = torch.where(order < 0, 0.0, p)
    y = torch.zeros_like(x)

    def weights(name, at, rows, cols):
        w = s[name][at:at + rows]
        return w.double() if s[name + "_scale"] is None else _exact_unpack(w, s[name + "_scale"][at:at + rows], cols)

    for e in torch.unique(order).tolist():
        if e < 0:
            continue
        row, place = torch.nonzero(order == e, as_tuple=True)
        at, wide = e * h * (1 + s["gated"]), h * (1 + s["gated"])
        v = torch.mm(x[row], weights("up", at, wide, f).t())
        if s["up_b"] is not None:
            v += s["up_b"][at:at + wide].double()
        v = _exact_act(s["act"], v[:, :h]) * (v[:, h:] if s["gated"] else 1.0)
        v = torch.mm(v, weights("down", e * f, f, h).t())
        if s["down_b"] is not None:
            v += s["down_b"][e * f:(e + 1) * f].double()
        y[row] += v * p[row, place].unsqueeze(1)
    return y, order.int(), p


def exact(case, seed):
    s = prepare(case, seed)
    return {"rows": _exact_rows, "product": _exact_product, "experts": _exact_experts}[case["kind"]](s)
