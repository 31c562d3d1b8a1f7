"""The operators of a deep, served network over the graph layers, as timed cases.

Between two Gathers such a network transforms its vertices in 8-bit integers,
adds the block's result to the residual stream and normalises it; after the
last one it answers with log probabilities.

Kinds of case
  product  act(rs * (x w^T) + b) on 8-bit integers with a scale per row of x
           (a vertex) and per row of w (an output channel): the rows come as
           8-bit integers with their scales, or as float32 / bfloat16 values
           that the call quantises.  x: m x k, w: n x k, out: m x n.  deg: rs is
           the degree scaling deg^-1/2 of a GCN transform.
  block    y = x + c * ch * act(gate) * post(block), z = pre(y): the norm after
           a block, its gate, channel scale and residual scale, the residual
           sum, and the norm before the next block; z "i8" is quantised by rows.
  labels   log probability of each row's label, the row's entropy, and its
           top_k classes with their log probabilities.  masked: part of the
           classes is -inf (not allowed), some rows are all -inf, and some rows
           have no label (-1).

Rows whose largest magnitude is A have the scale s = A / 127 rounded to float32
(2^-126 at least) and hold rint(x / s), ties to even.
"""
import math

import torch

own = False
DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2, "i8": 1}
TINY = 2.0 ** -126


# --------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------
def _product(m, k, n, x, out, act="none", bias=True, deg=False, **kw):
    return dict(kind="product", m=m, k=k, n=n, x=x, out=out, act=act, bias=bias, deg=deg, **kw)


def _block(m, f, x, block, z, post, pre, gate="none", channel=False, **kw):
    return dict(kind="block", m=m, f=f, x=x, block=block, z=z, post=post, pre=pre, gate=gate,
                channel=channel, **kw)


def _labels(m, c, dtype, top_k, masked=False, **kw):
    return dict(kind="labels", m=m, c=c, dtype=dtype, top_k=top_k, masked=masked, **kw)


def listed():
    return [
        # one vertex asked for: latency, the weights are read for a single row
        _product(1, 1024, 1024, "f32", "f32", "relu", name="product_one_vertex"),
        # the first transform of a 1M-vertex GCN, 602 raw features in bfloat16
        _product(1 << 20, 602, 128, "bf16", "bf16", deg=True, bias=False, name="product_gcn_1m_602"),
        # a hidden transform whose rows the norm before it has quantised, a ragged vertex count
        _product(40001, 1024, 1024, "i8", "bf16", "relu", name="product_hidden_40k"),
        # the largest product: wide vertices, all of the matrix cores
        _product(32768, 4096, 4096, "i8", "bf16", name="product_wide_33k"),
        # one vertex through a block's end: latency
        _block(1, 128, "f32", "f32", "f32", "rms", "rms", name="block_one_vertex"),
        # the hidden width of a GCN over 1M vertices, bfloat16, gated, both norms
        _block(1 << 20, 128, "bf16", "bf16", "bf16", "layer", "layer", "sigmoid", True, name="block_gcn_1m"),
        # an odd width, float32 stream with bfloat16 blocks, no norm after the block
        _block(100003, 602, "f32", "bf16", "bf16", "none", "rms", "tanh", name="block_odd_100k"),
        # wide vertices whose next transform runs in 8 bits: z leaves quantised
        _block(32768, 4096, "f32", "bf16", "i8", "rms", "rms", "sigmoid", name="block_wide_i8"),
        # one vertex classified: latency
        _labels(1, 41, "f32", 5, name="labels_one_vertex"),
        # every vertex of the 2.1M-vertex graph over 41 classes
        _labels(1 << 21, 41, "bf16", 3, name="labels_2m_41"),
        # link prediction for a few queries: one row scores every vertex of a graph
        _labels(8, 262147, "f32", 10, name="labels_links_8"),
        # link prediction in bulk, candidates that are no answer masked out
        _labels(4099, 100003, "bf16", 20, True, name="labels_links_4k"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["product", "block", "labels"])
    if kind == "product":
        x = rng.choice(["i8", "bf16", "f32"])
        k, n = _log_int(rng, 1, 4096), _log_int(rng, 1, 4096)
        most = min(1 << 20, (1 << 39) // (k * n), (1 << 29) // max(k, n))
        return _product(_log_int(rng, 1, max(1, most)), k, n, x, rng.choice(["f32", "bf16"]),
                        rng.choice(["none", "relu", "elu", "sigmoid", "tanh"]), rng.random() < 0.5,
                        rng.random() < 0.3)
    if kind == "block":
        f = _log_int(rng, 1, 8192)
        x, block = rng.choice([("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
        return _block(_log_int(rng, 1, min(1 << 21, (1 << 27) // f)), f, x, block, rng.choice([block, "i8"]),
                      rng.choice(["none", "rms", "layer"]), rng.choice(["rms", "layer"]),
                      rng.choice(["none", "linear", "sigmoid", "tanh"]), rng.random() < 0.5)
    c = _log_int(rng, 1, 1 << 18)
    return _labels(_log_int(rng, 1, min(1 << 21, (1 << 28) // c)), c, rng.choice(["f32", "bf16"]),
                   rng.randint(0, 32), rng.random() < 0.5)


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------
def _rows(t, dtype):
    """t in a buffer whose row pitch is a multiple of 16 bytes, as the library's matrices are"""
    es = torch.empty(0, dtype=dtype).element_size()
    ld = -(-t.shape[1] * es // 16) * 16 // es
    buf = torch.zeros((t.shape[0], ld), dtype=dtype, device=t.device)
    buf[:, :t.shape[1]] = t
    return buf[:, :t.shape[1]]


def _ints(shape, gen):
    """8-bit rows as a quantiser leaves them: a bell whose far end is 127"""
    return (torch.randn(shape, generator=gen, device=DEV) * 36).round_().clamp_(-127, 127)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(case)
    m = case["m"]

    def vector(n, mean=0.0, dev=0.1):
        return torch.randn(n, generator=g, device=DEV) * dev + mean

    if case["kind"] == "product":
        k, n = case["k"], case["n"]
        s["w"] = _rows(_ints((n, k), g), torch.int8)
        s["w_scale"] = (torch.rand(n, generator=g, device=DEV) + 0.5) / (36 * math.sqrt(k))
        if case["x"] == "i8":
            s["rows"] = _rows(_ints((m, k), g), torch.int8)
            s["x_scale"] = (torch.rand(m, generator=g, device=DEV) + 0.5) / 36
        else:
            x = torch.randn((m, k), generator=g, device=DEV)
            x *= torch.rand((m, 1), generator=g, device=DEV) * 2 + 0.1
            if m > 4:
                x[m // 3] = 0  # a vertex without features
            s["rows"], s["x_scale"] = _rows(x, DTYPES[case["x"]]), None
        s["b"] = vector(n) if case["bias"] else None
        s["degrees"] = (torch.randint(0, 200, (m,), generator=g, device=DEV, dtype=torch.int32)
                        if case["deg"] else None)
        return s
    if case["kind"] == "block":
        f = case["f"]

        def matrix(dtype, dev):
            return _rows(torch.randn((m, f), generator=g, device=DEV) * dev, DTYPES[dtype])

        s["stream"] = matrix(case["x"], 1.5)
        s["made"] = matrix(case["block"], 0.7)
        s["gates"] = matrix(case["block"], 1.0) if case["gate"] != "none" else None
        s["channels"] = vector(f, 0.5) if case["channel"] else None
        for name in ("post", "pre"):
            s[name + "_w"] = vector(f, 1.0) if case[name] != "none" else None
            s[name + "_b"] = vector(f) if case[name] == "layer" else None
        s["res_scale"], s["eps"] = 0.7, 1e-5
        return s
    c = case["c"]
    x = torch.randn((m, c), generator=g, device=DEV, dtype=DTYPES[case["dtype"]]) * 3
    s["to"] = torch.randint(0, c, (m,), generator=g, device=DEV, dtype=torch.int32)
    if case["masked"]:
        for at in range(0, m, max(1, (1 << 27) // c)):  # (in pieces: the mask's random numbers are large)
            part = x[at:at + max(1, (1 << 27) // c)]
            part.masked_fill_(torch.rand(part.shape, generator=g, device=DEV) < 0.3, -math.inf)
        if m > 8:
            x[m // 2] = -math.inf  # nothing is allowed
            s["to"][m // 5] = -1   # nothing is known
    s["logits"] = _rows(x, DTYPES[case["dtype"]])
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


def _quantise(x):
    """(whole numbers, scales) of rows; the quotients in 64 bits: many lie next to a half"""
    top = x.abs().amax(1, keepdim=True).double()
    scale = (top / 127).float().clamp_min(TINY)
    return torch.round(x.double() / scale.double()).clamp_(-127, 127), scale


def _plain_product(s):
    q, scale = s["rows"].float(), s["x_scale"]
    if scale is None:
        q, scale = _quantise(s["rows"])
        q, scale = q.float(), scale[:, 0]
    v = (q @ s["w"].float().T) * scale[:, None] * s["w_scale"]
    if s["degrees"] is not None:
        d = s["degrees"].float()
        v = v * torch.where(d > 0, 1 / torch.sqrt(d), torch.zeros_like(d))[:, None]
    if s["b"] is not None:
        v = v + s["b"]
    return _act(s["act"], v).to(DTYPES[s["out"]])


def _norm(kind, v, w, b, eps):
    if kind == "none":
        return v
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    v = v / torch.sqrt((v * v).mean(1, keepdim=True) + eps) * w
    return v if b is None else v + b


def _plain_block(s):
    u = _norm(s["post"], s["made"].float(), s["post_w"], s["post_b"], s["eps"]) * s["res_scale"]
    if s["channels"] is not None:
        u = u * s["channels"]
    if s["gates"] is not None:
        u = u * _act(s["gate"], s["gates"].float())
    y = s["stream"].float() + u
    z = _norm(s["pre"], y, s["pre_w"], s["pre_b"], s["eps"])
    y = y.to(DTYPES[s["x"]])
    if s["z"] != "i8":
        return y, z.to(DTYPES[s["z"]])
    q, scale = _quantise(z)
    # what the whole numbers stand for, in bfloat16: rows that two computations of z
    # differ in by 2^-24 may differ by a whole step where a quotient is next to a half
    return y, (q.float() * scale).to(torch.bfloat16), scale[:, 0]


def _plain_labels(s):
    x, to, k = s["logits"].float(), s["to"].long(), s["top_k"]
    m, c = x.shape
    top = x.amax(1, keepdim=True)
    empty = top == -math.inf
    shift = x - torch.where(empty, torch.zeros_like(top), top)
    e = torch.exp(shift)
    total = e.sum(1, keepdim=True)
    log_total = torch.log(total)
    weighted = torch.where(e > 0, e * shift, torch.zeros_like(e)).sum(1, keepdim=True)
    entropy = torch.where(empty, torch.zeros_like(total), log_total - weighted / total)[:, 0]
    logp = shift.gather(1, to.clamp_min(0)[:, None]) - log_total
    logp = torch.where(empty, torch.full_like(logp, -math.inf), logp)[:, 0]
    logp = torch.where(to < 0, torch.zeros_like(logp), logp)
    # by value and, where equal, by index: both in one whole number
    bits = (x + 0.0).view(torch.int32).long()
    bits = torch.where(bits < 0, bits ^ 0x7fffffff, bits)
    key = bits * (1 << 32) + torch.arange(c - 1, -1, -1, device=x.device)
    del e, bits
    best = torch.topk(key, min(k, c), dim=1).values
    index = c - 1 - (best & 0xffffffff)
    value = shift.gather(1, index) - log_total
    gone = torch.isneginf(x.gather(1, index))
    index = torch.where(gone, torch.full_like(index, -1), index)
    value = torch.where(gone, torch.full_like(value, -math.inf), value)
    if k > c:
        index = torch.cat([index, index.new_full((m, k - c), -1)], 1)
        value = torch.cat([value, value.new_full((m, k - c), -math.inf)], 1)
    return logp, entropy, index.int(), value


def _own_product(s):
    from paper_2009_00804_amd import layers as LY

    return LY.quant_linear(s["rows"], s["w"], s["w_scale"], x_scale=s["x_scale"], bias=s["b"], act=s["act"],
                           row_scale_deg=s["degrees"], out_dtype=DTYPES[s["out"]])


def _own_block(s):
    from paper_2009_00804_amd import layers as LY

    y, z, scale = LY.block_norm(
        s["made"], s["stream"], post=s["post"], post_weight=s["post_w"], post_bias=s["post_b"],
        gate=s["gates"], gate_act="none" if s["gate"] == "linear" else s["gate"],
        channel_scale=s["channels"], res_scale=s["res_scale"], pre=s["pre"], pre_weight=s["pre_w"],
        pre_bias=s["pre_b"], eps=s["eps"], quantize=s["z"] == "i8")
    if s["z"] != "i8":
        return y, z
    return y, torch.mul(z, scale[:, None], out=torch.empty(z.shape, dtype=torch.bfloat16, device=z.device)), scale


def _own_labels(s):
    from paper_2009_00804_amd import layers as LY

    return LY.label_log_probs(s["logits"], s["to"], top_k=s["top_k"])


def run(state):
    if own:
        return {"product": _own_product, "block": _own_block, "labels": _own_labels}[state["kind"]](state)
    return {"product": _plain_product, "block": _plain_block, "labels": _plain_labels}[state["kind"]](state)


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------
def work(case):
    m = case["m"]
    if case["kind"] == "product":
        k, n = case["k"], case["n"]
        b = m * k * SIZE[case["x"]] + n * k + m * n * SIZE[case["out"]] + 4 * n
        b += 4 * m * ((case["x"] == "i8") + case["deg"]) + 4 * n * case["bias"]
        return {"bytes": b, "flops": 2 * m * k * n}
    if case["kind"] == "block":
        f = case["f"]
        b = m * f * (2 * SIZE[case["x"]] + SIZE[case["block"]] * (1 + (case["gate"] != "none")) + SIZE[case["z"]])
        return {"bytes": b + 4 * m * (case["z"] == "i8"), "flops": 20 * m * f}
    return {"bytes": m * case["c"] * SIZE[case["dtype"]] + 4 * m * (3 + 2 * case["top_k"]),
            "flops": 8 * m * case["c"]}


# --------------------------------------------------------------------------
# the definition in 64 bits
# --------------------------------------------------------------------------
def _exact_rows(x):
    """What 8-bit rows stand for: (whole numbers, scales), both float64"""
    step = torch.clamp(torch.div(x.abs().max(dim=1)[0], 127.0).to(torch.float32), min=TINY).double().unsqueeze(1)
    return torch.round(x / step).clamp(-127, 127), step


def _exact_act(name, v):
    return {"relu": lambda: v.clamp(min=0), "elu": lambda: torch.nn.functional.elu(v),
            "sigmoid": lambda: torch.sigmoid(v), "tanh": lambda: torch.tanh(v)}.get(name, lambda: v)()


def _exact_product(s):
    w = s["w"].double() * s["w_scale"].double().unsqueeze(1)
    out = []
    rows = max(1, (1 << 27) // max(s["k"], s["n"]))
    for at in range(0, s["m"], rows):
        x = s["rows"][at:at + rows].double()
        if s["x_scale"] is None:
            q, step = _exact_rows(x)
            x = q * step
        else:
            x = x * s["x_scale"][at:at + rows].double().unsqueeze(1)
        v = torch.mm(x, w.t())
        if s["degrees"] is not None:
            d = s["degrees"][at:at + rows].double().unsqueeze(1)
            v = v * torch.where(d > 0, d.clamp(min=1).pow(-0.5), 0.0)
        if s["b"] is not None:
            v += s["b"].double()
        out.append(_exact_act(s["act"], v))
    return torch.cat(out)


def _exact_norm(kind, v, w, b, eps):
    if kind == "none":
        return v
    centre = v.mean(dim=1, keepdim=True) if kind == "layer" else 0.0
    spread = (v - centre).pow(2).mean(dim=1, keepdim=True)
    v = (v - centre) * (spread + eps).rsqrt() * w.double()
    return v if b is None else v + b.double()


def _exact_block(s):
    u = _exact_norm(s["post"], s["made"].double(), s["post_w"], s["post_b"], s["eps"])
    if s["gates"] is not None:
        u = u * _exact_act(s["gate"], s["gates"].double())
    if s["channels"] is not None:
        u = u * s["channels"].double()
    y = s["stream"].double() + s["res_scale"] * u
    z = _exact_norm(s["pre"], y, s["pre_w"], s["pre_b"], s["eps"])
    if s["z"] != "i8":
        return y, z
    q, step = _exact_rows(z)
    return y, q * step, step.squeeze(1)


def _exact_labels(s):
    k, c = s["top_k"], s["c"]
    outs = []
    rows = max(1, (1 << 26) // c)
    for at in range(0, s["m"], rows):
        x, to = s["logits"][at:at + rows].double(), s["to"][at:at + rows].long()
        empty = torch.isneginf(x).all(dim=1, keepdim=True)
        p = torch.softmax(x, dim=1)
        logp = torch.log_softmax(x, dim=1)
        h = -torch.where(p > 0, p * logp, 0.0).sum(dim=1)
        h[empty[:, 0]] = 0.0
        logp = torch.where(empty, -math.inf, logp)
        at_label = torch.where(to < 0, 0.0, logp.gather(1, to.clamp(min=0).unsqueeze(1)).squeeze(1))
        order = torch.sort(x, dim=1, descending=True, stable=True)[1][:, :k]
        best = logp.gather(1, order)
        order = order.masked_fill(torch.isneginf(best), -1)
        pad = max(0, k - c)
        outs.append((at_label, h, torch.nn.functional.pad(order, (0, pad), value=-1).int(),
                     torch.nn.functional.pad(best, (0, pad), value=-math.inf)))
    return tuple(torch.cat(t) for t in zip(*outs))


def exact(case, seed):
    s = prepare(case, seed)
    return {"product": _exact_product, "block": _exact_block, "labels": _exact_labels}[case["kind"]](s)
