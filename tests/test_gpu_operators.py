"""8-bit rows and products, block norms and label log probabilities against
their definitions in float64, each within the roundings its float32 steps make."""
import ctypes as C

import numpy as np
import pytest
import torch

from gpu_util import device, graph, lib
from helpers import edges_to_csr

pytestmark = pytest.mark.gpu

U = 2.0 ** -24            # half a step of float32, relative
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
TINY = 2.0 ** -126
FLOATS = [torch.float32, torch.bfloat16]


def LY():
    lib()
    from paper_2009_00804_amd import layers

    return layers


def padded(t, dtype=None, fill=None, extra=0):
    """t on the GPU in a buffer with 16-byte rows whose padding holds ``fill``"""
    dtype = dtype or t.dtype
    step = 16 // dtype.itemsize
    ld = (t.shape[1] + step - 1) // step * step + extra * step
    if fill is None:
        fill = 77 if dtype == torch.int8 else float("nan")
    buf = torch.full((t.shape[0], ld), fill, dtype=dtype, device=device())
    buf[:, :t.shape[1]] = t.to(device()).to(dtype)
    return buf[:, :t.shape[1]]


def padding_of(t):
    """the columns of t's buffer past its own"""
    return t.as_strided((t.shape[0], t.stride(0) - t.shape[1]), t.stride(), t.storage_offset() + t.shape[1])


def gen(seed):
    return torch.Generator().manual_seed(seed)


# --------------------------------------------------------------------------
# 8-bit rows
# --------------------------------------------------------------------------
def rows_exact(x):
    """(q, scale) of float64 rows by the definition"""
    top = x.abs().amax(1, keepdim=True)
    s = torch.clamp((top / 127).float(), min=TINY)
    q = torch.round(x / s.double())
    bad = ~torch.isfinite(top)
    return torch.where(bad, 0.0, q).to(torch.int8), torch.where(bad, float("nan"), s)[:, 0]


def special_rows(k, g):
    """rows at which a quantiser can go wrong"""
    r = [torch.zeros(k), torch.full((k,), 1e-42), torch.randn(k, generator=g) * 1e-39,
         torch.randn(k, generator=g) * 1e37, torch.full((k,), -0.0)]
    ties = torch.arange(k).float() % 254 - 126.5  # scale 1: every value next to or on a half
    ties[0] = 127.0
    near = torch.nextafter(ties, torch.full((k,), 1e9))
    near[0] = 127.0
    r += [ties, near, torch.nextafter(ties, -torch.full((k,), 1e9)).clamp(-127, 127)]
    r[-1][0] = 127.0
    for bad in (float("nan"), float("inf"), -float("inf")):
        b = torch.randn(k, generator=g)
        b[k // 2] = bad
        r.append(b)
    scale = (torch.rand(1, generator=g) + 0.5).item()  # ties about a scale that is no power of two
    t = (torch.arange(k).float() % 100 + 0.5) * scale
    t[0] = 127 * scale
    r.append(t)
    return torch.stack(r)


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("k", [1, 7, 8, 17, 64, 65, 128, 200, 256, 300, 512, 602, 1024, 1500, 2048, 4096, 5001,
                               8192, 9001, 20000])
def test_quantize_rows_exactly(k, dtype):
    S = lib()
    g = gen(k)
    x = torch.cat([torch.randn(13, k, generator=g) * 3, special_rows(k, g)]).to(dtype)
    want_q, want_s = rows_exact(x.double())
    xd = padded(x, extra=1)
    q = padded(torch.full(x.shape, 99, dtype=torch.int8), extra=1)
    scale = torch.full((x.shape[0] + 1,), -5.0, device=device())
    S.saga_quantize_rows(S.dtype_code(dtype), S.cmat(xd), S.mat(q), scale.data_ptr(), S.stream_handle())
    torch.cuda.synchronize()
    got_s = scale[:-1].cpu()
    assert torch.equal(torch.isnan(got_s), torch.isnan(want_s))
    assert torch.equal(got_s.nan_to_num(1), want_s.nan_to_num(1))
    assert torch.equal(q.cpu(), want_q)
    assert scale[-1] == -5.0 and bool((padding_of(q) == 77).all())


def test_quantize_many_rows_and_none():
    L = LY()
    x = torch.randn(70001, 24, generator=gen(3))
    want_q, want_s = rows_exact(x.double())
    q, s = L.quantize_rows(x.to(device()))
    assert torch.equal(q.cpu(), want_q) and torch.equal(s.cpu(), want_s)
    q, s = L.quantize_rows(x[:0].to(device()))
    assert q.shape == (0, 24) and s.shape == (0,)


# --------------------------------------------------------------------------
# product
# --------------------------------------------------------------------------
ACTS = {"none": lambda v: v, "relu": lambda v: v.clamp(min=0), "elu": lambda v: torch.where(v > 0, v, torch.expm1(v)),
        "sigmoid": torch.sigmoid, "tanh": torch.tanh}


def product_exact(q, s, w, ws, bias, act, deg):
    """(float64 result, magnitude of what is added up in it)"""
    v = (q.double() @ w.double().T) * s.double()[:, None] * ws.double()
    if deg is not None:
        d = deg.double()[:, None]
        v = v * torch.where(d > 0, d.clamp(min=1) ** -0.5, 0.0)
    mag = v.abs()
    if bias is not None:
        v = v + bias.double()
        mag = mag + bias.double().abs()
    return ACTS[act](v), mag


def check_product(got, want, mag, dtype):
    """Before the activation: the sum to float32, two scales, the degree's root, quotient
    and product, the bias: seven roundings of at most U each.  The activations have
    slopes of at most 1 and float32 functions that are a few U of their values (at
    most about 1 where they are curved) off: 8 U.  Then the rounding to the output's type."""
    err = (got.double().cpu() - want).abs()
    tol = 8 * U * mag + 8 * U * (1 + want.abs()) + (HALF[dtype] * want.abs() if dtype != torch.float32 else 0)
    worst = (err / tol).max().item() if err.numel() else 0
    assert worst <= 1, worst


SIZES = [(1, 1, 1), (1, 1024, 1000), (2, 100, 70), (7, 602, 41), (16, 16, 16), (33, 17, 5), (31, 127, 32), (128, 128, 128),
         (129, 130, 257), (300, 602, 128), (513, 257, 41), (1000, 64, 33), (70, 4096, 65), (257, 1000, 300),
         (64, 129, 64), (2000, 15, 129), (9, 5000, 700), (4099, 144, 4096), (3, 40000, 33),
         # wider and longer than the kernel for few rows takes: every tile shape, fused and not
         (17003, 130, 13), (17003, 1, 30), (20000, 257, 41), (17100, 602, 128), (16500, 64, 65), (9000, 640, 70),
         (16390, 641, 100), (17000, 1248, 16), (16400, 1000, 300), (17001, 77, 500), (18000, 1249, 20),
         (1300, 2100, 11008), (1290, 2048, 11010)]


@pytest.mark.parametrize("m,k,n", SIZES)
@pytest.mark.parametrize("out", FLOATS)
def test_product_of_8bit_rows(m, k, n, out):
    L = LY()
    g = gen(m * 7 + k + n)
    q = torch.randint(-128, 128, (m, k), generator=g, dtype=torch.int8)
    w = torch.randint(-128, 128, (n, k), generator=g, dtype=torch.int8)
    s, ws = torch.rand(m, generator=g) + 0.1, (torch.rand(n, generator=g) + 0.1) / (5000 * k ** 0.5)
    act = list(ACTS)[(m + n) % 5]
    bias = torch.randn(n, generator=g) if k % 2 else None
    deg = torch.randint(0, 9, (m,), generator=g, dtype=torch.int32) if n % 2 else None
    want, mag = product_exact(q, s, w, ws, bias, act, deg)
    d = device()
    got = L.quant_linear(padded(q, extra=1), padded(w), ws.to(d), x_scale=s.to(d),
                         bias=None if bias is None else bias.to(d), act=act,
                         row_scale_deg=None if deg is None else deg.to(d), out_dtype=out)
    check_product(got, want, mag, out)


def test_float_product_leaves_what_is_not_its_own():
    S = lib()
    g = gen(6)
    for m, k, n in [(5, 40, 13), (17000, 30, 29), (17001, 200, 75), (9001, 700, 10), (3000, 70, 130)]:
        x = padded(torch.randint(-127, 128, (m, k), generator=g).float())
        x[:, 0] = 127.0  # scale 1: the rows hold themselves
        w = padded(torch.randint(-9, 9, (n, k), generator=g, dtype=torch.int8))
        ws = torch.ones(n, device=device())
        for dtype in FLOATS:
            out = padded(torch.full((m + 2, n), 5.0), dtype, fill=7.0, extra=1)
            op = S.saga_quant_op(S.SAGA_F32, S.dtype_code(dtype), 0, None)
            nbytes = S.saga_apply_vertex_quant_workspace_size(op, m, k, n)
            space = S.workspace(nbytes + 256, device())
            space.fill_(33)
            S.saga_apply_vertex_quant(op, S.cmat(x), None, S.cmat(w), ws.data_ptr(), None, S.mat(out, rows=m),
                                      space.data_ptr() if nbytes else None, nbytes, S.stream_handle())
            torch.cuda.synchronize()
            assert torch.equal(out[:m].cpu(), (x.cpu().double() @ w.cpu().double().T).to(dtype))
            assert bool((out[m:] == 5).all()) and bool((padding_of(out) == 7).all())
            assert bool((space[nbytes:] == 33).all())


@pytest.mark.parametrize("m,k,n", SIZES)
@pytest.mark.parametrize("dtype", FLOATS)
def test_product_of_float_rows(m, k, n, dtype):
    """the call quantises exactly as quantize_rows does"""
    L = LY()
    g = gen(m + k * 3 + n)
    x = torch.randn(m, k, generator=g).to(dtype)
    x[m // 2] *= 0 if m > 2 else 1
    q, s = rows_exact(x.double())
    w = torch.randint(-127, 128, (n, k), generator=g, dtype=torch.int8)
    ws = (torch.rand(n, generator=g) + 0.1) / (100 * k ** 0.5)
    want, mag = product_exact(q, s, w, ws, None, "none", None)
    got = L.quant_linear(padded(x), padded(w), ws.to(device()))
    assert got.dtype == dtype
    check_product(got, want, mag, dtype)


@pytest.mark.parametrize("m", [65536, 131137])
@pytest.mark.parametrize("k,n", [(1, 1), (13, 41), (64, 64), (100, 32), (127, 100), (128, 128), (129, 32), (200, 41), (256, 65),
                                 (256, 128)])
@pytest.mark.parametrize("dtype", FLOATS)
def test_product_of_many_short_rows(m, k, n, dtype):
    """workgroups that take several tiles of rows; a row without a number, one of zeros,
    the last row alone in its tile, and nothing written around the result"""
    S = lib()
    g = gen(m + k * 3 + n)
    x = torch.randn(m, k, generator=g).to(dtype)
    x[77], x[m - 3, k // 2] = 0, float("nan")
    x[1::2] *= 300  # (a row that got a neighbour's scale would show)
    q, s = rows_exact(torch.nan_to_num(x.double()))
    w = torch.randint(-127, 128, (n, k), generator=g, dtype=torch.int8)
    ws = (torch.rand(n, generator=g) + 0.1) / (30000 * k ** 0.5)
    bias = torch.randn(n, generator=g) if n % 2 else None
    deg = torch.randint(0, 9, (m,), generator=g, dtype=torch.int32) if k % 2 else None
    want, mag = product_exact(q, s, w, ws, bias, "none", deg)
    keep = torch.arange(m) != m - 3
    wd, wsd = padded(w), ws.to(device())
    bd, degd = (None if v is None else v.to(device()) for v in (bias, deg))
    for out_dtype in FLOATS:
        for extra in (0, 1):
            xd = padded(x, extra=extra)
            out = padded(torch.full((m + 70, n), 5.0), out_dtype, fill=7.0, extra=extra)
            op = S.saga_quant_op(S.dtype_code(dtype), S.dtype_code(out_dtype), 0, None if deg is None else degd.data_ptr())
            assert S.saga_apply_vertex_quant_workspace_size(op, m, k, n) == 0
            S.saga_apply_vertex_quant(op, S.cmat(xd), None, S.cmat(wd), wsd.data_ptr(),
                                      None if bias is None else bd.data_ptr(), S.mat(out, rows=m), None, 0,
                                      S.stream_handle())
            torch.cuda.synchronize()
            assert bool(out[m - 3].isnan().all())
            check_product(out[:m].cpu()[keep], want[keep], mag[keep], out_dtype)
            assert bool((out[m:] == 5).all())
            if out.stride(0) > n:
                assert bool((padding_of(out) == 7).all())


@pytest.mark.parametrize("m,n", [(1, 40), (130, 40), (1500, 130)])
def test_product_sums_reach_31_bits(m, n):
    L = LY()
    k = 131071
    q = torch.full((m, k), -128, dtype=torch.int8)
    w = torch.full((n, k), -128, dtype=torch.int8)
    w[n // 2:] = 127
    got = L.quant_linear(padded(q), padded(w), torch.ones(n, device=device()),
                         x_scale=torch.ones(m, device=device()))
    want = (q[:1].double() @ w.double().T).float().expand(m, n)
    assert torch.equal(got.cpu(), want)


def test_product_leaves_what_is_not_its_own():
    """columns past N and rows past M keep what they held"""
    S = lib()
    g = gen(5)
    for m, k, n in [(5, 40, 13), (200, 40, 75), (130, 200, 130), (20000, 40, 13), (17000, 30, 29), (17000, 200, 75),
                    (3000, 70, 130)]:
        q = padded(torch.randint(-9, 9, (m, k), generator=g, dtype=torch.int8))
        w = padded(torch.randint(-9, 9, (n, k), generator=g, dtype=torch.int8))
        s, ws = torch.ones(m, device=device()), torch.ones(n, device=device())
        for dtype in FLOATS:
            out = padded(torch.full((m + 2, n), 5.0), dtype, fill=7.0, extra=1)
            op = S.saga_quant_op(S.SAGA_I8, S.dtype_code(dtype), 0, None)
            S.saga_apply_vertex_quant(op, S.cmat(q), s.data_ptr(), S.cmat(w), ws.data_ptr(), None,
                                      S.mat(out, rows=m), None, 0, S.stream_handle())
            torch.cuda.synchronize()
            want = (q.cpu().double() @ w.cpu().double().T)
            assert torch.equal(out[:m].cpu(), want.to(dtype))
            assert bool((out[m:] == 5).all()) and bool((padding_of(out) == 7).all())


def test_product_with_rows_that_hold_no_number():
    L = LY()
    x = torch.randn(40, 100, generator=gen(8))
    x[3, 5] = float("nan")
    x[17, 99] = float("inf")
    w = torch.randint(-9, 9, (50, 100), generator=gen(9), dtype=torch.int8)
    got = L.quant_linear(padded(x), padded(w), torch.ones(50, device=device())).cpu()
    bad = torch.isnan(got).all(1)
    assert bad.nonzero().flatten().tolist() == [3, 17]
    assert bool(torch.isfinite(got[~bad]).all())
    assert L.quant_linear(padded(x)[:0], padded(w), torch.ones(50, device=device())).shape == (0, 50)


# --------------------------------------------------------------------------
# block norm
# --------------------------------------------------------------------------
N_SUM = 48  # roundings a row sum of up to 16384 values goes through: 16 a lane, 10 steps between lanes, and room


def norm_exact(kind, v, dv, w, b, eps):
    """(norm of v, bound of its error) for values known to within dv"""
    if kind == "none":
        return v, dv
    f = v.shape[1]
    centre = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    if kind == "layer":  # the mean: N_SUM roundings of the values' mean magnitude
        dc = dv.mean(1, keepdim=True) + N_SUM * U * v.abs().mean(1, keepdim=True)
        dv = dv + dc + U * (v - centre).abs()
    t = v - centre
    spread = t.pow(2).mean(1, keepdim=True) + eps
    r = spread ** -0.5
    # r: by Cauchy-Schwarz d(spread) / (2 spread) <= rms(dv) / sqrt(spread), and the sum's
    # own roundings, root and quotient
    rel = dv.pow(2).mean(1, keepdim=True).sqrt() * r + (N_SUM + 4) * U
    o = t * r
    do = dv * r + o.abs() * (rel + U)
    w = torch.ones(f, dtype=torch.float64) if w is None else w.double()
    o2 = o * w
    do = do * w.abs() + U * o2.abs()
    if b is not None:
        o2 = o2 + b.double()
        do = do + U * o2.abs()
    return o2, do


def block_exact(c):
    u, du = norm_exact(c["post"], c["block"].double(), torch.zeros(c["block"].shape, dtype=torch.float64),
                       c["post_w"], c["post_b"], c["eps"])
    if c["ch"] is not None:
        u, du = u * c["ch"].double(), du * c["ch"].double().abs() + U * (u * c["ch"].double()).abs()
    if c["gate"] is not None:
        a = ACTS[c["act"]](c["gate"].double())
        da = 8 * U * (1 + a.abs())
        u, du = u * a, du * a.abs() + da * u.abs() + U * (u * a).abs()
    u, du = u * c["res"], du * abs(c["res"]) + 2 * U * abs(c["res"]) * u.abs()
    y = u if c["x"] is None else u + c["x"].double()
    dy = du + U * y.abs()
    z, dz = norm_exact(c["pre"], y, dy, c["pre_w"], c["pre_b"], c["eps"])
    return y, dy, z, dz


def near(got, want, bound, dtype):
    err = (got.double().cpu() - want).abs()
    tol = 1.01 * bound + HALF[dtype] * (want.abs() + bound) + 1e-38
    worst = (err / tol).max().item() if err.numel() else 0
    assert worst <= 1, worst


def block_case(m, f, x, b, post, pre, gate, seed, ch=True, shift=0.0):
    g = gen(seed)

    def vec(mean):
        return torch.randn(f, generator=g) * 0.3 + mean

    return dict(block=(torch.randn(m, f, generator=g) + shift).to(b),
                x=None if x is None else (torch.randn(m, f, generator=g) * 2).to(x),
                gate=None if gate is None else torch.randn(m, f, generator=g).to(b), act=gate or "none",
                post=post, pre=pre, post_w=vec(1.0), post_b=vec(0.0) if post == "layer" else None,
                pre_w=vec(1.0) if seed % 2 else None, pre_b=vec(0.0), ch=vec(0.5) if ch else None, res=-0.7, eps=1e-5)


def run_block(c, quantize, **kw):
    d = device()

    def vec(v):
        return None if v is None else v.to(d)

    return LY().block_norm(padded(c["block"]), None if c["x"] is None else padded(c["x"], extra=1),
                           post=c["post"], post_weight=vec(c["post_w"]), post_bias=vec(c["post_b"]),
                           gate=None if c["gate"] is None else padded(c["gate"], extra=2), gate_act=c["act"],
                           channel_scale=vec(c["ch"]), res_scale=c["res"], pre=c["pre"],
                           pre_weight=vec(c["pre_w"]), pre_bias=vec(c["pre_b"]), eps=c["eps"],
                           quantize=quantize, **kw)


def check_block(c, quantize):
    y, dy, z, dz = block_exact(c)
    gy, gz, gs = run_block(c, quantize)
    near(gy, y, dy, gy.dtype)
    if not quantize:
        near(gz, z, dz, gz.dtype)
        return
    top, dtop = z.abs().amax(1), dz.amax(1)
    want_s = (top / 127).clamp(min=TINY)
    gs, gz = gs.double().cpu(), gz.double().cpu()
    assert bool(((gs - want_s).abs() <= dtop / 127 * 1.01 + 2 * U * want_s).all())
    # a whole number stands for what is at most half a step (and z's own error) away
    assert bool(((gz * gs[:, None] - z).abs() <= 0.5 * gs[:, None] * (1 + 4 * U) + 1.01 * dz + 128 * U * gs[:, None]).all())
    assert bool((gz.abs().amax(1) == 127).all()) or c["block"].shape[1] == 0 or bool((top == 0).any())


WIDTHS = [1, 2, 7, 8, 9, 41, 64, 65, 128, 130, 256, 257, 512, 602, 1024, 1027, 2048, 2050, 4096, 5003, 8192, 9000, 16384]


@pytest.mark.parametrize("quantize", [False, True])
@pytest.mark.parametrize("f", WIDTHS)
def test_block_norm_widths(f, quantize):
    types = [(torch.float32, torch.float32), (torch.float32, torch.bfloat16), (torch.bfloat16, torch.bfloat16)]
    for i, (x, b) in enumerate(types):
        kinds = [("rms", "rms"), ("layer", "layer"), ("none", "rms"), ("rms", "layer"), ("layer", "none")]
        post, pre = kinds[(f + i) % 5]
        if f == 1 and "layer" in (post, pre):
            post, pre = "rms", "rms"  # (a single value less its mean is 0)
        gate = [None, "none", "sigmoid", "tanh", "relu", "elu"][(f + 2 * i) % 6]
        check_block(block_case(3 if f > 2000 else 37, f, x, b, post, pre, gate, f + i, ch=i != 1), quantize)


@pytest.mark.parametrize("post", ["none", "rms", "layer"])
@pytest.mark.parametrize("pre", ["none", "rms", "layer"])
@pytest.mark.parametrize("f", [96, 700, 3000])
def test_block_norm_kinds(f, post, pre):
    check_block(block_case(21, f, torch.float32, torch.bfloat16, post, pre, "sigmoid", f + 1), False)
    check_block(block_case(21, f, None, torch.float32, post, pre, None, f, ch=False), True)


def test_block_norm_far_from_zero():
    """a layer norm of values whose mean is many times their spread"""
    check_block(block_case(33, 500, torch.float32, torch.float32, "layer", "rms", None, 4, shift=100.0), False)


def test_block_norm_many_rows():
    check_block(block_case(40009, 40, torch.float32, torch.bfloat16, "rms", "rms", "sigmoid", 2), False)


def test_block_norm_rows_without_values():
    """zero rows: eps keeps the norm finite; an 8-bit row of zeros has the least scale"""
    for f in (24, 300, 2500):
        c = block_case(5, f, torch.float32, torch.float32, "rms", "rms", None, 6, ch=False)
        c["block"][1] = 0
        c["x"][1] = 0
        c["pre_b"] = None
        c["post_b"] = None
        y, z, s = run_block(c, True)
        assert bool((y[1] == 0).all()) and bool((z[1] == 0).all()) and s[1].item() == TINY
        c["block"][2, f // 2] = float("nan")
        y, z, s = run_block(c, True)
        assert bool(torch.isnan(y[2]).all()) and bool((z[2] == 0).all()) and bool(torch.isnan(s[2]))
        assert not bool(torch.isnan(s[3])) and bool(torch.isfinite(y[3]).all())


@pytest.mark.parametrize("f", [130, 3000])
def test_block_norm_outputs_apart_and_in_place(f):
    """y alone, z alone, y in place of x: the same bits; padding untouched"""
    S, L = lib(), LY()
    c = block_case(19, f, torch.float32, torch.bfloat16, "rms", "layer", "tanh", 11)
    y, z, _ = run_block(c, False)
    d = device()
    x = padded(c["x"], fill=3.0, extra=1)
    block, gate = padded(c["block"]), padded(c["gate"])
    keep = [c["post_w"].to(d), c["pre_w"].to(d), c["pre_b"].to(d), c["ch"].to(d)]
    op = S.saga_block_op(S.SAGA_BF16, S.SAGA_F32, S.saga_norm_desc(1, 1e-5, keep[0].data_ptr(), None),
                         S.saga_norm_desc(2, 1e-5, keep[1].data_ptr(), keep[2].data_ptr()), S.ACT["tanh"], -0.7,
                         keep[3].data_ptr())
    none = S.saga_mat(None, 0, 0, 0)
    y2 = padded(torch.zeros(19, f), torch.float32, fill=9.0, extra=1)
    z2 = padded(torch.zeros(19, f), torch.bfloat16, fill=9.0, extra=1)
    S.saga_block_norm(op, S.cmat(block), S.cmat(gate), S.cmat(x), S.mat(y2), none, None, S.stream_handle())
    S.saga_block_norm(op, S.cmat(block), S.cmat(gate), S.cmat(x), none, S.mat(z2), None, S.stream_handle())
    torch.cuda.synchronize()
    assert torch.equal(y2, y) and torch.equal(z2, z)
    assert bool((padding_of(y2) == 9).all()) and bool((padding_of(z2) == 9).all())
    S.saga_block_norm(op, S.cmat(block), S.cmat(gate), S.cmat(x), S.mat(x), S.mat(z2), None, S.stream_handle())
    torch.cuda.synchronize()
    assert torch.equal(x, y) and bool((padding_of(x) == 3).all())


# --------------------------------------------------------------------------
# label log probabilities
# --------------------------------------------------------------------------
def labels_exact(x, to, k):
    """the definition in float64, and the mean distance from the largest logit (the
    exponents' arguments, whose roundings the sums take over)"""
    m, c = x.shape
    x = x.double()
    bad = torch.isnan(x).any(1) | (x == float("inf")).any(1)
    empty = (x == -float("inf")).all(1) & ~bad
    safe = torch.where((bad | empty)[:, None], 0.0, x)
    lse = torch.logsumexp(safe, 1, keepdim=True)
    lp = safe - lse
    p = torch.exp(lp)
    ent = -torch.where(p > 0, p * lp, 0.0).sum(1)
    dist = torch.where(p > 0, p * (safe.amax(1, keepdim=True) - safe), 0.0).sum(1)
    nan = torch.full_like(lp, float("nan"))
    lp = torch.where(bad[:, None], nan, torch.where(empty[:, None], -float("inf"), lp))
    ent = torch.where(bad, nan[:, 0], torch.where(empty, 0.0, ent))
    at = to.long().clamp(0, c - 1)
    logp = lp.gather(1, at[:, None])[:, 0]
    logp = torch.where(to < 0, 0.0, torch.where(to >= c, float("nan"), logp))
    order = torch.sort(torch.where(bad[:, None], -float("inf"), x), dim=1, descending=True, stable=True)
    kk = min(k, c)
    idx, val = order.indices[:, :kk], lp.gather(1, order.indices[:, :kk])
    gone = order.values[:, :kk] == -float("inf")
    idx = torch.where(gone, -1, idx)
    val = torch.where(gone, -float("inf"), val)
    idx = torch.nn.functional.pad(idx, (0, k - kk), value=-1)
    val = torch.nn.functional.pad(val, (0, k - kk), value=-float("inf"))
    val = torch.where(bad[:, None], float("nan"), val)
    return logp, ent, idx, val, dist


def same(got, want, tol):
    got = got.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    inf = torch.isinf(want)
    assert torch.equal(torch.isinf(got), inf) and torch.equal(got[inf], want[inf])
    ok = torch.isfinite(want)
    err = (got - want).abs()[ok] / tol.expand_as(want)[ok]
    assert err.numel() == 0 or err.max().item() <= 1, err.max().item()


def check_labels(x, to, k, dtype):
    """Every e^d has a relative error of at most (2 |d| + 4) U (the argument's product and
    rounding, the function), so log S is off by (2 D + 4) U with D = sum p |d|, plus the sum's
    own roundings (32 a step and lane, rescalings, 6 or more joins: 128 U) and the
    logarithm's (4 U of its value).  log p: two more differences of that size.  H: T / S has
    both sums' errors, relative to at most 1 + D, and its quotient."""
    logp, ent, idx, val, dist = labels_exact(x, to, k)
    got = LY().label_log_probs(padded(x, dtype), to.to(device()), top_k=k)
    scale = 140 + 6 * dist
    size = torch.where(torch.isfinite(logp), logp.abs(), torch.zeros_like(logp))
    same(got[0], logp, U * (scale + 4 * (size + torch.log(torch.tensor(2.0 + x.shape[1])))))
    same(got[1], ent, U * 2 * scale * (1 + dist + ent.nan_to_num(0)))
    assert got[2].dtype == torch.int32 and torch.equal(got[2].cpu().long(), idx)
    size = torch.where(torch.isfinite(val), val.abs(), torch.zeros_like(val))
    same(got[3], val, U * (scale[:, None] + 4 * (size + torch.log(torch.tensor(2.0 + x.shape[1])))))


def logits_for(m, c, dtype, seed, special=True):
    g = gen(seed)
    x = torch.randn(m, c, generator=g) * 3
    if special and m >= 12:
        x[1] = 2.5                                    # all equal
        x[2] = torch.arange(c).float() / 64           # ascending: the best come last
        x[3] = -torch.arange(c).float() / 64
        x[4] = (x[4] / 3).round()                     # many ties
        x[5, torch.rand(c, generator=g) < 0.6] = -float("inf")
        x[6] = -float("inf")
        x[7] = -float("inf")
        x[7, c - 1] = -40.0                           # one class is left
        x[8, c // 2] = float("nan")
        x[9, c // 3] = float("inf")
        x[10] = x[10] * 30 + 1000                     # far from zero, nearly certain
        x[11] = torch.tensor([0.0, -0.0]).repeat(c // 2 + 1)[:c]
    x = x.to(dtype)
    to = torch.randint(0, c, (m,), generator=g, dtype=torch.int32)
    if m > 3:
        to[0], to[m - 1] = -1, c
    return x, to


CLASSES = [1, 2, 3, 7, 8, 31, 32, 33, 41, 64, 65, 128, 129, 200, 256, 257, 511, 512, 513, 1000, 2047, 2048, 2049,
           4097, 6145, 8192, 8193, 20000, 70001]


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("c", CLASSES)
def test_labels_classes(c, dtype):
    for m, k in ((13, 5), (1, 32), (30, 1), (5, 0), (40, 20)):
        check_labels(*logits_for(m, c, dtype, c + m), k, dtype)


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("m,c,k", [(3000, 41, 3), (70000, 5, 2), (1024, 9000, 20), (1500, 2500, 10), (1023, 8500, 7),
                                   (300, 30000, 32), (2, 300001, 31)])
def test_labels_many_rows(m, c, k, dtype):
    check_labels(*logits_for(m, c, dtype, m + c), k, dtype)


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("m,c,ks", [(16400, 41, (1, 2, 3, 5, 8, 12, 20, 32)), (17000, 64, (4, 19, 31)),
                                    (3000, 60, (7, 32)), (700, 250, (8, 20)), (600, 1000, (10, 32)), (50, 5000, (20,))])
def test_labels_equal_logits(m, c, ks, dtype):
    """few distinct values: every place among the best is decided by the column"""
    g = gen(m + c)
    x = torch.randint(-4, 5, (m, c), generator=g).float() / 2
    x[torch.rand(m, c, generator=g) < 0.1] = -float("inf")
    to = torch.randint(0, c, (m,), generator=g, dtype=torch.int32)
    for k in ks:
        check_labels(x.to(dtype), to, k, dtype)


def test_labels_some_outputs():
    L = LY()
    x, to = logits_for(20, 600, torch.float32, 1)
    xd, td = padded(x), to.to(device())
    a = L.label_log_probs(xd, td, top_k=4)
    b = L.label_log_probs(xd, None, top_k=4, entropy=False)
    assert b[0] is None and b[1] is None and torch.equal(a[2], b[2])
    c = L.label_log_probs(xd, td)
    assert torch.equal(a[0].nan_to_num(3), c[0].nan_to_num(3)) and c[2].shape == (20, 0)
    e = L.label_log_probs(xd[:0], td[:0], top_k=4)
    assert e[0].shape == (0,) and e[2].shape == (0, 4)


# --------------------------------------------------------------------------
# together, streams and graphs
# --------------------------------------------------------------------------
def small_graph(n, deg, seed):
    rng = np.random.default_rng(seed)
    src, dst = rng.integers(0, n, n * deg), rng.integers(0, n, n * deg)
    rp, col, _ = edges_to_csr(n, src.tolist(), dst.tolist())
    return graph(rp, col), rp, col


def deep_weights(f_in, f, classes, depth, seed):
    g = gen(seed)

    def mat(a, b):
        return torch.randn(a, b, generator=g) / a ** 0.5

    def vec(n, mean=0.0):
        return torch.randn(n, generator=g) * 0.1 + mean

    return dict(W_in=mat(f_in, f), b_in=vec(f), norm=vec(f, 1.0), W_out=mat(f, classes), b_out=vec(classes),
                blocks=[dict(W=mat(f, f), W_g=mat(f, f), b=vec(f), b_g=vec(f), pre=vec(f, 1.0), post=vec(f, 1.0))
                        for _ in range(depth)])


@pytest.mark.parametrize("dtype", FLOATS)
def test_residual_gcn(dtype):
    """The network against float64 stages: each on the values the stage before it gave,
    within its own roundings; and the network gives the stages' results bit for bit."""
    L = LY()
    d = device()
    n, f_in, f, classes = 203, 50, 48, 11
    gr, rp, col = small_graph(n, 6, 3)
    w = deep_weights(f_in, f, classes, 2, 5)
    net = L.ResidualGCN(gr, w, dtype=dtype, res_scale=0.5)
    x = torch.randn(n, f_in, generator=gen(9))
    to = torch.randint(0, classes, (n,), generator=gen(10), dtype=torch.int32)
    xd = padded(x)

    def product(z, zs, pair, out):
        wq, ws, b = (t.cpu() for t in pair)
        q, s = rows_exact(z.double().cpu()) if zs is None else (z.cpu(), zs.cpu())
        got = L.quant_linear(z, pair[0], pair[1], x_scale=zs, bias=pair[2], out_dtype=out)
        check_product(got, *product_exact(q, s, wq, ws, b, "none", None), out)
        return got

    def end(block, x0, post, gate, pre, x_dtype=None):
        # y is rounded once, from the same sum z is computed of
        got = L.block_norm(block, x0, post="rms" if post is not None else "none",
                           post_weight=post, gate=gate, gate_act="sigmoid" if gate is not None else "none",
                           res_scale=0.5 if post is not None else 1.0, pre="rms", pre_weight=pre, quantize=True,
                           x_dtype=x_dtype)
        c = dict(block=block.cpu(), x=None if x0 is None else x0.cpu(), gate=None if gate is None else gate.cpu(),
                 act="sigmoid", post="rms" if post is not None else "none", pre="rms",
                 post_w=None if post is None else post.cpu(), post_b=None, pre_w=pre.cpu(), pre_b=None, ch=None,
                 res=0.5 if post is not None else 1.0, eps=1e-5)
        y, dy, z, dz = block_exact(c)
        near(got[0], y, dy, got[0].dtype)
        s = got[2].double().cpu()[:, None]
        assert bool(((got[1].double().cpu() * s - z).abs() <= 0.5 * s + 1.01 * dz + 128 * U * s).all())
        return got

    wide = xd
    h = product(wide, None, net.first, dtype)
    norms = [b["pre"] for b in net.blocks] + [net.norm]
    h, z, zs = end(h, None, None, None, norms[0], torch.float32)
    d_in = np.diff(rp).astype(np.float64)
    d_out = np.bincount(col, minlength=n).astype(np.float64)
    inv = lambda v: np.where(v > 0, np.maximum(v, 1) ** -0.5, 0.0)  # noqa: E731
    adj = np.zeros((n, n))
    for v in range(n):
        for u in col[rp[v]:rp[v + 1]]:
            adj[v, u] += 1
    adj = torch.from_numpy(inv(d_in)[:, None] * adj * inv(d_out))
    for blk, norm in zip(net.blocks, norms[1:]):
        vg = product(z, zs, blk["both"], dtype)
        m = net.gather(vg[:, :f], blk["bias"])
        v = vg[:, :f].double().cpu()
        b = blk["bias"].double().cpu()
        near(m, torch.relu(adj @ v + b), (d_in.max() + 8) * U * (adj @ v.abs() + b.abs()), dtype)
        h, z, zs = end(m, h, blk["post"], vg[:, f:], norm)
    logits = product(z, zs, net.last, torch.float32)
    check_labels(logits.cpu(), to, 3, torch.float32)
    want = L.label_log_probs(logits, to.to(d), top_k=3)
    got = net(xd, to.to(d), top_k=3)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_residual_gcn_captured():
    """the whole network in a graph, replayed on new features"""
    L = LY()
    n, f_in, f = 500, 40, 64
    gr, _, _ = small_graph(n, 5, 8)
    net = L.ResidualGCN(gr, deep_weights(f_in, f, 9, 3, 6), res_scale=0.3)
    x = padded(torch.randn(n, f_in, generator=gen(1)))
    net(x, top_k=2)
    torch.cuda.synchronize()
    gph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gph):
        got = net(x, top_k=2)
    for turn in range(3):
        x.copy_(torch.randn(n, f_in, generator=gen(2 + turn)).to(device()))
        want = net(x, top_k=2)
        torch.cuda.synchronize()
        gph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got[1:], want[1:]))


def everything(L, t):
    """one call of each operator on the tensors t"""
    out = [L.quant_linear(t["x"], t["w"], t["ws"], act="tanh")]
    out += [L.quant_linear(t["few"], t["w"], t["ws"])]
    out += list(L.block_norm(t["block"], t["x"], post="rms", gate=t["gate"], gate_act="sigmoid", pre="layer",
                             quantize=True))
    out += [L.quant_linear(out[-2], t["w"], t["ws"], x_scale=out[-1])]
    out += list(L.label_log_probs(t["wide"], t["to"], top_k=9))
    out += list(L.label_log_probs(t["x"], t["to_x"], top_k=9))
    return out


def tensors(seed, m=300, f=200, n=96, c=40000):
    g = gen(seed)
    d = device()
    return dict(x=padded(torch.randn(m, f, generator=g)), few=padded(torch.randn(2, f, generator=g)),
                block=padded(torch.randn(m, f, generator=g)), gate=padded(torch.randn(m, f, generator=g)),
                w=padded(torch.randint(-127, 128, (n, f), generator=g, dtype=torch.int8)),
                ws=torch.rand(n, generator=g).to(d) / 1000, wide=padded(torch.randn(7, c, generator=g)),
                to=torch.randint(0, c, (7,), generator=g, dtype=torch.int32).to(d),
                to_x=torch.randint(0, f, (m,), generator=g, dtype=torch.int32).to(d))


def test_streams_and_repeats():
    """two streams at once and again: the same bits"""
    L = LY()
    a, b = tensors(1), tensors(2)
    want_a, want_b = everything(L, a), everything(L, b)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for s in (s1, s2):
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        with torch.cuda.stream(s1):
            got_a = everything(L, a)
        with torch.cuda.stream(s2):
            got_b = everything(L, b)
        torch.cuda.synchronize()
        for got, want in ((got_a, want_a), (got_b, want_b)):
            assert all(torch.equal(x, y) for x, y in zip(got, want))
    # the stream argument
    got = L.quant_linear(a["x"], a["w"], a["ws"], act="tanh", stream=s1)
    s1.synchronize()
    assert torch.equal(got, want_a[0])


def test_two_captured_graphs():
    """graphs replayed several times, eager work between, new inputs in the same places"""
    L = LY()
    a, b = tensors(1), tensors(2)
    everything(L, a)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for t in (a, b):
        gph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gph):
            outs.append(everything(L, t))
        graphs.append(gph)
    for turn in range(4):
        for t, seed in ((a, 10 + turn), (b, 20 + turn)):
            new = tensors(seed)
            for k in ("x", "few", "block", "gate", "wide"):
                t[k].copy_(new[k])
        want = [everything(L, t) for t in (a, b)]
        torch.cuda.synchronize()
        for gph in graphs:
            gph.replay()
        torch.cuda.synchronize()
        for got, w in zip(outs, want):
            assert all(torch.equal(x, y) for x, y in zip(got, w))


def test_largest_offsets():
    """rows that lie more than 2^31 elements into their matrix"""
    L = LY()
    m, f = 1100000, 2048
    x = torch.zeros((m, f), dtype=torch.bfloat16, device=device())
    assert m * f > 2 ** 31
    tail = torch.randn(3, f, generator=gen(4)).to(torch.bfloat16)
    x[-3:] = tail.to(device())
    q, s = L.quantize_rows(x)
    want_q, want_s = rows_exact(tail.double())
    assert torch.equal(q[-3:].cpu(), want_q) and torch.equal(s[-3:].cpu(), want_s)
    assert bool((q[:5] == 0).all())
    w = torch.randint(-127, 128, (40, f), generator=gen(5), dtype=torch.int8)
    ws = torch.full((40,), 1e-4)
    want, mag = product_exact(want_q, want_s, w, ws, None, "none", None)
    check_product(L.quant_linear(q, w.to(device()), ws.to(device()), x_scale=s)[-3:], want, mag, torch.float32)
    check_product(L.quant_linear(x, w.to(device()), ws.to(device()), out_dtype=torch.float32)[-3:], want, mag,
                  torch.float32)
    del q
    logp, ent, idx, val = L.label_log_probs(x, torch.zeros(m, dtype=torch.int32, device=device()), top_k=2)
    small = L.label_log_probs(tail.to(device()), torch.zeros(3, dtype=torch.int32, device=device()), top_k=2)
    for g, w_ in zip((logp, ent, idx, val), small):
        assert torch.allclose(g[-3:].double(), w_.double(), rtol=64 * U, atol=64 * U)
    assert idx[0].tolist() == [0, 1]
    y, z, _ = L.block_norm(x, x, pre="rms", in_place=False)
    y3, z3, _ = L.block_norm(tail.to(device()), tail.to(device()), pre="rms")
    assert torch.equal(y[-3:], y3) and torch.equal(z[-3:], z3)


def test_torch_entry_points_refuse():
    """what the tensors themselves give away, and what the library answers"""
    S, L = lib(), LY()
    d = device()
    x = torch.zeros(4, 32, device=d)
    w, ws = torch.zeros(8, 32, dtype=torch.int8, device=d), torch.ones(8, device=d)
    for f in (lambda: L.quant_linear(x.double(), w, ws), lambda: L.quant_linear(x, w.cpu(), ws),
              lambda: L.quant_linear(x, w[:, :16], ws), lambda: L.quant_linear(x, w, ws[:4]),
              lambda: L.quant_linear(x, w, ws, out_dtype=torch.float16),
              lambda: L.quant_linear(x, w, ws, row_scale_deg=torch.ones(4, device=d)),
              lambda: L.block_norm(x, x[:2]), lambda: L.block_norm(x, x.cpu()),
              lambda: L.block_norm(x, gate=x.bfloat16()), lambda: L.block_norm(x, in_place=True),
              lambda: L.block_norm(x, x, pre="rms", pre_weight=torch.ones(31, device=d)),
              lambda: L.label_log_probs(x, torch.zeros(4, dtype=torch.int64, device=d)),
              lambda: L.label_log_probs(x.t())):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: L.quant_linear(x, w, ws, x_scale=torch.ones(4, device=d)),          # float rows have no scale
              lambda: L.quant_linear(x.to(torch.int8), w, ws),                          # 8-bit rows need one
              lambda: L.quantize_rows(torch.zeros(4, 31, device=d)),                      # 124-byte rows
              lambda: L.block_norm(x, x, pre="rms", eps=0.0), lambda: L.label_log_probs(x, top_k=33),
              lambda: L.label_log_probs(x, entropy=False), lambda: L.quantize_rows(x[:1].expand(4, 32)),
              lambda: L.block_norm(x, x.bfloat16(), pre="rms")):
        with pytest.raises(S.SagaError):
            f()
    torch.cuda.synchronize()
