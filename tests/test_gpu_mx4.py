"""4-bit rows, their products and layers of experts against their definitions in
float64, each within the roundings its float32 steps make."""
import ctypes as C
import math

import pytest
import torch

from gpu_util import device, lib

pytestmark = pytest.mark.gpu

U = 2.0 ** -24            # half a step of float32, relative
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
FLOATS = [torch.float32, torch.bfloat16]
NAN, INF = float("nan"), float("inf")
VALUES = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)


def LY():
    lib()
    from paper_2009_00804_amd import layers

    return layers


def gen(seed):
    return torch.Generator().manual_seed(seed)


def padded(t, dtype=None, fill=None, extra=0, unit=16):
    """t on the GPU in a buffer whose rows are whole ``unit`` bytes and whose padding holds ``fill``"""
    dtype = dtype or t.dtype
    step = unit // dtype.itemsize
    ld = (t.shape[1] + step - 1) // step * step + extra * step
    if fill is None:
        fill = 0xff if dtype == torch.uint8 else NAN
    buf = torch.full((t.shape[0], ld), fill, dtype=dtype, device=device())
    buf[:, :t.shape[1]] = t.to(device()).to(dtype)
    return buf[:, :t.shape[1]]


def padding_of(t):
    """the columns of t's buffer past its own"""
    return t.as_strided((t.shape[0], t.stride(0) - t.shape[1]), t.stride(), t.storage_offset() + t.shape[1])


# --------------------------------------------------------------------------
# the format, by its definition
# --------------------------------------------------------------------------
def rows_exact(x):
    """(codes 0..15, scale bytes, values) of float64 rows"""
    m, k = x.shape
    v = torch.nn.functional.pad(x, (0, -k % 32)).view(m, -1, 32)
    top = v.abs().amax(2, keepdim=True)
    bad = ~torch.isfinite(top)
    clean = torch.where(bad, 0.0, top)
    e = torch.where(clean > 0, torch.frexp(clean)[1] - 3, torch.full_like(clean, -127).int()).clamp(min=-127)
    t = torch.ldexp(torch.where(bad, 0.0, v), -e)
    d = (t.abs()[..., None] - VALUES).abs()
    near = d.amin(3, keepdim=True)
    even = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7])  # of two equally near numbers the one of even mantissa
    code = even[(d[..., even] == near).int().argmax(3)]
    value = VALUES[code] * torch.where(torch.signbit(t), -1.0, 1.0) * torch.ldexp(torch.ones_like(clean), e)
    code = code + 8 * torch.signbit(t).int()
    byte = torch.where(bad, 255, e + 127)[..., 0].to(torch.uint8)
    value = torch.where(bad, NAN, value)
    return code.view(m, -1)[:, :k], byte, value.view(m, -1)[:, :k]


def packed(code):
    c = torch.nn.functional.pad(code, (0, code.shape[1] % 2)).view(code.shape[0], -1, 2)
    return (c[..., 0] | c[..., 1] << 4).to(torch.uint8)


def special_rows(k, g):
    """rows at which a quantiser can go wrong"""
    r = [torch.zeros(k), torch.full((k,), 1e-42), torch.randn(k, generator=g) * 1e-39,
         torch.randn(k, generator=g) * 1e-37, torch.randn(k, generator=g) * 1e37, torch.full((k,), -0.0),
         torch.full((k,), 3.4e38), torch.full((k,), 2.0 ** -126)]
    halves = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 7.9])
    ties = halves[torch.arange(k) % 10] * torch.where(torch.arange(k) % 20 < 10, 1.0, -1.0)
    ties[::32] = 4.0  # scale 1 in every block
    for s in (1.0, 2.0 ** 40, 2.0 ** -90):
        r += [ties * s, torch.nextafter(ties, torch.full((k,), 1e9)) * s,
              torch.nextafter(ties, -torch.full((k,), 1e9)) * s]
    for bad in (NAN, INF, -INF):
        b = torch.randn(k, generator=g)
        b[k // 2] = bad
        r.append(b)
    return torch.stack(r)


def values_of(code):
    return VALUES[code & 7] * torch.where(code > 7, -1.0, 1.0)


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("k", [1, 2, 7, 8, 31, 32, 33, 63, 64, 65, 100, 128, 256, 602, 1000, 1024, 1025, 2047, 4096,
                               5001, 20000])
def test_rows_exactly(k, dtype):
    S = lib()
    g = gen(k)
    x = torch.cat([torch.randn(13, k, generator=g) * 3, special_rows(k, g)]).to(dtype)
    code, byte, value = rows_exact(x.double())
    xd = padded(x, extra=1)
    q = padded(torch.full((x.shape[0], (k + 1) // 2), 99, dtype=torch.uint8), fill=77, extra=1)
    s = padded(torch.full((x.shape[0], (k + 31) // 32), 99, dtype=torch.uint8), fill=77, extra=1, unit=4)
    S.saga_quantize_rows_mx(S.dtype_code(dtype), S.cmat(xd), S.mat(q), S.mat(s), S.stream_handle())
    torch.cuda.synchronize()
    assert torch.equal(s.cpu(), byte)
    got = q.cpu().int()
    got = torch.stack([got & 15, got >> 4], 2).view(x.shape[0], -1)
    assert torch.equal(values_of(got[:, :k].long()), values_of(code.long()))  # (a zero of either sign)
    if k % 2:
        assert bool((got[:, k] == 0).all())
    assert bool((padding_of(q) == 77).all()) and bool((padding_of(s) == 77).all())
    # and back
    y = padded(torch.full((x.shape[0], k), 5.0), dtype=dtype, fill=3.0, extra=1)
    S.saga_dequantize_rows_mx(S.dtype_code(dtype), S.cmat(q), S.cmat(s), S.mat(y), S.stream_handle())
    torch.cuda.synchronize()
    want = value.to(dtype)
    got = y.cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got.nan_to_num(1), want.nan_to_num(1))
    assert bool((padding_of(y) == 3.0).all())


@pytest.mark.parametrize("dtype,k", [(torch.float32, 515), (torch.bfloat16, 1031)])
def test_values_that_no_cache_holds(dtype, k):
    """More than 256 MiB of values: the same as of the same rows a few at a time."""
    L = LY()
    m = (256 << 20) // (k * dtype.itemsize) + 77
    q = torch.randint(0, 256, (m, (k + 1) // 2), dtype=torch.uint8, device=device())
    s = torch.randint(0, 255, (m, (k + 31) // 32), dtype=torch.uint8, device=device())
    q, s = padded(q.cpu()), padded(s.cpu(), unit=4)
    x = L.dequantize_rows_mx4(q, s, k, dtype=dtype)
    for i in range(0, m, 50000):
        part = L.dequantize_rows_mx4(q[i:i + 50000], s[i:i + 50000], k, dtype=dtype)
        assert torch.equal(x[i:i + 50000], part)


def test_many_rows_and_none():
    L = LY()
    x = torch.randn(70001, 40, generator=gen(3))
    code, byte, value = rows_exact(x.double())
    q, s = L.quantize_rows_mx4(x.to(device()))
    assert torch.equal(s.cpu(), byte)
    assert torch.equal(L.dequantize_rows_mx4(q, s, dtype=torch.float32).cpu().double(), value)
    assert L.dequantize_rows_mx4(q, s, 39).shape == (70001, 39)
    q, s = L.quantize_rows_mx4(x[:0].to(device()))
    assert q.shape == (0, 20) and s.shape == (0, 2)
    assert L.dequantize_rows_mx4(q, s).shape == (0, 40)


# --------------------------------------------------------------------------
# product
# --------------------------------------------------------------------------
ACTS = {"none": lambda v: v, "relu": lambda v: v.clamp(min=0), "elu": lambda v: torch.where(v > 0, v, torch.expm1(v)),
        "sigmoid": torch.sigmoid, "tanh": torch.tanh}


def four_bits(x):
    """(q, scale, values) of float rows: on the GPU with garbage behind every row, and float64"""
    code, byte, value = rows_exact(x.double())
    return padded(packed(code)), padded(byte, unit=4), value


def check_product(got, x, w, bias, act, deg):
    """x, w: float64.  A sum of k products is exact products added in float32: at most one
    rounding for each 32 products and one for each sum of sums (here at most k / 32 + 16),
    relative to the sum of magnitudes; the degree's root, quotient and product and the
    bias are four more.  The activations have slopes of at most 1 and float32 functions that
    are a few U of their values (at most about 1 where they are curved) off: 8 U.  Then
    the rounding to the output's type."""
    v, mag = x @ w.T, x.abs() @ w.abs().T
    if deg is not None:
        d = deg.double()[:, None]
        rs = torch.where(d > 0, d.clamp(min=1) ** -0.5, 0.0)
        v, mag = v * rs, mag * rs
    if bias is not None:
        v = v + bias.double()
        mag = mag + bias.double().abs()
    want = ACTS[act](v)
    err = (got.double().cpu() - want).abs()
    tol = (x.shape[1] / 32 + 20) * U * mag + 8 * U * (1 + want.abs())
    if got.dtype != torch.float32:
        tol = tol + HALF[got.dtype] * want.abs()
    worst = (err / tol).max().item() if err.numel() else 0
    assert worst <= 1, worst


SIZES = [(1, 1, 1), (1, 1024, 1024), (3, 17, 5), (16, 128, 16), (17, 129, 33), (40, 602, 128), (64, 4096, 100),
         (100, 47, 256), (129, 256, 64), (257, 1025, 200), (1000, 64, 41), (500, 2000, 300), (300, 96, 1030),
         (5000, 200, 128), (2, 20000, 24), (4100, 33, 7)]


@pytest.mark.parametrize("m,k,n", SIZES)
@pytest.mark.parametrize("kind", ["mx4", torch.float32, torch.bfloat16])
def test_product(m, k, n, kind):
    L = LY()
    g = gen(m * 7 + k * 3 + n)
    x = torch.randn(m, k, generator=g) * (torch.rand(m, 1, generator=g) * 4 + 0.01)
    x[m // 2] = 0 if m > 2 else x[m // 2]
    w = torch.randn(n, k, generator=g) * torch.exp(torch.randn(n, 1, generator=g))
    bias = torch.randn(n, generator=g)
    deg = torch.randint(0, 9, (m,), generator=g, dtype=torch.int32)
    q, s, w64 = four_bits(w)
    x = x if kind == "mx4" else x.to(kind)
    xq, xs, x64 = four_bits(x)
    xd = xq if kind == "mx4" else padded(x, extra=1)
    scale = xs if kind == "mx4" else None
    i = 0
    for act in ACTS:
        for out in FLOATS:
            b, d = (bias if i % 2 else None), (deg if i % 3 == 0 else None)
            i += 1
            got = L.mx4_linear(xd, q, s, x_scale=scale, bias=None if b is None else b.to(device()), act=act,
                               row_scale_deg=None if d is None else d.to(device()), out_dtype=out)
            assert got.dtype == out and got.shape == (m, n)
            check_product(got, x64, w64, b, act, d)


@pytest.mark.parametrize("m,k,n", [(40001, 70, 33), (70000, 602, 128), (66000, 256, 40), (20000, 130, 700),
                                   (3000, 1024, 1024), (9000, 640, 520), (2000, 4096, 2048), (33000, 1300, 130)])
@pytest.mark.parametrize("kind", ["mx4", torch.float32, torch.bfloat16])
def test_large_products(m, k, n, kind):
    """many rows: the library's own 4-bit rows (tested by themselves) as the reference's, checked on the GPU"""
    L = LY()
    g = torch.Generator(device=device()).manual_seed(m + k)
    x = torch.randn(m, k, generator=g, device=device())
    w = torch.randn(n, k, generator=g, device=device())
    x = padded(x, dtype=torch.float32 if kind == "mx4" else kind)
    q, s = L.quantize_rows_mx4(padded(w))
    xq, xs = L.quantize_rows_mx4(x)
    x64 = L.dequantize_rows_mx4(xq, xs, k, dtype=torch.float32).double()
    w64 = L.dequantize_rows_mx4(q, s, k, dtype=torch.float32).double()
    got = L.mx4_linear(xq if kind == "mx4" else x, q, s, x_scale=xs if kind == "mx4" else None, act="relu",
                       out_dtype=torch.bfloat16)
    mag = x64.abs() @ w64.abs().T
    want = (x64 @ w64.T).clamp(min=0)
    tol = (k / 32 + 20) * U * mag + 8 * U * (1 + want) + HALF[torch.bfloat16] * want
    assert ((got.double() - want).abs() / tol).max().item() <= 1


@pytest.mark.parametrize("kind", ["mx4", torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,k,n", [(5, 100, 20), (300, 300, 40), (3000, 256, 260), (70000, 100, 30), (600, 1500, 600)])
def test_rows_without_numbers(m, k, n, kind):
    """a block with a NaN or an infinity makes its row NaN, whatever the activation, and no other"""
    L = LY()
    g = gen(k)
    x = torch.randn(m, k, generator=g).to(torch.float32 if kind == "mx4" else kind)
    clean = x.clone()
    bad = [1, m // 2, m - 1]
    x[1, 0], x[m // 2, k - 1], x[m - 1, k // 2] = NAN, INF, -INF
    w = torch.randn(n, k, generator=g)
    q, s = L.quantize_rows_mx4(padded(w))
    for act in ("none", "relu"):
        def run(t):
            t = padded(t)
            if kind != "mx4":
                return L.mx4_linear(t, q, s, act=act, out_dtype=torch.float32).cpu()
            tq, ts = L.quantize_rows_mx4(t)
            return L.mx4_linear(tq, q, s, x_scale=ts, act=act).cpu()
        got, other = run(x), run(clean)
        assert bool(torch.isnan(got[bad]).all())
        keep = torch.ones(m, dtype=torch.bool)
        keep[bad] = False
        assert torch.equal(got[keep], other[keep])


def test_channels_without_numbers():
    L = LY()
    w = torch.randn(50, 200, generator=gen(1))
    w[7, 199], w[30, 3] = NAN, INF
    q, s = L.quantize_rows_mx4(padded(w))
    got = L.mx4_linear(padded(torch.randn(33, 200, generator=gen(2))), q, s, act="relu").cpu()
    assert bool(torch.isnan(got[:, [7, 30]]).all()) and int(torch.isnan(got).sum()) == 2 * 33


def test_float_rows_as_their_own_four_bits():
    """a float row gives what its 4-bit form gives, to the bit, wherever one kernel takes both"""
    L = LY()
    for m, k, n in ((1, 70, 30), (20, 1024, 64), (48, 333, 100)):
        x, w = padded(torch.randn(m, k, generator=gen(m))), padded(torch.randn(n, k, generator=gen(n)))
        q, s = L.quantize_rows_mx4(w)
        xq, xs = L.quantize_rows_mx4(x)
        assert torch.equal(L.mx4_linear(x, q, s), L.mx4_linear(xq, q, s, x_scale=xs))


# --------------------------------------------------------------------------
# experts
# --------------------------------------------------------------------------
def route_exact(x, router, bias, top_k, renorm):
    logits = x.double() @ router.double().T
    if bias is not None:
        logits = logits + bias.double()
    order = torch.sort(logits, dim=1, descending=True, stable=True)[1][:, :top_k]
    mine = logits.gather(1, order)
    closed = mine == -INF
    p = torch.softmax(mine, 1) if renorm else torch.softmax(logits, 1).gather(1, order)
    return torch.where(closed, -1, order), torch.where(closed, 0.0, p)


def experts_exact(x, index, p, up, down, up_b, down_b, e, act, gated, dtype):
    """(y, tolerance): the float32 steps of each product counted as in check_product, a product of
    float32 rows being three terms or less and 8 terms of k an instruction; the values between
    them held to 2^-16 (dtype bfloat16) or 2^-24, activations 8 U, weights 16 U"""
    m, f = x.shape
    wide, h, n = up.shape[0] // e, up.shape[0] // e // (2 if gated else 1), down.shape[0] // e
    x, up, down = x.double(), up.double(), down.double()
    y, tol, total = x.new_zeros(m, n), x.new_zeros(m, n), x.new_zeros(m, n)
    split = 2.0 ** -16 if dtype == torch.bfloat16 else U
    for i in range(e):
        share = torch.where(index == i, p, 0.0).sum(1, keepdim=True)
        w, d = up[i * wide:(i + 1) * wide], down[i * n:(i + 1) * n]
        v, mag = x @ w.T, x.abs() @ w.abs().T
        if up_b is not None:
            b = up_b.double()[i * wide:(i + 1) * wide]
            v, mag = v + b, mag + b.abs()
        off = (3 * f / 8 + 20) * U * mag
        hid = ACTS[act](v[:, :h])
        hid_off = off[:, :h] + 8 * U * (1 + hid.abs())
        if gated:
            hid_off = hid_off * (v[:, h:].abs() + off[:, h:]) + hid.abs() * off[:, h:]
            hid = hid * v[:, h:]
        hid_off = hid_off + (split + U) * (hid.abs() + hid_off)
        z, zmag = hid @ d.T, (hid.abs() + hid_off) @ d.abs().T
        z_off = hid_off @ d.abs().T + (3 * h / 8 + 20) * U * zmag
        if down_b is not None:
            z = z + down_b.double()[i * n:(i + 1) * n]
        y += share * z
        total += share * z.abs()
        tol += share * (z_off + 16 * U * z.abs())
    tol += 20 * U * total + 1e-30
    if dtype != torch.float32:
        tol = tol + HALF[dtype] * (y.abs() + tol)
    return y, tol


class Layer:
    def __init__(self, seed, f, h, n, e, weights, gated=False, biases=False, router_dtype=torch.float32, closed=()):
        L = LY()
        g = gen(seed)
        self.e, self.h, self.n, self.gated = e, h, n, gated
        wide = h * (2 if gated else 1)
        self.router = (torch.randn(e, f, generator=g) / math.sqrt(f)).to(router_dtype)
        self.up = torch.randn(e * wide, f, generator=g) / math.sqrt(f)
        self.down = torch.randn(e * n, h, generator=g) / math.sqrt(h)
        vec = lambda k: torch.randn(k, generator=g) * 0.3  # noqa: E731
        self.router_b = vec(e) if biases or closed else None
        for c in closed:
            self.router_b[c] = -INF
        self.up_b, self.down_b = (vec(e * wide), vec(e * n)) if biases else (None, None)
        self.kw = {}
        if weights == "mx4":
            (uq, us, self.up), (dq, ds, self.down) = four_bits(self.up), four_bits(self.down)
            self.up_d, self.down_d = uq, dq
            self.kw = dict(up_scale=us, down_scale=ds)
        else:
            self.up, self.down = self.up.bfloat16(), self.down.bfloat16()
            self.up_d, self.down_d = padded(self.up, extra=1), padded(self.down, extra=1)
        for name in ("router_b", "up_b", "down_b"):
            v = getattr(self, name)
            self.kw[{"router_b": "router_bias", "up_b": "up_bias", "down_b": "down_bias"}[name]] = (
                None if v is None else v.to(device()))
        self.router_d = padded(self.router)
        self.L = L

    def __call__(self, x, **kw):
        return self.L.expert_layer(x, self.router_d, self.up_d, self.down_d, gated=self.gated, **self.kw, **kw)

    def check(self, x, top_k, act="relu", renorm=True, got=None):
        y, index, weight = got or self(padded(x), top_k=top_k, act=act, renormalise=renorm)
        want_i, want_p = route_exact(x, self.router, self.router_b, top_k, renorm)
        assert index.dtype == torch.int32 and torch.equal(index.cpu().long(), want_i)
        # differences of float64 logits rounded once, at most 80 or so: e^d is off by d U; exponential,
        # sum and quotient a few U more
        assert ((weight.cpu().double() - want_p).abs() <= 100 * U * want_p + 1e-36).all()
        want, tol = experts_exact(x, want_i, want_p, self.up, self.down, self.up_b, self.down_b, self.e, act,
                                  self.gated, x.dtype)
        worst = ((y.cpu().double() - want).abs() / tol).max().item()
        assert worst <= 1, worst


EXPERT_SIZES = [  # rows, f, h, n, experts, top_k
    (1, 1, 1, 1, 1, 1), (1, 128, 256, 128, 4, 1), (1, 33, 65, 17, 5, 5), (2, 130, 31, 50, 70, 3),
    (5, 64, 100, 602, 3, 2), (17, 602, 129, 41, 16, 2), (16, 1000, 300, 8, 9, 4), (40, 256, 500, 200, 8, 1),
    (64, 200, 70, 64, 64, 2), (100, 96, 513, 40, 4, 3), (200, 48, 64, 48, 2, 2), (300, 20, 40, 30, 100, 16),
]


@pytest.mark.parametrize("m,f,h,n,e,top_k", EXPERT_SIZES)
@pytest.mark.parametrize("weights", ["mx4", "bf16"])
@pytest.mark.parametrize("dtype", FLOATS)
def test_experts(m, f, h, n, e, top_k, weights, dtype):
    g = gen(m + f)
    x = torch.randn(m, f, generator=g).to(dtype)
    for i, (gated, biases) in enumerate([(False, False), (True, False), (False, True), (True, True)]):
        layer = Layer(m * 31 + i, f, h, n, e, weights, gated, biases,
                      router_dtype=FLOATS[i % 2], closed=[1] if e > 2 and i == 3 else ())
        act = ["relu", "sigmoid", "elu", "tanh"][(i + m) % 4]
        layer.check(x, top_k, act, renorm=(i + f) % 3 != 0)


@pytest.mark.parametrize("m,f,h,n,e,top_k", [(3, 130, 20000, 140, 4, 1), (40, 602, 1100, 300, 20, 2),
                                             (200, 200, 2100, 130, 8, 2), (600, 1000, 700, 515, 24, 4),
                                             (700, 129, 4500, 100, 4, 1), (1024, 64, 130, 1030, 256, 3)])
@pytest.mark.parametrize("weights", ["mx4", "bf16"])
@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("gated", [False, True])
def test_large_layers(m, f, h, n, e, top_k, weights, dtype, gated):
    """weights enough for the kernels that are bounded by them, one row to hundreds an expert"""
    layer = Layer(m, f, h, n, e, weights, gated, biases=gated)
    layer.check(torch.randn(m, f, generator=gen(m)).to(dtype), top_k, "sigmoid" if gated else "relu")


@pytest.mark.parametrize("m,f,h,n,e,top_k", [(1, 2000, 4096, 33, 8, 2), (2, 1024, 1024, 40, 8, 4),
                                             (2, 1032, 1032, 40, 8, 4), (2, 1024, 512, 40, 8, 4),
                                             (3, 128, 100, 40, 9, 2), (4, 256, 250, 70, 4, 2),
                                             (4, 264, 258, 70, 4, 2), (16, 130, 220, 50, 9, 4), (16, 130, 110, 50, 9, 4),
                                             (16, 40, 64, 20, 40, 4), (16, 130, 230, 50, 9, 4)])
@pytest.mark.parametrize("weights", ["mx4", "bf16"])
@pytest.mark.parametrize("dtype", FLOATS)
def test_few_rows_two_kernels_or_four(m, f, h, n, e, top_k, weights, dtype):
    """sizes on both sides of what the kernels of few rows take and of where they choose themselves"""
    for gated in (False, True):
        layer = Layer(m + h, f, h, n, e, weights, gated, biases=True)
        layer.check(torch.randn(m, f, generator=gen(m + f)).to(dtype), top_k, "tanh")


def at_the_end(t):
    """t on the GPU, pitch a multiple of 16 bytes, as the last rows of 24 MiB that are an allocation"""
    ld = (t.shape[1] * t.element_size() + 15) // 16 * 16 // t.element_size()
    buf = torch.empty((24 << 20) // t.element_size(), dtype=t.dtype, device=device())
    rows = buf[buf.numel() - t.shape[0] * ld:].view(t.shape[0], ld)
    rows.fill_(NAN)
    rows[:, :t.shape[1]] = t.to(device())
    return rows[:, :t.shape[1]]


@pytest.mark.parametrize("k", [1, 3, 4, 12, 33, 36, 100, 129, 132])
@pytest.mark.parametrize("dtype", FLOATS)
def test_last_rows_of_an_allocation(k, dtype):
    """nothing past the last row's pitch is read: rows are whole 16 bytes, four columns of float32"""
    L = LY()
    for m in (1, 5, 20, 4099):
        x = torch.randn(m, k, generator=gen(k + m)).to(dtype)
        code, byte, value = rows_exact(x.double())
        xd = at_the_end(x)
        q, s = L.quantize_rows_mx4(xd)
        assert torch.equal(s.cpu(), byte)
        wq, ws, w = four_bits(torch.randn(70, k, generator=gen(k)))
        y = L.mx4_linear(xd, wq, ws, out_dtype=torch.float32).cpu().double()
        want, size = value @ w.double().t(), value.abs() @ w.double().abs().t()
        assert ((y - want).abs() <= (k + 8) * U * size + 1e-30).all()  # (exact products, k float32 sums)
    for m in (1, 3, 16, 40):
        layer = Layer(m + k, k, 40, 24, 5, "mx4", True, True)
        x = torch.randn(m, k, generator=gen(m)).to(dtype)
        layer.check(x, 2, got=layer(at_the_end(x), top_k=2))


def test_more_rows_than_one_run():
    """more than 1024 rows: the kernels run for each part, rows of one expert more than a tile"""
    layer = Layer(5, 40, 50, 24, 6, "mx4", True, True)
    x = torch.randn(2500, 40, generator=gen(6))
    layer.check(x, 2, "sigmoid")
    empty = layer(padded(x)[:0], top_k=2)
    assert empty[0].shape == (0, 24) and empty[1].shape == (0, 2)


def test_equal_logits_go_to_the_first():
    layer = Layer(5, 64, 32, 16, 130, "bf16")
    layer.router[:] = layer.router[0]
    layer.router_d = padded(layer.router)
    _, index, weight = layer(padded(torch.randn(9, 64, generator=gen(6))), top_k=4)
    assert torch.equal(index.cpu(), torch.arange(4, dtype=torch.int32).expand(9, 4))
    assert ((weight - 0.25).abs() <= 4 * U).all()


@pytest.mark.parametrize("renorm", [True, False])
def test_closed_experts(renorm):
    x = torch.randn(50, 64, generator=gen(6))
    layer = Layer(5, 64, 32, 16, 5, "mx4", biases=True, closed=[0, 2, 3])
    layer.check(x, 4, renorm=renorm)
    _, index, weight = layer(padded(x), top_k=4, renormalise=renorm)
    assert bool((index[:, 2:] == -1).all()) and bool((weight[:, 2:] == 0).all())
    layer = Layer(5, 64, 32, 16, 5, "mx4", biases=True, closed=range(5))
    y, index, weight = layer(padded(x), top_k=2, renormalise=renorm)
    assert bool((y == 0).all()) and bool((index == -1).all()) and bool((weight == 0).all())


@pytest.mark.parametrize("dtype", FLOATS)
def test_expert_rows_without_numbers(dtype):
    layer = Layer(5, 70, 33, 40, 6, "mx4", True)
    x = torch.randn(40, 70, generator=gen(6)).to(dtype)
    clean = padded(x)
    want = layer(clean, top_k=2)
    x[3, 69], x[20, 0], x[39, 5] = NAN, INF, -INF
    y, index, weight = layer(padded(x), top_k=2)
    bad = [3, 20, 39]
    keep = [i for i in range(40) if i not in bad]
    assert bool(torch.isnan(y[bad]).all()) and bool(torch.isnan(weight[bad]).all()) and bool((index[bad] == -1).all())
    for a, b in zip((y, index, weight), want):
        assert torch.equal(a[keep], b[keep])


@pytest.mark.parametrize("m,f,e", [(5, 70, 6), (16, 600, 9), (1, 70, 3)])
@pytest.mark.parametrize("weights", ["mx4", "bf16"])
@pytest.mark.parametrize("dtype", FLOATS)
def test_few_rows_without_numbers_or_experts(m, f, e, weights, dtype):
    """the kernels of few rows, with the choice in the first of them and without"""
    layer = Layer(5, f, 33, 40, e, weights, True, biases=True, closed=[1])
    x = torch.randn(m, f, generator=gen(6)).to(dtype)
    want = layer(padded(x), top_k=2)
    layer.check(x, 2, got=want)
    bad = [0] if m == 1 else [0, m - 1]
    x[0, f - 1] = NAN
    if m > 1:
        x[m - 1, 0] = -INF
    y, index, weight = layer(padded(x), top_k=2)
    assert bool(torch.isnan(y[bad]).all()) and bool(torch.isnan(weight[bad]).all()) and bool((index[bad] == -1).all())
    keep = [i for i in range(m) if i not in bad]
    for a, b in zip((y, index, weight), want):
        assert torch.equal(a[keep], b[keep])
    closed = Layer(5, f, 33, 40, e, weights, True, biases=True, closed=range(e))
    y, index, weight = closed(padded(x[:0] if m == 1 else x[1:-1]), top_k=2)
    assert bool((y == 0).all()) and bool((index == -1).all()) and bool((weight == 0).all())


def test_a_router_without_numbers():
    """a NaN in an expert's row of the router: no row has a choice"""
    for m in (3, 50):
        layer = Layer(5, 64, 32, 16, 5, "mx4")
        layer.router_d[2, 7] = NAN
        y, index, weight = layer(padded(torch.randn(m, 64, generator=gen(6))), top_k=2)
        assert bool(torch.isnan(y).all()) and bool((index == -1).all()) and bool(torch.isnan(weight).all())


@pytest.mark.parametrize("m,f,h,e", [(300, 200, 300, 60), (90, 300, 4000, 64), (200, 128, 3000, 12)])
@pytest.mark.parametrize("weights", ["mx4", "bf16"])
@pytest.mark.parametrize("dtype", FLOATS)
def test_all_rows_take_one_expert(m, f, h, e, weights, dtype):
    """far more rows of one expert than of the mean: more tiles than one of it, none of others"""
    layer = Layer(5, f, h, 70, e, weights, True, closed=[i for i in range(e) if i not in (1, 2)])
    layer.check(torch.randn(m, f, generator=gen(6)).to(dtype), 2, "tanh")


def test_hidden_values_beyond_float32():
    """an expert whose values between the products overflow gives no number, others theirs"""
    layer = Layer(5, 64, 40, 24, 4, "bf16")
    layer.up_d[40:80] *= 1e38
    x = torch.randn(50, 64, generator=gen(6))
    y, index, _ = layer(padded(x), top_k=1)
    took = (index[:, 0] == 1).cpu()
    assert took.any() and not took.all()
    assert bool(torch.isfinite(y.cpu()[~took]).all())


def test_wide_pitches():
    """rows far apart, and part of wider buffers, give what rows next to each other give"""
    L = LY()
    g = gen(4)
    x, w = torch.randn(70, 200, generator=g), torch.randn(90, 200, generator=g)
    q, s = L.quantize_rows_mx4(padded(w))
    want = L.mx4_linear(padded(x), q, s)
    far_q, far_s = padded(q.cpu(), extra=700), padded(s.cpu(), extra=900, unit=4)
    assert torch.equal(L.mx4_linear(padded(x, extra=4001), far_q, far_s), want)
    xq, xs = L.quantize_rows_mx4(padded(x, extra=33))
    big_q = torch.full((140, 512), 0xff, dtype=torch.uint8, device=device())
    big_s = torch.full((140, 64), 0xff, dtype=torch.uint8, device=device())
    big_q[::2, 16:116], big_s[::2, 4:11] = xq, xs
    assert torch.equal(L.mx4_linear(big_q[::2, 16:116], far_q, far_s, x_scale=big_s[::2, 4:11]), want)


def test_two_calls_at_once():
    """two streams, each with calls of its own sizes: the bits of one call alone"""
    L = LY()
    layer = Layer(5, 96, 130, 96, 8, "mx4", True, True)
    q, s = L.quantize_rows_mx4(padded(torch.randn(96, 96, generator=gen(1)) / 10))
    xs = [padded(torch.randn(m, 96, generator=gen(m))) for m in (9, 1500)]
    want = [[t.clone() for t in chain(L, layer, x, q, s)] for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        got = []
        for st, x in zip(streams, xs):
            with torch.cuda.stream(st):
                got.append(chain(L, layer, x, q, s))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(p, r) for p, r in zip(a, b))


def test_experts_that_no_row_takes_may_hold_anything():
    layer = Layer(5, 64, 48, 32, 4, "bf16", closed=[2])
    layer.up_d[2 * 48:3 * 48] = NAN
    layer.down_d[2 * 32:3 * 32] = NAN
    layer.check(torch.randn(7, 64, generator=gen(6)), 3)


# --------------------------------------------------------------------------
# how they are called
# --------------------------------------------------------------------------
def chain(L, layer, x, q, s):
    """a transform of float rows, its result in 4 bits, another transform, experts"""
    h = L.mx4_linear(x, q, s, act="relu")
    hq, hs = L.quantize_rows_mx4(h)
    h = L.mx4_linear(hq, q, s, x_scale=hs, out_dtype=torch.float32)
    return (h, *layer(h, top_k=2, act="sigmoid"))


def test_streams_and_graphs():
    """the operators as they are used together: on another stream, and captured, replayed
    with new inputs and eager work between; two captured graphs share nothing"""
    L = LY()
    layer = Layer(5, 96, 130, 96, 8, "mx4", True, True)
    q, s = L.quantize_rows_mx4(padded(torch.randn(96, 96, generator=gen(1)) / 10))
    xs = [padded(torch.randn(m, 96, generator=gen(m))) for m in (1, 37)]
    want = [[t.clone() for t in chain(L, layer, x, q, s)] for x in xs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = chain(L, layer, xs[1], q, s)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(got, want[1]):
        assert torch.equal(a, b)
    y = L.mx4_linear(xs[1], q, s, act="relu", stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, L.mx4_linear(xs[1], q, s, act="relu"))
    graphs, outs, ins = [], [], [x.clone() for x in xs]
    ins = [padded(x.cpu()) for x in xs]
    for x in ins:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs.append(chain(L, layer, x, q, s))
        graphs.append(gr)
    for turn in range(4):
        for i in (0, 1) if turn % 2 else (1, 0):
            fresh = torch.randn(xs[i].shape, generator=gen(100 * turn + i)).to(device())
            ins[i].copy_(fresh)
            eager = [t.clone() for t in chain(L, layer, ins[i], q, s)]
            graphs[i].replay()
            torch.cuda.synchronize()
            for a, b in zip(outs[i], eager):
                assert torch.equal(a, b)


def test_refused_tensors():
    L = LY()
    x = padded(torch.randn(4, 64))
    q, s = L.quantize_rows_mx4(x)
    with pytest.raises(ValueError, match="w_scale"):
        L.mx4_linear(x, q, None)
    with pytest.raises(ValueError, match="x_scale"):
        L.mx4_linear(q, q, s)
    with pytest.raises(ValueError, match="x_scale"):
        L.mx4_linear(x, q, s, x_scale=s)
    with pytest.raises(ValueError, match="w: shape"):
        L.mx4_linear(x, q[:, :31], s)
    with pytest.raises(ValueError, match="w_scale: shape"):
        L.mx4_linear(x, q, s[:, :1])
    with pytest.raises(ValueError, match="scale"):
        L.mx4_linear(x, q, s.int())
    with pytest.raises(ValueError, match="bias"):
        L.mx4_linear(x, q, s, bias=torch.zeros(5, device=device()))
    with pytest.raises(lib().SagaError, match="shape"):
        L.dequantize_rows_mx4(q, s, 60)
    layer = Layer(5, 64, 48, 32, 4, "mx4")
    with pytest.raises(ValueError, match="router"):
        L.expert_layer(x, layer.router_d[:, :63], layer.up_d, layer.down_d, **layer.kw)
    with pytest.raises(ValueError, match="no multiple"):
        L.expert_layer(x, layer.router_d, layer.up_d[:-1], layer.down_d, **layer.kw)
    with pytest.raises(ValueError, match="up_scale"):
        L.expert_layer(x, layer.router_d, layer.up_d, layer.down_d)
    with pytest.raises(lib().SagaError, match="top_k"):
        layer(x, top_k=5)


# --------------------------------------------------------------------------
# in a network
# --------------------------------------------------------------------------
def network(bits, dtype, gated, seed=7, n=203, f_in=50, f=72, classes=11, depth=2, e=6, h=40):
    import numpy as np

    from gpu_util import graph
    from helpers import edges_to_csr

    rng = np.random.default_rng(seed)
    rp, col, _ = edges_to_csr(n, rng.integers(0, n, n * 6).tolist(), rng.integers(0, n, n * 6).tolist())
    g = gen(seed)
    mat = lambda *s: torch.randn(*s, generator=g) / s[-2] ** 0.5  # noqa: E731
    vec = lambda *s: torch.randn(*s, generator=g) * 0.1  # noqa: E731
    w = dict(W_in=mat(f_in, f), b_in=vec(f), norm=vec(f) + 1, W_out=mat(f, classes), b_out=vec(classes),
             blocks=[dict(W=mat(f, f), W_g=mat(f, f), b=vec(f), b_g=vec(f), pre=vec(f) + 1, post=vec(f) + 1)
                     for _ in range(depth)],
             experts=dict(norm=vec(f) + 1, router=mat(f, e), up=mat(e, f, h), down=mat(e, h, f), top_k=2, act="sigmoid",
                          b_router=vec(e), b_up=vec(e, h), b_down=vec(e, f)))
    if gated:
        w["experts"].update(gate=mat(e, f, h), b_gate=vec(e, h))
    gr = graph(rp, col)
    x = torch.randn(n, f_in, generator=g)
    return LY().ResidualGCN(gr, w, dtype=dtype, res_scale=0.5, bits=bits), w, padded(x)


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("bits,gated", [(4, True), (4, False), (8, True)])
def test_network_of_experts(bits, dtype, gated):
    """Each stage that a tested operator does is taken from it; the network has the stages' bits,
    its experts' layer is the definition's on the rows that enter it, and vertices asked for
    have the answers that they have among all."""
    L = LY()
    net, w, x = network(bits, dtype, gated)
    f, n = net.f, x.shape[0]
    seen = {}
    real = L.expert_layer

    def watch(z, *args, **kw):
        seen["z"], seen["out"] = z, real(z, *args, **kw)
        return seen["out"]

    L.expert_layer = watch
    try:
        logits = net.logits(x)
    finally:
        L.expert_layer = real
    # by hand
    lin = (lambda z, t, zs, out: L.mx4_linear(z, t[0], t[1], bias=t[2], out_dtype=out)) if bits == 4 else (
        lambda z, t, zs, out: L.quant_linear(z, t[0], t[1], x_scale=zs, bias=t[2], out_dtype=out))
    norms = [b["pre"] for b in net.blocks] + [net.experts["norm"]]
    h, z, zs = L.block_norm(lin(x, net.first, None, dtype), None, x_dtype=torch.float32, pre="rms",
                            pre_weight=norms[0], quantize=bits == 8)
    for i, b in enumerate(net.blocks):
        vg = lin(z, b["both"], zs, dtype)
        m = net.gather(vg[:, :f], b["bias"])
        h, z, zs = L.block_norm(m, h, post="rms", post_weight=b["post"], gate=vg[:, f:], gate_act="sigmoid",
                                res_scale=0.5, pre="rms", pre_weight=norms[i + 1],
                                quantize=bits == 8 and i + 1 < len(net.blocks))
    assert torch.equal(z, seen["z"])
    # the experts, from the weights as given
    ex = w["experts"]
    up, down = ex["up"].transpose(1, 2), ex["down"].transpose(1, 2).reshape(-1, ex["up"].shape[2])
    up_b = ex["b_up"]
    if gated:
        up, up_b = torch.cat([ex["gate"].transpose(1, 2), up], 1), torch.cat([ex["b_gate"], ex["b_up"]], 1)
    up = up.reshape(-1, f)
    up, down = (rows_exact(t.double())[2] if bits == 4 else t.bfloat16().double() for t in (up, down))
    zc = z.cpu()
    index, p = route_exact(zc, ex["router"].T, ex["b_router"], 2, True)
    y, got_i, got_p = seen["out"]
    assert torch.equal(got_i.cpu().long(), index)
    want, tol = experts_exact(zc, index, p, up, down, up_b.reshape(-1), ex["b_down"].reshape(-1), ex["router"].shape[1],
                              "sigmoid", gated, dtype)
    assert ((y.cpu().double() - want).abs() / tol).max().item() <= 1
    _, z, zs = L.block_norm(y, h, res_scale=0.5, pre="rms", pre_weight=net.norm, quantize=bits == 8)
    assert torch.equal(lin(z, net.last, zs, torch.float32), logits)
    # some vertices, one of them twice
    to = torch.randint(0, 11, (5,), generator=gen(3), dtype=torch.int32).to(device())
    ask = torch.tensor([n - 1, 0, 7, 7, 100], device=device())
    some = net(x, to, 3, vertices=ask)
    every = L.label_log_probs(net.logits(x, ask), to, 3)
    for a, b in zip(some, every):
        assert torch.equal(a, b)
    # (few rows go through other kernels: the same values within the tolerances of both, through
    # a norm and a quantiser that may turn them by a step)
    near = net.logits(x, ask) - logits[ask]
    assert near.abs().max().item() <= 0.25 * logits.abs().max().item()


def test_network_in_four_bits_captured():
    L = LY()
    net, _, x = network(4, torch.bfloat16, True)
    ask = torch.tensor([3, 50, 77], device=device())
    net(x, top_k=2, vertices=ask)
    torch.cuda.synchronize()
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        got = net(x, top_k=2, vertices=ask)
    for turn in range(3):
        x.copy_(torch.randn(x.shape, generator=gen(40 + turn)).to(device()))
        want = net(x, top_k=2, vertices=ask)
        torch.cuda.synchronize()
        gr.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got[1:], want[1:]))


@pytest.mark.parametrize("ids", [torch.int32, torch.int64])
@pytest.mark.parametrize("bits,experts", [(4, True), (8, True), (4, False), (8, False)])
def test_vertices_outside_the_graph(bits, experts, ids):
    """an id that is no vertex's has NaN for logits, the others what they have without it"""
    net, w, x = network(bits, torch.bfloat16, True)
    if not experts:
        net = LY().ResidualGCN(net.graph, {k: v for k, v in w.items() if k != "experts"}, res_scale=0.5, bits=bits)
    n, far = x.shape[0], torch.iinfo(ids)
    ask = torch.tensor([5, -1, n - 1, n, far.max, 0, far.min, 5], dtype=ids).to(device())
    good = [0, 2, 5, 7]
    bad = [1, 3, 4, 6]
    got = net.logits(x, ask)
    clean = ask.clone()
    clean[bad] = 9
    want = net.logits(x, clean)
    assert bool(torch.isfinite(want).all())
    assert torch.equal(got[good], want[good]) and bool(torch.isnan(got[bad]).all())
    logp, entropy, index, top = net(x, torch.zeros(8, dtype=torch.int32, device=device()), 2, vertices=ask)
    assert bool(torch.isnan(logp[bad]).all()) and bool((index[bad] == -1).all())
    assert bool(torch.isfinite(logp[good]).all()) and bool((index[good] >= 0).all())
    assert net.logits(x, ask[:0]).shape == (0, want.shape[1])
    for wrong in (ask.cpu(), ask.float(), ask[None], [1, 2]):
        with pytest.raises(ValueError, match="vertices"):
            net.logits(x, wrong)


def test_network_refusals():
    with pytest.raises(ValueError, match="bits"):
        network(6, torch.bfloat16, True)
