"""4-bit products and layers of experts at sizes that take each of their kernels with every
epilogue, slice and remainder: against the definitions in float64, as in test_gpu_mx4."""
import pytest
import torch

from gpu_util import device
from test_gpu_mx4 import ACTS, FLOATS, HALF, LY, U, Layer, experts_exact, four_bits, gen, network, padded, route_exact

pytestmark = pytest.mark.gpu


# --------------------------------------------------------------------------
# values between the products that float32 does not hold
# --------------------------------------------------------------------------
def overflowing(m, f, h, n, e, top_k, weights, gated, channel, seed=11):
    """(a layer, x, rows that take expert 1): row i takes the experts i, i + 1.. of e; both last columns of x are
    2; nothing overflows yet.  `overflow` puts 2^127 into both columns of one channel of expert 1."""
    layer = Layer(seed, f, h, n, e, weights, gated)
    layer.router[:] = 0
    layer.router[torch.arange(e), torch.arange(e)] = 1.0
    layer.router_d = padded(layer.router)
    x = torch.randn(m, f, generator=gen(seed + 1))
    x[:, :e] = 0
    rows = torch.arange(m)
    for j in range(top_k):
        x[rows, (rows + j) % e] = 8.0 - j
    x[:, f - 2:] = 2.0
    took = ((1 - rows) % e) < top_k
    wide = h * (2 if gated else 1)
    at = wide + (h if gated else 0) + channel  # (gated: the up, behind all gates of the expert)

    def overflow():
        row = layer.up[at:at + 1].double().clone()
        row[:, f - 2:] = 2.0 ** 127
        if weights == "mx4":
            q, s, value = four_bits(row)
            layer.up_d[at], layer.kw["up_scale"][at] = q[0], s[0]
            layer.up[at] = value[0]
        else:
            layer.up_d[at] = row[0].bfloat16().to(device())
            layer.up[at] = row[0].bfloat16()
        return layer.up[at].double()

    return layer, x, took, overflow


@pytest.mark.parametrize("m,f,h,n,e,top_k", [
    (4, 40, 40, 24, 4, 1), (3, 40, 40, 24, 4, 2),          # two kernels, the first chooses
    (16, 600, 33, 40, 4, 1), (9, 70, 65, 17, 8, 2),        # two kernels
    (40, 70, 100, 50, 4, 2),                               # 16 channels a workgroup
    (64, 130, 1100, 140, 32, 2),                           # weights by way of registers, a few rows an expert
    (200, 130, 1100, 140, 32, 2), (400, 130, 1100, 140, 32, 2), (700, 130, 1100, 140, 32, 2),  # tiles
])
@pytest.mark.parametrize("weights", ["mx4", "bf16"])
@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("gated", [False, True])
def test_hidden_values_that_overflow(m, f, h, n, e, top_k, weights, dtype, gated):
    """a value between the products beyond float32 makes its row NaN, all of it, and leaves the others their bits"""
    act = "sigmoid" if gated else "relu"
    for channel in (0, h - 1):
        layer, x, took, overflow = overflowing(m, f, h, n, e, top_k, weights, gated, channel)
        x = x.to(dtype)
        xd = padded(x)
        want = [t.clone() for t in layer(xd, top_k=top_k, act=act)]
        assert torch.equal(want[1].cpu().long(), route_exact(x, layer.router, None, top_k, True)[0])
        assert bool(torch.isfinite(want[0]).all())
        v = x.double() @ overflow()
        assert took.any() and not took.all() and bool((v[took] >= 2.0 ** 128).all())
        y, index, weight = layer(xd, top_k=top_k, act=act)
        assert torch.equal(index, want[1]) and torch.equal(weight, want[2])
        assert bool(torch.isnan(y.cpu()[took]).all())
        assert torch.equal(y.cpu()[~took], want[0].cpu()[~took])


FAMILIES = [(3, 64, 40, 24, 4), (16, 600, 33, 40, 4), (60, 70, 100, 50, 4), (64, 130, 1100, 140, 32),
            (200, 130, 1100, 140, 32), (400, 130, 1100, 140, 32), (700, 130, 1100, 140, 32)]  # rows, f, h, n, experts


@pytest.mark.parametrize("m,f,h,n,e", FAMILIES)
@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("gated", [False, True])
def test_blocks_of_weights_without_numbers(m, f, h, n, e, dtype, gated):
    """the scale byte 255 in a 4-bit expert: in a down's row that channel of the rows that take the expert is NaN, in an
    up's row all channels are; no other row sees it, nor does a byte behind the last block"""
    layer = Layer(m, f, h, n, e, "mx4", gated)
    x = padded(torch.randn(m, f, generator=gen(m)).to(dtype))
    act = "sigmoid" if gated else "none"
    want, index, weight = (t.cpu() for t in layer(x, top_k=2, act=act))
    took = (index == 1).any(1)
    assert took.any() and not took.all() and bool(torch.isfinite(want).all())
    scale = layer.kw["down_scale"]
    old = scale[n + 7, (h - 1) // 32].clone()
    scale[n + 7, (h - 1) // 32] = 255
    y = layer(x, top_k=2, act=act)[0].cpu()
    assert bool(torch.isnan(y[took, 7]).all())
    y[took, 7] = want[took, 7]
    assert torch.equal(y, want)
    scale[n + 7, (h - 1) // 32] = old
    wide = h * (2 if gated else 1)
    layer.kw["up_scale"][wide + wide - 1, 0] = 255
    y, i2, w2 = (t.cpu() for t in layer(x, top_k=2, act=act))
    assert torch.equal(i2, index) and torch.equal(w2, weight)
    assert bool(torch.isnan(y[took]).all()) and torch.equal(y[~took], want[~took])


@pytest.mark.parametrize("m,f,h,n,e", FAMILIES)
@pytest.mark.parametrize("dtype", FLOATS)
def test_smallest_scales_of_weights(m, f, h, n, e, dtype):
    """4-bit weights whose scales are at and next to the smallest, 2^-127, which no normal float32 is"""
    layer = Layer(m, f, h, n, e, "mx4")
    uq, us, up = four_bits(torch.randn(e * h, f, generator=gen(m)) * 2.0 ** -125)
    assert int((us == 0).sum()) > 0 and int((us == 1).sum()) > 0
    layer.up, layer.up_d, layer.kw["up_scale"] = up, uq, us
    layer.router *= 2.0 ** -120
    layer.router_d = padded(layer.router)
    x = (torch.randn(m, f, generator=gen(m + 1)) * 2.0 ** 120).to(dtype)
    layer.check(x, 2, "none")


# --------------------------------------------------------------------------
# products: every kernel with every epilogue
# --------------------------------------------------------------------------
def check_sums(got, v, mag, k, bias, act, deg):
    """check_product's roundings, on the GPU: v and mag are the sums and those of magnitudes in float64"""
    if deg is not None:
        d = deg.double()[:, None]
        rs = torch.where(d > 0, d.clamp(min=1) ** -0.5, 0.0)
        v, mag = v * rs, mag * rs
    if bias is not None:
        v = v + bias.double()
        mag = mag + bias.double().abs()
    want = ACTS[act](v)
    tol = (k / 32 + 20) * U * mag + 8 * U * (1 + want.abs())
    if got.dtype != torch.float32:
        tol = tol + HALF[got.dtype] * want.abs()
    worst = ((got.double() - want).abs() / tol).max().item()
    assert worst <= 1, worst


@pytest.mark.parametrize("kind,m,k,n", [
    ("mx4", 20011, 1101, 700), ("mx4", 20011, 513, 700), ("mx4", 21500, 640, 750),    # 256 x 256
    ("mx4", 20011, 1101, 130), ("mx4", 16500, 390, 200), ("mx4", 40003, 640, 300),    # 128 x 128
    ("mx4", 66001, 515, 40), ("mx4", 40001, 300, 64),                                 # 128 x 64
    ("mx4", 40001, 333, 29), ("mx4", 66001, 700, 32), ("mx4", 40001, 128, 3),         # 128 x 32
    ("mx4", 3001, 2100, 333), ("mx4", 300, 1100, 2030),                               # 64 x 64
    (torch.bfloat16, 20011, 650, 700), (torch.float32, 9001, 1300, 1030),             # rounded first, then tiles
    # float rows past a w in LDS: up to the longest rows that fit, and rounded first from there on
    (torch.bfloat16, 4111, 2000, 128), (torch.float32, 4111, 2048, 100), (torch.bfloat16, 4111, 2049, 128),
    (torch.float32, 4111, 4224, 64), (torch.bfloat16, 4111, 4225, 64), (torch.bfloat16, 4100, 8300, 32),
    (torch.float32, 4100, 16896, 16), (torch.bfloat16, 4100, 16897, 9),
])
def test_tiles_and_their_epilogues(kind, m, k, n):
    """float32 and bfloat16 results, bias and degrees or none, every activation, ragged sizes; of 4-bit rows (the
    library's own, tested by themselves) the product in float64"""
    L = LY()
    g = torch.Generator(device=device()).manual_seed(m + k + n)
    rand = lambda *s: torch.randn(*s, generator=g, device=device())  # noqa: E731
    x = padded(rand(m, k) * (torch.rand(m, 1, generator=g, device=device()) * 3 + 0.1),
               dtype=torch.float32 if kind == "mx4" else kind)
    q, s = L.quantize_rows_mx4(padded(rand(n, k) * torch.exp(rand(n, 1) - 4)))
    q, s = padded(q, extra=1), padded(s, unit=4, extra=1)
    xq, xs = L.quantize_rows_mx4(x)
    x64 = L.dequantize_rows_mx4(xq, xs, k, dtype=torch.float32).double()
    w64 = L.dequantize_rows_mx4(q, s, k, dtype=torch.float32).double()
    v, mag = x64 @ w64.T, x64.abs() @ w64.abs().T
    bias, deg = rand(n), torch.randint(0, 9, (m,), generator=g, device=device(), dtype=torch.int32)
    xd, scale = (xq, xs) if kind == "mx4" else (x, None)
    i = 0
    for act in ACTS:
        for out in FLOATS:
            b, d = (bias if i % 2 == 0 else None), (deg if i % 3 else None)
            i += 1
            got = L.mx4_linear(xd, q, s, x_scale=scale, bias=b, act=act, row_scale_deg=d, out_dtype=out)
            assert got.dtype == out and got.shape == (m, n)
            check_sums(got, v, mag, k, b, act, d)


@pytest.mark.parametrize("m,k,n", [(3, 100, 40), (60, 1100, 130), (300, 1100, 2030), (4111, 333, 100), (40001, 333, 29),
                                   (20011, 700, 130), (20011, 700, 700)])
@pytest.mark.parametrize("kind", ["mx4", torch.float32, torch.bfloat16])
@pytest.mark.parametrize("power", [-125, 123])
def test_scales_far_apart(kind, m, k, n, power):
    """rows and weights at opposite ends of the scales, the smallest of which is 2^-127"""
    L = LY()
    g = torch.Generator(device=device()).manual_seed(m + k + n)
    x = torch.randn(m, k, generator=g, device=device()) * 2.0 ** power
    x = padded(x, dtype=torch.float32 if kind == "mx4" else kind)
    q, s = L.quantize_rows_mx4(padded(torch.randn(n, k, generator=g, device=device()) * 2.0 ** -power))
    xq, xs = L.quantize_rows_mx4(x)
    assert power > 0 or m < 100 or int(xs.min()) == 0
    x64 = L.dequantize_rows_mx4(xq, xs, k, dtype=torch.float32).double()
    w64 = L.dequantize_rows_mx4(q, s, k, dtype=torch.float32).double()
    xd, scale = (xq, xs) if kind == "mx4" else (x, None)
    got = L.mx4_linear(xd, q, s, x_scale=scale, out_dtype=torch.float32)
    check_sums(got, x64 @ w64.T, x64.abs() @ w64.abs().T, k, None, "none", None)


# --------------------------------------------------------------------------
# experts: slices, the same bits again
# --------------------------------------------------------------------------
@pytest.mark.parametrize("m,f,h,n,e,top_k", [
    (1024 + 7, 96, 100, 50, 512, 2),                # a few rows an expert; the remainder by the kernels of few rows
    (1024 + 16, 100, 1400, 130, 24, 2),             # tiles, down in parts of k; a few rows an expert
    (1024 + 200, 100, 1400, 130, 24, 2), (2500, 130, 1400, 260, 24, 2),
    (1024 + 1, 40, 3000, 70, 12, 4),
])
@pytest.mark.parametrize("weights", ["mx4", "bf16"])
@pytest.mark.parametrize("dtype", FLOATS)
def test_more_rows_than_one_run_takes(m, f, h, n, e, top_k, weights, dtype):
    """slices that share a workspace, each by the kernels that its own rows take"""
    layer = Layer(m, f, h, n, e, weights, False, True)
    layer.check(torch.randn(m, f, generator=gen(m)).to(dtype), top_k, "relu")
    layer = Layer(m, f, h // 2, n, e, weights, True, False)
    layer.check(torch.randn(m, f, generator=gen(m)).to(dtype), top_k, "sigmoid")


@pytest.mark.parametrize("m,f,h,n,e,top_k", [(1, 128, 256, 128, 4, 1), (1, 1024, 2048, 512, 8, 2), (19, 602, 500, 602, 16, 2),
                                             (64, 512, 1024, 512, 64, 2), (300, 512, 1024, 512, 32, 4),
                                             (600, 256, 700, 256, 2, 1)])
@pytest.mark.parametrize("weights", ["mx4", "bf16"])
@pytest.mark.parametrize("dtype", FLOATS)
def test_the_same_bits_again(m, f, h, n, e, top_k, weights, dtype):
    """no result depends on the order in which workgroups run: repeated calls, other work between them, and workspaces
    that held something else"""
    layer = Layer(m, f, h, n, e, weights, True, True)
    x = padded(torch.randn(m, f, generator=gen(m)).to(dtype))
    want = [t.clone() for t in layer(x, top_k=top_k, act="sigmoid")]
    other = padded(torch.randn(m, f, generator=gen(m + 1)).to(dtype))
    for turn in range(4):
        if turn % 2:
            layer(other, top_k=top_k, act="tanh")
            torch.empty(64 << 20, dtype=torch.uint8, device=device()).fill_(0xff)
        got = layer(x, top_k=top_k, act="sigmoid")
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("m,f,h,n,e,top_k", [(304, 602, 900, 400, 2, 2), (1024, 300, 520, 300, 1, 1), (260, 1000, 700, 1000, 4, 4),
                                             (1500, 128, 256, 128, 2, 1), (130, 4096, 260, 33, 1, 1),
                                             (304, 130, 3100, 130, 2, 2), (304, 130, 1530, 130, 8, 2),
                                             (200, 100, 2000, 70, 12, 3), (150, 64, 4100, 50, 3, 1), (140, 64, 4100, 50, 3, 1)])
@pytest.mark.parametrize("weights", ["mx4", "bf16"])
@pytest.mark.parametrize("dtype", FLOATS)
def test_few_experts_of_many_rows(m, f, h, n, e, top_k, weights, dtype):
    """hundreds of rows of each expert, on both sides of where the kernels of many rows take them"""
    for gated in (False, True):
        layer = Layer(m + e, f, h, n, e, weights, gated, gated)
        layer.check(torch.randn(m, f, generator=gen(m)).to(dtype), top_k, "sigmoid" if gated else "relu")


# --------------------------------------------------------------------------
# in a network
# --------------------------------------------------------------------------
@pytest.mark.parametrize("bits,gated", [(4, True), (4, False), (8, True)])
def test_all_vertices_asked_for(bits, gated):
    """asked for all its vertices, in whatever order, a network says of each to the bit what it says unasked"""
    net, _, x = network(bits, torch.bfloat16, gated)
    every = net.logits(x)
    assert bool(torch.isfinite(every).all())
    order = torch.randperm(x.shape[0], generator=gen(2)).to(device())
    assert torch.equal(net.logits(x, order), every[order])
    assert torch.equal(net.logits(x, order.int()), every[order])


@pytest.mark.parametrize("m,f,h,n,e", [(3, 64, 40, 24, 4), (16, 600, 33, 40, 4), (60, 70, 100, 50, 4), (64, 130, 1100, 140, 32),
                                       (400, 130, 1100, 140, 32)])
@pytest.mark.parametrize("weights", ["mx4", "bf16"])
@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("power", [-100, -112, -122, -132])
def test_tiny_rows(m, f, h, n, e, weights, dtype, power):
    """Rows far below the numbers around 1: the terms that hold a float32 end at 2^-133, bfloat16's smallest number,
    so a column is off by that at most.  (Large ups bring the values between the products back to normal ones.)"""
    layer = Layer(m, f, h, n, e, weights)
    large = min(-power, 120)
    layer.up *= 2.0 ** large
    if weights == "mx4":
        layer.kw["up_scale"] += large
    else:
        layer.up_d *= 2.0 ** large
    x = (torch.randn(m, f, generator=gen(m)) * 2.0 ** power).to(dtype)
    y, index, weight = layer(padded(x), top_k=2, act="none")
    want_i, want_p = route_exact(x, layer.router, None, 2, True)
    assert torch.equal(index.cpu().long(), want_i)
    want, tol = experts_exact(x, want_i, want_p, layer.up, layer.down, None, None, e, "none", False, dtype)
    if dtype == torch.float32:
        for i in range(e):
            up, down = layer.up[i * h:(i + 1) * h].double().abs(), layer.down[i * n:(i + 1) * n].double().abs()
            share = torch.where(want_i == i, want_p, 0.0).sum(1, keepdim=True)
            tol += share * (2.0 ** -133 * up.sum(1) @ down.T)
    assert ((y.cpu().double() - want).abs() <= tol).all()
