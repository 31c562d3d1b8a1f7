"""8-bit products, block norms and label log probabilities at the far ends of what
their calls allow: long rows, rows without a number, large magnitudes, ordinary
torch tensors, other streams."""
import pytest
import torch

from gpu_util import device, lib
from test_gpu_operators import ACTS, FLOATS, LY, U, gen, padded, product_exact, rows_exact

pytestmark = pytest.mark.gpu


# --------------------------------------------------------------------------
# long rows: the sums' error does not grow with the number of classes
# --------------------------------------------------------------------------
def long_rows(c):
    """rows whose float32 sums go wrong if every term is added to the running sum (few
    distinct values: all roundings to one side) or if the sum is rescaled often (a
    largest value that grows all the time)"""
    g = gen(c)
    at = torch.arange(c, dtype=torch.float64)
    two = torch.where(torch.rand(c, generator=g) < 0.1, 0.0, -1.1)
    one_top = torch.full((c,), -3.3)
    one_top[c - 7] = 0.5
    three = torch.tensor([0.0, -0.7, -2.9])[torch.randint(0, 3, (c,), generator=g)]
    return torch.stack([two, one_top, three, torch.full((c,), 0.3), (at * (8.0 / c) - 4).float(),
                        (at * (60.0 / c) - 30).float(), (4 - at * (8.0 / c)).float(), torch.randn(c, generator=g) * 3])


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("times,c", [(64, 100003), (64, 1 << 18), (64, 1 << 20), (1, 1 << 20), (1, (1 << 22) + 5)])
def test_labels_sums_of_long_rows(times, c, dtype):
    """With D = sum p |x - m| and D2 = sum p (x - m)^2, in units of 2^-24.  The sums are
    about a value r that is at most 2 below the largest so far.  A term e^(x - r): the
    difference, its product with log2 e (rounded twice) and the function, 2.3 |x - r| + 4, at
    most 2.3 |x - m| + 8.6.  A rescaling by e^-d, d >= 2: 2.3 d + 3, at most 3.8 d, over all of a
    term's steps 3.8 |x - m|.  The joins of lanes, waves and ranges: 2.3 |x - m| again, scale
    factors of 7.6 (from r to m), 3 and 3, and 22 additions.  A tile's terms are added in
    float32, 8 additions at most, the tiles' sums in float64 and rounded once.  So S is within
    9 D + 54 of itself, T within 9 D2 / D + 54; log S adds 3 of its own value, log p another
    2 of its, and T / S one."""
    x = long_rows(c).to(dtype)
    patterns = x.shape[0]
    m = times * patterns
    to = (torch.arange(m, dtype=torch.int64) * 7919 % c).int()
    xd = x.to(device())
    big = padded(torch.empty(0, c, dtype=dtype))  # (its pitch)
    big = torch.zeros((m, big.stride(0)), dtype=dtype, device=device())[:, :c]
    for t in range(times):
        big[t * patterns:(t + 1) * patterns] = xd
    got = LY().label_log_probs(big, to.to(device()), top_k=2)
    logp, ent = (v.double().cpu().view(times, patterns) for v in got[:2])
    for r in range(patterns):
        v = x[r].double()
        d = v - v.max()
        e = torch.exp(d)
        s = e.sum()
        log_s, dist = torch.log(s), -(e * d).sum() / s
        dist2 = (e * d * d).sum() / s
        want = (v - v.max() - log_s)[to.view(times, patterns)[:, r].long()]
        tol = U * (9 * dist + 54 + 3 * log_s + 2 * want.abs() + 1)
        assert ((logp[:, r] - want).abs() / tol).max() <= 1, (r, (logp[:, r] - want).abs().max() / U)
        tol = U * ((9 * dist + 54) * (1 + dist) + 9 * dist2 + 54 * dist + 3 * log_s + dist + 2 * (log_s + dist))
        assert ((ent[:, r] - log_s - dist).abs() / tol).max() <= 1, (r, (ent[:, r] - log_s - dist).abs().max() / U)
        order = torch.sort(v, descending=True, stable=True).indices[:2]
        assert bool((got[2].view(times, patterns, 2)[:, r].cpu().long() == order).all()), r


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("m,k,n", [(7, 100, 50), (70, 1024, 1024), (17000, 602, 41), (17000, 200, 300), (65600, 100, 64),
                                   (65600, 200, 128), (300, 1400, 600), (20000, 1300, 300)])
def test_product_rows_without_a_number_in_every_activation(m, k, n, act):
    """a row that holds a NaN or an infinity answers NaN, whatever the activation, from
    every kernel: float rows, and the 8-bit rows and scales quantize_rows makes of them"""
    L = LY()
    bad = [0, m // 2, m - 1]
    for dtype in FLOATS:
        x = torch.randn(m, k, generator=gen(m + k)).to(dtype)
        for i, v in zip(bad, (float("nan"), float("inf"), -float("inf"))):
            x[i, (i * 7) % k] = v
        x = padded(x)
        w = padded(torch.randint(-9, 9, (n, k), generator=gen(n), dtype=torch.int8))
        ws = torch.full((n,), 0.01, device=device())
        q, s = L.quantize_rows(x)
        for out in FLOATS:
            for got in (L.quant_linear(x, w, ws, act=act, out_dtype=out),
                        L.quant_linear(q, w, ws, x_scale=s, act=act, out_dtype=out)):
                empty = torch.isnan(got)
                assert empty.all(1).nonzero().flatten().tolist() == bad
                assert empty.any(1).sum().item() == len(bad)


def test_product_relu_of_zeros():
    """+0 for what is not above 0, from -0 too"""
    L = LY()
    x = padded(torch.full((5, 40), -1.0))
    w = padded(torch.cat([torch.zeros(20, 40), torch.ones(20, 40)]).to(torch.int8))
    got = L.quant_linear(x, w, torch.full((40,), -0.0, device=device()), act="relu")
    assert bool((got == 0).all()) and not bool(torch.signbit(got).any())


@pytest.mark.parametrize("m,k,n", [(3, 100, 50), (70, 1024, 1024), (17000, 602, 41), (17000, 200, 300), (65600, 100, 64),
                                   (65600, 200, 128), (300, 1400, 600), (20000, 1300, 300)])
def test_product_of_rows_of_large_magnitude(m, k, n):
    """Finite results are finite and within the product's roundings: large rows (up to
    3e38) by small weights, whole numbers times the row's scale being past float32, and
    small rows by large weights."""
    L = LY()
    g = gen(m + n)
    w = torch.randint(-127, 128, (n, k), generator=g, dtype=torch.int8)
    unit = (torch.rand(n, generator=g) + 0.5) / k
    deg = torch.randint(0, 9, (m,), generator=g, dtype=torch.int32)
    for dtype in FLOATS:
        base = torch.randn(m, k, generator=g).clamp_(-4, 4)
        for size, weight in ((6e37, 1e-6), (1e34, 1e-3), (1e30, 1.0), (1e-30, 1e30), (1e-34, 1e36), (1.0, 1e30)):
            x = (base * size).to(dtype)
            x[m // 2] = base[m // 2].to(dtype)  # an ordinary row between them
            ws = unit * weight
            q, s = rows_exact(x.double())
            want, mag = product_exact(q, s, w, ws, None, "none", deg)
            assert bool(torch.isfinite(want.float()).all())
            xd, wd, wsd, degd = padded(x), padded(w), ws.to(device()), deg.to(device())
            qd, sd = L.quantize_rows(xd)
            for got in (L.quant_linear(xd, wd, wsd, row_scale_deg=degd, out_dtype=torch.float32),
                        L.quant_linear(qd, wd, wsd, x_scale=sd, row_scale_deg=degd, out_dtype=torch.float32)):
                err = (got.double().cpu() - want).abs()
                # the sum to float32, two scales, the degree's root, quotient and product: seven roundings
                assert bool((err <= 8 * U * mag + 2.0 ** -149).all()), (size, (err / (U * mag + 1e-45)).max())


# --------------------------------------------------------------------------
# the torch entry points
# --------------------------------------------------------------------------
def test_arguments_by_name():
    """the same bits by name as by place"""
    L = LY()
    d = device()
    x, block, gate = (padded(torch.randn(30, 50, generator=gen(i))) for i in range(3))
    w = padded(torch.randint(-127, 128, (20, 50), generator=gen(4), dtype=torch.int8))
    ws, to = torch.rand(20, generator=gen(5)).to(d), torch.randint(0, 50, (30,), generator=gen(6), dtype=torch.int32).to(d)
    q, s = L.quantize_rows(x)
    for a, b in ((L.quantize_rows(x=x), (q, s)),
                 ([L.quant_linear(w_scale=ws, w=w, x=x, act="elu")], [L.quant_linear(x, w, ws, act="elu")]),
                 ([L.quant_linear(x=q, x_scale=s, w=w, w_scale=ws)], [L.quant_linear(q, w, ws, s)]),
                 (L.block_norm(block=block, x=x, pre="rms", gate=gate)[:2], L.block_norm(block, x, pre="rms", gate=gate)[:2]),
                 (L.block_norm(block, x=x, pre="rms", quantize=True), L.block_norm(block, x, pre="rms", quantize=True)),
                 (L.label_log_probs(logits=x, labels=to, top_k=3, entropy=True), L.label_log_probs(x, to, 3, True))):
        assert len(a) == len(b) and all(torch.equal(g, h) for g, h in zip(a, b))


def test_memory_on_another_stream():
    """What a call on ``stream`` still reads, and what it returned to work on the current
    stream, is not handed out again while that work is under way"""
    L = LY()
    d = device()
    torch.cuda.synchronize()
    m, f, n = 400, 512, 256
    side = torch.cuda.Stream()
    w = padded(torch.randint(-127, 128, (n, f), generator=gen(1), dtype=torch.int8))
    ws = torch.rand(n, generator=gen(2)).to(d)
    host = torch.randn(m, f, generator=gen(3))
    busy = torch.zeros(4096, 4096, dtype=torch.bfloat16, device=d)
    sink = torch.empty_like(busy)
    keep = host.to(d)
    calls = [lambda x, **kw: (L.quant_linear(x, w, ws, **kw),), lambda x, **kw: (L.quant_linear(x=x, w=w, w_scale=ws, **kw),),
             lambda x, **kw: L.quantize_rows(x, **kw), lambda x, **kw: L.block_norm(x, x=keep, gate=x, pre="rms", **kw)[:2],
             lambda x, **kw: L.block_norm(keep, gate=x, pre="rms", **kw)[:2],
             lambda x, **kw: L.label_log_probs(logits=x, **kw)[1:2]]
    for call in calls:
        want = call(keep.clone())
        call(keep.clone(), stream=side)
        with torch.cuda.stream(side):
            torch.mm(busy, busy, out=sink)
        torch.cuda.synchronize()
        x = host.to(d)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(100):
                torch.mm(busy, busy, out=sink)
        got = call(x, stream=side)
        at = x.untyped_storage().data_ptr()
        del x
        others = [torch.empty(m, f, device=d) for _ in range(8)]
        assert side.query() or at not in [t.untyped_storage().data_ptr() for t in others]
        del others
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        del got, want
    # a result, read on the current stream and dropped
    want = L.quant_linear(keep, w, ws) * 2.0
    torch.mm(busy, busy, out=sink)
    torch.cuda.synchronize()
    got = L.quant_linear(keep, w, ws, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(100):
        torch.mm(busy, busy, out=sink)
    total = got * 2.0
    at = got.untyped_storage().data_ptr()
    del got
    with torch.cuda.stream(side):
        others = [torch.empty(m, n, device=d) for _ in range(8)]
    assert torch.cuda.current_stream().query() or at not in [t.untyped_storage().data_ptr() for t in others]
    torch.cuda.synchronize()
    assert torch.equal(total, want)


def test_captured_with_the_stream_argument():
    """a side stream inside a capture, joined again"""
    L = LY()
    d = device()
    x = padded(torch.randn(40, 96, generator=gen(1)))
    w = padded(torch.randint(-127, 128, (64, 96), generator=gen(2), dtype=torch.int8))
    ws = torch.rand(64, generator=gen(3)).to(d)
    L.quant_linear(x, w, ws)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    gph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gph):
        side.wait_stream(torch.cuda.current_stream())
        out = L.quant_linear(x, w, ws, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        top = L.label_log_probs(out, top_k=3)
    for turn in range(3):
        x.copy_(torch.randn(40, 96, generator=gen(5 + turn)).to(d))
        want = L.quant_linear(x, w, ws)
        tops = L.label_log_probs(want, top_k=3)
        torch.cuda.synchronize()
        gph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and all(torch.equal(a, b) for a, b in zip(top[1:], tops[1:]))


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("k", [1, 5, 41, 602, 5001])
def test_single_and_no_rows_as_they_come(k, dtype):
    """one row of any width, from the first or in the middle of a vector, and no row"""
    L = LY()
    d = device()
    n = 21
    flat = torch.randn(64 + k, generator=gen(k)).to(dtype).to(d)
    x, block, gate = flat[:k][None], flat[16:16 + k].unsqueeze(0), flat[32:32 + k].view(1, k)
    w = padded(torch.randint(-127, 128, (n, k), generator=gen(4), dtype=torch.int8))
    ws, one = torch.rand(n, generator=gen(5)).to(d), torch.rand(1, generator=gen(6)).to(d)
    to = torch.zeros(1, dtype=torch.int32, device=d)
    wide, wb, wg = padded(x), padded(block), padded(gate)
    q, s = L.quantize_rows(x)
    byte = torch.randint(-127, 128, (1, k), generator=gen(7), dtype=torch.int8).to(d)  # w of one channel
    for a, b in ((L.quantize_rows(x), L.quantize_rows(wide)),
                 ([L.quant_linear(x, w, ws)], [L.quant_linear(wide, w, ws)]),
                 ([L.quant_linear(q, w, ws, s)], [L.quant_linear(wide, w, ws, out_dtype=torch.float32)]),
                 ([L.quant_linear(x, byte, one)], [L.quant_linear(wide, padded(byte), one)]),
                 (L.block_norm(block, x, gate=gate, post="layer", pre="rms", quantize=True),
                  L.block_norm(wb, wide, gate=wg, post="layer", pre="rms", quantize=True)),
                 (L.label_log_probs(x, to, 4), L.label_log_probs(wide, to, 4))):
        assert all(torch.equal(g.nan_to_num(3.0), h.nan_to_num(3.0)) for g, h in zip(a, b))
    # in place: nothing behind the row is written
    rest = flat[k:].clone()
    y, z, _ = L.block_norm(wb, x, pre="rms", in_place=True)
    y2, z2, _ = L.block_norm(wb, wide, pre="rms")
    assert y.data_ptr() == x.data_ptr() and torch.equal(y, y2) and torch.equal(z, z2)
    assert torch.equal(flat[k:], rest)
    # no rows
    none = torch.empty(0, k, dtype=dtype, device=d)
    assert L.quantize_rows(none)[0].shape == (0, k) and L.quant_linear(none, w, ws).shape == (0, n)
    assert L.block_norm(none, none, pre="rms")[1].shape == (0, k)
    assert L.label_log_probs(none, top_k=2)[2].shape == (0, 2)
    # more rows have a pitch, and it is checked
    two = torch.empty(2 * k, dtype=dtype, device=d).view(2, k)
    if k % (16 // dtype.itemsize):
        with pytest.raises(lib().SagaError, match="multiple of 16"):
            L.quantize_rows(two)


def test_no_gradients():
    """inference only: results without history, x in place neither part of a graph nor
    changed behind a graph's back"""
    L = LY()
    x, block = (padded(torch.randn(6, 24, generator=gen(i))) for i in range(2))
    want = L.block_norm(block, x, pre="rms")
    leaf = block.detach().clone().requires_grad_()
    got = L.block_norm(leaf, x, pre="rms")
    assert not got[0].requires_grad and not got[1].requires_grad and torch.equal(got[0], want[0])
    assert not L.label_log_probs(leaf)[1].requires_grad and not L.quantize_rows(leaf)[1].requires_grad
    for t in (x.clone().requires_grad_(), x.clone().requires_grad_() * 1.0):
        with pytest.raises(ValueError, match="requires grad"):
            L.block_norm(block, t, pre="rms", in_place=True)
        assert torch.equal(t, x)
        with torch.no_grad():
            assert torch.equal(L.block_norm(block, t, pre="rms", in_place=True)[0], want[0])
    scale = torch.ones(24, device=x.device, requires_grad=True)
    t = x.clone()
    out = (t * scale).sum()  # its backward pass needs t
    L.block_norm(block, t, pre="rms", in_place=True)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.backward()
    with torch.inference_mode():
        t = x.clone()
        assert torch.equal(L.block_norm(block, t, pre="rms", in_place=True)[0], want[0])


@pytest.mark.parametrize("act", ["none", "relu", "elu", "sigmoid", "tanh"])
def test_gates_to_their_last_places(act):
    """Gates alone (y = act(gate)), relative to their own size, in units of 2^-24.  e^x by
    the card's exponential: 2.3 |x| + 4 (argument, its product with log2 e, the function), a
    reciprocal 2, an addition 1.  sigmoid: 2.3 |x| + 7.  tanh from 0.3 on, q = 2 / (e^2x + 1): a
    share e / (e + 1) of 4.6 |x| + 4, and 3 more, times q, over tanh x: at x = -0.3, where q is
    largest, (0.35 * 5.4 + 3) * 1.29 / 0.29 = 22, and 2 for the last difference over 0.29: 29
    in all; falling from there on both sides; below, four multiply-adds and the term left
    out (0.9): 6.  ELU: expm1f, 4.  What is below 2^-126 may be 0."""
    L = LY()
    sizes = torch.cat([torch.logspace(-8, 0, 3000), torch.linspace(0.25, 0.35, 2000), torch.linspace(1, 100, 3193)])
    g = torch.cat([sizes, -sizes]).view(2, 8193)[:, :8192].contiguous()
    y, _, _ = L.block_norm(torch.ones(2, 8192, device=device()), gate=g.to(device()), gate_act=act)
    want = ACTS[act](g.double())
    units = {"none": 0, "relu": 0, "elu": 4, "sigmoid": 7, "tanh": 32}[act] + (2.3 * g.double().abs() if act == "sigmoid" else 0)
    err = (y.double().cpu() - want).abs()
    assert bool((err <= U * units * want.abs() + 2.0 ** -126).all()), (err / (U * want.abs() + 1e-45)).max()
