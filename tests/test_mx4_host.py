"""Refusals of 4-bit rows, their products and layers of experts: every bad call returns
from validation, on the host, before anything is launched."""
import inspect
import os
import shutil
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A, B, D, E, F, G, H, I, J = (i << 34 for i in range(1, 10))  # addresses far apart, never read


@pytest.fixture(scope="module")
def S():
    import paper_2009_00804_amd.saga as S

    if not os.path.exists(S.LIB_PATH):
        from paper_2009_00804_amd import build

        build.build()
    S.lib()
    return S


def refused(S, status, text, f, *args):
    with pytest.raises(S.SagaError) as e:
        f(*args)
    assert e.value.status == status, e.value
    assert text in str(e.value), e.value


def test_rows_refusals(S):
    ok = dict(dtype=0, x=(A, 4, 41, 44), q=(B, 4, 21, 32), s=(D, 4, 2, 4))

    def call(status, text, **kw):
        a = {**ok, **kw}
        refused(S, status, text, S.saga_quantize_rows_mx, a["dtype"], S.saga_cmat(*a["x"]), S.saga_mat(*a["q"]),
                S.saga_mat(*a["s"]), None)
        refused(S, status, text, S.saga_dequantize_rows_mx, a["dtype"], S.saga_cmat(*a["q"]), S.saga_cmat(*a["s"]),
                S.saga_mat(*a["x"]), None)

    call(S.SAGA_EINVAL, "bad dtype", dtype=2)
    call(S.SAGA_EINVAL, "bad dtype", dtype=3)
    call(S.SAGA_EINVAL, "x: null", x=(None, 4, 41, 44))
    call(S.SAGA_EINVAL, "q: null", q=(None, 4, 21, 32))
    call(S.SAGA_EINVAL, "scale: null", s=(None, 4, 2, 4))
    call(S.SAGA_EINVAL, "multiple of 16", x=(A, 4, 41, 42))
    call(S.SAGA_EINVAL, "16-byte aligned", x=(A + 4, 4, 41, 44))
    call(S.SAGA_EINVAL, "multiple of 16", q=(B, 4, 21, 24))
    call(S.SAGA_EINVAL, "16-byte aligned", q=(B + 8, 4, 21, 32))
    call(S.SAGA_EINVAL, "multiple of 4", s=(D, 4, 2, 6))
    call(S.SAGA_EINVAL, "4-byte aligned", s=(D + 2, 4, 2, 4))
    call(S.SAGA_EINVAL, "shape", q=(B, 4, 20, 32))
    call(S.SAGA_EINVAL, "shape", q=(B, 5, 21, 32))
    call(S.SAGA_EINVAL, "shape", s=(D, 4, 1, 4))
    call(S.SAGA_EINVAL, "shape", s=(D, 3, 2, 4))
    call(S.SAGA_EINVAL, "ld", x=(A, 4, 41, 40))
    call(S.SAGA_EINVAL, "rows", x=(A, -1, 41, 44), q=(B, -1, 21, 32), s=(D, -1, 2, 4))
    call(S.SAGA_EINVAL, "columns", x=(A, 4, 0, 44))
    call(S.SAGA_EINVAL, "out of range", x=(A, 1 << 60, 41, 44), q=(B, 1 << 60, 21, 32), s=(D, 1 << 60, 2, 4))
    call(S.SAGA_EUNSUPPORTED, "columns", x=(A, 1, 1 << 31, 1 << 31))
    call(S.SAGA_EINVAL, "overlaps", q=(A + 64, 4, 21, 32))
    call(S.SAGA_EINVAL, "overlaps", s=(A + 64, 4, 2, 4))
    refused(S, S.SAGA_EINVAL, "two outputs", S.saga_quantize_rows_mx, 0, S.saga_cmat(*ok["x"]),
            S.saga_mat(*ok["q"]), S.saga_mat(B + 64, 4, 2, 4), None)
    S.saga_quantize_rows_mx(0, S.saga_cmat(None, 0, 41, 44), S.saga_mat(None, 0, 21, 32), S.saga_mat(None, 0, 2, 4), None)
    S.saga_dequantize_rows_mx(1, S.saga_cmat(None, 0, 21, 32), S.saga_cmat(None, 0, 2, 4), S.saga_mat(None, 0, 41, 48),
                              None)


def test_product_refusals(S):
    ok = dict(a_dtype=3, out_dtype=0, act=0, deg=None, a=(A, 5, 20, 32), sa=(B, 5, 2, 4), w=(D, 7, 20, 32),
              sw=(E, 7, 2, 4), bias=None, out=(F, 5, 7, 8), ws=None, nws=0)

    def call(status, text, **kw):
        a = {**ok, **kw}
        op = S.saga_mx_op(a["a_dtype"], a["out_dtype"], a["act"], a["deg"])
        refused(S, status, text, S.saga_apply_vertex_mx, op, S.saga_cmat(*a["a"]), S.saga_cmat(*a["sa"]),
                S.saga_cmat(*a["w"]), S.saga_cmat(*a["sw"]), a["bias"], S.saga_mat(*a["out"]), a["ws"], a["nws"], None)

    none = (None, 0, 0, 0)
    call(S.SAGA_EINVAL, "a_dtype", a_dtype=2)
    call(S.SAGA_EINVAL, "a_dtype", a_dtype=4)
    call(S.SAGA_EINVAL, "out_dtype", out_dtype=3)
    call(S.SAGA_EINVAL, "activation", act=5)
    call(S.SAGA_EINVAL, "activation", act=-1)
    call(S.SAGA_EINVAL, "m must", a=(A, -1, 20, 32))
    call(S.SAGA_EINVAL, "k and n", a=(A, 5, 0, 32))
    call(S.SAGA_EINVAL, "k and n", w=(D, 0, 20, 32))
    k = (1 << 20) + 2
    call(S.SAGA_EUNSUPPORTED, "too large", a=(A, 5, k // 2, k))
    call(S.SAGA_EUNSUPPORTED, "too large", a_dtype=0, a=(A, 5, k, k), sa=none)
    call(S.SAGA_EUNSUPPORTED, "too large", a=(A, 5, 1 << 62, 1 << 62))
    call(S.SAGA_EUNSUPPORTED, "too large", w=(D, (1 << 28) + 1, 20, 32))
    call(S.SAGA_EUNSUPPORTED, "2^23", a=(A, 5, 20, 1 << 23))
    call(S.SAGA_EUNSUPPORTED, "2^23", w=(D, 7, 20, 1 << 23))
    call(S.SAGA_EUNSUPPORTED, "2^23", sw=(E, 7, 2, 1 << 23))
    call(S.SAGA_EINVAL, "shape", w=(D, 7, 21, 32))
    call(S.SAGA_EINVAL, "shape", sw=(E, 7, 1, 4))
    call(S.SAGA_EINVAL, "shape", sw=(E, 6, 2, 4))
    call(S.SAGA_EINVAL, "shape", sa=(B, 4, 2, 4))
    call(S.SAGA_EINVAL, "columns", sa=none)
    call(S.SAGA_EINVAL, "shape", out=(F, 5, 8, 8))
    call(S.SAGA_EINVAL, "shape", out=(F, 4, 7, 8))
    call(S.SAGA_EINVAL, "null", a=(None, 5, 20, 32))
    call(S.SAGA_EINVAL, "w_scale: null", sw=(None, 7, 2, 4))
    call(S.SAGA_EINVAL, "multiple of 4", sw=(E, 7, 2, 3))
    call(S.SAGA_EINVAL, "4-byte", sa=(B + 1, 5, 2, 4))
    call(S.SAGA_EINVAL, "misaligned", bias=G + 1)
    call(S.SAGA_EINVAL, "misaligned", deg=G + 2)
    call(S.SAGA_EINVAL, "multiple of 16", a=(A, 5, 20, 24))
    call(S.SAGA_EINVAL, "multiple of 16", out=(F, 5, 7, 7))
    call(S.SAGA_EINVAL, "overlaps", out=(A, 5, 7, 8))
    call(S.SAGA_EINVAL, "overlaps", out=(B, 5, 7, 8))
    call(S.SAGA_EINVAL, "overlaps", out=(D + 64, 5, 7, 8))
    call(S.SAGA_EINVAL, "overlaps", out=(E, 5, 7, 8))
    call(S.SAGA_EINVAL, "overlaps", bias=F + 16)
    # float rows: no scales, and a workspace where kernels of their own quantise them
    call(S.SAGA_EINVAL, "a_scale is for", a_dtype=0, a=(A, 5, 39, 40))
    call(S.SAGA_EINVAL, "shape", a_dtype=0, a=(A, 5, 41, 44), sa=none)
    assert S.saga_apply_vertex_mx_workspace_size(S.saga_mx_op(3, 0, 0, None), 20000, 4096, 4096) == 0
    m, k, n = 6000, 1300, 600
    big = dict(a_dtype=0, sa=none, a=(A, m, k, 1312), w=(D, n, 650, 656), sw=(E, n, 41, 44), out=(F, m, n, 608))
    need = S.saga_apply_vertex_mx_workspace_size(S.saga_mx_op(0, 0, 0, None), m, k, n)
    assert need >= m * 656 + m * 44
    call(S.SAGA_EWORKSPACE, "need", **big)
    call(S.SAGA_EWORKSPACE, "need", **big, ws=G, nws=need - 1)
    call(S.SAGA_EINVAL, "256", **big, ws=G + 16, nws=need)
    for other in (A, D, E, F):
        call(S.SAGA_EINVAL, "overlap", **big, ws=other, nws=need)
    with pytest.raises(S.SagaError):
        S.saga_apply_vertex_mx_workspace_size(S.saga_mx_op(0, 0, 0, None), 5, 0, 7)
    assert S.lib().saga_apply_vertex_mx_workspace_size(None, 1, 1, 1, None) == S.SAGA_EINVAL


def test_expert_refusals(S):
    # 4 gated experts: 40 columns, 24 hidden channels, 10 out; 6 rows, 2 choices
    ok = dict(dtype=0, rd=1, wd=3, e=4, k=2, act=1, gated=1, renorm=1, x=(A, 6, 40, 40), out=(B, 6, 10, 12), i=D, p=E,
              r=(F, 4, 40, 40), rb=None, up=(G, 192, 20, 32), us=(G + (1 << 30), 192, 2, 4), ub=None,
              down=(H, 40, 12, 16), ds=(H + (1 << 30), 40, 1, 4), db=None, ws=I, nws=1 << 30)

    def call(status, text, **kw):
        a = {**ok, **kw}
        op = S.saga_expert_op(*(a[n] for n in ("dtype", "rd", "wd", "e", "k", "act", "gated", "renorm")))
        w = S.saga_expert_weights(S.saga_cmat(*a["r"]), a["rb"], S.saga_cmat(*a["up"]), S.saga_cmat(*a["us"]), a["ub"],
                                  S.saga_cmat(*a["down"]), S.saga_cmat(*a["ds"]), a["db"])
        refused(S, status, text, S.saga_apply_vertex_experts, op, w, S.saga_cmat(*a["x"]), S.saga_mat(*a["out"]),
                a["i"], a["p"], a["ws"], a["nws"], None)

    none = (None, 0, 0, 0)
    call(S.SAGA_EINVAL, "bad dtype", dtype=2)
    call(S.SAGA_EINVAL, "router_dtype", rd=3)
    call(S.SAGA_EINVAL, "weight_dtype", wd=0)
    call(S.SAGA_EINVAL, "weight_dtype", wd=2)
    call(S.SAGA_EINVAL, "activation", act=5)
    call(S.SAGA_EINVAL, "experts must", e=0)
    call(S.SAGA_EINVAL, "experts must", e=1025)
    call(S.SAGA_EINVAL, "experts must", e=-4)
    call(S.SAGA_EINVAL, "top_k", k=0)
    call(S.SAGA_EINVAL, "top_k", k=5)
    call(S.SAGA_EINVAL, "top_k", e=24, k=17, up=(G, 192, 20, 32), r=(F, 24, 40, 40))
    call(S.SAGA_EINVAL, "0 or 1", gated=2)
    call(S.SAGA_EINVAL, "0 or 1", renorm=-1)
    call(S.SAGA_EINVAL, "m must", x=(A, -6, 40, 40))
    call(S.SAGA_EINVAL, "f, h and n", x=(A, 6, 0, 40))
    call(S.SAGA_EINVAL, "f, h and n", out=(B, 6, 0, 12))
    call(S.SAGA_EINVAL, "no multiple", up=(G, 191, 20, 32))
    call(S.SAGA_EINVAL, "no multiple", up=(G, 0, 20, 32))
    wide = (1 << 16) + 16
    call(S.SAGA_EUNSUPPORTED, "too large", x=(A, 6, wide, wide))
    call(S.SAGA_EUNSUPPORTED, "too large", up=(G, 8 * wide, 20, 32))
    call(S.SAGA_EUNSUPPORTED, "too large", out=(B, 6, wide, wide))
    call(S.SAGA_EUNSUPPORTED, "2^23", up=(G, 192, 20, 1 << 23))
    call(S.SAGA_EUNSUPPORTED, "2^23", down=(H, 40, 12, 1 << 23))
    call(S.SAGA_EINVAL, "x: null", x=(None, 6, 40, 40))
    call(S.SAGA_EINVAL, "out: null", out=(None, 6, 10, 12))
    call(S.SAGA_EINVAL, "out: shape", out=(B, 5, 10, 12))
    call(S.SAGA_EINVAL, "router: shape", r=(F, 4, 39, 40))
    call(S.SAGA_EINVAL, "router: row pitch", r=(F, 4, 40, 41))
    call(S.SAGA_EINVAL, "up: shape", up=(G, 192, 21, 32))
    call(S.SAGA_EINVAL, "down: shape", down=(H, 39, 12, 16))
    call(S.SAGA_EINVAL, "down: shape", down=(H, 40, 13, 16))
    call(S.SAGA_EINVAL, "up_scale: shape", us=(G + (1 << 30), 191, 2, 4))
    call(S.SAGA_EINVAL, "down_scale: shape", ds=(H + (1 << 30), 40, 2, 4))
    call(S.SAGA_EINVAL, "up_scale: 0 columns", us=none)
    call(S.SAGA_EINVAL, "4-bit weights", wd=1, up=(G, 192, 40, 40), down=(H, 40, 24, 24))
    call(S.SAGA_EINVAL, "up: shape", wd=1, us=none, ds=none)
    call(S.SAGA_EINVAL, "misaligned", rb=J + 2)
    call(S.SAGA_EINVAL, "misaligned", ub=J + 1)
    call(S.SAGA_EINVAL, "misaligned", db=J + 3)
    call(S.SAGA_EINVAL, "index: null", i=None)
    call(S.SAGA_EINVAL, "weight: null", p=None)
    op = S.saga_expert_op(0, 1, 3, 4, 2, 1, 1, 1)
    need = S.saga_apply_vertex_experts_workspace_size(op, 6, 40, 24, 10)
    assert need > 0 and S.saga_apply_vertex_experts_workspace_size(op, 0, 40, 24, 10) == 0
    call(S.SAGA_EWORKSPACE, "need", nws=need - 1)
    call(S.SAGA_EWORKSPACE, "need", ws=None)
    call(S.SAGA_EINVAL, "256", ws=I + 16)
    for other in ("x", "r", "up", "us", "down", "ds"):
        call(S.SAGA_EINVAL, "overlaps an input", ws=ok[other][0], nws=need)
        call(S.SAGA_EINVAL, "overlaps an input", i=ok[other][0])
    call(S.SAGA_EINVAL, "overlaps an input", out=(A, 6, 10, 12))
    call(S.SAGA_EINVAL, "two outputs", out=(E, 6, 10, 12))
    call(S.SAGA_EINVAL, "two outputs", p=D + 4)
    call(S.SAGA_EINVAL, "two outputs", ws=B, nws=need)
    with pytest.raises(S.SagaError):
        S.saga_apply_vertex_experts_workspace_size(op, 6, 40, 0, 10)
    assert S.lib().saga_apply_vertex_experts(None, None, S.saga_cmat(*none), S.saga_mat(*none), None, None, None, 0,
                                             None) == S.SAGA_EINVAL


def test_the_workspace_is_that_of_one_run(S):
    """(rows beyond 1024 go through it again)"""
    op = S.saga_expert_op(0, 1, 3, 4, 2, 1, 1, 1)
    assert (S.saga_apply_vertex_experts_workspace_size(op, 1024, 400, 240, 100)
            == S.saga_apply_vertex_experts_workspace_size(op, 1 << 30, 400, 240, 100))


def test_every_argument_by_its_name():
    """the torch entry points take each argument by the name that they show, and refuse
    tensors that are not on the GPU"""
    from paper_2009_00804_amd import layers as L

    x = torch.zeros(4, 64)
    q, s = torch.zeros(8, 32, dtype=torch.uint8), torch.zeros(8, 2, dtype=torch.uint8)
    given = {"x": x, "q": q, "scale": s, "columns": None, "dtype": torch.bfloat16, "w": q, "w_scale": s,
             "x_scale": None, "bias": None, "act": "none", "row_scale_deg": None, "out_dtype": None, "router": x,
             "up": q, "down": q, "up_scale": s, "down_scale": s, "router_bias": None, "up_bias": None,
             "down_bias": None, "top_k": 1, "gated": False, "renormalise": True, "stream": None}
    for f in (L.quantize_rows_mx4, L.dequantize_rows_mx4, L.mx4_linear, L.expert_layer):
        names = list(inspect.signature(f).parameters)
        assert names[-1] == "stream"
        with pytest.raises(ValueError, match="on the GPU"):
            f(**{n: given[n] for n in names})
        with pytest.raises(ValueError, match="on the GPU"):
            f(given[names[0]], **{n: given[n] for n in names[1:]})
        with pytest.raises(TypeError, match="tensor"):
            f(3)


@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
def test_vertices_outside_the_graph(dtype):
    """ids that name no row get one of the rows there are, and are told apart"""
    from paper_2009_00804_amd import layers as L

    far = torch.iinfo(dtype)
    ids = torch.tensor([3, -1, 0, 7, 6, far.max, far.min, 6], dtype=dtype)
    at, off = L._asked(ids, 7, ids.device)
    assert off.tolist() == [False, True, False, True, False, True, True, False]
    assert int(at.min()) >= 0 and int(at.max()) <= 6
    assert torch.equal(at[~off], ids[~off])
    t = torch.arange(35).view(7, 5).float()
    got = L._rows_at(t, at)
    assert got.stride() == (8, 1) and torch.equal(got[~off], t[[3, 0, 6, 6]])
    assert torch.equal(L._rows_at(t[:, 0], at)[~off], torch.tensor([15.0, 0, 30, 30]))
    at, off = L._asked(ids[:0], 0, ids.device)  # (no vertex of none)
    assert at.numel() == 0 and off.numel() == 0 and L._rows_at(t[:0], at).shape == (0, 5)


def test_vertices_refused():
    from paper_2009_00804_amd import layers as L

    cpu = torch.device("cpu")
    for bad in ([0, 1], 3, torch.tensor(3), torch.tensor([[1, 2]]), torch.tensor([True, False]), torch.tensor([1.0]),
                torch.tensor([1], dtype=torch.int16), torch.tensor([1], dtype=torch.uint8),
                torch.zeros(2, dtype=torch.int64, device="meta")):
        with pytest.raises(ValueError, match="vertices"):
            L._asked(bad, 7, cpu)
    with pytest.raises(ValueError, match="vertices: the graph has none"):
        L._asked(torch.tensor([0]), 0, cpu)


def test_pitches_of_scales():
    from paper_2009_00804_amd import layers as L

    s = torch.zeros(1, 5, dtype=torch.uint8)
    assert L._matrix(s, "s", s, (torch.uint8,), unit=4).ld == 8
    s = torch.zeros(3, 8, dtype=torch.uint8)[:, :5]
    assert L._matrix(s, "s", s, (torch.uint8,), unit=4).ld == 8
    _, m = L._out(3, 5, torch.uint8, s, 4)
    assert (m.cols, m.ld) == (5, 8)


@pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"),
                    reason="ROCm toolchain absent")
def test_refusals_clean_under_asan_and_ubsan():
    from paper_2009_00804_amd import build as B_

    lib = B_.build_sanitized()
    env = dict(os.environ, LD_PRELOAD=B_.asan_runtime(), ASAN_OPTIONS="detect_leaks=0:halt_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    code = ("import sys, pytest\n"
            "import paper_2009_00804_amd.saga as S\n"
            f"S.LIB_PATH = {lib!r}\n"
            "sys.exit(pytest.main(['-q', '-s', '-p', 'no:cacheprovider', '-k', 'refusals and not clean',\n"
            "                      'tests/test_mx4_host.py']))\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    out = r.stdout + r.stderr
    assert "AddressSanitizer" not in out and "runtime error:" not in out, out[-6000:]
    assert r.returncode == 0 and " passed" in out, out[-6000:]
