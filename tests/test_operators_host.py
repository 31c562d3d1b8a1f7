"""Refusals of the 8-bit products, block norms and label log probabilities: every
bad call returns from validation, on the host, before anything is launched."""
import ctypes as C
import os
import shutil
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A, B, D, E, F, G = (i << 32 for i in range(1, 7))  # addresses far apart, never read


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


def cm(S, p, r, c, ld):
    return S.saga_cmat(p, r, c, ld)


def mm(S, p, r, c, ld):
    return S.saga_mat(p, r, c, ld)


def test_quantize_rows_refusals(S):
    ok = dict(dtype=0, x=(A, 4, 10, 12), q=(B, 4, 10, 16), scale=D)

    def call(status, text, **kw):
        a = {**ok, **kw}
        refused(S, status, text, S.saga_quantize_rows, a["dtype"], cm(S, *a["x"]), mm(S, *a["q"]), a["scale"], None)

    call(S.SAGA_EINVAL, "bad dtype", dtype=2)
    call(S.SAGA_EINVAL, "null", x=(None, 4, 10, 12))
    call(S.SAGA_EINVAL, "null", q=(None, 4, 10, 16))
    call(S.SAGA_EINVAL, "null", scale=None)
    call(S.SAGA_EINVAL, "misaligned", scale=D + 2)
    call(S.SAGA_EINVAL, "multiple of 16", x=(A, 4, 10, 13))
    call(S.SAGA_EINVAL, "multiple of 16", q=(B, 4, 10, 12))
    call(S.SAGA_EINVAL, "16-byte aligned", x=(A + 4, 4, 10, 12))
    call(S.SAGA_EINVAL, "ld", x=(A, 4, 10, 8))
    call(S.SAGA_EINVAL, "shape", q=(B, 5, 10, 16))
    call(S.SAGA_EINVAL, "shape", q=(B, 4, 11, 16))
    call(S.SAGA_EINVAL, "rows", x=(A, -1, 10, 12), q=(B, -1, 10, 16))
    call(S.SAGA_EINVAL, "columns", x=(A, 4, 0, 12), q=(B, 4, 0, 16))
    call(S.SAGA_EINVAL, "out of range", x=(A, 1 << 60, 10, 12), q=(B, 1 << 60, 10, 16))
    call(S.SAGA_EUNSUPPORTED, "columns", x=(A, 1, 1 << 31, 1 << 31), q=(B, 1, 1 << 31, 1 << 31))
    call(S.SAGA_EINVAL, "overlaps", q=(A + 32, 4, 10, 16))
    call(S.SAGA_EINVAL, "overlap", scale=B)
    call(S.SAGA_EINVAL, "overlaps", scale=A + 16)
    S.saga_quantize_rows(0, cm(S, None, 0, 10, 12), mm(S, None, 0, 10, 16), None, None)  # nothing to do


def test_product_refusals(S):
    ok = dict(a_dtype=2, out_dtype=0, act=0, deg=None, a=(A, 5, 40, 48), sa=B, w=(D, 7, 40, 48), sw=E, bias=None,
              out=(F, 5, 7, 8), ws=None, nws=0)

    def call(status, text, **kw):
        a = {**ok, **kw}
        op = S.saga_quant_op(a["a_dtype"], a["out_dtype"], a["act"], a["deg"])
        refused(S, status, text, S.saga_apply_vertex_quant, op, cm(S, *a["a"]), a["sa"], cm(S, *a["w"]), a["sw"],
                a["bias"], mm(S, *a["out"]), a["ws"], a["nws"], None)

    call(S.SAGA_EINVAL, "a_dtype", a_dtype=3)
    call(S.SAGA_EINVAL, "out_dtype", out_dtype=2)
    call(S.SAGA_EINVAL, "activation", act=5)
    call(S.SAGA_EINVAL, "activation", act=-1)
    call(S.SAGA_EINVAL, "m must", a=(A, -1, 40, 48))
    call(S.SAGA_EINVAL, "k and n", a=(A, 5, 0, 48))
    call(S.SAGA_EINVAL, "k and n", w=(D, 0, 40, 48))
    call(S.SAGA_EUNSUPPORTED, "too large", a=(A, 5, 131072, 131072), w=(D, 7, 131072, 131072))
    call(S.SAGA_EUNSUPPORTED, "too large", w=(D, (1 << 28) + 1, 40, 48), out=(F, 5, (1 << 28) + 1, (1 << 28) + 4))
    call(S.SAGA_EUNSUPPORTED, "2^23", a=(A, 5, 40, 1 << 23))
    call(S.SAGA_EUNSUPPORTED, "2^23", w=(D, 7, 40, 1 << 23))
    call(S.SAGA_EINVAL, "shape", w=(D, 7, 41, 48))
    call(S.SAGA_EINVAL, "shape", out=(F, 5, 8, 8))
    call(S.SAGA_EINVAL, "shape", out=(F, 4, 7, 8))
    call(S.SAGA_EINVAL, "null", a=(None, 5, 40, 48))
    call(S.SAGA_EINVAL, "a_scale: null", sa=None)
    call(S.SAGA_EINVAL, "w_scale: null", sw=None)
    call(S.SAGA_EINVAL, "misaligned", bias=G + 1)
    call(S.SAGA_EINVAL, "misaligned", deg=G + 2)
    call(S.SAGA_EINVAL, "multiple of 16", a=(A, 5, 40, 40))
    call(S.SAGA_EINVAL, "multiple of 16", out=(F, 5, 7, 7))
    call(S.SAGA_EINVAL, "overlaps", out=(A, 5, 7, 8))
    call(S.SAGA_EINVAL, "overlaps", out=(D + 64, 5, 7, 8))
    call(S.SAGA_EINVAL, "overlaps", out=(E, 5, 7, 8))
    # float rows: no scales, and a workspace where a kernel of its own quantises them
    call(S.SAGA_EINVAL, "a_scale is for", a_dtype=0)
    m, k, n = 2000, 1300, 600
    big = dict(a_dtype=0, sa=None, a=(A, m, k, 1312), w=(D, n, k, 1312), out=(F, m, n, 608))
    need = S.saga_apply_vertex_quant_workspace_size(S.saga_quant_op(0, 0, 0, None), m, k, n)
    assert need >= m * 1312 + m * 4
    assert S.saga_apply_vertex_quant_workspace_size(S.saga_quant_op(2, 0, 0, None), m, k, n) == 0
    call(S.SAGA_EWORKSPACE, "need", **big)
    call(S.SAGA_EWORKSPACE, "need", **big, ws=G, nws=need - 1)
    call(S.SAGA_EINVAL, "256", **big, ws=G + 16, nws=need)
    call(S.SAGA_EINVAL, "overlap", **big, ws=F, nws=need)
    call(S.SAGA_EINVAL, "overlap", **big, ws=A, nws=need)
    call(S.SAGA_EINVAL, "overlap", **big, ws=D, nws=need)
    with pytest.raises(S.SagaError):
        S.saga_apply_vertex_quant_workspace_size(S.saga_quant_op(0, 0, 0, None), 5, 0, 7)
    assert S.lib().saga_apply_vertex_quant_workspace_size(None, 1, 1, 1, None) == S.SAGA_EINVAL


def test_block_norm_refusals(S):
    inf, nan = float("inf"), float("nan")
    ok = dict(dtype=0, x_dtype=0, post=(1, 1e-5, None, None), pre=(2, 1e-5, None, None), act=0, ch=None,
              block=(A, 6, 20, 20), gate=(None, 0, 0, 0), x=(B, 6, 20, 20), y=(D, 6, 20, 20), z=(E, 6, 20, 20), zs=None)

    def call(status, text, **kw):
        a = {**ok, **kw}
        op = S.saga_block_op(a["dtype"], a["x_dtype"], S.saga_norm_desc(*a["post"]), S.saga_norm_desc(*a["pre"]),
                             a["act"], 1.0, a["ch"])
        refused(S, status, text, S.saga_block_norm, op, cm(S, *a["block"]), cm(S, *a["gate"]), cm(S, *a["x"]),
                mm(S, *a["y"]), mm(S, *a["z"]), a["zs"], None)

    call(S.SAGA_EINVAL, "dtype", dtype=2)
    call(S.SAGA_EINVAL, "dtype", x_dtype=-1)
    call(S.SAGA_EUNSUPPORTED, "stream", x_dtype=1)
    call(S.SAGA_EINVAL, "activation", act=9)
    call(S.SAGA_EINVAL, "bad norm", post=(3, 1e-5, None, None))
    call(S.SAGA_EINVAL, "bad norm", pre=(-1, 1e-5, None, None))
    for eps in (0.0, -1.0, inf, nan):
        call(S.SAGA_EINVAL, "eps", pre=(1, eps, None, None))
    call(S.SAGA_EINVAL, "misaligned", pre=(1, 1e-5, G + 1, None))
    call(S.SAGA_EINVAL, "misaligned", ch=G + 3)
    wide = 16385
    call(S.SAGA_EUNSUPPORTED, "too large", block=(A, 6, wide, wide + 3), x=(B, 6, wide, wide + 3),
         y=(D, 6, wide, wide + 3), z=(E, 6, wide, wide + 3))
    call(S.SAGA_EINVAL, "columns", block=(A, 6, 0, 20))
    call(S.SAGA_EINVAL, "null", block=(None, 6, 20, 20))
    call(S.SAGA_EINVAL, "shape", gate=(F, 5, 20, 20))
    call(S.SAGA_EINVAL, "shape", x=(B, 6, 19, 20))
    call(S.SAGA_EINVAL, "shape", y=(D, 7, 20, 20))
    call(S.SAGA_EINVAL, "shape", z=(E, 6, 21, 24))
    call(S.SAGA_EINVAL, "multiple of 16", block=(A, 6, 20, 21))
    call(S.SAGA_EINVAL, "multiple of 16", z=(E, 6, 20, 20), zs=F)  # 8-bit rows: 20 bytes
    call(S.SAGA_EINVAL, "neither", y=(None, 0, 0, 0), z=(None, 0, 0, 0))
    call(S.SAGA_EINVAL, "z_scale without", z=(None, 0, 0, 0), zs=F)
    call(S.SAGA_EINVAL, "overlaps an input", y=(A, 6, 20, 20))
    call(S.SAGA_EINVAL, "overlaps an input", z=(B, 6, 20, 20))
    call(S.SAGA_EINVAL, "overlaps an input", y=(B + 16, 6, 20, 20))       # near x, but not x itself
    call(S.SAGA_EINVAL, "overlaps an input", y=(B, 6, 20, 24))            # x's base, another ld
    call(S.SAGA_EINVAL, "two outputs", z=(D + 64, 6, 20, 20))
    call(S.SAGA_EINVAL, "overlaps an input", pre=(1, 1e-5, E + 16, None))
    call(S.SAGA_EINVAL, "overlap", z=(E, 6, 20, 32), zs=E + 64)


def test_label_refusals(S):
    ok = dict(dtype=0, x=(A, 8, 100, 100), labels=B, logp=D, ent=E, k=3, ti=F, tl=G, ws=None, nws=0)

    def call(status, text, **kw):
        a = {**ok, **kw}
        refused(S, status, text, S.saga_label_log_probs, a["dtype"], cm(S, *a["x"]), a["labels"], a["logp"], a["ent"],
                a["k"], a["ti"], a["tl"], a["ws"], a["nws"], None)

    call(S.SAGA_EINVAL, "dtype", dtype=2)
    call(S.SAGA_EINVAL, "top_k", k=-1)
    call(S.SAGA_EINVAL, "top_k", k=33)
    call(S.SAGA_EINVAL, "logits", x=(A, 8, 0, 100))
    call(S.SAGA_EINVAL, "logits", x=(A, -8, 100, 100))
    call(S.SAGA_EUNSUPPORTED, "classes", x=(A, 8, (1 << 30) + 1, (1 << 30) + 4))
    call(S.SAGA_EINVAL, "null", x=(None, 8, 100, 100))
    call(S.SAGA_EINVAL, "multiple of 16", x=(A, 8, 100, 101))
    call(S.SAGA_EINVAL, "16-byte aligned", x=(A + 4, 8, 100, 100))
    call(S.SAGA_EINVAL, "both or neither", logp=None)
    call(S.SAGA_EINVAL, "both or neither", labels=None)
    call(S.SAGA_EINVAL, "null", ti=None)
    call(S.SAGA_EINVAL, "null", tl=None)
    call(S.SAGA_EINVAL, "misaligned", ent=E + 1)
    call(S.SAGA_EINVAL, "no output", labels=None, logp=None, ent=None, k=0)
    call(S.SAGA_EINVAL, "overlaps", logp=A + 400)
    call(S.SAGA_EINVAL, "two outputs", tl=F + 4)
    call(S.SAGA_EINVAL, "overlaps", ent=B)
    # few long rows are split: a workspace
    c = 100000
    need = S.saga_label_log_probs_workspace_size(0, 8, c, 3)
    assert need > 0 and S.saga_label_log_probs_workspace_size(0, 8, 100, 3) == 0
    call(S.SAGA_EWORKSPACE, "need", x=(A, 8, c, c))
    call(S.SAGA_EWORKSPACE, "need", x=(A, 8, c, c), ws=7 << 32, nws=need - 1)
    call(S.SAGA_EINVAL, "256", x=(A, 8, c, c), ws=(7 << 32) + 4, nws=need)
    call(S.SAGA_EINVAL, "overlap", x=(A, 8, c, c), ws=D, nws=need)
    call(S.SAGA_EINVAL, "overlap", x=(A, 8, c, c), ws=A, nws=need)
    assert S.lib().saga_label_log_probs_workspace_size(0, 1, 1, 1, None) == S.SAGA_EINVAL


def test_tensors_off_the_gpu_are_refused():
    from paper_2009_00804_amd import layers as L

    x = torch.zeros(4, 16)
    w, ws = torch.zeros(8, 16, dtype=torch.int8), torch.ones(8)
    for f in (lambda: L.quantize_rows(x), lambda: L.quant_linear(x, w, ws), lambda: L.block_norm(x, x),
              lambda: L.label_log_probs(x, torch.zeros(4, dtype=torch.int32))):
        with pytest.raises(ValueError, match="on the GPU"):
            f()


def test_tensor_checks():
    """types, shapes and strides, as the torch entry points check them"""
    from paper_2009_00804_amd import layers as L

    x = torch.zeros(4, 16)
    for bad in (x.double(), x[0], x.t(), x[:, ::2]):
        with pytest.raises(ValueError, match="x"):
            L._matrix(bad, "x", bad, (torch.float32,))
    with pytest.raises(ValueError, match="shape"):
        L._matrix(x, "x", x, (torch.float32,), (4, 15))
    for bad in (torch.zeros(5), torch.zeros(4).double(), torch.zeros(8)[::2]):
        with pytest.raises(ValueError, match="v"):
            L._vector(bad, "v", x, 4)
    assert L._vector(None, "v", x, 4) is None and L._matrix(None, "x", x, ()).ptr is None


def test_every_argument_by_its_name():
    """the torch entry points take each argument by the name that they show"""
    import inspect

    from paper_2009_00804_amd import layers as L

    x = torch.zeros(4, 16)
    w, ws = torch.zeros(8, 16, dtype=torch.int8), torch.ones(8)
    to = torch.zeros(4, dtype=torch.int32)
    given = {"x": x, "w": w, "w_scale": ws, "x_scale": None, "bias": None, "act": "none", "row_scale_deg": None,
             "out_dtype": None, "block": x, "post": "none", "post_weight": None, "post_bias": None, "gate": None,
             "gate_act": "none", "channel_scale": None, "res_scale": 1.0, "pre": "none", "pre_weight": None,
             "pre_bias": None, "eps": 1e-5, "quantize": False, "in_place": False, "x_dtype": None, "logits": x,
             "labels": to, "top_k": 2, "entropy": True, "stream": None}
    for f in (L.quantize_rows, L.quant_linear, L.block_norm, L.label_log_probs):
        names = list(inspect.signature(f).parameters)
        assert names[-1] == "stream"
        with pytest.raises(ValueError, match="on the GPU"):  # (past the binding of the arguments)
            f(**{n: given[n] for n in names})
        with pytest.raises(ValueError, match="on the GPU"):
            f(given[names[0]], **{n: given[n] for n in names[1:]})
        with pytest.raises(TypeError, match=f"required positional argument.*'{names[0]}'"):
            f()
        with pytest.raises(TypeError, match="tensor"):
            f(3)
        with pytest.raises(TypeError, match="tensor"):
            f(**{names[0]: None})


def test_a_single_row_has_no_pitch():
    from paper_2009_00804_amd import layers as L

    for t in (torch.zeros(1, 41), torch.zeros(41)[None], torch.zeros(41, 1).t(), torch.zeros(0, 41), torch.zeros(9, 41)[4:5]):
        m = L._matrix(t, "x", t, (torch.float32,))
        assert (m.rows, m.cols, m.ld) == (t.shape[0], 41, 44)
    t = torch.zeros(1, 41, dtype=torch.bfloat16)
    assert L._matrix(t, "x", t, (torch.bfloat16,)).ld == 48
    t = torch.zeros(2, 41)
    assert L._matrix(t, "x", t, (torch.float32,)).ld == 41  # (which the library refuses)
    with pytest.raises(ValueError, match="neighbours"):
        L._matrix(torch.zeros(1, 82)[:, ::2], "x", t, (torch.float32,))


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
            "                      'tests/test_operators_host.py']))\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    out = r.stdout + r.stderr
    assert "AddressSanitizer" not in out and "runtime error:" not in out, out[-6000:]
    assert r.returncode == 0 and " passed" in out, out[-6000:]
