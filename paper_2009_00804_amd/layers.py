"""Layer and model compositions over the C ABI (torch only allocates).

``Layer`` binds a ``saga_layer_desc`` to device weights and preallocates its
workspace and output, so a forward pass enqueues kernels and nothing else.
The two-layer models of the workloads (GCN: ReLU then raw output; GAT:
concat + ELU then head mean) are sequences of such layers.

``quantize_rows``, ``quant_linear``, ``quantize_rows_mx4``, ``dequantize_rows_mx4``,
``mx4_linear``, ``expert_layer``, ``block_norm`` and ``label_log_probs`` call the operators
of a deep network on torch tensors; ``ResidualGCN`` is such a network, served with 8-bit
or 4-bit transforms and, if it has them, a layer of experts for the vertices asked for.
"""
from __future__ import annotations

import ctypes as C
import functools
import inspect

import torch

from . import saga as S


def _dev(t, device, dtype=None):
    if t is None:
        return None
    t = torch.as_tensor(t)
    return t.to(device=device, dtype=dtype or t.dtype).contiguous()


class Layer:
    """One SAGA-NN layer (Table I model) with preallocated buffers."""

    def __init__(self, graph: S.Graph, kind: str, in_feat: int, out_feat: int, weights: dict,
                 dtype=torch.float32, act="none", heads=1, head_mean=False, neg_slope=0.2,
                 edge_feat=0, out_ld=None, hidden=0, rel=None):
        dev = graph.row_ptr.device
        self.graph = graph
        self.dtype = dtype
        wdt = dtype
        kinds = {"gcn": S.SAGA_LAYER_GCN, "gat": S.SAGA_LAYER_GAT, "sage_pool": S.SAGA_LAYER_SAGE_POOL,
                 "gated_gru": S.SAGA_LAYER_GATED_GRU, "sage_lstm": S.SAGA_LAYER_SAGE_LSTM,
                 "rgcn": S.SAGA_LAYER_RGCN}
        self.w = {k: (_dev(v, dev, wdt if k in ("w", "w_pool", "w_self") else torch.float32))
                  for k, v in weights.items()}
        d = S.saga_layer_desc()
        d.kind = kinds[kind]
        d.dtype = S.dtype_code(dtype)
        d.in_feat = in_feat
        d.out_feat = out_feat
        d.heads = heads
        d.head_mean = int(head_mean)
        d.neg_slope = neg_slope
        d.act = S.ACT[act]
        d.edge_feat = edge_feat
        d.hidden = hidden
        for k in ("w", "b", "w_pool", "b_pool", "attn_l", "attn_r", "w_e", "b_e", "w_ih", "b_ih",
                  "w_hh", "b_hh", "w_self"):
            t = self.w.get(k)
            setattr(d, k, None if t is None else t.data_ptr())
        self.rel = rel  # keeps the RelGraph (and its device arrays) alive
        if rel is not None:
            d.rel = C.pointer(rel.rel)
        self.desc = d
        self.ws_bytes = S.saga_layer_workspace_size(graph.plan, d)
        self.ws = S.workspace(self.ws_bytes, dev)
        es = torch.tensor([], dtype=dtype).element_size()
        ld = out_ld or ((out_feat * es + 15) // 16 * 16) // es
        self.out_buf = torch.empty((graph.num_dst, ld), dtype=dtype, device=dev)
        self.out = self.out_buf[:, :out_feat]

    def __call__(self, x, edge_feat=None, stream=None):
        S.saga_layer(self.graph.plan, self.desc, S.cmat(x), S.cmat(edge_feat), S.mat(self.out),
                     C.c_void_p(self.ws.data_ptr()), self.ws.numel(), S.stream_handle(stream))
        return self.out


def gcn2(graph, W1, b1, W2, b2, dtype=torch.float32, out_ld=None):
    """2-layer GCN: ReLU after layer 1, raw output after layer 2."""
    l1 = Layer(graph, "gcn", W1.shape[0], W1.shape[1], {"w": W1, "b": b1}, dtype=dtype, act="relu")
    l2 = Layer(graph, "gcn", W2.shape[0], W2.shape[1], {"w": W2, "b": b2}, dtype=dtype, act="none",
               out_ld=out_ld)
    return [l1, l2]


def gat2(graph, g, dtype=torch.float32):
    """2-layer GAT: heads concatenated + ELU, then heads averaged."""
    K = g["heads"]
    F1 = g["W1"].shape[1]
    l1 = Layer(graph, "gat", g["W1"].shape[0], F1,
               {"w": g["W1"], "b": g["b1"], "attn_l": g["al1"], "attn_r": g["ar1"]},
               heads=K, act="elu", neg_slope=g["neg_slope"])
    l2 = Layer(graph, "gat", F1, g["W2"].shape[1] // K,
               {"w": g["W2"], "b": g["b2"], "attn_l": g["al2"], "attn_r": g["ar2"]},
               heads=K, head_mean=True, act="none", neg_slope=g["neg_slope"])
    return [l1, l2]


def sage_pool(graph, g):
    F = g["W_pool"].shape[0]
    return [Layer(graph, "sage_pool", F, g["W"].shape[1],
                  {"w": g["W"], "b": g["b"], "w_pool": g["W_pool"], "b_pool": g["b_pool"]})]


def gated_gru(graph, g):
    F = g["H"].shape[1]
    return [Layer(graph, "gated_gru", F, F,
                  {"w_e": g["W_e"], "b_e": g["b_e"], "w_ih": g["W_ih"], "b_ih": g["b_ih"],
                   "w_hh": g["W_hh"], "b_hh": g["b_hh"]}, edge_feat=g["E_feat"].shape[1])]


def sage_lstm(graph, g):
    """GraphSAGE layer with the LSTM Gather: out = [x | LSTM(in-edges)] W + b."""
    F, G4 = g["W_ih"].shape
    return [Layer(graph, "sage_lstm", F, g["W"].shape[1],
                  {"w": g["W"], "b": g["b"], "w_ih": g["W_ih"], "b_ih": g["b_ih"],
                   "w_hh": g["W_hh"], "b_hh": g["b_hh"]}, hidden=G4 // 4)]


def rgcn(graph, rel, g, dtype=torch.float32):
    """R-GCN layer: act(x_v W_self + b + sum over in-edges of x_u W_r / c(v, r))."""
    R, Fi, Fo = g["W_rel"].shape
    return [Layer(graph, "rgcn", Fi, Fo,
                  {"w": g["W_rel"].reshape(R * Fi, Fo), "w_self": g["W_self"], "b": g["b"]},
                  dtype=dtype, act=g.get("act", "none"), rel=rel)]


def run(layers, x, edge_feat=None, stream=None):
    h = x
    for l in layers:
        h = l(h, edge_feat=edge_feat, stream=stream)
    return h


# --------------------------------------------------------------------------
# operators of a deep network on torch tensors
#
# Matrices are 2-D, on one GPU, each row's columns neighbours; a matrix begins on 16 bytes
# and its rows lie a multiple of 16 bytes apart (S.padded_empty makes such a buffer, and
# every matrix returned here is one; a single row needs no pitch).  Others are
# refused, not copied.  The scales of 4-bit rows lie a multiple of 4 bytes apart and begin
# on 4.  Vectors are contiguous: float32, labels and degrees int32.
# Errors: ValueError for what the tensors give away, S.SagaError from the library.
#
# Inference only, as the library: results have no history, whether the inputs require
# grad or not.
# --------------------------------------------------------------------------
def _placed(f):
    """Runs f on its first tensor's device and on ``stream`` (None: torch's
    current stream of that device).  Outputs and workspaces are allocated there,
    so calls on different streams or in different graphs share none.  The caller
    orders ``stream`` with the work before and after, as for torch's own operators."""
    parameters = inspect.signature(f).parameters
    first = next(iter(parameters))

    @functools.wraps(f)
    def call(*args, stream=None, **kw):
        if not args and first not in kw:
            return f(*args, **kw)  # (Python's own TypeError)
        x = args[0] if args else kw[first]
        if not isinstance(x, torch.Tensor):
            raise TypeError(f"{f.__name__}: {first}: a tensor is needed, got {type(x).__name__}")
        if not x.is_cuda:
            raise ValueError(f"{f.__name__}: tensors on the GPU are needed, got one on {x.device}")
        if stream is None and x.get_device() == torch._C._cuda_getDevice():
            return f(*args, **kw)
        here = torch.cuda.current_stream(x.device)
        with torch.cuda.device(x.device), torch.cuda.stream(stream):
            if torch.cuda.current_device() != x.device.index:
                raise ValueError(f"{f.__name__}: the stream belongs to another device than {x.device}")
            out = f(*args, **kw)
        if stream is not None and stream != here:
            # memory freed by the caller waits for this call, results for the caller's reads
            for ts, reader in (((*args, *kw.values()), stream), (out if isinstance(out, tuple) else (out,), here)):
                for t in ts:
                    if isinstance(t, torch.Tensor):
                        t.record_stream(reader)
        return out

    call.__signature__ = inspect.Signature(
        [*parameters.values(), inspect.Parameter("stream", inspect.Parameter.KEYWORD_ONLY, default=None)])
    return call


def _matrix(t, name, like, dtypes, shape=None, unit=16):
    """saga_cmat of a 2-D tensor on the device of ``like``"""
    if t is None:
        return S.saga_cmat(None, 0, 0, 0)
    size = t.shape
    if len(size) != 2 or t.dtype not in dtypes or t.get_device() != like.get_device():
        raise ValueError(f"{name}: a 2-D tensor of {dtypes} on {like.device} is needed, got "
                         f"{tuple(size)} {t.dtype} on {t.device}")
    if shape is not None and size != shape:
        raise ValueError(f"{name}: shape {tuple(size)}, expected {tuple(shape)}")
    rows, cols = size
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError(f"{name}: the columns of a row have to be neighbours")
    if rows <= 1:  # no pitch to speak of
        ld = _whole(cols, t.dtype, unit)
    return S.saga_cmat(t.data_ptr(), rows, cols, ld)


def _vector(t, name, like, n, dtype=torch.float32):
    """address of a contiguous vector of n values on the device of ``like``"""
    if t is None:
        return None
    if t.dtype != dtype or t.get_device() != like.get_device() or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name}: {n} contiguous values of {dtype} on {like.device} are needed, got "
                         f"{tuple(t.shape)} {t.dtype} on {t.device}")
    return t.data_ptr()


def _whole(cols, dtype, unit=16):
    """cols rounded up to whole 16 bytes (or ``unit``)"""
    a = unit // dtype.itemsize
    return (cols + a - 1) // a * a


def _out(rows, cols, dtype, like, unit=16):
    """(view, saga_mat) of a new matrix with 16-byte rows (or a multiple of ``unit`` bytes)"""
    ld = _whole(cols, dtype, unit)
    buf = like.new_empty((rows, ld), dtype=dtype)
    return (buf if ld == cols else buf[:, :cols]), S.saga_mat(buf.data_ptr(), rows, cols, ld)


def _stream(t):
    """hipStream_t of torch's current stream on t's device"""
    return torch._C._cuda_getCurrentRawStream(t.get_device())


def _space(nbytes, like):
    return like.new_empty(nbytes, dtype=torch.uint8) if nbytes else None


# (workspace sizes depend on types and sizes alone)
@functools.lru_cache(maxsize=1024)
def _quant_bytes(a_dtype, out_dtype, m, k, n):
    return S.saga_apply_vertex_quant_workspace_size(S.saga_quant_op(a_dtype, out_dtype, 0, None), m, k, n)


@functools.lru_cache(maxsize=1024)
def _label_bytes(dtype, m, c, top_k):
    return S.saga_label_log_probs_workspace_size(dtype, m, c, top_k)


@functools.lru_cache(maxsize=1024)
def _mx_bytes(a_dtype, out_dtype, m, k, n):
    return S.saga_apply_vertex_mx_workspace_size(S.saga_mx_op(a_dtype, out_dtype, 0, None), m, k, n)


@functools.lru_cache(maxsize=1024)
def _expert_bytes(*sizes):
    return S.saga_apply_vertex_experts_workspace_size(S.saga_expert_op(*sizes[:-4]), *sizes[-4:])


_FLOATS = (torch.float32, torch.bfloat16)
_BYTES = (torch.int8,)
_NIBBLES = (torch.uint8,)
_NONE = S.saga_cmat(None, 0, 0, 0)


def _four_bit(q, scale, name, scale_name, like, shape=None):
    """saga_cmats of 4-bit rows and their scales, whose rows lie a multiple of 4 bytes apart"""
    cq = _matrix(q, name, like, _NIBBLES, shape)
    if scale is None:
        raise ValueError(f"{scale_name}: 4-bit rows need their scales")
    return cq, _matrix(scale, scale_name, like, _NIBBLES, (cq.rows, (cq.cols + 15) // 16), 4)


@_placed
def quantize_rows(x):
    """(q, scale): the 8-bit rows of x and their float32 scales."""
    cx = _matrix(x, "x", x, _FLOATS)
    q, mq = _out(x.shape[0], x.shape[1], torch.int8, x)
    scale = x.new_empty(x.shape[0], dtype=torch.float32)
    S.saga_quantize_rows(S.dtype_code(x.dtype), cx, mq, scale.data_ptr(), _stream(x))
    return q, scale


@_placed
def quant_linear(x, w, w_scale, x_scale=None, bias=None, act="none", row_scale_deg=None, out_dtype=None):
    """act(rs * (x w^T) + bias) in 8-bit integers: w and w_scale hold one output
    channel a row; x is 8-bit rows with x_scale, or float rows that the call
    quantises.  out_dtype: x's own, float32 for 8-bit rows."""
    m, k = x.shape
    i8 = x.dtype == torch.int8
    if out_dtype is None:
        out_dtype = torch.float32 if i8 else x.dtype
    cx = _matrix(x, "x", x, _BYTES if i8 else _FLOATS)
    n = w.shape[0]
    cw = _matrix(w, "w", x, _BYTES, (n, k))
    op = S.saga_quant_op(S.SAGA_I8 if i8 else S.dtype_code(x.dtype), S.dtype_code(out_dtype), S.ACT[act],
                         _vector(row_scale_deg, "row_scale_deg", x, m, torch.int32))
    nbytes = _quant_bytes(op.a_dtype, op.out_dtype, m, k, n)
    out, mo = _out(m, n, out_dtype, x)
    ws = _space(nbytes, x)
    S.saga_apply_vertex_quant(op, cx, _vector(x_scale, "x_scale", x, m), cw,
                              _vector(w_scale, "w_scale", x, n), _vector(bias, "bias", x, n), mo,
                              ws.data_ptr() if nbytes else None, nbytes, _stream(x))
    return out


@_placed
def quantize_rows_mx4(x):
    """(q, scale): the 4-bit rows of x, two columns a byte, and a scale byte for every
    32 columns."""
    m, k = x.shape
    cx = _matrix(x, "x", x, _FLOATS)
    q, mq = _out(m, (k + 1) // 2, torch.uint8, x)
    scale, ms = _out(m, (k + 31) // 32, torch.uint8, x, 4)
    S.saga_quantize_rows_mx(S.dtype_code(x.dtype), cx, mq, ms, _stream(x))
    return q, scale


@_placed
def dequantize_rows_mx4(q, scale, columns=None, dtype=torch.bfloat16):
    """The values that 4-bit rows stand for, as float32 or bfloat16; columns: how many
    (all that q's bytes hold, or one less)."""
    if columns is None:
        columns = 2 * q.shape[1]
    cq, cs = _four_bit(q, scale, "q", "scale", q)
    x, mx = _out(q.shape[0], columns, dtype, q)
    S.saga_dequantize_rows_mx(S.dtype_code(dtype), cq, cs, mx, _stream(q))
    return x


@_placed
def mx4_linear(x, w, w_scale, x_scale=None, bias=None, act="none", row_scale_deg=None, out_dtype=None):
    """act(rs * (x w^T) + bias) on 4-bit rows: w and w_scale hold one output channel a
    row; x is 4-bit rows with x_scale, or float rows that the call quantises.
    out_dtype: x's own, float32 for 4-bit rows."""
    m, k = x.shape
    mx = x.dtype == torch.uint8
    if mx:
        k *= 2
    if out_dtype is None:
        out_dtype = torch.float32 if mx else x.dtype
    n = w.shape[0]
    if mx:
        cx, cxs = _four_bit(x, x_scale, "x", "x_scale", x)
    elif x_scale is not None:
        raise ValueError("x_scale: for 4-bit rows (float rows are quantised by the call)")
    else:
        cx, cxs = _matrix(x, "x", x, _FLOATS), _NONE
    cw, cws = _four_bit(w, w_scale, "w", "w_scale", x, (n, (k + 1) // 2))
    op = S.saga_mx_op(S.SAGA_MX4 if mx else S.dtype_code(x.dtype), S.dtype_code(out_dtype), S.ACT[act],
                      _vector(row_scale_deg, "row_scale_deg", x, m, torch.int32))
    nbytes = _mx_bytes(op.a_dtype, op.out_dtype, m, k, n)
    out, mo = _out(m, n, out_dtype, x)
    ws = _space(nbytes, x)
    S.saga_apply_vertex_mx(op, cx, cxs, cw, cws, _vector(bias, "bias", x, n), mo,
                           ws.data_ptr() if nbytes else None, nbytes, _stream(x))
    return out


@_placed
def expert_layer(x, router, up, down, *, up_scale=None, down_scale=None, router_bias=None, up_bias=None,
                 down_bias=None, top_k=1, act="relu", gated=False, renormalise=True):
    """(y, index, weight): y = sum over each row's top_k experts of weight *
    (act(x up^T) down^T), the experts chosen by x router^T.  up and down hold the experts'
    weights one below the other, an output channel a row, in bfloat16 or, with
    up_scale and down_scale, in 4 bits; gated: up holds each expert's gate above its up, and
    an expert is (act(x gate^T) * (x up^T)) down^T."""
    m, f = x.shape
    e = router.shape[0]
    per = e * (2 if gated else 1)
    mx = up.dtype == torch.uint8
    h, n = (up.shape[0] // per, down.shape[0] // e) if e else (0, 0)
    if not e or h * per != up.shape[0] or n * e != down.shape[0]:
        raise ValueError(f"{up.shape[0]} rows of up and {down.shape[0]} of down are no multiple of {e} experts'")
    w = S.saga_expert_weights()
    cx = _matrix(x, "x", x, _FLOATS)
    w.router = _matrix(router, "router", x, _FLOATS, (e, f))
    if mx:
        w.up, w.up_scale = _four_bit(up, up_scale, "up", "up_scale", x, (per * h, (f + 1) // 2))
        w.down, w.down_scale = _four_bit(down, down_scale, "down", "down_scale", x, (e * n, (h + 1) // 2))
    elif up_scale is not None or down_scale is not None:
        raise ValueError("up_scale, down_scale: for 4-bit weights")
    else:
        w.up = _matrix(up, "up", x, (torch.bfloat16,), (per * h, f))
        w.down = _matrix(down, "down", x, (torch.bfloat16,), (e * n, h))
    w.router_bias = _vector(router_bias, "router_bias", x, e)
    w.up_bias = _vector(up_bias, "up_bias", x, per * h)
    w.down_bias = _vector(down_bias, "down_bias", x, e * n)
    op = S.saga_expert_op(S.dtype_code(x.dtype), S.dtype_code(router.dtype), S.SAGA_MX4 if mx else S.SAGA_BF16, e,
                          top_k, S.ACT[act], bool(gated), bool(renormalise))
    nbytes = _expert_bytes(*(getattr(op, name) for name, _ in op._fields_), m, f, h, n)
    y, my = _out(m, n, x.dtype, x)
    index = x.new_empty((m, top_k), dtype=torch.int32)
    weight = x.new_empty((m, top_k), dtype=torch.float32)
    ws = _space(nbytes, x)
    S.saga_apply_vertex_experts(op, w, cx, my, index.data_ptr(), weight.data_ptr(),
                                ws.data_ptr() if nbytes else None, nbytes, _stream(x))
    return y, index, weight


@_placed
def block_norm(block, x=None, *, post="none", post_weight=None, post_bias=None, gate=None, gate_act="none",
               channel_scale=None, res_scale=1.0, pre="none", pre_weight=None, pre_bias=None, eps=1e-5,
               quantize=False, in_place=False, x_dtype=None):
    """(y, z, z_scale): y = x + res_scale * channel_scale * act(gate) * post(block)
    and z = pre(y), quantised to 8-bit rows with z_scale if ``quantize`` (else
    z_scale is None).  x_dtype: the type of y where there is no x; in_place: y is
    written into x."""
    m, f = block.shape
    cb = _matrix(block, "block", block, _FLOATS)
    if x is not None:
        x_dtype = x.dtype
    elif x_dtype is None:
        x_dtype = block.dtype
    cx = _matrix(x, "x", block, _FLOATS, block.shape)
    cg = _matrix(gate, "gate", block, (block.dtype,), block.shape)
    op = S.saga_block_op(
        S.dtype_code(block.dtype), S.dtype_code(x_dtype),
        S.saga_norm_desc(S.NORM[post], eps, _vector(post_weight, "post_weight", block, f),
                         _vector(post_bias, "post_bias", block, f)),
        S.saga_norm_desc(S.NORM[pre], eps, _vector(pre_weight, "pre_weight", block, f),
                         _vector(pre_bias, "pre_bias", block, f)),
        S.ACT[gate_act], res_scale, _vector(channel_scale, "channel_scale", block, f))
    if in_place:
        if x is None:
            raise ValueError("in_place: there is no x")
        if x.requires_grad and torch.is_grad_enabled():
            raise ValueError("in_place: x requires grad, and no gradient passes through this call")
        y, my = x, S.saga_mat(cx.ptr, cx.rows, cx.cols, cx.ld)
    else:
        y, my = _out(m, f, x_dtype, block)
    z, mz = _out(m, f, torch.int8 if quantize else block.dtype, block)
    zs = block.new_empty(m, dtype=torch.float32) if quantize else None
    S.saga_block_norm(op, cb, cg, cx, my, mz, zs.data_ptr() if quantize else None, _stream(block))
    if in_place:  # (a backward pass that saved x sees that it has changed)
        torch.autograd.graph.increment_version(x)
    return y, z, zs


@_placed
def label_log_probs(logits, labels=None, top_k=0, entropy=True):
    """(logp, entropy, top_index, top_logp) of rows of logits; logp is None without
    labels, entropy None if it is not asked for."""
    m, c = logits.shape
    cl = _matrix(logits, "logits", logits, _FLOATS)
    code = S.dtype_code(logits.dtype)
    at = _vector(labels, "labels", logits, m, torch.int32)
    nbytes = _label_bytes(code, m, c, top_k)
    ws = _space(nbytes, logits)
    lp = logits.new_empty(m, dtype=torch.float32) if labels is not None else None
    h = logits.new_empty(m, dtype=torch.float32) if entropy else None
    ti = logits.new_empty((m, top_k), dtype=torch.int32)
    tl = logits.new_empty((m, top_k), dtype=torch.float32)
    S.saga_label_log_probs(code, cl, at, lp.data_ptr() if labels is not None else None,
                           h.data_ptr() if entropy else None, top_k, ti.data_ptr() if top_k else None,
                           tl.data_ptr() if top_k else None, ws.data_ptr() if nbytes else None, nbytes,
                           _stream(logits))
    return lp, h, ti, tl


def _asked(vertices, n, device):
    """(at, off): the rows of n that ``vertices`` names, and which of its ids name none (at: any row).  Without a look
    at the ids from the host, so that a call can be captured."""
    if not isinstance(vertices, torch.Tensor) or vertices.dim() != 1 or vertices.dtype not in (
            torch.int32, torch.int64) or vertices.device != device:
        raise ValueError(f"vertices: a vector of int32 or int64 on {device} is needed, got " + (
            f"{tuple(vertices.shape)} {vertices.dtype} on {vertices.device}" if isinstance(vertices, torch.Tensor)
            else type(vertices).__name__))
    if n == 0 and vertices.numel():
        raise ValueError("vertices: the graph has none")
    at = vertices.clamp(0, max(n - 1, 0))
    return at, at != vertices


def _rows_at(t, at):
    """rows ``at`` of a matrix, in one with 16-byte rows; values ``at`` of a vector"""
    rows = t.index_select(0, at)
    return rows if t.dim() == 1 else _out(at.numel(), t.shape[1], t.dtype, t)[0].copy_(rows)


class ResidualGCN:
    """A deep GCN with a gated residual stream, its transforms in 8-bit integers (bits=8) or
    microscaled 4-bit floating point (bits=4).

        h = x W_in + b_in
        per block:  z = pre(h) quantised;  [v | g] = z [W | W_g] + [0 | b_g]
                    m = relu(d_in^-1/2 A d_out^-1/2 v + b)
                    h = h + res_scale * sigmoid(g) * post(m)
        experts:    h = h + res_scale * expert_layer(experts.norm(h))
        logits = norm(h) W_out + b_out

    weights: W_in (F_in x F), b_in, blocks: a list of dicts with W, W_g (F x F),
    b, b_g, pre, post (norm weights, F), then norm (F), W_out (F x classes), b_out;
    float32 tensors or arrays.  The weights are quantised once, one scale per
    output channel (per 32 of its weights).  F is a multiple of 8.  The stream h is
    float32, blocks are ``dtype``; all norms are RMS norms.

    experts (may be absent): a dict with norm (F), router (F x E), up (E x F x H), down
    (E x H x F), top_k, act, and, each of which may be absent, gate (E x F x H: gated
    experts), b_router (E), b_up, b_gate (E x H) and b_down (E x F).  They are kept in
    bfloat16, or in 4 bits with the transforms.  They are meant for the vertices that are asked
    for: every 1,024 rows read the experts' weights again."""

    def __init__(self, graph: S.Graph, weights: dict, dtype=torch.bfloat16, res_scale=1.0, eps=1e-5, bits=8):
        dev = graph.row_ptr.device
        if bits not in (4, 8):
            raise ValueError(f"bits has to be 4 or 8, got {bits}")
        self.graph, self.dtype, self.res_scale, self.eps, self.bits = graph, dtype, res_scale, eps, bits
        quantise = quantize_rows if bits == 8 else quantize_rows_mx4

        def vector(v):
            return None if v is None else _dev(v, dev, torch.float32).reshape(-1)

        def matrix(rows, dtype=torch.float32):
            wide, _ = _out(rows.shape[0], rows.shape[1], dtype, rows)
            return wide.copy_(rows)

        def transform(w, b):
            return (*quantise(matrix(_dev(w, dev, torch.float32).t())), vector(b))

        self.f = f = weights["blocks"][0]["W"].shape[0] if weights["blocks"] else weights["W_out"].shape[0]
        if f % 8:
            raise ValueError(f"the hidden width has to be a multiple of 8, got {f}")
        self.first = transform(weights["W_in"], weights["b_in"])
        self.blocks = []
        for b in weights["blocks"]:
            w, w_g = (_dev(b[k], dev, torch.float32) for k in ("W", "W_g"))
            gate_bias = torch.cat([torch.zeros(f, device=dev), vector(b["b_g"])])
            self.blocks.append(dict(both=transform(torch.cat([w, w_g], 1), gate_bias), bias=vector(b["b"]),
                                    pre=vector(b["pre"]), post=vector(b["post"])))
        self.norm = vector(weights["norm"])
        self.last = transform(weights["W_out"], weights["b_out"])
        self.experts = None
        if weights.get("experts"):
            x = weights["experts"]
            up, down = (_dev(x[k], dev, torch.float32).transpose(1, 2) for k in ("up", "down"))
            up_bias, gated = x.get("b_up"), x.get("gate") is not None
            if gated:
                up = torch.cat([_dev(x["gate"], dev, torch.float32).transpose(1, 2), up], 1)
                if (up_bias is None) != (x.get("b_gate") is None):
                    raise ValueError("experts: b_gate and b_up go together")
                if up_bias is not None:
                    up_bias = torch.cat([_dev(x[k], dev, torch.float32) for k in ("b_gate", "b_up")], 1)
            kw = dict(router_bias=vector(x.get("b_router")), up_bias=vector(up_bias),
                      down_bias=vector(x.get("b_down")), top_k=x["top_k"], act=x["act"], gated=gated)
            up, down = up.reshape(-1, f), down.reshape(-1, down.shape[2])
            if bits == 4:
                (up, kw["up_scale"]), (down, kw["down_scale"]) = (quantize_rows_mx4(matrix(w)) for w in (up, down))
            else:
                up, down = (matrix(w, torch.bfloat16) for w in (up, down))
            router = matrix(_dev(x["router"], dev, torch.float32).t())
            self.experts = dict(norm=vector(x["norm"]), args=(router, up, down), kw=kw)
        self.op = S.saga_edge_op()
        self.op.msg, self.op.reduce, self.op.dtype = S.SAGA_MSG_SRC_NORM, S.SAGA_RED_SUM, S.dtype_code(dtype)
        self.op.heads, self.op.dst_norm, self.op.act = 1, 1, S.SAGA_ACT_RELU
        self.ws_bytes = S.saga_gather_workspace_size(graph.plan, self.op, f)

    def gather(self, v, bias):
        """relu(d_in^-1/2 A d_out^-1/2 v + bias)"""
        out, mo = _out(self.graph.num_dst, self.f, self.dtype, v)
        ws = S.workspace(self.ws_bytes, v.device)
        inputs = S.saga_edge_inputs()
        inputs.src = S.cmat(v)
        inputs.bias = bias.data_ptr()
        S.saga_scatter_apply_edge_gather(self.graph.plan, self.op, inputs, mo, C.c_void_p(ws.data_ptr()),
                                         ws.numel(), S.stream_handle())
        return out

    def transform(self, x, weights, x_scale=None, out_dtype=torch.float32):
        """x W + b in the network's bits; x: floats, or 8-bit rows with their scales"""
        w, ws, b = weights
        if self.bits == 4:
            return mx4_linear(x, w, ws, bias=b, out_dtype=out_dtype)
        return quant_linear(x, w, ws, x_scale=x_scale, bias=b, out_dtype=out_dtype)

    def logits(self, x, vertices=None):
        """x: num_vertices x F_in (float32 or bfloat16) on the graph's device; vertices: those
        whose logits are wanted (int32 or int64; None: all), in their order; an id that is no vertex of
        the graph has NaN for logits"""
        if x.device != self.graph.row_ptr.device:
            raise ValueError(f"x is on {x.device}, the graph on {self.graph.row_ptr.device}")
        with torch.cuda.device(x.device):
            # (4-bit transforms quantise on their way, experts take floats)
            ends = [self.norm] if self.experts is None else [self.experts["norm"], self.norm]
            norms = [blk["pre"] for blk in self.blocks] + ends
            whole = [self.bits == 8] * len(self.blocks) + [self.bits == 8 and self.experts is None]
            h = self.transform(x, self.first, out_dtype=self.dtype)
            h, z, zs = block_norm(h, None, x_dtype=torch.float32, pre="rms", pre_weight=norms[0], eps=self.eps,
                                  quantize=whole[0])
            for i, blk in enumerate(self.blocks):
                vg = self.transform(z, blk["both"], zs, self.dtype)
                m = self.gather(vg[:, :self.f], blk["bias"])
                h, z, zs = block_norm(m, h, post="rms", post_weight=blk["post"], gate=vg[:, self.f:],
                                      gate_act="sigmoid", res_scale=self.res_scale, pre="rms",
                                      pre_weight=norms[i + 1], eps=self.eps, quantize=whole[i + 1], in_place=True)
            if vertices is not None:
                at, off = _asked(vertices, h.shape[0], h.device)
                h = _rows_at(h, at) if self.experts is not None else None
                z, zs = _rows_at(z, at), None if zs is None else _rows_at(zs, at)
                # (a row of NaN, or of 8-bit numbers whose scale is NaN, is NaN from here on)
                (z if zs is None else zs[:, None]).masked_fill_(off[:, None], float("nan"))
            if self.experts is not None:
                y, _, _ = expert_layer(z, *self.experts["args"], **self.experts["kw"])
                _, z, zs = block_norm(y, h, res_scale=self.res_scale, pre="rms", pre_weight=self.norm,
                                      eps=self.eps, quantize=self.bits == 8)
            return self.transform(z, self.last, zs)

    def __call__(self, x, labels=None, top_k=1, vertices=None):
        """(logp, entropy, top_index, top_logp) of every vertex, or of those asked for
        (labels: one of each of them)"""
        return label_log_probs(self.logits(x, vertices), labels, top_k)
