"""Object layer over the binding: owns torch device tensors and handles, computes nothing itself."""
from __future__ import annotations

from typing import NamedTuple

import numpy as np
import torch

from . import binding as B


class Context:
    """A library context on `device`, bound to torch's current stream on that device."""

    def __init__(self, device: int = 0):
        self.device = device
        self.torch_device = torch.device("cuda", device)
        torch.cuda.set_device(device)
        self.stream = torch.cuda.current_stream(device)
        self.handle = B.grf_ctx_create(device, self.stream.cuda_stream)

    def close(self):
        if self.handle:
            B.grf_ctx_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def launches(self) -> int:
        return B.grf_ctx_launch_count(self.handle)


class DeviceGraph:
    """CSR of W resident on the device."""

    def __init__(self, graph, device: int = 0):
        dev = torch.device("cuda", device)
        self.N = graph.N
        self.rowptr = torch.from_numpy(np.ascontiguousarray(graph.rowptr, dtype=np.int32)).to(dev)
        self.col = torch.from_numpy(np.ascontiguousarray(graph.col, dtype=np.int32)).to(dev)
        self.w = torch.from_numpy(np.ascontiguousarray(graph.w, dtype=np.float32)).to(dev)


class Features:
    def __init__(self, ctx: Context, handle: int):
        self.ctx, self.handle = ctx, handle

    def free(self):
        if self.handle:
            B.grf_features_free(self.handle)
            self.handle = None

    def shape(self, which: int):
        rows, cols, nnz, *_ = B.grf_features_view(self.handle, which)
        return rows, cols, nnz

    def to_host(self, which: int):
        """(rowptr, col, val) numpy copies of Phi (0), Psi (1) or Psi^T (2)."""
        rows, cols, nnz = self.shape(which)
        dev = torch.device("cuda", self.ctx.device)
        rp = torch.empty(rows + 1, dtype=torch.int32, device=dev)
        c = torch.empty(max(nnz, 1), dtype=torch.int32, device=dev)
        v = torch.empty(max(nnz, 1), dtype=torch.float32, device=dev)
        B.grf_features_copy(self.ctx.handle, self.handle, which, rp, c, v)
        torch.cuda.synchronize(self.ctx.device)
        return rp.cpu().numpy(), c[:nnz].cpu().numpy(), v[:nnz].cpu().numpy()


def sample(ctx: Context, g: DeviceGraph, seed, n_walks, p_halt, max_len, f_phi, f_psi=None,
           features: Features | None = None) -> Features:
    h = B.grf_sample(ctx.handle, g.N, g.rowptr, g.col, g.w, seed, n_walks, p_halt, max_len, f_phi, f_psi,
                     features.handle if features else None)
    if features:
        features.handle = h
        return features
    return Features(ctx, h)


def features_from_csr(ctx: Context, N, R, phi, psi) -> Features:
    """phi, psi: (rowptr, col, val) numpy triples."""
    dev = torch.device("cuda", ctx.device)

    def up(t):
        rp, c, v = t
        c = np.ascontiguousarray(c, dtype=np.int32); v = np.ascontiguousarray(v, dtype=np.float32)
        if c.size == 0:
            c = np.zeros(1, np.int32); v = np.zeros(1, np.float32)
        return (torch.from_numpy(np.ascontiguousarray(rp, dtype=np.int32)).to(dev),
                torch.from_numpy(c).to(dev), torch.from_numpy(v).to(dev))

    a, b = up(phi), up(psi)
    return Features(ctx, B.grf_features_from_csr(ctx.handle, N, R, *a, *b))


def masked_linear_attn(ctx: Context, feat: Features, phiQ, phiK, V, workspace=None, want_den=False,
                       workspace_bytes=None):
    """phiQ, phiK [G,N,m], V [G,N,d] CUDA tensors (fp32 or bf16).  Returns out, or (out, den)."""
    G, N, m = phiQ.shape
    d = V.shape[2]
    dt = B.dtype_code(phiQ)
    R = feat.shape(0)[1]
    if workspace is None:
        nbytes = workspace_bytes or B.grf_attn_workspace_bytes(G, R, m, d, dt)
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=phiQ.device)
    out = torch.empty_like(V)
    den = torch.empty((G, N), dtype=torch.float32, device=V.device) if want_den else None
    B.grf_masked_linear_attn(ctx.handle, feat.handle, G, N, m, d, dt, phiQ, phiK, V, out, den, workspace,
                             workspace.numel())
    return (out, den) if want_den else out


def masked_attn_asym(ctx: Context, feat: Features, Q, K, V, softmax=False, want_den=False):
    """Alg. 2 (asymmetric features: the mask estimate is Phi).  Q, K [G,N,m], V [G,N,d] CUDA tensors."""
    G, N, m = Q.shape
    d = V.shape[2]
    out = torch.empty_like(V)
    den = torch.empty((G, N), dtype=torch.float32, device=V.device) if want_den else None
    B.grf_masked_attn_asym(ctx.handle, feat.handle, G, N, m, d, B.dtype_code(Q),
                           B.GRF_KERNEL_SOFTMAX if softmax else B.GRF_KERNEL_LINEAR, Q, K, V, out, den)
    return (out, den) if want_den else out


def masked_attn_mhat(ctx: Context, feat: Features, phiQ, phiK, V, want_den=False):
    """Eqs. 1-2 over the materialised mask (call B.grf_features_materialise first).  bf16, d = 64."""
    G, N, m = phiQ.shape
    d = V.shape[2]
    out = torch.empty_like(V)
    den = torch.empty((G, N), dtype=torch.float32, device=V.device) if want_den else None
    B.grf_masked_attn_mhat(ctx.handle, feat.handle, G, N, m, d, B.dtype_code(phiQ), phiQ, phiK, V, out, den)
    return (out, den) if want_den else out


INT32_MAX = 2**31 - 1
ORDERS = {"full": B.GRF_ORDER_FULL, "causal": B.GRF_ORDER_CAUSAL, "prefix": B.GRF_ORDER_PREFIX}


def relative_buckets(n_buckets: int = 32, max_distance: int = 128) -> np.ndarray:
    """Smallest distance of each bucket of a learned relative position bias (half of them exact, half logarithmic)."""
    return B.grf_relative_buckets(n_buckets, max_distance)


class SoftmaxSaved(NamedTuple):
    """What softmax_attn keeps of its rows for softmax_attn_backward."""
    lse: torch.Tensor                   # [B, H, Nq] fp32
    rest: torch.Tensor | None           # [B, H, Nq, d] bf16: what rounding took from out (None in fp32)


def _tokens(t, device, shape, name):
    """Address of an int32 device array of the given shape."""
    if t.dtype != torch.int32 or t.device != device or tuple(t.shape) != shape or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous int32 tensor {shape} on {device}")
    return t.data_ptr()


def _set_strides(to, t, name):
    """A descriptor's strides of [batch, heads, tokens, dim] whose last axis is contiguous."""
    s = t.stride()
    if len(s) != 4:
        raise ValueError(f"{name}: expected four axes")
    if s[3] != 1 and t.shape[3] > 1:
        raise ValueError(f"{name}: the last axis must be contiguous")
    # (all zeros would mean "contiguous": an axis of one token, head or sequence is never stepped over, so any stride does)
    if s[0] == s[1] == s[2] == 0 and t.shape[0] * t.shape[1] * t.shape[2] > 1:
        raise ValueError(f"{name}: a tensor broadcast along every axis")
    to[0], to[1], to[2] = s[0], s[1], s[2]


def _softmax_desc(ctx, q, k, v, scale, cap, mask, k_len, q_start, prefix, q_doc, k_doc, slopes, table, first, two_sided):
    q_shape, k_shape = q.shape, k.shape
    if mask not in ORDERS:
        raise ValueError(f"mask: expected one of {', '.join(ORDERS)}")
    if len(q_shape) != 4 or len(k_shape) != 4 or v.shape != k_shape:
        raise ValueError("expected q [B, H, Nq, d] and k, v [B, KV, Nk, d]")
    batch, heads, n_q, dim = q_shape
    kv_heads, n_k = k_shape[1], k_shape[2]
    if n_q > INT32_MAX or n_k > INT32_MAX:
        raise ValueError("too many tokens")
    dtype, device = q.dtype, ctx.torch_device
    if k_shape[0] != batch or k_shape[3] != dim or k.dtype != dtype or v.dtype != dtype:
        raise ValueError("q, k and v disagree in batch, dim or type")
    if not (q.is_cuda and k.is_cuda and v.is_cuda and q.get_device() == k.get_device() == v.get_device() == ctx.device):
        raise ValueError(f"expected tensors on {device}")
    s = B.SoftmaxDesc(batch, heads, kv_heads, n_q, n_k, dim, B.dtype_code(q), dim ** -0.5 if scale is None else scale, cap, ORDERS[mask])
    _set_strides(s.q_stride, q, "q")
    _set_strides(s.k_stride, k, "k")
    _set_strides(s.v_stride, v, "v")
    if k_len is not None:
        s.k_len = _tokens(k_len, device, (batch,), "k_len")
    if q_start is not None:
        s.q_start = _tokens(q_start, device, (batch,), "q_start")
    if prefix is not None:
        s.prefix = _tokens(prefix, device, (batch,), "prefix")
    if q_doc is not None:
        s.q_doc = _tokens(q_doc, device, (batch, n_q), "q_doc")
    if k_doc is not None:
        s.k_doc = _tokens(k_doc, device, (batch, n_k), "k_doc")
    if slopes is not None and table is not None:
        raise ValueError("slopes or a table, not both")
    if slopes is not None:
        if slopes.dtype != torch.float32 or slopes.device != device or tuple(slopes.shape) != (heads,) or not slopes.is_contiguous():
            raise ValueError(f"slopes: expected a contiguous float32 tensor ({heads},) on {device}")
        s.bias, s.slopes = B.GRF_BIAS_SLOPES, slopes.data_ptr()
    if table is not None:
        if first is None or not 1 <= len(first) <= B.GRF_MAX_BUCKETS:
            raise ValueError(f"a table needs first, the smallest distance of each of 1 .. {B.GRF_MAX_BUCKETS} buckets")
        n = len(first)
        shape = (heads, n * (2 if two_sided else 1))
        if table.dtype != dtype or table.get_device() != ctx.device or tuple(table.shape) != shape or not table.is_contiguous():
            raise ValueError(f"table: expected a contiguous {dtype} tensor {shape} on {device}")
        s.bias, s.table, s.two_sided = B.GRF_BIAS_BUCKETS, table.data_ptr(), int(two_sided)
        B.set_distances(s, first)
    return s


def _like(t):
    """Contiguous, whatever t's strides are (torch.empty takes twice as long, and a call on few tokens is bound by the host)."""
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def _scratch(nbytes, ctx):
    """A workspace for one call.  It belongs to the context's stream, so that its memory goes to nobody else while the call runs, whichever
    stream is the current one."""
    if not nbytes:
        return None
    if torch.cuda.current_stream(ctx.device) == ctx.stream:
        return torch.empty(nbytes, dtype=torch.uint8, device=ctx.torch_device)
    with torch.cuda.stream(ctx.stream):
        return torch.empty(nbytes, dtype=torch.uint8, device=ctx.torch_device)


def _bytes(workspace):
    return 0 if workspace is None else workspace.numel() * workspace.element_size()


def softmax_attn(ctx: Context, q, k, v, scale=None, cap=0.0, mask="full", k_len=None, q_start=None, prefix=None, q_doc=None,
                 k_doc=None, slopes=None, table=None, first=None, two_sided=False, want_lse=False, out=None, workspace=None):
    """Softmax attention over tokens in an order (grf_softmax_attn).  q [B, H, Nq, d], k, v [B, KV, Nk, d]: CUDA tensors (fp32 or bf16),
    the last axis contiguous, the others of any strides, 0 among them, that are whole 16 bytes, as addresses are; d a multiple of 8 up to 128; KV divides H.  mask: "full", "causal", "prefix" (with prefix [B]).  k_len, q_start,
    prefix [B], q_doc [B, Nq], k_doc [B, Nk]: int32.  A bias by distance: slopes [H] (fp32), or table [H, len(first)] (twice as many
    columns when two_sided) with first as relative_buckets gives it.  Returns out [B, H, Nq, d]; with want_lse (out, SoftmaxSaved),
    which the backward pass takes."""
    s = _softmax_desc(ctx, q, k, v, scale, cap, mask, k_len, q_start, prefix, q_doc, k_doc, slopes, table, first, two_sided)
    if out is None:
        out = _like(q)
    elif out.shape != q.shape or out.dtype != q.dtype or out.device != q.device:
        raise ValueError("out: expected the shape, type and device of q")
    else:
        _set_strides(s.out_stride, out, "out")
    lse = q.new_empty(q.shape[:3], dtype=torch.float32) if want_lse else None
    if workspace is None:
        workspace = _scratch(B.grf_softmax_attn_workspace_bytes(ctx.handle, s, False), ctx)
    rest = _like(q) if want_lse and q.dtype == torch.bfloat16 else None
    B.grf_softmax_attn(ctx.handle, s, q, k, v, out, lse, rest, workspace, _bytes(workspace))
    return (out, SoftmaxSaved(lse, rest)) if want_lse else out


def softmax_attn_backward(ctx: Context, q, k, v, out, saved, dout, scale=None, cap=0.0, mask="full", k_len=None, q_start=None,
                          prefix=None, q_doc=None, k_doc=None, slopes=None, table=None, first=None, two_sided=False,
                          want_dtable=True, workspace=None):
    """Gradients of softmax_attn from its out and SoftmaxSaved and the gradient dout of out (strides as of q): (dq, dk, dv, dtable), dtable None
    without a table.  Gradients of broadcast or shared k, v are those of the tensors as they are passed."""
    s = _softmax_desc(ctx, q, k, v, scale, cap, mask, k_len, q_start, prefix, q_doc, k_doc, slopes, table, first, two_sided)
    for name, t in (("out", out), ("dout", dout)):
        if t.shape != q.shape or t.dtype != q.dtype or t.device != q.device:
            raise ValueError(f"{name}: expected the shape, type and device of q")
    lse, rest = saved
    if lse.shape != q.shape[:3] or lse.dtype != torch.float32 or lse.device != q.device:
        raise ValueError("lse: expected float32 [B, H, Nq]")
    if rest is not None and (rest.shape != q.shape or rest.dtype != q.dtype or rest.device != q.device):
        raise ValueError("rest: expected the shape, type and device of q")
    _set_strides(s.out_stride, out, "out")
    _set_strides(s.dout_stride, dout, "dout")
    dq, dk, dv = _like(q), _like(k), _like(v)
    dtable = torch.empty_like(table) if table is not None and want_dtable else None
    if workspace is None:
        workspace = _scratch(B.grf_softmax_attn_workspace_bytes(ctx.handle, s, True), ctx)
    B.grf_softmax_attn_backward(ctx.handle, s, q, k, v, out, lse, rest, dout, dq, dk, dv, dtable, workspace, _bytes(workspace))
    return dq, dk, dv, dtable


def _first_position(ctx, t, n_q, n_k, q_start):
    """Where the queries begin; checked, with the device of t."""
    if not t.is_cuda or t.get_device() != ctx.device:
        raise ValueError(f"expected a tensor on {ctx.torch_device}")
    start = n_k - n_q if q_start is None else q_start
    if n_q > INT32_MAX or n_k > INT32_MAX or not -INT32_MAX - 1 <= start <= INT32_MAX:
        raise ValueError("n_q, n_k and q_start: expected 32-bit integers")
    return start


def relative_bias(ctx: Context, table, first, n_q, n_k, two_sided=False, q_start=None):
    """Rows [H, n_q, n_k] of the learned relative position bias table [H, len(first)] (twice as many columns when two_sided); the
    queries are the last of the n_k tokens unless q_start says where they begin."""
    heads = table.shape[0]
    if tuple(table.shape) != (heads, len(first) * (2 if two_sided else 1)):
        raise ValueError("table: expected one column per bucket and side")
    start = _first_position(ctx, table, n_q, n_k, q_start)
    rows = table.new_empty((heads, n_q, n_k))
    B.grf_relative_bias(ctx.handle, heads, n_q, n_k, start, first, two_sided, B.dtype_code(table), table, rows)
    return rows


def relative_bias_backward(ctx: Context, drows, first, two_sided=False, q_start=None, workspace=None):
    """Gradient [H, columns] of relative_bias's table from drows [B, H, n_q, n_k] (or [H, n_q, n_k]), summed over the batch."""
    if drows.dim() == 3:
        drows = drows[None]
    batch, heads, n_q, n_k = drows.shape
    start = _first_position(ctx, drows, n_q, n_k, q_start)
    dtable = drows.new_empty((heads, len(first) * (2 if two_sided else 1)))
    if workspace is None:
        workspace = _scratch(B.grf_relative_bias_workspace_bytes(heads, n_q, n_k, len(first), two_sided), ctx)
    B.grf_relative_bias_backward(ctx.handle, batch, heads, n_q, n_k, start, first, two_sided, B.dtype_code(drows), drows, dtable, workspace,
                                 _bytes(workspace))
    return dtable
