"""Layer operators around the quantised products, on torch device tensors: block-scaled fp8 quantiser and product, the
norms, gate and residual between two branches of a transformer block with their gradients, and rotary positions.

As in the package's other functions torch supplies memory and the stream, and every step runs in the library's kernels.
Tensors may be views: the last dimension has to be contiguous, the others have any stride that does not lie on itself.
``stream`` is a torch.cuda.Stream (default: the current one of the tensors' device); tensors made here are marked as used
by it when it is another.
"""
from __future__ import annotations

from ._lib import (SC_BF16, SC_BLOCK_1X128, SC_BLOCK_128X1_T, SC_BLOCK_128X128, SC_E4M3, SC_E5M2, SC_F16, SC_F32, SC_FP8_BLOCK,
                   SC_INT8, SC_NORM_LAYER, SC_NORM_NONE, SC_NORM_RMS, SC_OK, SC_ROPE_HALVES, SC_ROPE_NEIGHBOURS, ScError,
                   ScFp8GemmDesc, ScNormDesc, ScRopeDesc, sc_fp8_gemm, sc_fp8_gemm_workspace_size, sc_fp8_quantize,
                   sc_residual_norm, sc_residual_norm_backward, sc_residual_norm_backward_workspace_size, sc_rope)

_types = {}


def _type(t, name, allowed):
    """The library's number of a tensor's (or a) dtype, which has to be one of ``allowed``."""
    if not _types:
        import torch
        _types.update({torch.float32: SC_F32, torch.bfloat16: SC_BF16, torch.float16: SC_F16, torch.float8_e4m3fn: SC_E4M3,
                       torch.float8_e5m2: SC_E5M2, torch.int8: SC_INT8})
    n = _types.get(t)
    if n not in allowed:
        raise TypeError("%s: %s is not served" % (name, t))
    return n


FLOATS, FP8 = (SC_F32, SC_BF16, SC_F16), (SC_E4M3, SC_E5M2)


def _on(t, name, dev):
    if not t.is_cuda or t.device != dev:
        raise ValueError("%s must be on %s" % (name, dev))


def _rows(t, name, dev, shape=None):
    """(row stride, batch stride) of [rows, n] or [batch, rows, n] with a contiguous last dimension."""
    _on(t, name, dev)
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    if t.dim() not in (2, 3):
        raise ValueError("%s must be [rows, n] or [batch, rows, n]" % name)
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError("%s: the last dimension must be contiguous" % name)
    # (a stride of a dimension with one entry says nothing, and torch gives any)
    ld = t.stride(-2) if t.shape[-2] > 1 else max(t.shape[-1], 1)
    return ld, t.stride(0) if t.dim() == 3 and t.shape[0] > 1 else 0


class _Call:
    """Device, stream and outputs of one call."""

    def __init__(self, dev, stream):
        import torch
        if dev.type != "cuda":
            raise ValueError("tensors must be on a GPU")
        self.dev, self.stream, self.torch = dev, stream, torch
        self.foreign = stream is not None and stream != torch.cuda.current_stream(dev)
        self.handle = int(stream.cuda_stream) if stream is not None else torch._C._cuda_getCurrentRawStream(dev.index)

    def empty(self, shape, dtype):
        t = self.torch.empty(shape, dtype=dtype, device=self.dev)
        if self.foreign:
            t.record_stream(self.stream)
        return t

    def workspace(self, nbytes, given=None):
        """(address, bytes) of a workspace; ``given`` is grown where it is too small."""
        if nbytes == 0:
            return 0, 0
        if given is None:
            from . import Workspace
            given = Workspace(nbytes, self.dev)
        else:
            given.ensure(nbytes)
        if self.foreign:
            given._buf.record_stream(self.stream)
        return given.ptr, given.nbytes

    def run(self, function, name, *args):
        cuda = self.torch.cuda
        if self.dev.index != cuda.current_device():
            with cuda.device(self.dev):
                rc = function(*args, self.handle)
        else:
            rc = function(*args, self.handle)
        if rc != SC_OK:
            raise ScError(rc, name)


def _ptr(t):
    return t.data_ptr() if t is not None else 0


def fp8_quantize(X, *, dtype=None, block: int = SC_BLOCK_1X128, stream=None):
    """8-bit floats of X [rows, K] or [batch, rows, K] (float32, bfloat16, float16) with an fp32 scale for each block.

    ``dtype``: torch.float8_e4m3fn (default) or torch.float8_e5m2.  Returns (Q, scale): SC_BLOCK_1X128 Q like X and
    scale [.., rows, ceil(K/128)]; SC_BLOCK_128X128 scale [.., ceil(rows/128), ceil(K/128)]; SC_BLOCK_128X1_T the
    transpose's rows, Q [.., K, rows] and scale [.., K, ceil(rows/128)].
    """
    import torch
    dtype = torch.float8_e4m3fn if dtype is None else dtype
    c = _Call(X.device, stream)
    ld, st = _rows(X, "X", c.dev)
    tx, tq = _type(X.dtype, "X", FLOATS), _type(dtype, "dtype", FP8)
    lead, (rows, K) = tuple(X.shape[:-2]), X.shape[-2:]
    batch = lead[0] if lead else 1
    kb, rb = -(-K // SC_FP8_BLOCK), -(-rows // SC_FP8_BLOCK)
    turned = block == SC_BLOCK_128X1_T
    qs, ss = ((K, rows), (K, rb)) if turned else ((rows, K), (rb if block == SC_BLOCK_128X128 else rows, kb))
    Q, scale = c.empty(lead + qs, dtype), c.empty(lead + ss, torch.float32)
    c.run(sc_fp8_quantize, "sc_fp8_quantize", batch, rows, K, tx, X.data_ptr(), ld, st, tq, block, Q.data_ptr(), qs[1],
          qs[0] * qs[1], scale.data_ptr(), ss[1], ss[0] * ss[1])
    return Q, scale


def _scale_rows(s, name, dev, rows, kb, lead):
    """Rows that share a scale (1 or 128), row stride and batch stride of a scale tensor."""
    import torch
    if s.dtype != torch.float32:
        raise TypeError("%s must be float32" % name)
    per = 1 if s.dim() >= 2 and s.shape[-2] == rows else SC_FP8_BLOCK
    ld, st = _rows(s, name, dev, lead + (rows if per == 1 else -(-rows // SC_FP8_BLOCK), kb))
    return per, ld, st


def fp8_gemm(A, sA, B, sB, *, bias=None, out=None, out_dtype=None, workspace=None, stream=None):
    """out = (sA . A) (sB . B)^T (+ bias) of 8-bit floats with a scale for each block of 128 elements of a row.

    A [M, K] or [batch, M, K], B [N, K] or [batch or 1, N, K] (torch.float8_e4m3fn or float8_e5m2 each); sA float32
    [.., M, ceil(K/128)] or [.., ceil(M/128), ceil(K/128)], sB alike, as ``fp8_quantize`` gives them; bias float32 [N] or
    [batch, N].  ``out_dtype`` (default bfloat16) or ``out`` with rows of any stride.  Returns out [.., M, N].
    """
    import torch
    c = _Call(A.device, stream)
    d = ScFp8GemmDesc()
    d.typeA, d.typeB = _type(A.dtype, "A", FP8), _type(B.dtype, "B", FP8)
    d.lda, d.strideA = _rows(A, "A", c.dev)
    lead, (M, K) = tuple(A.shape[:-2]), A.shape[-2:]
    batch = lead[0] if lead else 1
    d.ldb, d.strideB = _rows(B, "B", c.dev)
    N = B.shape[-2]
    leadB = tuple(B.shape[:-2])
    if B.shape[-1] != K or (leadB and leadB[0] not in (1, batch)):
        raise ValueError("A is [batch, M, K], B must be [batch or 1, N, K]")
    kb = -(-K // SC_FP8_BLOCK)
    d.rowsA, d.ldsA, d.strideSA = _scale_rows(sA, "sA", c.dev, M, kb, lead)
    d.rowsB, d.ldsB, d.strideSB = _scale_rows(sB, "sB", c.dev, N, kb, leadB)
    d.batch, d.M, d.N, d.K = batch, M, N, K
    if bias is not None:
        _on(bias, "bias", c.dev)
        if bias.dtype != torch.float32:
            raise TypeError("bias must be float32")
        if tuple(bias.shape) not in ((N,), (batch, N)) or (N > 1 and bias.stride(-1) != 1):
            raise ValueError("bias must be [N] or [batch, N] with a contiguous last dimension")
        d.strideBias = bias.stride(0) if bias.dim() == 2 and batch > 1 else 0
    if out is None:
        out = c.empty(lead + (M, N), torch.bfloat16 if out_dtype is None else out_dtype)
    elif out_dtype is not None and out.dtype != out_dtype:
        raise TypeError("out must be %s" % out_dtype)
    d.typeO = _type(out.dtype, "out", FLOATS)
    d.ldo, d.strideO = _rows(out, "out", c.dev, lead + (M, N))
    ws, nbytes = c.workspace(sc_fp8_gemm_workspace_size(d), workspace)
    c.run(sc_fp8_gemm, "sc_fp8_gemm", d, A.data_ptr(), sA.data_ptr(), B.data_ptr(), sB.data_ptr(), _ptr(bias), out.data_ptr(),
          ws, nbytes)
    return out


_PARAMS = ("post_weight", "post_bias", "gate", "pre_weight", "pre_bias")


def _norm_desc(c, x, y, dtype_h, post, pre, post_eps, pre_eps, res_scale, post_offset, pre_offset, params):
    d = ScNormDesc()
    d.batch = x.shape[0] if x.dim() == 3 else 1
    d.rows, d.D = x.shape[-2:]
    d.post, d.pre = post, pre
    d.typeX = _type(x.dtype, "x", FLOATS)
    d.typeY = _type(y.dtype, "y", FLOATS) if y is not None else d.typeX
    d.typeH = dtype_h
    d.eps_post, d.eps_pre, d.scale_res, d.off_post, d.off_pre = post_eps, pre_eps, res_scale, post_offset, pre_offset
    D, batch = d.D, d.batch
    d.ldx = d.ldy = d.ldxo = d.ldh = max(D, 1)
    d.lds = -(-D // SC_FP8_BLOCK)
    kind = None
    for name, p, field in zip(_PARAMS, params, ("stride_post_w", "stride_post_b", "stride_gate", "stride_pre_w", "stride_pre_b")):
        if p is None:
            continue
        _on(p, name, c.dev)
        if kind is not None and p.dtype != kind:
            raise TypeError("the parameters must have one type")
        kind = p.dtype
        if tuple(p.shape) not in ((D,), (1, D), (batch, D)) or (D > 1 and p.stride(-1) != 1):
            raise ValueError("%s must be [D], [1, D] or [batch, D] with a contiguous last dimension" % name)
        if p.dim() == 2 and p.shape[0] > 1:
            if p.stride(0) == 0:
                raise ValueError("%s: pass a shared parameter as [D]" % name)
            setattr(d, field, p.stride(0))
    d.typeP = _type(kind, "parameters", FLOATS) if kind is not None else SC_F32
    return d


def residual_norm(x, y=None, *, post: int = SC_NORM_NONE, pre: int = SC_NORM_LAYER, post_weight=None, post_bias=None,
                  gate=None, pre_weight=None, pre_bias=None, res_scale: float = 1.0, post_offset: float = 0.0,
                  pre_offset: float = 0.0, post_eps: float = 1e-6, pre_eps: float = 1e-6, out_dtype=None, want_x: bool = True,
                  want_h: bool = True, want_rowmax: bool = False, inplace: bool = False, stream=None):
    """The seam between two branches of a transformer block: xo = res_scale x + gate u with u = n_post(y) (post_offset +
    post_weight) + post_bias, and h = n_pre(xo) (pre_offset + pre_weight) + pre_bias.

    x, y [rows, D] or [batch, rows, D] (float32, bfloat16, float16); parameters of one type, each [D] (or [1, D]) or a row
    for each batch entry [batch, D]; ``post``, ``pre``: SC_NORM_NONE, SC_NORM_RMS or SC_NORM_LAYER.  ``out_dtype`` of h: a float
    type (default x's), torch.int8 (rows with a scale, operands of ``gemm``) or torch.float8_e4m3fn / float8_e5m2 (blocks of
    128, operands of ``fp8_gemm``).  ``inplace`` writes xo over x.  Returns (xo, h, scale, rowmax), None for what is not
    there.
    """
    import torch
    c = _Call(x.device, stream)
    out_dtype = x.dtype if out_dtype is None else out_dtype
    th = _type(out_dtype, "out_dtype", FLOATS + FP8 + (SC_INT8,))
    params = (post_weight, post_bias, gate, pre_weight, pre_bias)
    ldx, sx = _rows(x, "x", c.dev)
    d = _norm_desc(c, x, y, th, post, pre, post_eps, pre_eps, res_scale, post_offset, pre_offset, params)
    d.ldx, d.strideX = ldx, sx
    if y is not None:
        d.ldy, d.strideY = _rows(y, "y", c.dev, x.shape)
    lead, D = tuple(x.shape[:-1]), d.D
    xo = None
    if want_x:
        xo = x if inplace else c.empty(lead + (D,), x.dtype)
        d.ldxo, d.strideXO = _rows(xo, "xo", c.dev)
    elif inplace:
        raise ValueError("inplace writes xo: want_x must be set")
    h = scale = rowmax = None
    if want_h:
        h = c.empty(lead + (D,), out_dtype)
        d.ldh, d.strideH = _rows(h, "h", c.dev)
        if th == SC_INT8:
            scale, d.strideS = c.empty(lead, torch.float32), d.rows
            rowmax = c.empty(lead, torch.float32) if want_rowmax else None
        elif th in FP8:
            scale, d.strideS = c.empty(lead + (d.lds,), torch.float32), d.rows * d.lds
    if want_rowmax and rowmax is None:
        raise ValueError("rowmax comes with an int8 h")
    c.run(sc_residual_norm, "sc_residual_norm", d, x.data_ptr(), _ptr(y), *(_ptr(p) for p in params), _ptr(xo), _ptr(h),
          _ptr(scale), _ptr(rowmax))
    return xo, h, scale, rowmax


def residual_norm_backward(xo, y=None, *, dxo=None, dh=None, post: int = SC_NORM_NONE, pre: int = SC_NORM_LAYER,
                           post_weight=None, post_bias=None, gate=None, pre_weight=None, pre_bias=None,
                           res_scale: float = 1.0, post_offset: float = 0.0, pre_offset: float = 0.0,
                           post_eps: float = 1e-6, pre_eps: float = 1e-6, want_x: bool = True, want_params: bool = True,
                           workspace=None, stream=None):
    """Gradients of ``residual_norm`` from those of its outputs: ``dxo`` [.., D] of x's type and ``dh`` [.., D] of a float type
    (None = zero), at the stored xo and the branch y.  The other arguments are the forward pass's.

    Returns a dict: "x" and "y" with the types of xo and y, and, for each parameter given, its gradient in float32 with
    the parameter's shape (summed over the rows, and over the batch where it is shared).
    """
    import torch
    c = _Call(xo.device, stream)
    params = (post_weight, post_bias, gate, pre_weight, pre_bias)
    th = _type(dh.dtype, "dh", FLOATS) if dh is not None else SC_F32
    ldxo, sxo = _rows(xo, "xo", c.dev)
    d = _norm_desc(c, xo, y, th, post, pre, post_eps, pre_eps, res_scale, post_offset, pre_offset, params)
    d.ldxo, d.strideXO = ldxo, sxo
    if y is not None:
        d.ldy, d.strideY = _rows(y, "y", c.dev, xo.shape)
    elif post != SC_NORM_NONE or any(p is not None for p in params[:3]):
        raise ValueError("a branch's norm and gate need y")
    if dxo is not None:
        if dxo.dtype != xo.dtype:
            raise TypeError("dxo must have xo's type")
        d.lddxo, d.strideDXO = _rows(dxo, "dxo", c.dev, xo.shape)
    if dh is not None:
        d.ldh, d.strideH = _rows(dh, "dh", c.dev, xo.shape)
    got = {}
    dx = dy = None
    if want_x:
        dx = got["x"] = c.empty(tuple(xo.shape), xo.dtype)
        d.ldx, d.strideX = _rows(dx, "dx", c.dev)
    if y is not None:
        dy = got["y"] = c.empty(tuple(y.shape), y.dtype)
        d.lddy, d.strideDY = _rows(dy, "dy", c.dev)
    sums = []
    for name, p in zip(_PARAMS, params):
        g = None
        if p is not None and want_params:
            g = got[name] = c.empty(tuple(p.shape), torch.float32)
        sums.append(g)
    ws, nbytes = c.workspace(sc_residual_norm_backward_workspace_size(d) if any(g is not None for g in sums) else 0, workspace)
    c.run(sc_residual_norm_backward, "sc_residual_norm_backward", d, xo.data_ptr(), _ptr(y), *(_ptr(p) for p in params[:4]),
          _ptr(dxo), _ptr(dh), _ptr(dx), _ptr(dy), *(_ptr(g) for g in sums), ws, nbytes)
    return got


def rope_table(dims, base: float = 10000.0, shared: bool = False, device="cuda"):
    """(freq float64, axis int32) of ``rope`` for axes with ``dims`` elements each (even numbers).

    ``shared`` false: every axis has a ladder of its own, base^(-2j/d) for pair j of its d elements; true: one ladder over all
    pairs, base^(-2p/sum(dims)), whose sections turn with one axis each.
    """
    import torch
    if any(d < 0 or d % 2 for d in dims):
        raise ValueError("dims must be even")
    total = sum(dims)
    freq, axis = [], []
    for a, d in enumerate(dims):
        for j in range(d // 2):
            freq.append(base ** (-2.0 * len(freq) / total) if shared else base ** (-2.0 * j / d))
            axis.append(a)
    return torch.tensor(freq, dtype=torch.float64, device=device), torch.tensor(axis, dtype=torch.int32, device=device)


def _heads(t, name, dev):
    """[batch, tokens, heads, D] strides of [tokens, heads, D] or [batch, tokens, heads, D]."""
    _on(t, name, dev)
    if t.dim() not in (3, 4):
        raise ValueError("%s must be [tokens, heads, D] or [batch, tokens, heads, D]" % name)
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError("%s: the last dimension must be contiguous" % name)
    return (t.stride(0) if t.dim() == 4 else 0), t.stride(-3), t.stride(-2)


def _rope(c, x, pos, freq, axis, interleaved, inverse):
    import torch
    d = ScRopeDesc()
    d.strideXB, d.strideXT, d.strideXH = _heads(x, "x", c.dev)
    d.batch = x.shape[0] if x.dim() == 4 else 1
    d.tokens, d.heads, d.D = x.shape[-3:]
    d.typeX = _type(x.dtype, "x", FLOATS)
    for t, name, dtype in ((pos, "pos", torch.int32), (freq, "freq", torch.float64), (axis, "axis", torch.int32)):
        _on(t, name, c.dev)
        if t.dtype != dtype:
            raise TypeError("%s must be %s" % (name, dtype))
    if freq.dim() != 1 or axis.shape != freq.shape or not freq.is_contiguous() or not axis.is_contiguous():
        raise ValueError("freq and axis must be contiguous [pairs]")
    lead = tuple(pos.shape[:-2])
    if pos.dim() not in (2, 3) or pos.shape[-1] != d.tokens or (lead and lead[0] not in (1, d.batch)) or \
            (d.tokens > 1 and pos.stride(-1) != 1):
        raise ValueError("pos must be [axes, tokens] or [batch, axes, tokens] with a contiguous last dimension")
    d.pairs, d.axes = freq.shape[0], pos.shape[-2]
    d.stridePB = pos.stride(0) if lead and lead[0] > 1 else 0
    d.stridePA = pos.stride(-2)
    d.pairing = SC_ROPE_NEIGHBOURS if interleaved else SC_ROPE_HALVES
    d.inverse = 1 if inverse else 0
    return d


def rope(x, pos, freq, axis, *, interleaved: bool = False, inverse: bool = False, out=None, out_dtype=None, stream=None):
    """Rotary positions with several axes: pair p of a token turns by pos[axis[p]] freq[p].

    x [tokens, heads, D] or [batch, tokens, heads, D] (float32, bfloat16, float16; a view of joined queries, keys and values
    will do), pos int32 [axes, tokens] or [batch, axes, tokens], freq float64 and axis int32 [pairs] (``rope_table``).
    Pairs are elements (p, pairs + p), or (2p, 2p + 1) where ``interleaved``; elements behind them pass.  ``inverse`` turns
    back: the gradient of x from that of the result.  ``out`` may be x itself.  Returns out, like x.
    """
    c = _Call(x.device, stream)
    d = _rope(c, x, pos, freq, axis, interleaved, inverse)
    if out is None:
        out = c.empty(tuple(x.shape), x.dtype if out_dtype is None else out_dtype)
    elif tuple(out.shape) != tuple(x.shape) or (out_dtype is not None and out.dtype != out_dtype):
        raise ValueError("out must be like x, of out_dtype")
    d.typeO = _type(out.dtype, "out", FLOATS)
    d.strideOB, d.strideOT, d.strideOH = _heads(out, "out", c.dev)
    c.run(sc_rope, "sc_rope", d, x.data_ptr(), pos.data_ptr(), freq.data_ptr(), axis.data_ptr(), out.data_ptr(), 0, 0)
    return out


def rope_quantize(x, pos, freq, axis, *, interleaved: bool = False, want_rowmax: bool = False, stream=None):
    """``rope`` with its result as int8 rows by head, the operands of ``gemm`` for attention scores.

    Returns (Q int8 [.., heads, tokens, D], scale float32 [.., heads, tokens], rowmax alike or None).
    """
    import torch
    c = _Call(x.device, stream)
    d = _rope(c, x, pos, freq, axis, interleaved, False)
    lead = tuple(x.shape[:-3])
    H, T, D = d.heads, d.tokens, d.D
    Q = c.empty(lead + (H, T, D), torch.int8)
    scale = c.empty(lead + (H, T), torch.float32)
    rowmax = c.empty(lead + (H, T), torch.float32) if want_rowmax else None
    d.typeO = SC_INT8
    d.strideOB, d.strideOT, d.strideOH = H * T * D, D, T * D
    d.strideSB, d.strideST, d.strideSH = H * T, 1, T
    c.run(sc_rope, "sc_rope", d, x.data_ptr(), pos.data_ptr(), freq.data_ptr(), axis.data_ptr(), Q.data_ptr(),
          scale.data_ptr(), _ptr(rowmax))
    return Q, scale, rowmax
