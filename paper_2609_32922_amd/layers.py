"""Layer operators around the quantised products, on torch device tensors: block-scaled fp8 quantiser and product, the
norms, gate and residual between two branches of a transformer block with their gradients, and rotary positions.

As in the package's other functions torch supplies memory and the stream, and every step runs in the library's kernels.
Tensors may be views: the last dimension has to be contiguous, the others have any stride that does not lie on itself.
``stream`` is a torch.cuda.Stream of the tensors' device (default: the current one).  What is made here comes from that stream's
memory and is marked as used by the current one too; as with any stream, the inputs have to be ready on it and to live until it has
read them.

Nothing here is recorded by autograd.  Where gradients are recorded (torch.is_grad_enabled) and a tensor of a forward call requires
one, the call is refused: call it under torch.no_grad(), and ``residual_norm_backward`` or ``rope(inverse=True)`` for the gradients.
"""
from __future__ import annotations

import ctypes

from ._lib import (SC_BF16, SC_BLOCK_1X128, SC_BLOCK_128X1_T, SC_BLOCK_128X128, SC_E4M3, SC_E5M2, SC_F16, SC_F32, SC_FP8_BLOCK,
                   SC_INT8, SC_NORM_LAYER, SC_NORM_NONE, SC_NORM_RMS, SC_OK, SC_ROPE_HALVES, SC_ROPE_NEIGHBOURS, ScError,
                   ScFp8GemmDesc, ScNormDesc, ScRopeDesc, load, sc_fp8_gemm_workspace_size,
                   sc_residual_norm_backward_workspace_size)

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

# The kernels of a small call take less time than checking its arguments in Python, so what the shapes, strides, types and
# options of a call come to (the checks passed, the filled descriptor, what its results look like) is kept for the next call
# with the same ones.  Nothing of the tensors themselves is.
_PLANS_MOST = 1024
_plans = {}


def _keep(key, plan):
    if len(_plans) >= _PLANS_MOST:
        _plans.clear()
    _plans[key] = plan
    return plan


def _form(t):
    return (t.shape, t.stride(), t.dtype, t.device) if t is not None else None


class _Plan:
    """A checked call: its device, and the library's function with the arguments that do not change."""

    def __init__(self, dev, name):
        if dev.type != "cuda":
            raise ValueError("tensors must be on a GPU")
        self.dev, self.index, self.name = dev, dev.index, name
        self.function = getattr(load(), name)

    def run(self, *args):
        """The call on the current stream of its device."""
        import torch
        if torch._C._cuda_getDevice() == self.index:
            rc = self.function(*args, torch._C._cuda_getCurrentRawStream(self.index))
        else:
            with torch.cuda.device(self.dev):
                rc = self.function(*args, torch._C._cuda_getCurrentRawStream(self.index))
        if rc != SC_OK:
            raise ScError(rc, self.name)


def _on_stream(stream, dev, call):
    """``call()``, which makes tensors and works on the current stream, on ``stream``.

    Memory that the current stream's tensors have left may still be in use by work that waits there, which ``stream`` knows
    nothing of.  So what the call makes has to be the other stream's memory, and is marked as used by the current one, on which its
    user goes on.
    """
    import torch
    if stream.device != dev:
        raise ValueError("stream must be one of %s" % dev)
    now = torch.cuda.current_stream(dev)
    if stream == now:
        return call()
    with torch.cuda.stream(stream):
        got = call()
    for t in got.values() if isinstance(got, dict) else got if isinstance(got, tuple) else (got,):
        if t is not None:
            t.record_stream(now)
    return got


def _workspace(dev, nbytes, given):
    """(address, bytes, what holds it) of a workspace for the current stream; ``given`` is grown where it is too small."""
    import torch
    if given is not None:
        given.ensure(nbytes).use(dev)
        return given.ptr, given.nbytes, given
    buf = torch.empty(nbytes + 256, dtype=torch.uint8, device=dev)
    return (buf.data_ptr() + 255) // 256 * 256, nbytes, buf


def _unrecorded():
    """Of a call where gradients are recorded and a tensor requires one: it would be lost without a word."""
    raise ValueError("a tensor requires a gradient, and autograd does not record this call: call it under torch.no_grad()")


def _written(t):
    """Tells autograd that a caller's tensor has changed, as torch's own writes do."""
    import torch
    if not t.is_inference():
        torch.autograd.graph.increment_version(t)


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


def _ptr(t):
    return t.data_ptr() if t is not None else None


def _quantize_plan(key, X, dtype, block):
    import torch
    p = _Plan(X.device, "sc_fp8_quantize")
    ld, st = _rows(X, "X", p.dev)
    tx, tq = _type(X.dtype, "X", FLOATS), _type(dtype, "dtype", FP8)
    lead, (rows, K) = tuple(X.shape[:-2]), X.shape[-2:]
    kb, rb = -(-K // SC_FP8_BLOCK), -(-rows // SC_FP8_BLOCK)
    turned = block == SC_BLOCK_128X1_T
    qs, ss = ((K, rows), (K, rb)) if turned else ((rows, K), (rb if block == SC_BLOCK_128X128 else rows, kb))
    p.q_shape, p.s_shape, p.f32 = lead + qs, lead + ss, torch.float32
    p.head, p.mid = (lead[0] if lead else 1, rows, K, tx), (ld, st, tq, block)
    p.q_strides, p.s_strides = (qs[1], qs[0] * qs[1]), (ss[1], ss[0] * ss[1])
    return _keep(key, p)


def fp8_quantize(X, *, dtype=None, block: int = SC_BLOCK_1X128, stream=None):
    """8-bit floats of X [rows, K] or [batch, rows, K] (float32, bfloat16, float16) with an fp32 scale for each block.

    ``dtype``: torch.float8_e4m3fn (default) or torch.float8_e5m2.  Returns (Q, scale): SC_BLOCK_1X128 Q like X and
    scale [.., rows, ceil(K/128)]; SC_BLOCK_128X128 scale [.., ceil(rows/128), ceil(K/128)]; SC_BLOCK_128X1_T the
    transpose's rows, Q [.., K, rows] and scale [.., K, ceil(rows/128)].
    """
    import torch
    if stream is not None:
        return _on_stream(stream, X.device, lambda: fp8_quantize(X, dtype=dtype, block=block))
    if torch.is_grad_enabled() and X.requires_grad:
        _unrecorded()
    if dtype is None:
        dtype = torch.float8_e4m3fn
    key = ("quantize", X.shape, X.stride(), X.dtype, X.device, dtype, block)
    p = _plans.get(key) or _quantize_plan(key, X, dtype, block)
    Q, scale = torch.empty(p.q_shape, dtype=dtype, device=p.dev), torch.empty(p.s_shape, dtype=p.f32, device=p.dev)
    p.run(*p.head, X.data_ptr(), *p.mid, Q.data_ptr(), *p.q_strides, scale.data_ptr(), *p.s_strides)
    return Q, scale


def _scale_rows(s, name, dev, rows, kb, lead):
    """Rows that share a scale (1 or 128), row stride and batch stride of a scale tensor."""
    import torch
    if s.dtype != torch.float32:
        raise TypeError("%s must be float32" % name)
    per = 1 if s.dim() >= 2 and s.shape[-2] == rows else SC_FP8_BLOCK
    ld, st = _rows(s, name, dev, lead + (rows if per == 1 else -(-rows // SC_FP8_BLOCK), kb))
    return per, ld, st


def _gemm_plan(key, A, sA, B, sB, bias, out, out_dtype):
    import torch
    p = _Plan(A.device, "sc_fp8_gemm")
    d = ScFp8GemmDesc()
    d.typeA, d.typeB = _type(A.dtype, "A", FP8), _type(B.dtype, "B", FP8)
    d.lda, d.strideA = _rows(A, "A", p.dev)
    lead, (M, K) = tuple(A.shape[:-2]), A.shape[-2:]
    batch = lead[0] if lead else 1
    d.ldb, d.strideB = _rows(B, "B", p.dev)
    N = B.shape[-2]
    leadB = tuple(B.shape[:-2])
    if B.shape[-1] != K or (leadB and leadB[0] not in (1, batch)):
        raise ValueError("A is [batch, M, K], B must be [batch or 1, N, K]")
    kb = -(-K // SC_FP8_BLOCK)
    d.rowsA, d.ldsA, d.strideSA = _scale_rows(sA, "sA", p.dev, M, kb, lead)
    d.rowsB, d.ldsB, d.strideSB = _scale_rows(sB, "sB", p.dev, N, kb, leadB)
    d.batch, d.M, d.N, d.K = batch, M, N, K
    if bias is not None:
        _on(bias, "bias", p.dev)
        if bias.dtype != torch.float32:
            raise TypeError("bias must be float32")
        if tuple(bias.shape) not in ((N,), (batch, N)) or (N > 1 and bias.stride(-1) != 1):
            raise ValueError("bias must be [N] or [batch, N] with a contiguous last dimension")
        d.strideBias = bias.stride(0) if bias.dim() == 2 and batch > 1 else 0
    p.shape, p.dtype = lead + (M, N), torch.bfloat16 if out_dtype is None else out_dtype
    if out is None:
        d.typeO = _type(p.dtype, "out", FLOATS)
        d.ldo, d.strideO = max(N, 1), M * N
    else:
        if out_dtype is not None and out.dtype != out_dtype:
            raise TypeError("out must be %s" % out_dtype)
        d.typeO = _type(out.dtype, "out", FLOATS)
        d.ldo, d.strideO = _rows(out, "out", p.dev, p.shape)
    p.nbytes, p.desc, p.ref = sc_fp8_gemm_workspace_size(d), d, ctypes.byref(d)
    return _keep(key, p)


def fp8_gemm(A, sA, B, sB, *, bias=None, out=None, out_dtype=None, workspace=None, stream=None):
    """out = (sA . A) (sB . B)^T (+ bias) of 8-bit floats with a scale for each block of 128 elements of a row.

    A [M, K] or [batch, M, K], B [N, K] or [batch or 1, N, K] (torch.float8_e4m3fn or float8_e5m2 each); sA float32
    [.., M, ceil(K/128)] or [.., ceil(M/128), ceil(K/128)], sB alike, as ``fp8_quantize`` gives them; bias float32 [N] or
    [batch, N].  ``out_dtype`` (default bfloat16) or ``out`` with rows of any stride.  float32 and float16 results have float32
    products and sums throughout; bfloat16 ones of more than 16 rows take the matrix cores' 8-bit products at twice the rate, which
    may lose up to 7 2^-13 of the sum of the products' magnitudes.  Returns out [.., M, N].
    """
    import torch
    if stream is not None:
        return _on_stream(stream, A.device, lambda: fp8_gemm(A, sA, B, sB, bias=bias, out=out, out_dtype=out_dtype, workspace=workspace))
    if torch.is_grad_enabled() and (A.requires_grad or sA.requires_grad or B.requires_grad or sB.requires_grad or
                                    (bias is not None and bias.requires_grad) or (out is not None and out.requires_grad)):
        _unrecorded()
    key = ("gemm", A.shape, A.stride(), A.dtype, A.device, sA.shape, sA.stride(), sA.dtype, sA.device, B.shape, B.stride(), B.dtype,
           B.device, sB.shape, sB.stride(), sB.dtype, sB.device, out_dtype, _form(bias), _form(out))
    p = _plans.get(key) or _gemm_plan(key, A, sA, B, sB, bias, out, out_dtype)
    given = out is not None
    if not given:
        out = torch.empty(p.shape, dtype=p.dtype, device=p.dev)
    ws = (None, 0, None) if p.nbytes == 0 else _workspace(p.dev, p.nbytes, workspace)
    p.run(p.ref, A.data_ptr(), sA.data_ptr(), B.data_ptr(), sB.data_ptr(), _ptr(bias), out.data_ptr(), ws[0], ws[1])
    if given:
        _written(out)
    return out


_PARAMS = ("post_weight", "post_bias", "gate", "pre_weight", "pre_bias")


def _norm_desc(c, x, y, dtype_h, post, pre, numbers, params):
    d = ScNormDesc()
    d.batch = x.shape[0] if x.dim() == 3 else 1
    d.rows, d.D = x.shape[-2:]
    d.post, d.pre = post, pre
    d.typeX = _type(x.dtype, "x", FLOATS)
    d.typeY = _type(y.dtype, "y", FLOATS) if y is not None else d.typeX
    d.typeH = dtype_h
    d.eps_post, d.eps_pre, d.scale_res, d.off_post, d.off_pre = numbers
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


def _norm_plan(key, x, y, params, post, pre, numbers, out_dtype, want_x, want_h, want_rowmax, inplace):
    import torch
    p = _Plan(x.device, "sc_residual_norm")
    th = _type(out_dtype, "out_dtype", FLOATS + FP8 + (SC_INT8,))
    ldx, sx = _rows(x, "x", p.dev)
    d = _norm_desc(p, x, y, th, post, pre, numbers, params)
    d.ldx, d.strideX = ldx, sx
    if y is not None:
        d.ldy, d.strideY = _rows(y, "y", p.dev, x.shape)
    lead, D = tuple(x.shape[:-1]), d.D
    if inplace and not want_x:
        raise ValueError("inplace writes xo: want_x must be set")
    if want_rowmax and not (want_h and th == SC_INT8):
        raise ValueError("rowmax comes with an int8 h")
    d.ldxo, d.strideXO = (ldx, sx) if inplace else (max(D, 1), d.rows * D)
    d.ldh, d.strideH = max(D, 1), d.rows * D
    d.strideS = d.rows * d.lds if th in FP8 else d.rows
    p.shape, p.h_dtype, p.f32 = tuple(x.shape), out_dtype, torch.float32
    p.s_shape = None if not want_h or th in FLOATS else lead if th == SC_INT8 else lead + (d.lds,)
    p.desc, p.ref = d, ctypes.byref(d)
    return _keep(key, p)


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
    if stream is not None:
        return _on_stream(stream, x.device, lambda: residual_norm(
            x, y, post=post, pre=pre, post_weight=post_weight, post_bias=post_bias, gate=gate, pre_weight=pre_weight, pre_bias=pre_bias,
            res_scale=res_scale, post_offset=post_offset, pre_offset=pre_offset, post_eps=post_eps, pre_eps=pre_eps,
            out_dtype=out_dtype, want_x=want_x, want_h=want_h, want_rowmax=want_rowmax, inplace=inplace))
    if torch.is_grad_enabled() and (
            x.requires_grad or (y is not None and y.requires_grad) or (post_weight is not None and post_weight.requires_grad) or
            (post_bias is not None and post_bias.requires_grad) or (gate is not None and gate.requires_grad) or
            (pre_weight is not None and pre_weight.requires_grad) or (pre_bias is not None and pre_bias.requires_grad)):
        _unrecorded()
    if out_dtype is None:
        out_dtype = x.dtype
    key = ("norm", x.shape, x.stride(), x.dtype, x.device, _form(y), _form(post_weight), _form(post_bias), _form(gate),
           _form(pre_weight), _form(pre_bias), post, pre, res_scale, post_offset, pre_offset, post_eps, pre_eps, out_dtype, want_x,
           want_h, want_rowmax, inplace)
    p = _plans.get(key) or _norm_plan(key, x, y, (post_weight, post_bias, gate, pre_weight, pre_bias), post, pre,
                                      (post_eps, pre_eps, res_scale, post_offset, pre_offset), out_dtype, want_x, want_h,
                                      want_rowmax, inplace)
    dev = p.dev
    xo = None if not want_x else x if inplace else torch.empty(p.shape, dtype=x.dtype, device=dev)
    h = torch.empty(p.shape, dtype=out_dtype, device=dev) if want_h else None
    scale = torch.empty(p.s_shape, dtype=p.f32, device=dev) if p.s_shape is not None else None
    rowmax = torch.empty(p.s_shape, dtype=p.f32, device=dev) if want_rowmax else None
    p.run(p.ref, x.data_ptr(), _ptr(y), _ptr(post_weight), _ptr(post_bias), _ptr(gate), _ptr(pre_weight), _ptr(pre_bias), _ptr(xo),
          _ptr(h), _ptr(scale), _ptr(rowmax))
    if inplace:
        _written(x)
    return xo, h, scale, rowmax


def _backward_plan(key, xo, y, dxo, dh, params, post, pre, numbers, want_x, want_params):
    p = _Plan(xo.device, "sc_residual_norm_backward")
    th = _type(dh.dtype, "dh", FLOATS) if dh is not None else SC_F32
    ldxo, sxo = _rows(xo, "xo", p.dev)
    d = _norm_desc(p, xo, y, th, post, pre, numbers, params)
    D = max(d.D, 1)
    d.ldxo, d.strideXO = ldxo, sxo
    if y is not None:
        d.ldy, d.strideY = _rows(y, "y", p.dev, xo.shape)
    elif post != SC_NORM_NONE or any(q is not None for q in params[:3]):
        raise ValueError("a branch's norm and gate need y")
    if dxo is not None:
        if dxo.dtype != xo.dtype:
            raise TypeError("dxo must have xo's type")
        d.lddxo, d.strideDXO = _rows(dxo, "dxo", p.dev, xo.shape)
    if dh is not None:
        d.ldh, d.strideH = _rows(dh, "dh", p.dev, xo.shape)
    d.ldx = d.lddy = D
    d.strideX = d.strideDY = d.rows * d.D
    p.shape = tuple(xo.shape)
    # the parameters' gradients, made together by their shapes
    p.sums = {}
    if want_params:
        for name, q in zip(_PARAMS, params):
            if q is not None:
                p.sums.setdefault(tuple(q.shape), []).append(name)
    p.nbytes = sc_residual_norm_backward_workspace_size(d) if p.sums else 0
    p.desc, p.ref = d, ctypes.byref(d)
    return _keep(key, p)


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
    if stream is not None:
        return _on_stream(stream, xo.device, lambda: residual_norm_backward(
            xo, y, dxo=dxo, dh=dh, post=post, pre=pre, post_weight=post_weight, post_bias=post_bias, gate=gate, pre_weight=pre_weight,
            pre_bias=pre_bias, res_scale=res_scale, post_offset=post_offset, pre_offset=pre_offset, post_eps=post_eps,
            pre_eps=pre_eps, want_x=want_x, want_params=want_params, workspace=workspace))
    key = ("back", xo.shape, xo.stride(), xo.dtype, xo.device, _form(y), _form(dxo), _form(dh), _form(post_weight), _form(post_bias),
           _form(gate), _form(pre_weight), _form(pre_bias), post, pre, res_scale, post_offset, pre_offset, post_eps, pre_eps, want_x,
           want_params)
    p = _plans.get(key) or _backward_plan(key, xo, y, dxo, dh, (post_weight, post_bias, gate, pre_weight, pre_bias), post, pre,
                                          (post_eps, pre_eps, res_scale, post_offset, pre_offset), want_x, want_params)
    dev = p.dev
    got = {}
    if want_x:
        got["x"] = torch.empty(p.shape, dtype=xo.dtype, device=dev)
    if y is not None:
        got["y"] = torch.empty(p.shape, dtype=y.dtype, device=dev)
    for shape, names in p.sums.items():
        got.update(zip(names, torch.empty((len(names),) + shape, dtype=torch.float32, device=dev).unbind(0)))
    ws = (None, 0, None) if p.nbytes == 0 else _workspace(dev, p.nbytes, workspace)
    g = got.get
    p.run(p.ref, xo.data_ptr(), _ptr(y), _ptr(post_weight), _ptr(post_bias), _ptr(gate), _ptr(pre_weight), _ptr(dxo), _ptr(dh),
          _ptr(g("x")), _ptr(g("y")), _ptr(g("post_weight")), _ptr(g("post_bias")), _ptr(g("gate")), _ptr(g("pre_weight")),
          _ptr(g("pre_bias")), ws[0], ws[1])
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


def _rope_plan(key, x, pos, freq, axis, interleaved, inverse, out, out_dtype, quantised):
    import torch
    p = _Plan(x.device, "sc_rope")
    d = ScRopeDesc()
    d.strideXB, d.strideXT, d.strideXH = _heads(x, "x", p.dev)
    d.batch = x.shape[0] if x.dim() == 4 else 1
    d.tokens, d.heads, d.D = x.shape[-3:]
    d.typeX = _type(x.dtype, "x", FLOATS)
    for t, name, dtype in ((pos, "pos", torch.int32), (freq, "freq", torch.float64), (axis, "axis", torch.int32)):
        _on(t, name, p.dev)
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
    H, T, D = d.heads, d.tokens, d.D
    if quantised:
        p.shape, p.s_shape = tuple(x.shape[:-3]) + (H, T, D), tuple(x.shape[:-3]) + (H, T)
        d.typeO = SC_INT8
        d.strideOB, d.strideOT, d.strideOH = H * T * D, D, T * D
        d.strideSB, d.strideST, d.strideSH = H * T, 1, T
    elif out is None:
        p.shape, p.dtype = tuple(x.shape), x.dtype if out_dtype is None else out_dtype
        d.typeO = _type(p.dtype, "out", FLOATS)
        d.strideOB, d.strideOT, d.strideOH = T * H * D, H * D, D
    else:
        if tuple(out.shape) != tuple(x.shape) or (out_dtype is not None and out.dtype != out_dtype):
            raise ValueError("out must be like x, of out_dtype")
        d.typeO = _type(out.dtype, "out", FLOATS)
        d.strideOB, d.strideOT, d.strideOH = _heads(out, "out", p.dev)
    p.desc, p.ref = d, ctypes.byref(d)
    return _keep(key, p)


def rope(x, pos, freq, axis, *, interleaved: bool = False, inverse: bool = False, out=None, out_dtype=None, stream=None):
    """Rotary positions with several axes: pair p of a token turns by pos[axis[p]] freq[p].

    x [tokens, heads, D] or [batch, tokens, heads, D] (float32, bfloat16, float16; a view of joined queries, keys and values
    will do), pos int32 [axes, tokens] or [batch, axes, tokens], freq float64 and axis int32 [pairs] (``rope_table``).
    Pairs are elements (p, pairs + p), or (2p, 2p + 1) where ``interleaved``; elements behind them pass.  ``inverse`` turns
    back: the gradient of x from that of the result.  ``out`` may be x itself.  Returns out, like x.
    """
    import torch
    if stream is not None:
        return _on_stream(stream, x.device, lambda: rope(x, pos, freq, axis, interleaved=interleaved, inverse=inverse, out=out,
                                                         out_dtype=out_dtype))
    if torch.is_grad_enabled() and (x.requires_grad or freq.requires_grad or (out is not None and out.requires_grad)):
        _unrecorded()
    key = ("rope", x.shape, x.stride(), x.dtype, x.device, pos.shape, pos.stride(), pos.dtype, pos.device, freq.shape, freq.dtype,
           freq.device, axis.shape, axis.dtype, axis.device, freq.stride(), axis.stride(), interleaved, inverse, out_dtype, _form(out))
    p = _plans.get(key) or _rope_plan(key, x, pos, freq, axis, interleaved, inverse, out, out_dtype, False)
    given = out is not None
    if not given:
        out = torch.empty(p.shape, dtype=p.dtype, device=p.dev)
    p.run(p.ref, x.data_ptr(), pos.data_ptr(), freq.data_ptr(), axis.data_ptr(), out.data_ptr(), None, None)
    if given:
        _written(out)
    return out


def rope_quantize(x, pos, freq, axis, *, interleaved: bool = False, want_rowmax: bool = False, stream=None):
    """``rope`` with its result as int8 rows by head, the operands of ``gemm`` for attention scores.

    Returns (Q int8 [.., heads, tokens, D], scale float32 [.., heads, tokens], rowmax alike or None).
    """
    import torch
    if stream is not None:
        return _on_stream(stream, x.device, lambda: rope_quantize(x, pos, freq, axis, interleaved=interleaved, want_rowmax=want_rowmax))
    if torch.is_grad_enabled() and (x.requires_grad or freq.requires_grad):
        _unrecorded()
    key = ("rope int8", x.shape, x.stride(), x.dtype, x.device, pos.shape, pos.stride(), pos.dtype, pos.device, freq.shape, freq.dtype,
           freq.device, axis.shape, axis.dtype, axis.device, freq.stride(), axis.stride(), interleaved)
    p = _plans.get(key) or _rope_plan(key, x, pos, freq, axis, interleaved, False, None, None, True)
    Q = torch.empty(p.shape, dtype=torch.int8, device=p.dev)
    scale = torch.empty(p.s_shape, dtype=torch.float32, device=p.dev)
    rowmax = torch.empty(p.s_shape, dtype=torch.float32, device=p.dev) if want_rowmax else None
    p.run(p.ref, x.data_ptr(), pos.data_ptr(), freq.data_ptr(), axis.data_ptr(), Q.data_ptr(), scale.data_ptr(), _ptr(rowmax))
    return Q, scale, rowmax
