"""The layer operators in 64 bits, from their definitions, for the tests (plain torch on the CPU or the GPU)."""
import math

import torch

U = 2.0 ** -24                     # half a step of float32, relative
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11,
        torch.float8_e4m3fn: 2.0 ** -4, torch.float8_e5m2: 2.0 ** -3}
LEAST = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25,   # half the least step
         torch.float8_e4m3fn: 2.0 ** -10, torch.float8_e5m2: 2.0 ** -17}
TOP = {torch.float8_e4m3fn: 448.0, torch.float8_e5m2: 57344.0}


def fp8_quantize32(x, dtype, block_rows):
    """The quantiser's formula in float32, step by step as the header has it; bit for bit what the library gives."""
    x = x.float()
    rows, K = x.shape[-2:]
    rb, kb = -(-rows // block_rows), -(-K // 128)
    full = torch.zeros((*x.shape[:-2], rb * block_rows, kb * 128), dtype=torch.float32, device=x.device)
    full[..., :rows, :K] = x
    b = full.reshape(*x.shape[:-2], rb, block_rows, kb, 128)
    m = torch.nan_to_num(b.abs(), nan=0.0, posinf=math.inf).amax(dim=(-3, -1))
    top = torch.full_like(m, TOP[dtype])
    s = torch.where(m > 0, torch.maximum(m / top, torch.full_like(m, 2.0 ** -126)), torch.zeros_like(m))
    inv = torch.where(m > 0, torch.ones_like(m) / s, torch.zeros_like(m))
    y = b * inv[..., :, None, :, None]
    y = torch.where(torch.isnan(y), y, y.clamp(-TOP[dtype], TOP[dtype]))
    y = y.reshape(*x.shape[:-2], rb * block_rows, kb * 128)[..., :rows, :K]
    return y.to(dtype), s


def wide(s, per, rows, K):
    return s.double().repeat_interleave(128, -1)[..., :K].repeat_interleave(per, -2)[..., :rows, :]


def fp8_gemm(A, sA, perA, B, sB, perB, bias=None):
    """(product, sum of the terms' magnitudes) in float64"""
    M, K = A.shape[-2:]
    N = B.shape[-2]
    a = A.float().double() * wide(sA, perA, M, K)
    b = B.float().double() * wide(sB, perB, N, K)
    o = torch.matmul(a, b.transpose(-1, -2).contiguous())
    mag = torch.matmul(a.abs(), b.abs().transpose(-1, -2).contiguous())
    if bias is not None:
        t = bias.double() if bias.dim() == 1 else bias.double()[:, None, :]
        o, mag = o + t, mag + t.abs()
    return o, mag


def gemm_tolerance(mag, K, dtype, out):
    """Sums of 128 products and then of the blocks, in any order, and two scales: each of the 128 + blocks + 4 roundings is off
    by at most one step of the sum of magnitudes (the matrix cores need not round to nearest), then the result's rounding.
    16-bit results: of each eight products the seven smaller ones may also lose up to 2^-13 of the largest one's power of
    two, which is at most the sum of the eight magnitudes."""
    eights = 0.0 if dtype == torch.float32 else 7 * 2.0 ** -13
    return (eights + (128 + -(-K // 128) + 4) * 2 * U) * mag + HALF[dtype] * out.abs() + LEAST[dtype]


def gemm_norm_ratio(got, ref):
    """Error of a 16-bit result over that of the 64-bit one rounded to its type, in the 2-norm.  What eight products lose has
    no more than a twentieth of a bfloat16 rounding's norm and a third of a float16 one's, so by squares the ratio is at
    most 1.01 and 1.06 where there are enough values to average over."""
    near = ref.to(got.dtype).double()
    return float((got.double() - ref).norm() / (near - ref).norm())


def row(p, x):
    """A parameter [D], [1, D] or [batch, D] against [.., rows, D]."""
    return p.double() if p.dim() == 1 else p.double()[:, None, :] if x.dim() == 3 else p.double()


def normal(v, kind, eps):
    if kind == 0:
        return v
    if kind == 2:
        v = v - v.mean(-1, keepdim=True)
    return v / torch.sqrt((v * v).mean(-1, keepdim=True) + eps)


def residual_norm(x, y, p, post, pre, *, res_scale=1.0, post_offset=0.0, pre_offset=0.0, post_eps=1e-6, pre_eps=1e-6):
    xo = res_scale * x
    if y is not None:
        u = normal(y, post, post_eps)
        if "post_weight" in p:
            u = u * (post_offset + row(p["post_weight"], x))
        if "post_bias" in p:
            u = u + row(p["post_bias"], x)
        xo = xo + (u * row(p["gate"], x) if "gate" in p else u)
    h = normal(xo, pre, pre_eps)
    if "pre_weight" in p:
        h = h * (pre_offset + row(p["pre_weight"], x))
    if "pre_bias" in p:
        h = h + row(p["pre_bias"], x)
    return xo, h


# Roundings of one normalised element: sums over a row run through at most 20 values a thread, 6 steps across lanes and
# 16 across waves, and the mean, the deviation, the weight and the bias add a dozen more.
DEPTH = 64


def norm_error(v, err, kind, eps):
    """Bound of a float32 norm's error where its input is off by at most err: (bound, normalised row, 1 / deviation)."""
    n = normal(v, kind, eps)
    if kind == 0:
        return err, n, torch.ones_like(v[..., :1])
    c = v - v.mean(-1, keepdim=True) if kind == 2 else v
    r = 1.0 / torch.sqrt((c * c).mean(-1, keepdim=True) + eps)
    lost = err + DEPTH * U * (c.abs() + v.abs().mean(-1, keepdim=True))      # of a centred element
    # the deviation's own error: its squares' mean moves by at most 2 rms(c) rms(lost) (+ roundings)
    return r * lost + n.abs() * (DEPTH * U + r * torch.sqrt((lost * lost).mean(-1, keepdim=True))), n, r


def residual_norm_error(x, y, p, post, pre, *, res_scale=1.0, post_offset=0.0, pre_offset=0.0, post_eps=1e-6, pre_eps=1e-6):
    """Bounds of (xo, h) before their last rounding."""
    zero = torch.zeros_like(x)
    e_u = zero
    xo = res_scale * x
    mag = xo.abs()
    if y is not None:
        e_n, n, _ = norm_error(y, zero, post, post_eps)
        w = post_offset + row(p["post_weight"], x) if "post_weight" in p else torch.ones_like(x)
        b = row(p["post_bias"], x) if "post_bias" in p else zero
        g = row(p["gate"], x) if "gate" in p else torch.ones_like(x)
        u = n * w + b
        e_u = (e_n * w.abs() + 4 * U * ((n * w).abs() + b.abs())) * g.abs()
        xo, mag = xo + u * g, mag + (u * g).abs()
    e_x = e_u + 4 * U * mag
    e_n, n, _ = norm_error(xo, e_x, pre, pre_eps)
    w = pre_offset + row(p["pre_weight"], x) if "pre_weight" in p else torch.ones_like(x)
    b = row(p["pre_bias"], x) if "pre_bias" in p else zero
    return e_x, e_n * w.abs() + 4 * U * ((n * w).abs() + b.abs())


def rope(x, pos, freq, axis, interleaved, inverse):
    """x [batch, tokens, heads, D], pos [batch or 1, axes, tokens]"""
    P = freq.numel()
    out = x.double().clone()
    ok = (axis >= 0) & (axis < pos.shape[1])
    a = pos.double()[:, axis.clamp(0, pos.shape[1] - 1).long(), :] * (freq * ok)[None, :, None]
    a = a.transpose(1, 2)[:, :, None, :]
    c, s = torch.cos(a), torch.sin(a) * (-1.0 if inverse else 1.0)
    i, j = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if interleaved else (slice(0, P), slice(P, 2 * P))
    u, v = x.double()[..., i], x.double()[..., j]
    out[..., i], out[..., j] = u * c - v * s, u * s + v * c
    mag = x.double().abs().clone()
    mag[..., i] = mag[..., j] = u.abs() + v.abs()
    return out, mag
