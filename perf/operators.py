"""Timing cases of the layer operators around the quantised products, through the package's public functions:

* ``gemm``: ``fp8_gemm``, 8-bit float operands with an fp32 scale for each block of 128;
* ``quant``: ``fp8_quantize``, the operands of that product from float rows;
* ``norm``: ``residual_norm``, the seam between two branches of a transformer block (norm after the branch, gate,
  residual, norm before the next branch);
* ``grad``: ``residual_norm_backward``, its gradients;
* ``rope``: ``rope``, rotary positions with several axes.

With ``own`` false, ``run`` computes the same in plain torch operations, in 32 bits.
"""
from __future__ import annotations

import math

import torch

own = False

F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
F8_MAX = {"e4m3": 448.0, "e5m2": 57344.0}
FLOAT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "e4m3": 1, "e5m2": 1}
EPS = 1e-6


def _gemm(name, batch, M, N, K, A="e4m3", B="e4m3", rows_A=1, rows_B=128, out="bf16", bias=False, shared_B=True):
    return {"name": name, "op": "gemm", "batch": batch, "M": M, "N": N, "K": K, "A": A, "B": B, "rows_A": rows_A,
            "rows_B": rows_B, "out": out, "bias": bias, "shared_B": shared_B}


def _quant(name, rows, K, x, q, block):
    return {"name": name, "op": "quant", "rows": rows, "K": K, "x": x, "q": q, "block": block}


def _norm(name, op, batch, rows, D, x, y, h, post, pre, adaln):
    return {"name": name, "op": op, "batch": batch, "rows": rows, "D": D, "x": x, "y": y, "h": h, "post": post,
            "pre": pre, "adaln": adaln}


def _rope(name, batch, grid, H, Dh, dims, shared, interleaved, x, inverse):
    return {"name": name, "op": "rope", "batch": batch, "grid": grid, "H": H, "Dh": Dh, "dims": dims, "shared": shared,
            "interleaved": interleaved, "x": x, "inverse": inverse}


def listed():
    return [
        # one token through a DiT-XL/2 MLP: latency
        _gemm("gemm_1_token", 1, 1, 4608, 1152, bias=True),
        # one image of ViT-L/14 at 336 px into an odd number of classes from an odd width: rows on no boundary
        _gemm("gemm_577_odd", 1, 577, 1000, 1031, out="f32"),
        # the gradient of the DiT MLP's weights: contraction over 4096 tokens, gradients in e5m2
        _gemm("gemm_weight_gradient", 1, 4608, 1152, 4096, A="e5m2", rows_B=1, out="f32"),
        # ViT-L/14 MLP fc1 over 32 images: the largest product
        _gemm("gemm_vitl_fc1", 1, 18464, 4096, 1024),
        # the activations of that layer
        _quant("quant_vitl_rows", 18464, 1024, "bf16", "e4m3", "1x128"),
        # gradients of the DiT MLP laid along the tokens, for the gradient of its weights
        _quant("quant_transposed", 4096, 4608, "bf16", "e5m2", "128x1"),
        # one token of a model of width 4096, sandwich norms: latency
        _norm("norm_1_token", "norm", 1, 1, 4096, "bf16", "bf16", "bf16", "rms", "rms", False),
        # DiT-XL/2 seam, 32 images of 256 tokens: gate, LayerNorm, shift and scale per image, fp8 rows for the next product
        _norm("norm_dit_seam_fp8", "norm", 32, 256, 1152, "f32", "bf16", "e4m3", "none", "layer", True),
        # its gradients
        _norm("grad_dit_seam", "grad", 32, 256, 1152, "f32", "bf16", "bf16", "none", "layer", True),
        # sandwich norms at width 4096 with an odd number of rows
        _norm("grad_sandwich_4096", "grad", 1, 4099, 4096, "bf16", "bf16", "bf16", "rms", "rms", False),
        # queries and keys of one request's new token, three axes
        _rope("rope_1_token", 1, "1x1x1", 32, 128, "32,48,48", True, False, "bf16", False),
        # a video latent of 16 x 30 x 52 patches, 24 heads, each axis with frequencies of its own
        _rope("rope_video", 1, "16x30x52", 24, 128, "16,56,56", False, True, "bf16", False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["gemm", "gemm", "gemm", "heads", "quant", "norm", "grad", "rope"])
    if op == "gemm":
        while True:
            M, N, K = _log_int(rng, 1, 18464), _log_int(rng, 64, 8192), _log_int(rng, 48, 8192)
            if M * N * K <= 18464 * 4096 * 1024:
                break
        if rng.random() < 0.6:  # widths of layers are round
            N, K = max(64, N // 64 * 64), max(64, K // 64 * 64)
        grads = rng.random() < 0.3
        case = _gemm(None, 1, M, N, K, A="e5m2" if grads else "e4m3", rows_B=rng.choice([1, 128]) if grads else 128,
                     out=rng.choice(["bf16", "bf16", "f16", "f32"]), bias=rng.random() < 0.5)
    elif op == "heads":
        T, Dh = _log_int(rng, 49, 640), rng.choice([64, 72, 80, 128])
        N, K = rng.choice([(T, Dh), (Dh, T)])
        case = _gemm(None, rng.choice([12, 16, 64, 128]), T, N, K, rows_B=1, out=rng.choice(["bf16", "f32"]), shared_B=False)
    elif op == "quant":
        case = _quant(None, _log_int(rng, 1, 18464), _log_int(rng, 64, 1100), rng.choice(["f32", "bf16", "f16"]),
                      rng.choice(["e4m3", "e4m3", "e5m2"]), rng.choice(["1x128", "1x128", "128x128", "128x1"]))
    elif op in ("norm", "grad"):
        D = rng.choice([384, 768, 1024, 1152, 2048, 4096, _log_int(rng, 64, 8192)])
        adaln = rng.random() < 0.5
        batch = rng.choice([1, 2, 8, 32]) if adaln else 1
        rows = _log_int(rng, 1, max(1, 8192 * 1152 // (batch * D)))
        pre = rng.choice(["layer", "rms"])
        h = rng.choice(["bf16", "f16", "f32"] + (["e4m3", "e4m3"] if op == "norm" else []))
        case = _norm(None, op, batch, rows, D, rng.choice(["f32", "bf16"]), rng.choice(["bf16", "f16", "f32"]), h,
                     rng.choice(["none", "none", pre]), pre, adaln)
    else:
        dims, Dh = rng.choice([("32,48,48", 128), ("16,56,56", 128), ("32,32", 64), ("36,36", 72), ("16,24", 64), ("64,96,96", 256)])
        axes = dims.count(",") + 1
        side = _log_int(rng, 1, 48)
        grid = "%dx%d" % (side, _log_int(rng, 1, 48))
        if axes == 3:
            grid = "%dx%s" % (_log_int(rng, 1, 8), grid)
        case = _rope(None, rng.choice([1, 1, 2]), grid, rng.choice([3, 8, 12, 16]) if Dh <= 128 else rng.choice([2, 6]), Dh, dims,
                     rng.random() < 0.5, rng.random() < 0.5, rng.choice(["bf16", "f16", "f32"]), rng.random() < 0.4)
    del case["name"]
    return case


# ---------------------------------------------------------------- inputs

def _rand(shape, gen, kind="normal"):
    x = torch.randn(shape, generator=gen, device=gen.device)
    if kind == "outlier":  # activations: a few channels many times larger
        hot = torch.randint(0, shape[-1], (6,), generator=gen, device=gen.device)
        x[..., hot] *= 20.0
    return x


def _blocks(x, r):
    """`x` padded with zeros to whole blocks of r x 128 and seen as [..., rows/r, r, columns/128, 128]."""
    rows, cols = x.shape[-2:]
    x = torch.nn.functional.pad(x, (0, -cols % 128, 0, -rows % r))
    return x.reshape(*x.shape[:-2], (rows + r - 1) // r, r, (cols + 127) // 128, 128)


def _plain_quant(x, q, r):
    """Scales and 8-bit values of blocks of r x 128."""
    b = _blocks(x.float(), r)
    m = b.abs().amax(dim=(-3, -1))
    s = torch.where(m > 0, (m / torch.full_like(m, F8_MAX[q])).clamp(min=2.0 ** -126), m)
    inv = torch.where(m > 0, 1.0 / s, m)
    v = (b * inv[..., :, None, :, None]).clamp(-F8_MAX[q], F8_MAX[q])
    v = v.reshape(*v.shape[:-4], v.shape[-4] * r, -1)[..., :x.shape[-2], :x.shape[-1]]
    return v.to(F8[q]).contiguous(), s


def _wide(s, r, rows, cols):
    """Scales of blocks of r x 128, one for each element."""
    return s.repeat_interleave(128, -1)[..., :cols].repeat_interleave(r, -2)[..., :rows, :]


def _inv_freq(case):
    """Angle of each pair for a step of its axis, and the axis."""
    dims = [int(d) for d in case["dims"].split(",")]
    total = sum(dims)
    freq, axis = [], []
    for a, d in enumerate(dims):
        for j in range(d // 2):
            freq.append(10000.0 ** (-2.0 * len(freq) / total) if case["shared"] else 10000.0 ** (-2.0 * j / d))
            axis.append(a)
    return freq, axis


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]
    s = dict(case)
    if op == "gemm":
        M, N, K, nb = case["M"], case["N"], case["K"], case["batch"]
        a = _rand((nb, M, K) if nb > 1 else (M, K), gen, "outlier")
        b = 0.02 * _rand((nb, N, K) if nb > 1 and not case["shared_B"] else (N, K), gen)
        s["A8"], s["sA"] = _plain_quant(a, case["A"], case["rows_A"])
        s["B8"], s["sB"] = _plain_quant(b, case["B"], case["rows_B"])
        s["b"] = _rand((N,), gen) if case["bias"] else None
    elif op == "quant":
        s["X"] = _rand((case["rows"], case["K"]), gen, "outlier").to(FLOAT[case["x"]])
    elif op in ("norm", "grad"):
        nb, T, D = case["batch"], case["rows"], case["D"]
        groups = nb if case["adaln"] else 1
        s["X"] = _rand((nb, T, D), gen, "outlier").to(FLOAT[case["x"]])
        s["Y"] = _rand((nb, T, D), gen).to(FLOAT[case["y"]])
        p = {"gate": _rand((groups, D), gen), "pre_weight": 0.1 * _rand((groups, D), gen),
             "pre_bias": 0.1 * _rand((groups, D), gen) if case["pre"] == "layer" else None,
             "post_weight": 1.0 + 0.1 * _rand((D,), gen) if case["post"] != "none" else None}
        s["p"] = {k: v.to(torch.bfloat16) for k, v in p.items() if v is not None}
        if op == "grad":
            s["dX"] = _rand((nb, T, D), gen).to(FLOAT[case["x"]])
            s["dH"] = _rand((nb, T, D), gen).to(FLOAT[case["h"]])
    else:
        sides = [int(n) for n in case["grid"].split("x")]
        T = math.prod(sides)
        s["X"] = _rand((case["batch"], T, case["H"], case["Dh"]), gen).to(FLOAT[case["x"]])
        start = int(torch.randint(0, 100000, (1,), generator=gen, device="cuda").item())
        ax = torch.meshgrid(*[torch.arange(n, dtype=torch.int32, device="cuda") for n in sides], indexing="ij")
        pos = torch.stack([x.reshape(-1) for x in ax])
        s["pos"] = (pos + start).contiguous()  # text before the patches moves every axis on
        freq, axis = _inv_freq(case)
        s["freq"] = torch.tensor(freq, dtype=torch.float64, device="cuda")
        s["axis"] = torch.tensor(axis, dtype=torch.int32, device="cuda")
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    if own:
        return _run_own(s)
    return {"gemm": _plain_gemm, "quant": _plain_quant_op, "norm": _plain_norm, "grad": _plain_grad, "rope": _plain_rope}[s["op"]](s)


def _run_own(s):
    import paper_2609_32922_amd as scg
    op = s["op"]
    if op == "gemm":
        return scg.fp8_gemm(s["A8"], s["sA"], s["B8"], s["sB"], bias=s["b"], out_dtype=FLOAT[s["out"]])
    if op == "quant":
        block = {"1x128": scg.SC_BLOCK_1X128, "128x128": scg.SC_BLOCK_128X128, "128x1": scg.SC_BLOCK_128X1_T}[s["block"]]
        return scg.fp8_quantize(s["X"], dtype=F8[s["q"]], block=block)
    kinds = {"none": scg.SC_NORM_NONE, "rms": scg.SC_NORM_RMS, "layer": scg.SC_NORM_LAYER}
    if op == "norm":
        xo, h, scale, _ = scg.residual_norm(s["X"], s["Y"], post=kinds[s["post"]], pre=kinds[s["pre"]], post_eps=EPS, pre_eps=EPS,
                                            pre_offset=1.0, out_dtype={**FLOAT, **F8}[s["h"]], **s["p"])
        return (xo, h) if scale is None else (xo, h, scale)
    if op == "grad":
        return scg.residual_norm_backward(s["X"], s["Y"], dxo=s["dX"], dh=s["dH"], post=kinds[s["post"]], pre=kinds[s["pre"]],
                                          post_eps=EPS, pre_eps=EPS, pre_offset=1.0, **s["p"])
    return scg.rope(s["X"], s["pos"], s["freq"], s["axis"], interleaved=s["interleaved"], inverse=s["inverse"])


def _plain_gemm(s):
    M, N, K = s["M"], s["N"], s["K"]
    a = s["A8"].float() * _wide(s["sA"], s["rows_A"], M, K)
    b = s["B8"].float() * _wide(s["sB"], s["rows_B"], N, K)
    o = torch.matmul(a, b.transpose(-1, -2))
    if s["b"] is not None:
        o = o + s["b"]
    return o.to(FLOAT[s["out"]])


def _plain_quant_op(s):
    x = s["X"].t() if s["block"] == "128x1" else s["X"]
    return _plain_quant(x, s["q"], 128 if s["block"] == "128x128" else 1)


def _normal(x, kind):
    """`x` normalised, and 1 / its deviation."""
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return x * r, r


def _param(s, name):
    p = s["p"].get(name)
    return 0.0 if p is None else p.float()[:, None, :] if p.dim() == 2 else p.float()


def _plain_norm(s):
    x, u = s["X"].float(), s["Y"].float()
    if s["post"] != "none":
        u = _normal(u, s["post"])[0] * _param(s, "post_weight")
    xo = x + _param(s, "gate") * u
    h = _normal(xo, s["pre"])[0] * (1.0 + _param(s, "pre_weight")) + _param(s, "pre_bias")
    xo = xo.to(FLOAT[s["x"]])
    if s["h"] in F8:
        return (xo, *_plain_quant(h, s["h"], 1))
    return xo, h.to(FLOAT[s["h"]])


def _normal_back(d, n, r, kind):
    """The gradient before a norm from the one behind it, `n` and `r` as _normal gives them."""
    g = d - n * (d * n).mean(-1, keepdim=True)
    if kind == "layer":
        g = g - d.mean(-1, keepdim=True)
    return r * g


def _plain_grad(s):
    xo, y, g, dh = s["X"].float(), s["Y"].float(), s["dX"].float(), s["dH"].float()
    over = (1,) if s["adaln"] else (0, 1)
    as_groups = lambda t: t.sum(over).reshape(-1, s["D"])  # noqa: E731
    n, r = _normal(xo, s["pre"])
    got = {"pre_weight": as_groups(dh * n)}
    if s["pre"] == "layer":
        got["pre_bias"] = as_groups(dh)
    g = g + _normal_back(dh * (1.0 + _param(s, "pre_weight")), n, r, s["pre"])
    du = g * _param(s, "gate")
    if s["post"] == "none":
        got["gate"], dy = as_groups(g * y), du
    else:
        n, r = _normal(y, s["post"])
        w = _param(s, "post_weight")
        got["gate"], got["post_weight"] = as_groups(g * n * w), (du * n).sum((0, 1))
        dy = _normal_back(du * w, n, r, s["post"])
    return {"x": g.to(FLOAT[s["x"]]), "y": dy.to(FLOAT[s["y"]]), **got}


def _plain_rope(s):
    x = s["X"].float()
    angle = s["pos"].double().index_select(0, s["axis"]).t() * s["freq"]     # [T, pairs]; in 64 bits: far positions
    c, z = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]
    if s["inverse"]:
        z = -z
    P = angle.shape[1]
    if s["interleaved"]:
        u, v = x[..., 0:2 * P:2], x[..., 1:2 * P:2]
    else:
        u, v = x[..., :P], x[..., P:2 * P]
    a, b = u * c - v * z, u * z + v * c
    turned = torch.stack((a, b), -1).flatten(-2) if s["interleaved"] else torch.cat((a, b), -1)
    return torch.cat((turned, x[..., 2 * P:]), -1).to(FLOAT[s["x"]])


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    op = case["op"]
    if op == "gemm":
        nb, M, N, K = case["batch"], case["M"], case["N"], case["K"]
        kb = -(-K // 128)
        nB = 1 if case["shared_B"] else nb
        read = nb * M * K + nB * N * K + 4 * kb * (nb * -(-M // case["rows_A"]) + nB * -(-N // case["rows_B"]))
        return {"bytes": read + nb * M * N * BYTES[case["out"]] + (4 * N if case["bias"] else 0), "flops": 2 * nb * M * N * K}
    if op == "quant":
        n, r = case["rows"] * case["K"], {"1x128": 1, "128x128": 128, "128x1": 1}[case["block"]]
        return {"bytes": n * (BYTES[case["x"]] + 1) + 4 * n // (128 * r), "flops": 3 * n}
    if op in ("norm", "grad"):
        n = case["batch"] * case["rows"] * case["D"]
        params = (case["batch"] if case["adaln"] else 1) * case["D"] * (3 if case["pre"] == "layer" else 2)
        params += case["D"] if case["post"] != "none" else 0
        x, y, h = (BYTES[case[k]] for k in "xyh")
        if op == "norm":
            return {"bytes": n * (2 * x + y + h) + 2 * params + (n // 32 if case["h"] in F8 else 0), "flops": 12 * n}
        return {"bytes": n * (3 * x + 2 * y + h) + (2 + 4) * params, "flops": 30 * n}
    T = math.prod(int(v) for v in case["grid"].split("x"))
    n, axes = case["batch"] * T * case["H"] * case["Dh"], case["dims"].count(",") + 1
    return {"bytes": 2 * n * BYTES[case["x"]] + 4 * axes * T, "flops": 3 * n}


# ---------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "gemm":
        # block by block of the contraction, each with the product of its two scales
        A, B = s["A8"].float().double(), s["B8"].float().double()
        i = torch.arange(case["M"], device="cuda") // case["rows_A"]
        j = torch.arange(case["N"], device="cuda") // case["rows_B"]
        out = 0.0
        for k in range(s["sA"].shape[-1]):
            at = slice(128 * k, 128 * (k + 1))
            part = torch.matmul(A[..., at], B[..., at].transpose(-1, -2).contiguous())
            out = out + part * s["sA"].double()[..., i, k, None] * s["sB"].double()[..., j, k][..., None, :]
        return out if s["b"] is None else out + s["b"].double()
    if op == "quant":
        x = s["X"].double()
        v, top = _exact_blocks(x.t().contiguous() if case["block"] == "128x1" else x, case["q"], 128 if case["block"] == "128x128" else 1)
        # to the type's nearest value, ties to even: 3 (2) bits behind the leading one, the smallest exponent -6 (-14)
        bits, low = (3, -6) if case["q"] == "e4m3" else (2, -14)
        step = torch.pow(2.0, (torch.frexp(v).exponent.double() - 1).clamp(min=low) - bits)
        return torch.round(v / step) * step, top
    if op == "norm":
        with torch.no_grad():
            xo, h = _exact_seam(case, s["X"].double(), s["Y"].double(), {k: v.double() for k, v in s["p"].items()})
        return (xo, *_exact_blocks(h, case["h"], 1)) if case["h"] in F8 else (xo, h)
    if op == "grad":
        # torch's differentiation of the definition at the residual that the case gives
        leaf = lambda t: t.double().requires_grad_(True)  # noqa: E731
        y, p = leaf(s["Y"]), {k: leaf(v) for k, v in s["p"].items()}
        branch = _exact_branch(case, y, p)
        x = (s["X"].double() - branch.detach()).requires_grad_(True)
        xo = x + branch
        h = _exact_pre(case, xo, p)
        ((xo * s["dX"].double()).sum() + (h * s["dH"].double()).sum()).backward()
        return {"x": x.grad, "y": y.grad, **{k: v.grad for k, v in p.items()}}
    freq, axis = _inv_freq(case)
    x, P = s["X"].double(), len(freq)
    turn = torch.stack([s["pos"][a].double() * f for f, a in zip(freq, axis)], -1)[:, None, :]
    turn = torch.polar(torch.ones_like(turn), -turn if case["inverse"] else turn)
    if case["interleaved"]:
        z = torch.view_as_complex(x[..., :2 * P].reshape(*x.shape[:-1], P, 2).contiguous()) * turn
        x[..., :2 * P] = torch.view_as_real(z).reshape(*x.shape[:-1], 2 * P)
    else:
        z = torch.complex(x[..., :P].contiguous(), x[..., P:2 * P].contiguous()) * turn
        x[..., :P], x[..., P:2 * P] = z.real, z.imag
    return x


def _exact_blocks(x, q, r):
    """8-bit values before their rounding, and scales."""
    rows, cols = x.shape[-2:]
    rb, cb = -(-rows // r), -(-cols // 128)
    full = torch.zeros((*x.shape[:-2], rb * r, cb * 128), dtype=torch.float64, device=x.device)
    full[..., :rows, :cols] = x
    top = full.unflatten(-1, (cb, 128)).abs().max(-1).values.unflatten(-2, (rb, r)).max(-2).values
    s = top / F8_MAX[q]
    return full.div(s.clamp(min=1e-300).repeat_interleave(128, -1).repeat_interleave(r, -2))[..., :rows, :cols].contiguous(), s


def _exact_scaled(x, kind):
    centre = x.mean(-1, keepdim=True) if kind == "layer" else 0.0
    var = ((x - centre) ** 2).sum(-1, keepdim=True) / x.shape[-1]
    return (x - centre) / (var + EPS).sqrt()


def _exact_branch(case, y, p):
    u = y if case["post"] == "none" else _exact_scaled(y, case["post"]) * p["post_weight"]
    return u * p["gate"].unsqueeze(1)


def _exact_pre(case, xo, p):
    h = _exact_scaled(xo, case["pre"]) * (1.0 + p["pre_weight"].unsqueeze(1))
    return h + p["pre_bias"].unsqueeze(1) if "pre_bias" in p else h


def _exact_seam(case, x, y, p):
    xo = x + _exact_branch(case, y, p)
    return xo, _exact_pre(case, xo, p)
