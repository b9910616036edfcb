"""The layer operators on the GPU against their definitions in 64 bits (tests/layers_ref.py)."""
import sys
import types

import numpy as np
import pytest
import torch

import layers_ref as R

pytestmark = pytest.mark.gpu
E4, E5 = torch.float8_e4m3fn, torch.float8_e5m2
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def _note(msg):
    print("[gpu-case] " + msg, flush=True)
    sys.stdout.flush()


@pytest.fixture(scope="module")
def scg():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_32922_amd as scg
    scg.load()
    return scg


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(shape, gen, dtype=F32):
    return torch.randn(shape, generator=gen, device="cuda").to(dtype)


def _same_bytes(a, b):
    na, nb = torch.isnan(a.float()), torch.isnan(b.float())
    assert torch.equal(na, nb)
    same = (a.view(torch.uint8) == b.view(torch.uint8)) | na if a.element_size() == 1 else (a == b) | na
    assert bool(same.all()), "%d of %d differ" % (int((~same).sum()), same.numel())


def _within(got, ref, tol, what):
    d = (got.double() - ref).abs()
    bad = ~(d <= tol)
    assert not bool(bad.any()), "%s: %d of %d, worst %.3g against %.3g" % (
        what, int(bad.sum()), bad.numel(), float(d[bad].max()), float(tol.expand_as(d)[bad][d[bad].argmax()]))


# ---------------------------------------------------------------- quantiser

QUANT = [(1, 1, 1), (1, 70, 1023), (2, 130, 135), (1, 1, 128), (1, 3, 129), (1, 128, 1024), (2, 5, 777), (1, 300, 1000), (3, 129, 257), (1, 64, 4096), (1, 1000, 24)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("q", [E4, E5])
@pytest.mark.parametrize("batch,rows,K", QUANT)
def test_fp8_quantize(scg, batch, rows, K, q, dtype):
    _note("fp8_quantize %d x %d x %d %s %s" % (batch, rows, K, q, dtype))
    gen = _gen(rows * 1000 + K)
    x = _randn((batch, rows, K), gen) * torch.exp(2.0 * _randn((batch, rows, 1), gen))
    x[0, 0] = 0.0
    x = x.to(dtype)
    for block, per in ((scg.SC_BLOCK_1X128, 1), (scg.SC_BLOCK_128X128, 128), (scg.SC_BLOCK_128X1_T, 1)):
        Q, s = scg.fp8_quantize(x, dtype=q, block=block)
        src = x.transpose(1, 2).contiguous() if block == scg.SC_BLOCK_128X1_T else x
        Qr, sr = R.fp8_quantize32(src.cpu(), q, per)
        assert torch.equal(s.cpu(), sr)
        _same_bytes(Q.cpu(), Qr)
    Q2, s2 = scg.fp8_quantize(x[0], dtype=q)
    assert Q2.shape == (rows, K) and s2.shape == (rows, -(-K // 128))


@pytest.mark.parametrize("block,per", [(0, 1), (1, 128), (2, 1)])
def test_fp8_quantize_special_values(scg, block, per):
    # zeros, the least floats, NaN, infinities, a block of one value, the largest float
    _note("fp8_quantize special values, block %d" % block)
    x = torch.zeros(130, 264)
    x[1] = 1e-45
    x[2, :128] = torch.linspace(-3e38, 3e38, 128)
    x[3] = 7.0
    x[4, 5] = float("nan")
    x[4, 6] = 2.0
    x[5, 130] = float("inf")
    x[5, 131] = 1.0
    x[6, 200] = float("-inf")
    x[7] = 2.0 ** -140
    x[8] = float("nan")
    x[9, 3] = -0.0
    x[129, 263] = -1e-30
    for q in (E4, E5):
        Q, s = scg.fp8_quantize(x.cuda(), dtype=q, block=block)
        Qr, sr = R.fp8_quantize32(x.t().contiguous() if block == 2 else x, q, per)
        assert torch.equal(s.cpu(), sr)
        _same_bytes(Q.cpu(), Qr)


def test_fp8_quantize_views_and_untouched_bytes(scg):
    # rows inside a larger buffer, from an odd element on; what lies around the result stays as it was
    _note("fp8_quantize of views")
    gen = _gen(3)
    big = _randn((40, 700), gen, BF16)
    for view in (big[:, :512], big[:, 1:514], big[3:30, 8:264], big[5:6, 9:10]):
        for block, per in ((0, 1), (1, 128), (2, 1)):
            Q, s = scg.fp8_quantize(view, block=block)
            src = view.t() if block == 2 else view
            Qr, sr = R.fp8_quantize32(src.cpu().contiguous(), E4, per)
            assert torch.equal(s.cpu(), sr)
            _same_bytes(Q.cpu(), Qr)
    rows, K, ld = 130, 200, 333
    x = _randn((rows, K), gen)
    buf = torch.full((rows * ld + 7,), 0x55, dtype=torch.uint8, device="cuda")
    sc = torch.full((rows, 5), -7.0, device="cuda")
    rc = scg._lib.sc_fp8_quantize(1, rows, K, 0, x.data_ptr(), K, 0, 3, 0, buf.data_ptr() + 7, ld, 0, sc.data_ptr(), 5, 0, 0)
    assert rc == 0
    got = buf[7:].view(rows, ld)
    assert bool((buf[:7] == 0x55).all()) and bool((got[:, K:] == 0x55).all()) and bool((sc[:, 2:] == -7.0).all())
    _same_bytes(got[:, :K].contiguous().view(E4).cpu(), R.fp8_quantize32(x.cpu(), E4, 1)[0])


# ---------------------------------------------------------------- product

def _operand(shape, gen, dtype, per):
    x = _randn(shape, gen)
    x[..., :3] *= 20.0
    q, s = R.fp8_quantize32(x, dtype, per)
    return q.contiguous(), s.contiguous()


GEMM = [
    # batch, M, N, K, A, B, rows_A, rows_B, out, bias, shared
    (1, 1, 1, 1, E4, E4, 1, 1, F32, False, True),
    (1, 1, 4608, 1152, E4, E4, 1, 128, BF16, True, True),
    (1, 2, 130, 127, E4, E4, 1, 1, F32, True, True),
    (1, 7, 1000, 129, E5, E4, 1, 128, F32, False, True),
    (1, 16, 64, 4096, E4, E4, 1, 128, BF16, False, True),
    (1, 17, 300, 1031, E4, E5, 1, 1, F32, True, True),
    (1, 33, 500, 640, E4, E4, 128, 128, F16, False, True),
    (1, 64, 256, 2048, E5, E5, 1, 1, F32, False, True),
    (1, 100, 72, 8192, E4, E4, 1, 128, F32, True, True),
    (1, 129, 129, 257, E4, E4, 128, 1, F32, True, True),
    (1, 300, 300, 96, E4, E4, 1, 128, BF16, True, True),
    (1, 257, 513, 1024, E4, E4, 1, 128, F32, True, True),
    (1, 577, 1000, 1031, E4, E4, 1, 128, F32, False, True),
    (1, 1024, 1152, 1152, E5, E4, 1, 1, F32, False, True),
    (1, 2049, 770, 512, E4, E4, 1, 128, BF16, False, True),
    (1, 3000, 4100, 384, E4, E4, 1, 128, F32, True, True),
    (1, 4096, 4608, 1152, E4, E4, 1, 128, BF16, False, True),
    (1, 4608, 1152, 4099, E5, E4, 1, 1, F32, False, True),
    (3, 50, 70, 200, E4, E4, 1, 128, F32, True, True),
    (5, 65, 64, 64, E4, E5, 1, 1, BF16, False, False),
    (16, 577, 577, 64, E4, E4, 1, 1, F32, False, False),
    (12, 197, 64, 197, E4, E4, 1, 1, F32, True, False),
    (2, 700, 900, 260, E4, E4, 128, 128, F32, True, False),
    # a tile's stages by several blocks
    (1, 64, 256, 8192, E4, E4, 1, 128, F32, True, True),
    (1, 290, 383, 7233, E4, E4, 1, 128, F16, False, True),
    (2, 100, 130, 4099, E5, E4, 1, 1, BF16, True, False),
    (3, 17, 70, 5000, E4, E5, 128, 1, F32, True, True),
    (1, 40, 33, 262144, E4, E4, 1, 128, F32, True, True),
    (1, 16000, 2040, 1000, E4, E4, 1, 128, BF16, True, True),
    (1, 8000, 4000, 1016, E5, E4, 1, 1, F16, False, True),
    (2, 5000, 3000, 1024, E4, E4, 128, 1, BF16, True, False),
]


@pytest.mark.parametrize("case", GEMM, ids=lambda c: "%dx%dx%dx%d_%d_%d" % (c[0], c[1], c[2], c[3], c[6], c[7]))
def test_fp8_gemm(scg, case):
    batch, M, N, K, ta, tb, pa, pb, to, bias, shared = case
    _note("fp8_gemm %s" % (case,))
    gen = _gen(M + 7 * N + 31 * K)
    A, sA = _operand((batch, M, K) if batch > 1 else (M, K), gen, ta, pa)
    B, sB = _operand((batch, N, K) if batch > 1 and not shared else (N, K), gen, tb, pb)
    b = _randn((batch, N) if batch > 1 else (N,), gen) if bias else None
    got = scg.fp8_gemm(A, sA, B, sB, bias=b, out_dtype=to)
    ref, mag = R.fp8_gemm(A, sA, pa, B, sB, pb, b)
    _within(got, ref, R.gemm_tolerance(mag, K, to, ref), "product")
    if to != F32 and ref.numel() > 1000:
        assert R.gemm_norm_ratio(got, ref) <= (1.01 if to == BF16 else 1.06)
    again = scg.fp8_gemm(A, sA, B, sB, bias=b, out_dtype=to)
    assert torch.equal(got, again)


def test_fp8_gemm_exact_small_integers(scg):
    # products of small whole numbers with scales of powers of two: every sum is exact, so every bit counts
    _note("fp8_gemm exact integers")
    gen = _gen(5)
    for M, N, K in ((40, 50, 300), (256, 512, 512), (1, 96, 1024), (300, 513, 1000)):
        a = torch.randint(-4, 5, (M, K), generator=gen, device="cuda").float()
        b = torch.randint(-4, 5, (N, K), generator=gen, device="cuda").float()
        kb = -(-K // 128)
        sa = 2.0 ** torch.randint(-2, 3, (M, kb), generator=gen, device="cuda").float()
        sb = 2.0 ** torch.randint(-2, 3, (-(-N // 128), kb), generator=gen, device="cuda").float()
        got = scg.fp8_gemm(a.to(E4), sa, b.to(E4), sb, out_dtype=F32)
        ref, _ = R.fp8_gemm(a.to(E4), sa, 1, b.to(E4), sb, 128)
        assert torch.equal(got.double(), ref)


SMALL = [(1, 16, 128), (8, 64, 1024), (100, 72, 1024), (64, 256, 8192), (300, 300, 1000), (2000, 1411, 1024), (5000, 3000, 1024)]


@pytest.mark.parametrize("M,N,K,to", [(*c, t) for c in SMALL for t in (F32, F16, BF16) if t != BF16 or c[0] <= 16])
def test_fp8_gemm_small_products_beside_large_ones(scg, M, N, K, to):
    # of each eight neighbours two products are 2^16 and -2^16 and the others are small: every sum is a whole number that float32
    # and float16 hold, so nothing may be lost but its rounding to bfloat16
    _note("fp8_gemm small products %d x %d x %d" % (M, N, K))
    gen = _gen(K + M)
    a = torch.randint(-2, 3, (M, K), generator=gen, device="cuda").float()
    b = torch.randint(-2, 3, (N, K), generator=gen, device="cuda").float()
    a[:, 0::8] = a[:, 1::8] = b[:, 0::8] = 256.0
    b[:, 1::8] = -256.0
    one = lambda n: torch.ones(n, -(-K // 128), device="cuda")  # noqa: E731
    got = scg.fp8_gemm(a.to(E4), one(M), b.to(E4), one(N), out_dtype=to)
    ref, _ = R.fp8_gemm(a.to(E4), one(M), 1, b.to(E4), one(N), 1)
    assert float(ref.abs().max()) <= 2048.0 and torch.equal(got, ref.to(to))


def test_fp8_gemm_views(scg):
    # operands, scales and result inside larger buffers, from odd bytes on; the rest stays as it was
    _note("fp8_gemm of views")
    gen = _gen(6)
    for off, pad, M, N, K in ((0, 0, 150, 140, 256), (1, 3, 150, 140, 200), (16, 16, 270, 300, 384), (5, 11, 3, 333, 130), (16, 0, 40, 64, 256),
                               (5, 11, 1500, 1411, 200), (1, 15, 1500, 1411, 240), (16, 16, 1500, 1411, 224), (3, 2, 70, 99, 4000), (16, 0, 70, 99, 4000)):
        A0, B0 = (torch.randint(0, 120, (n, K + off + pad), generator=gen, device="cuda", dtype=torch.uint8) for n in (M, N))
        kb = -(-K // 128)
        sA0, sB0 = torch.rand((M, kb + 2), generator=gen, device="cuda"), torch.rand((-(-N // 128), kb + 1), generator=gen, device="cuda")
        A, B, sA, sB = A0.view(E4)[:, off:off + K], B0.view(E4)[:, off:off + K], sA0[:, 1:kb + 1], sB0[:, :kb]
        big = torch.full((M + 2, N + 9), -3.0, device="cuda")
        out = big[1:M + 1, 2:N + 2]
        scg.fp8_gemm(A, sA, B, sB, out=out)
        ref, mag = R.fp8_gemm(A, sA, 1, B, sB, 128)
        _within(out, ref, R.gemm_tolerance(mag, K, F32, ref), "product")
        big[1:M + 1, 2:N + 2] = -3.0
        assert bool((big == -3.0).all())


@pytest.mark.parametrize("to", [F32, BF16])
@pytest.mark.parametrize("M,N,K,ld", [(1500, 1411, 201, 208), (1500, 1411, 203, 256), (1500, 1411, 204, 208), (1500, 1411, 130, 144),
                                      (1500, 1411, 1031, 1040), (1500, 1411, 127, 128), (5000, 3001, 1029, 1040)])
def test_fp8_gemm_of_columns_of_padded_rows(scg, M, N, K, ld, to):
    # rows on 16 bytes whose last elements are no whole 16: these count in every row, a tile's last one too, and what lies behind does not
    _note("fp8_gemm %d x %d x %d of rows of %d" % (M, N, K, ld))
    gen = _gen(K)
    ops = []
    for n, per in ((M, 1), (N, 128)):
        x = _randn((n, K), gen)
        x[:, K - K % 16:] *= 30.0
        q, s = R.fp8_quantize32(x, E4, per)
        full = torch.full((n, ld), 0x7F, dtype=torch.uint8, device="cuda").view(E4)       # NaN behind K
        full[:, :K] = q
        ops += [full[:, :K], s]
    got = scg.fp8_gemm(*ops, out_dtype=to)
    ref, mag = R.fp8_gemm(ops[0], ops[1], 1, ops[2], ops[3], 128)
    _within(got, ref, R.gemm_tolerance(mag, K, to, ref), "product")


@pytest.mark.parametrize("to", [F32, BF16])
@pytest.mark.parametrize("M,N,K", [(5, 64, 128), (150, 72, 300), (70, 99, 4000), (700, 640, 256), (701, 643, 256)])
def test_fp8_gemm_into_rows_of_entries_in_turn(scg, M, N, K, to):
    # the result of [heads, rows, n] in memory as [rows, heads, n], with columns beside it that stay as they were
    _note("fp8_gemm into [rows, heads, n] %d x %d x %d %s" % (M, N, K, to))
    gen, H = _gen(M + N), 7
    A, sA = _operand((H, M, K), gen, E4, 1)
    B, sB = _operand((H, N, K), gen, E4, 1)
    want = scg.fp8_gemm(A, sA, B, sB, out_dtype=to)
    big = torch.full((M, H, N + 8), -3.0, dtype=to, device="cuda")
    out = big[:, :, :N].transpose(0, 1)
    got = scg.fp8_gemm(A, sA, B, sB, out=out)
    assert got is out and torch.equal(out, want) and bool((big[:, :, N:] == -3.0).all())


def test_fp8_gemm_lays_nothing_out_for_nothing(scg):
    # one operand off 16 bytes, the other with rows that would be laid out for the tiles which the first one keeps both from
    _note("fp8_gemm off 16 bytes beside odd rows")
    gen = _gen(18)
    M, N, K = 1500, 1411, 200
    odd, row = torch.zeros(M * 256 + 1, dtype=torch.uint8, device="cuda"), torch.zeros((N, 203), dtype=torch.uint8, device="cuda")
    (a, sA), (b, sB) = _operand((M, K), gen, E4, 1), _operand((N, K), gen, E4, 128)
    A, B = odd[1:].view(M, 256)[:, :K], row[:, :K]
    A.copy_(a.view(torch.uint8))
    B.copy_(b.view(torch.uint8))
    ws = scg.Workspace(1 << 20)
    ws._buf.fill_(0x3C)
    for x, sx, y, sy in ((A, sA, B, sB), (B, sB, A, sA)):
        got = scg.fp8_gemm(x.view(E4), sx, y.view(E4), sy, out_dtype=F32, workspace=ws)
        px, py = ((1, 128) if x is A else (128, 1))
        ref, mag = R.fp8_gemm(x.view(E4), sx, px, y.view(E4), sy, py)
        _within(got, ref, R.gemm_tolerance(mag, K, F32, ref), "product")
    assert bool((ws._buf == 0x3C).all())


def test_fp8_gemm_special_values(scg):
    # NaN and infinities reach their own rows and columns, and nothing else; what lies behind K never counts
    _note("fp8_gemm special values")
    gen = _gen(7)
    for M, N, K in ((20, 30, 200), (300, 300, 200), (40, 30, 200 + 256 * 16)):
        kb = -(-K // 128)
        A0 = torch.full((M, 128 * kb), 0x7F, dtype=torch.uint8, device="cuda").view(E4)       # NaN behind K
        B0 = torch.full((N, 128 * kb), 0x7F, dtype=torch.uint8, device="cuda").view(E4)
        A0[:, :K] = _randn((M, K), gen).to(E4)
        B0[:, :K] = _randn((N, K), gen).to(E4)
        A0[3, 150] = float("nan")
        sA, sB = torch.ones(M, kb, device="cuda"), torch.ones(N, kb, device="cuda")
        sB[5, 1] = float("inf")
        got = scg.fp8_gemm(A0[:, :K], sA, B0[:, :K], sB, out_dtype=F32)
        bad = ~torch.isfinite(got)
        want = torch.zeros_like(bad)
        want[3] = True
        want[:, 5] = True
        assert torch.equal(bad, want)


def test_fp8_gemm_empty(scg):
    _note("fp8_gemm empty")
    z = torch.zeros
    for M, N in ((0, 5), (5, 0), (0, 0)):
        out = scg.fp8_gemm(z(M, 64, device="cuda").to(E4), z(M, 1, device="cuda"), z(N, 64, device="cuda").to(E4),
                           z(N, 1, device="cuda"))
        assert out.shape == (M, N)
    # nothing to contract: the bias alone
    b = torch.arange(7.0, device="cuda")
    out = scg.fp8_gemm(z(3, 0, device="cuda").to(E4), z(3, 0, device="cuda"), z(7, 0, device="cuda").to(E4), z(7, 0, device="cuda"),
                       bias=b, out_dtype=F32)
    assert torch.equal(out, b.expand(3, 7))
    b = torch.arange(700.0, device="cuda")
    for M in (17, 3000):
        for to in (F32, BF16):
            out = scg.fp8_gemm(z(M, 0, device="cuda").to(E4), z(M, 0, device="cuda"), z(700, 0, device="cuda").to(E4),
                               z(6, 0, device="cuda"), bias=b, out_dtype=to)
            assert torch.equal(out, b.to(to).expand(M, 700))


def test_offsets_past_32_bits(scg):
    # rows that start past 2^31 elements (and bytes) from the first
    _note("offsets past 32 bits")
    gen = _gen(8)
    rows, K, ld = 530, 256, 1 << 23
    buf = torch.empty((rows - 1) * ld + K, dtype=torch.uint8, device="cuda")     # 4.4 GB
    A = torch.as_strided(buf, (rows, K), (ld, 1))
    q, s = _operand((rows, K), gen, E4, 1)
    A.copy_(q.view(torch.uint8))
    B, sB = _operand((260, K), gen, E4, 128)
    got = scg.fp8_gemm(A.view(E4), s, B, sB, out_dtype=F32)
    assert torch.equal(got, scg.fp8_gemm(q, s, B, sB, out_dtype=F32))
    got = scg.fp8_gemm(B, sB, A.view(E4), s, out_dtype=F32)
    assert torch.equal(got, scg.fp8_gemm(B, sB, q, s, out_dtype=F32))
    del buf, A
    big = torch.empty((rows - 1) * ld + K, dtype=BF16, device="cuda")            # 8.9 GB
    x = torch.as_strided(big, (rows, K), (ld, 1))
    src = _randn((rows, K), gen, BF16)
    x.copy_(src)
    for block in range(3):
        for a, b in zip(scg.fp8_quantize(x, block=block), scg.fp8_quantize(src, block=block)):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    for a, b in zip(scg.residual_norm(x, x), scg.residual_norm(src, src)):
        assert (a is None and b is None) or torch.equal(a, b)
    ga, gb = (scg.residual_norm_backward(v, v, dxo=v, dh=v) for v in (x, src))
    assert all(torch.equal(ga[k], gb[k]) for k in gb)
    pos = torch.arange(rows, dtype=torch.int32, device="cuda")[None]
    f, ax = scg.rope_table([64])
    assert torch.equal(scg.rope(x.view(rows, 4, 64), pos, f, ax), scg.rope(src.view(rows, 4, 64), pos, f, ax))


# ---------------------------------------------------------------- residual norm

def _params(names, D, gen, dtype, batch):
    """Every other parameter by batch entry."""
    p = {}
    for k, n in enumerate(names):
        shape = (batch, D) if batch > 1 and k % 2 == 0 else (D,)
        p[n] = (0.5 * _randn(shape, gen) + (1.0 if "weight" in n else 0.0)).to(dtype)
    return p


ALL = ("gate", "pre_weight", "post_weight", "pre_bias", "post_bias")
NORM = [
    # batch, rows, D, x, y, h, params, post, pre, names, kw
    (1, 1, 1, F32, F32, F32, F32, 0, 2, (), {}),
    (1, 1, 4096, BF16, BF16, BF16, BF16, 1, 1, ("gate", "pre_weight", "post_weight"), dict(pre_offset=1.0)),
    (2, 5, 64, F32, BF16, F32, F32, 0, 2, ("gate", "pre_weight", "pre_bias"), dict(pre_offset=1.0)),
    (3, 7, 1152, F32, BF16, BF16, BF16, 2, 2, ALL, dict(pre_offset=1.0, post_offset=1.0, res_scale=0.5)),
    (1, 9, 777, F16, F32, F16, F32, 1, 2, ALL, {}),
    (2, 3, 130, BF16, F16, F32, F16, 2, 1, ALL, dict(res_scale=-2.0)),
    (1, 6, 256, F32, F32, F32, F32, 0, 0, ("gate",), {}),
    (1, 4, 1280, F32, F32, F32, F32, 1, 1, ALL, {}),
    (1, 3, 1284, F32, F32, F32, F32, 1, 2, ALL, {}),
    (1, 5, 2048, BF16, BF16, F32, F32, 0, 1, ("pre_weight",), {}),
    (2, 3, 2500, F32, BF16, F32, F32, 2, 2, ALL, {}),
    (1, 3, 4100, F32, F32, BF16, BF16, 1, 1, ALL, {}),
    (1, 2, 8192, BF16, BF16, BF16, F32, 1, 1, ALL, {}),
    (1, 3, 8193, F32, F32, F32, F32, 2, 2, ALL, {}),
    (1, 21, 701, BF16, F16, F32, BF16, 1, 2, ALL, {}),
    (2, 5, 1023, F32, BF16, BF16, F32, 2, 1, ALL, {}),
    (1, 6, 2047, BF16, BF16, BF16, BF16, 1, 1, ALL, {}),
    (1, 5, 4095, F32, BF16, F32, F32, 1, 2, ALL, {}),
    (1, 3, 8191, BF16, BF16, BF16, F32, 2, 2, ALL, {}),
    (1, 2, 16384, F32, BF16, F32, F32, 1, 2, ALL, {}),
    (1, 1030, 96, F32, F32, F32, F32, 0, 2, ("gate", "pre_weight", "pre_bias"), {}),
]


def _norm_inputs(case, seed=0):
    batch, rows, D, tx, ty, th, tp, post, pre, names, kw = case
    gen = _gen(rows * 31 + D + seed)
    x = _randn((batch, rows, D), gen) * 3.0 + 1.0
    x[..., :2] *= 20.0
    y = _randn((batch, rows, D), gen) - 0.5
    x[0, 0] = 1.0                              # a constant row: no deviation
    y[0, 0] = 0.0                              # an empty branch
    return x.to(tx), y.to(ty), _params(names, D, gen, tp, batch), gen


@pytest.mark.parametrize("case", NORM, ids=lambda c: "%dx%dx%d_%d%d" % (c[0], c[1], c[2], c[7], c[8]))
def test_residual_norm(scg, case):
    batch, rows, D, tx, ty, th, tp, post, pre, names, kw = case
    _note("residual_norm %s" % (case,))
    x, y, p, _ = _norm_inputs(case)
    xo, h, scale, rowmax = scg.residual_norm(x, y, post=post, pre=pre, out_dtype=th, **p, **kw)
    assert scale is None and rowmax is None
    rx, rh = R.residual_norm(x.double(), y.double(), p, post, pre, **kw)
    ex, eh = R.residual_norm_error(x.double(), y.double(), p, post, pre, **kw)
    _within(xo, rx, ex + R.HALF[tx] * (rx.abs() + ex) + R.LEAST[tx], "xo")
    _within(h, rh, eh + R.HALF[th] * (rh.abs() + eh) + R.LEAST[th], "h")
    # quantised: exactly what the quantisers make of the float32 h
    _, h32, _, _ = scg.residual_norm(x, y, post=post, pre=pre, out_dtype=F32, want_x=False, **p, **kw)
    xo2, q, s, m = scg.residual_norm(x, y, post=post, pre=pre, out_dtype=torch.int8, want_rowmax=True, **p, **kw)
    qr, sr, mr = scg.quantize(h32, want_rowmax=True)
    assert torch.equal(xo, xo2) and torch.equal(q, qr) and torch.equal(s, sr) and torch.equal(m, mr)
    for t in (E4, E5):
        _, q, s, _ = scg.residual_norm(x, y, post=post, pre=pre, out_dtype=t, **p, **kw)
        qr, sr = scg.fp8_quantize(h32, dtype=t)
        assert torch.equal(s, sr)
        _same_bytes(q, qr)


def test_residual_norm_forms(scg):
    # no branch; xo alone; h alone; over x itself; two-dimensional; rows of a wider buffer from an odd element on
    _note("residual_norm forms")
    gen = _gen(1)
    x, y = _randn((6, 512), gen, BF16), _randn((6, 512), gen, BF16)
    g = _randn((512,), gen, BF16)
    xo, h, _, _ = scg.residual_norm(x, y, gate=g)
    a, none, _, _ = scg.residual_norm(x, y, gate=g, want_h=False)
    assert none is None and torch.equal(a, xo)
    none, b, _, _ = scg.residual_norm(x, y, gate=g, want_x=False)
    assert none is None and torch.equal(b, h)
    keep = x.clone()
    c, d, _, _ = scg.residual_norm(x, y, gate=g, inplace=True)
    assert c.data_ptr() == x.data_ptr() and torch.equal(c, xo) and torch.equal(d, h)
    x = keep
    e, f, _, _ = scg.residual_norm(x, res_scale=1.0)
    assert torch.equal(e, x)
    ref, err = R.normal(x.double(), 2, 1e-6), R.norm_error(x.double(), torch.zeros_like(x.double()), 2, 1e-6)[0]
    _within(f, ref, err + R.HALF[BF16] * (ref.abs() + err), "h of x alone")
    wide = torch.zeros((6, 1100), dtype=BF16, device="cuda")
    for off in (1, 4):
        vx, vy = wide[:, off:off + 512], wide[:, 520 + off:1032 + off]
        vx.copy_(x)
        vy.copy_(y)
        for t in (BF16, torch.int8, E4):
            u, v = (scg.residual_norm(s, t_, gate=g, out_dtype=t) for s, t_ in ((vx, vy), (x, y)))
            assert torch.equal(u[0], v[0])
            # (rows of another alignment may be summed in another order)
            if t == BF16:
                _within(u[1], v[1].double(), 2 * R.HALF[BF16] * v[1].double().abs() + 1e-4, "h of a view")
    for rows in (0, 3):
        z = torch.zeros((rows, 0 if rows else 8), device="cuda")
        xo, h, _, _ = scg.residual_norm(z, z)
        assert xo.shape == z.shape and h.shape == z.shape


@pytest.mark.parametrize("D", [64, 300, 777, 2500])
def test_int8_rows_of_special_values(scg, D):
    # NaN, infinities, zeros, the least and the largest floats: what the quantisers make of them
    _note("int8 rows of special values D=%d" % D)
    gen = _gen(D)
    x = _randn((12, D), gen)
    x[1, 3], x[2, 4], x[3, 5], x[4], x[5], x[6] = float("nan"), float("inf"), -float("inf"), 0.0, 1e-45, 3e38
    x[7, :2], x[8], x[9] = 1e-38, float("nan"), 2.0 ** -140
    _, q, s, m = scg.residual_norm(x, pre=0, out_dtype=torch.int8, want_rowmax=True)
    for a, b in zip((q, s, m), scg.quantize(x, want_rowmax=True)):
        assert torch.equal(a, b)
    for t in (E4, E5):
        _, q, s, _ = scg.residual_norm(x, pre=0, out_dtype=t)
        qr, sr = scg.fp8_quantize(x, dtype=t)
        assert torch.equal(s, sr)
        _same_bytes(q, qr)
    if D <= 256:
        f, ax = scg.rope_table([D])
        heads, pos = x.view(12, 1, D), torch.zeros(1, 12, dtype=torch.int32, device="cuda")
        turned = scg.rope(heads, pos, f, ax).transpose(0, 1).contiguous()
        for a, b in zip(scg.rope_quantize(heads, pos, f, ax, want_rowmax=True), scg.quantize(turned, want_rowmax=True)):
            assert torch.equal(a, b)


def test_residual_norm_over_rows_of_entries_in_turn(scg):
    # x as a view [batch, tokens, D] of a sequence-first buffer, written in place
    _note("residual_norm in place of a sequence-first buffer")
    gen = _gen(17)
    for T, B, D in ((33, 3, 1152), (40, 2, 777), (5, 4, 64)):
        buf = _randn((T, B, D + 8), gen, BF16)
        x, y, g = buf[:, :, :D].transpose(0, 1), _randn((B, T, D), gen, BF16), _randn((B, D), gen, BF16)
        keep, beside = x.clone(), buf[:, :, D:].clone()
        want = scg.residual_norm(keep, y, gate=g)
        xo, h, _, _ = scg.residual_norm(x, y, gate=g, inplace=True)
        assert xo is x and torch.equal(x, want[0]) and torch.equal(h, want[1]) and torch.equal(buf[:, :, D:], beside)


def test_residual_norm_special_values(scg):
    # NaN and infinities stay in their rows
    _note("residual_norm special values")
    gen = _gen(2)
    x, y = _randn((9, 300), gen), _randn((9, 300), gen)
    want = scg.residual_norm(x, y, pre=1)
    x[2, 7], y[4, 8], x[6, 0] = float("nan"), float("inf"), 1e38
    xo, h, _, _ = scg.residual_norm(x, y, pre=1)
    keep = [0, 1, 3, 5, 7, 8]
    assert torch.equal(xo[keep], want[0][keep]) and torch.equal(h[keep], want[1][keep])
    assert bool(torch.isnan(h[2]).all()) and not bool(torch.isfinite(h[4]).all())


@pytest.mark.parametrize("case", NORM, ids=lambda c: "%dx%dx%d_%d%d" % (c[0], c[1], c[2], c[7], c[8]))
def test_residual_norm_backward(scg, case):
    batch, rows, D, tx, ty, th, tp, post, pre, names, kw = case
    _note("residual_norm_backward %s" % (case,))
    xo, y, p, gen = _norm_inputs(case, 1)
    dxo, dh = _randn((batch, rows, D), gen, tx), _randn((batch, rows, D), gen, th)
    got = scg.residual_norm_backward(xo, y, dxo=dxo, dh=dh, post=post, pre=pre, **p, **kw)
    again = scg.residual_norm_backward(xo, y, dxo=dxo, dh=dh, post=post, pre=pre, **p, **kw)
    assert set(got) == {"x", "y"} | set(p) and all(torch.equal(got[k], again[k]) for k in got)
    _check_gradients(got, xo, y, p, dxo, dh, post, pre, kw)


def _check_gradients(got, xo, y, p, dxo, dh, post, pre, kw, tx=None):
    """Against the formula in 64 bits.  Bounds: an element of a norm's gradient r (d - n mean(d n) - mean(d)) has terms of size
    r |d|, r |n| mean|d n| and r mean|d|, each with DEPTH roundings and the error of n (norm_error); sums over rows have
    at most one rounding a row."""
    C, U = R.DEPTH, R.U
    x64, y64 = xo.double(), y.double()
    zero = torch.zeros_like(x64)
    rs = kw.get("res_scale", 1.0)

    def back(d, e_d, v, kind, eps=1e-6):
        if kind == 0:
            return d, e_d
        e_n, n, r = R.norm_error(v, zero, kind, eps)
        mean = lambda t: t.mean(-1, keepdim=True)  # noqa: E731
        g = d - n * mean(d * n) - (mean(d) if kind == 2 else 0.0)
        size = d.abs() + n.abs() * mean((d * n).abs()) + mean(d.abs())
        c = v - mean(v) if kind == 2 else v
        rel_r = C * U + r * torch.sqrt(mean((C * U * (c.abs() + mean(v.abs()))) ** 2))
        err = e_d + n.abs() * mean(e_d * n.abs()) + mean(e_d) + e_n * mean((d * n).abs()) + n.abs() * mean(d.abs() * e_n)
        return r * g, r * (err + (2 * C * U + rel_r) * size)

    def over(t, q):
        if q.dim() == 1:
            return t.sum((0, 1))
        return t.sum(1).reshape(q.shape)

    n_rows = xo.shape[0] * xo.shape[1]
    e_pre, n_pre, _ = R.norm_error(x64, zero, pre, 1e-6)
    w = kw.get("pre_offset", 0.0) + R.row(p["pre_weight"], x64) if "pre_weight" in p else torch.ones_like(x64)
    d64 = dh.double()
    g, e_g = back(d64 * w, 2 * U * (d64 * w).abs(), x64, pre)
    g, e_g = g + dxo.double(), e_g + 4 * U * (g.abs() + dxo.double().abs())
    n_row = n_rows + 8
    ref = {"x": (rs * g, abs(rs) * e_g + 2 * U * (rs * g).abs())}
    if "pre_weight" in p:
        ref["pre_weight"] = (d64 * n_pre, d64.abs() * e_pre)
    if "pre_bias" in p:
        ref["pre_bias"] = (d64, zero)
    gate = R.row(p["gate"], x64) if "gate" in p else torch.ones_like(x64)
    e_n, n, _ = R.norm_error(y64, zero, post, 1e-6)
    pw = kw.get("post_offset", 0.0) + R.row(p["post_weight"], x64) if "post_weight" in p else torch.ones_like(x64)
    pb = R.row(p["post_bias"], x64) if "post_bias" in p else zero
    u, e_u = n * pw + pb, e_n * pw.abs() + 4 * U * ((n * pw).abs() + pb.abs())
    du, e_du = g * gate, e_g * gate.abs() + 2 * U * (g * gate).abs()
    if "gate" in p:
        ref["gate"] = (g * u, e_g * u.abs() + g.abs() * e_u)
    if "post_weight" in p:
        ref["post_weight"] = (du * n, e_du * n.abs() + du.abs() * e_n)
    if "post_bias" in p:
        ref["post_bias"] = (du, e_du)
    ref["y"] = back(du * pw, e_du * pw.abs() + 2 * U * (du * pw).abs(), y64, post)
    for k, (v, e) in ref.items():
        if k not in got:
            continue
        if k in p:
            e = over(e + (n_row + 4) * U * v.abs(), p[k])
            _within(got[k], over(v, p[k]), e + 1e-30, k)
        else:
            t, g = got[k].dtype, got[k].double()
            if t == F16:   # 65504 is the largest, its step 32: from 65504 + 16 on the nearest float16 is an infinity
                g = torch.where(torch.isinf(g) & (v.abs() + e >= 65520.0) & (g.sign() == v.sign()), v, g)
            _within(g, v, e + R.HALF[t] * (v.abs() + e) + R.LEAST[t], k)


@pytest.mark.parametrize("names,kw", [((), {}), (("post_weight", "pre_weight"), dict(post_offset=1.0)), (("post_bias",), {})], ids=["bare", "weights", "bias"])
@pytest.mark.parametrize("D", [3, 64, 768, 777, 1024, 1152, 1300, 2500, 4100])
def test_residual_norm_backward_two_layer_norms_without_gate(scg, D, names, kw):
    # dh with a mean: the pre norm's gradient takes mean(d) off every element, and only off those of the row
    _note("residual_norm_backward two LayerNorms D=%d %s" % (D, names))
    for tx, rows in ((F32, 5), (BF16, 19)):
        case = (2, rows, D, tx, tx, tx, F32, 2, 2, names, kw)
        xo, y, p, gen = _norm_inputs(case, 4)
        dxo, dh = _randn((2, rows, D), gen, tx), (_randn((2, rows, D), gen) + 1.5).to(tx)
        got = scg.residual_norm_backward(xo, y, dxo=dxo, dh=dh, post=2, pre=2, **p, **kw)
        _check_gradients(got, xo, y, p, dxo, dh, 2, 2, kw)


def test_residual_norm_backward_forms(scg):
    # one gradient absent; parameters' gradients not wanted; no branch; many rows and chunks; no rows at all
    _note("residual_norm_backward forms")
    case = (2, 700, 256, F32, BF16, BF16, F32, 1, 2, ALL, {})
    xo, y, p, gen = _norm_inputs(case, 2)
    dxo, dh = _randn(tuple(xo.shape), gen), _randn(tuple(xo.shape), gen, BF16)
    zero = torch.zeros_like
    full = scg.residual_norm_backward(xo, y, dxo=dxo, dh=dh, post=1, pre=2, **p)
    _check_gradients(full, xo, y, p, dxo, dh, 1, 2, {})
    for a, b in ((dict(dh=dh), dict(dxo=zero(dxo), dh=dh)), (dict(dxo=dxo), dict(dxo=dxo, dh=zero(dh)))):
        ga, gb = (scg.residual_norm_backward(xo, y, post=1, pre=2, **p, **k) for k in (a, b))
        assert all(torch.equal(ga[k], gb[k]) for k in gb)
    some = scg.residual_norm_backward(xo, y, dxo=dxo, dh=dh, post=1, pre=2, want_params=False, want_x=False, **p)
    assert set(some) == {"y"} and torch.equal(some["y"], full["y"])
    alone = scg.residual_norm_backward(xo, dxo=dxo, dh=dh, pre=2, pre_weight=p["pre_weight"], pre_bias=p["pre_bias"])
    # (another kernel than the one with a norm behind the branch: the same sums, in roundings of its own)
    assert set(alone) == {"x", "pre_weight", "pre_bias"}
    _check_gradients(alone, xo, y, {k: p[k] for k in ("pre_weight", "pre_bias")}, dxo, dh, 0, 2, {})
    none = scg.residual_norm_backward(xo[:, :0], y[:, :0], dxo=dxo[:, :0], dh=dh[:, :0], post=1, pre=2, **p)
    assert all(bool((none[k] == 0).all()) for k in p) and none["x"].shape == (2, 0, 256)


def test_residual_norm_backward_in_place(scg):
    # dx over dxo, rows side by side and by several waves, four elements at a time and one
    _note("residual_norm_backward in place")
    for rows, D in ((701, 256), (530, 1152), (300, 2100), (67, 777)):
        xo, y, p, gen = _norm_inputs((1, rows, D, BF16, BF16, BF16, F32, 1, 2, ALL, {}), 3)
        dxo, dh = _randn((1, rows, D), gen, BF16), _randn((1, rows, D), gen, BF16)
        want = scg.residual_norm_backward(xo, y, dxo=dxo, dh=dh, post=1, pre=2, **{**p, "gate": None})
        d = scg._lib.ScNormDesc(batch=1, rows=rows, D=D, post=1, pre=2, typeX=1, typeY=1, typeP=0, typeH=1, eps_post=1e-6, eps_pre=1e-6, scale_res=1.0,
                           ldx=D, ldy=D, ldxo=D, ldh=D, lddxo=D, lddy=D)
        dy = torch.empty_like(y)
        w = {k: q.reshape(-1) for k, q in p.items()}
        assert all(q.numel() == D for q in w.values())
        rc = scg._lib.sc_residual_norm_backward(d, xo.data_ptr(), y.data_ptr(), w["post_weight"].data_ptr(), w["post_bias"].data_ptr(), 0,
                                                w["pre_weight"].data_ptr(), dxo.data_ptr(), dh.data_ptr(), dxo.data_ptr(), dy.data_ptr(), 0, 0,
                                                0, 0, 0, 0, 0, 0)
        assert rc == 0 and torch.equal(dxo, want["x"]) and torch.equal(dy, want["y"])


def test_residual_norm_backward_against_differences(scg):
    """The directional derivative of the kernel's own forward pass in float32.  A central difference of step t is off by
    t^2/6 of the third derivative, taken from differences of steps t and 2t in 64 bits, and by the outputs' errors over t."""
    _note("residual_norm_backward against differences")
    batch, rows, D = 2, 3, 200
    case = (batch, rows, D, F32, F32, F32, F32, 2, 1, ALL, {})
    x, y, p, gen = _norm_inputs(case, 3)
    x[0, 0], y[0, 0] = _randn((D,), gen), _randn((D,), gen)
    a, b = _randn((batch, rows, D), gen), _randn((batch, rows, D), gen)
    kw = dict(post=2, pre=1, **p)
    xo = scg.residual_norm(x, y, **kw)[0]
    grads = scg.residual_norm_backward(xo, y, dxo=a, dh=b, **kw)
    vx, vy, t = _randn(tuple(x.shape), gen), _randn(tuple(y.shape), gen), 2.0 ** -7

    def loss(own, h):
        xx, yy = x + h * vx, y + h * vy
        o, n = scg.residual_norm(xx, yy, **kw)[:2] if own else R.residual_norm(x.double() + h * vx.double(), y.double() + h * vy.double(), p, 2, 1)
        return float((o.double() * a.double()).sum() + (n.double() * b.double()).sum())

    slope = float((grads["x"].double() * vx.double()).sum() + (grads["y"].double() * vy.double()).sum())
    own = (loss(True, t) - loss(True, -t)) / (2 * t)
    d1, d2 = ((loss(False, s) - loss(False, -s)) / (2 * s) for s in (t, 2 * t))
    curve = abs(d2 - d1)                      # 3 (t^2 / 6) f''': three times what the step t is off by, to leading order
    ex, eh = R.residual_norm_error(x.double(), y.double(), p, 2, 1)
    # the inputs' own rounding at x + h v: half a step each, as large as a quarter of their share in the bounds
    noise = 2 * float((ex * a.double().abs()).sum() + (eh * b.double().abs()).sum()) / t
    assert abs(own - slope) <= curve + noise + 1e-3 * abs(slope) * R.U
    assert abs(d1 - slope) <= curve + noise


# ---------------------------------------------------------------- rotary positions

ROPE = [
    # batch, T, H, D, dims, x, out, interleaved, inverse
    (1, 1, 1, 2, [2], F32, F32, False, False),
    (1, 1, 32, 128, [32, 48, 48], BF16, BF16, False, False),
    (2, 13, 3, 64, [16, 24, 24], F32, F32, True, False),
    (1, 50, 5, 72, [36, 36], F16, F32, False, True),
    (3, 7, 4, 80, [10, 14, 6], F32, BF16, True, True),
    (1, 9, 2, 256, [64, 96, 96], BF16, BF16, False, False),
    (2, 5, 9, 65, [6, 10], F32, F32, False, False),
    (1, 33, 1, 7, [2], BF16, F16, True, False),
    (1, 4, 3, 96, [], F32, F32, False, False),
    (2, 300, 12, 64, [64], BF16, BF16, True, True),
]


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("case", ROPE, ids=lambda c: "%dx%dx%dx%d" % c[:4])
def test_rope(scg, case, shared):
    batch, T, H, D, dims, tx, to, inter, inv = case
    _note("rope %s shared=%s" % (case, shared))
    gen = _gen(T * 100 + D)
    x = _randn((batch, T, H, D), gen, tx)
    freq, axis = scg.rope_table(dims, shared=shared)
    nb = batch if shared else 1
    pos = torch.randint(-2 ** 31, 2 ** 31 - 1, (nb, max(len(dims), 1), T), generator=gen, device="cuda", dtype=torch.int64).to(torch.int32)
    pos[..., ::2] %= 1000
    got = scg.rope(x, pos if shared else pos[0], freq, axis, interleaved=inter, inverse=inv, out_dtype=to)
    ref, mag = R.rope(x, pos, freq, axis, inter, inv)
    # the reference's own angle in 64 bits, up to 2^31 radians, is off by up to 2^-22; kernel: cosine and sine off by 4 float32
    # roundings (argument and function), products and sum 3 more
    tol = (8 * R.U + (2.0 ** -21)) * mag + R.HALF[to] * ref.abs() + R.LEAST[to]
    _within(got, ref, tol, "rope")
    near = slice(0, None, 2)                 # tokens below 1000: the reference's angle is exact to 2^-43
    _within(got[:, near], ref[:, near], (8 * R.U * mag + R.HALF[to] * (ref.abs() + 8 * R.U * mag) + R.LEAST[to])[:, near], "near tokens")
    if tx == to:
        y = x.clone()
        assert torch.equal(scg.rope(y, pos if shared else pos[0], freq, axis, interleaved=inter, inverse=inv, out=y), got)
    # int8 rows by head: what the quantiser makes of the float32 result
    if not inv:
        f32 = scg.rope(x, pos if shared else pos[0], freq, axis, interleaved=inter, out_dtype=F32)
        Q, s, m = scg.rope_quantize(x, pos if shared else pos[0], freq, axis, interleaved=inter, want_rowmax=True)
        q, sr, mr = scg.quantize(f32.transpose(1, 2).contiguous().reshape(batch * H, T, D), want_rowmax=True)
        assert torch.equal(Q.reshape(q.shape), q) and torch.equal(s.reshape(sr.shape), sr) and torch.equal(m.reshape(mr.shape), mr)


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
def test_rope_of_unit_vectors(scg, inter, inverse):
    """(1, 0) turns to the cosine and the sine themselves: each within two steps of float32 (the function) and a rounding, also where
    one of the two is near zero and a rounding of the angle would be large beside it.  The reference's own angle, below 1000 in 64
    bits, is off by 2^-43."""
    _note("rope of unit vectors")
    freq, axis = scg.rope_table([128])
    pos = torch.arange(1000, dtype=torch.int32, device="cuda")[None]
    x = torch.zeros((1000, 2, 128), device="cuda")
    x[..., slice(0, None, 2) if inter else slice(0, 64)] = 1.0
    ref, _ = R.rope(x[None], pos[None], freq, axis, inter, inverse)
    for big in (x, x[:3]):
        n = big.shape[0]
        got = scg.rope(big.contiguous(), pos[:, :n], freq, axis, interleaved=inter, inverse=inverse)
        _within(got[None], ref[:, :n], 6 * R.U * ref[:, :n].abs() + 2.0 ** -41, "turned")


def test_rope_there_and_back_and_views(scg):
    _note("rope views")
    gen = _gen(4)
    T, Hq, Hk, D = 37, 6, 2, 64
    freq, axis = scg.rope_table([16, 24, 24])
    pos = torch.randint(0, 5000, (3, T), generator=gen, device="cuda", dtype=torch.int32)
    for off, inter in ((0, False), (0, True), (1, False), (1, True), (4, True)):
        buf = torch.zeros(T * (Hq + 2 * Hk) * D + off, dtype=BF16, device="cuda")
        qkv = buf[off:].view(T, Hq + 2 * Hk, D)
        qkv.copy_(_randn(tuple(qkv.shape), gen, BF16))
        keep = qkv.clone()
        turned = scg.rope(qkv[:, :Hq + Hk], pos, freq, axis, interleaved=inter)
        assert torch.equal(turned, scg.rope(keep[:, :Hq + Hk].contiguous(), pos, freq, axis, interleaved=inter))
        scg.rope(qkv[:, :Hq + Hk], pos, freq, axis, interleaved=inter, out=qkv[:, :Hq + Hk])
        assert torch.equal(qkv[:, :Hq + Hk], turned) and torch.equal(qkv[:, Hq + Hk:], keep[:, Hq + Hk:])
    # all heads by one thread, and a result that is stored past the caches, over its source
    far = torch.randint(0, 5000, (3, 9000), generator=gen, device="cuda", dtype=torch.int32)
    for inter in (False, True):
        x = _randn((9000, 131, D), gen, BF16)
        few = scg.rope(x[:300], far[:, :300], freq, axis, interleaved=inter), scg.rope(x[8700:], far[:, 8700:], freq, axis, interleaved=inter)
        scg.rope(x, far, freq, axis, interleaved=inter, out=x)
        assert torch.equal(x[:300], few[0]) and torch.equal(x[8700:], few[1])
    # the inverse is the transpose: <rope(x), g> = <x, rope_inverse(g)>
    x, g = _randn((T, Hq, D), gen), _randn((T, Hq, D), gen)
    l = (scg.rope(x, pos, freq, axis).double() * g.double()).sum()
    r = (x.double() * scg.rope(g, pos, freq, axis, inverse=True).double()).sum()
    assert abs(float(l - r)) <= 16 * R.U * float((x.double().abs() * g.double().abs()).sum() * 2)
    # an axis that is not there does not turn
    bad = axis.clone()
    bad[3], bad[5] = 3, -1
    ref, mag = R.rope(x[None], pos[None], freq, bad, False, False)
    _within(scg.rope(x, pos, freq, bad)[None], ref, 8 * R.U * mag + 1e-30, "axes outside")


def test_more_entries_than_a_grid_holds(scg):
    _note("40000 entries")
    gen, n = _gen(35), 40000
    x = _randn((n, 2, 136), gen)
    for block, per in ((0, 1), (1, 128), (2, 1)):
        Q, s = scg.fp8_quantize(x, block=block)
        Qr, sr = R.fp8_quantize32(x.transpose(1, 2).contiguous() if block == 2 else x, E4, per)
        assert torch.equal(s, sr)
        _same_bytes(Q, Qr)
    for M in (2, 17):
        A, sA = _operand((n, M, 130), gen, E4, 1)
        for lead in ((n,), ()):
            B, sB = _operand((*lead, 5, 130), gen, E4, 1)
            got = scg.fp8_gemm(A, sA, B, sB)
            ref, mag = R.fp8_gemm(A, sA, 1, B, sB, 1)
            _within(got, ref, R.gemm_tolerance(mag, 130, BF16, ref), "product")
    xo, y, p, gen = _norm_inputs((n, 2, 64, F32, F32, F32, F32, 2, 2, ALL, {}), 1)
    _, h, _, _ = scg.residual_norm(xo, y, post=2, pre=2, **p)
    ref, err = (f(xo.double(), y.double(), p, 2, 2)[1] for f in (R.residual_norm, R.residual_norm_error))
    _within(h, ref, err + R.HALF[F32] * (ref.abs() + err) + R.LEAST[F32], "h")
    assert torch.equal(scg.residual_norm(xo, y, post=2, pre=2, out_dtype=torch.int8, **p)[1], scg.quantize(h)[0])
    dxo, dh = _randn(tuple(xo.shape), gen), _randn(tuple(xo.shape), gen)
    _check_gradients(scg.residual_norm_backward(xo, y, dxo=dxo, dh=dh, post=2, pre=2, **p), xo, y, p, dxo, dh, 2, 2, {})
    f, ax = scg.rope_table([64])
    x = _randn((n, 3, 2, 64), gen)
    pos = torch.randint(0, 1000, (n, 1, 3), generator=gen, device="cuda", dtype=torch.int32)
    ref, mag = R.rope(x, pos, f, ax, False, False)
    _within(scg.rope(x, pos, f, ax), ref, 8 * R.U * mag + 1e-30, "rope")


# ---------------------------------------------------------------- together, streams, graphs

def _block(scg, s):
    """One seam of a block and the attention scores behind it: norm to fp8, product, rotary positions to int8, sc_gemm."""
    xo, h, sh, _ = scg.residual_norm(s["x"], s["y"], pre=scg.SC_NORM_LAYER, gate=s["gate"], pre_weight=s["scale"],
                                     pre_bias=s["shift"], pre_offset=1.0, out_dtype=E4)
    qk = scg.fp8_gemm(h, sh, s["W"], s["sW"], bias=s["b"], out_dtype=BF16)
    nb, T, n = qk.shape
    H, D = s["H"], s["D"]
    qk = qk.view(nb, T, 2 * H, D)
    Q, sq, _ = scg.rope_quantize(qk[:, :, :H], s["pos"], s["freq"], s["axis"])
    K, sk, _ = scg.rope_quantize(qk[:, :, H:], s["pos"], s["freq"], s["axis"])
    L = torch.full((nb * H, T), 32, dtype=torch.int32, device="cuda")
    scores, counts = scg.gemm(Q.view(nb * H, T, D), sq.view(nb * H, T), K.view(nb * H, T, D), sk.view(nb * H, T), L, L_max=32,
                              seed=3, want_counts=True)
    return {"xo": xo, "h": h, "sh": sh, "qk": qk, "Q": Q, "sq": sq, "K": K, "sk": sk, "scores": scores, "counts": counts}


def _block_state(scg, gen):
    nb, T, E, H, D = 2, 50, 384, 3, 64
    W, sW = scg.fp8_quantize(0.05 * _randn((2 * H * D, E), gen), block=scg.SC_BLOCK_128X128)
    freq, axis = scg.rope_table([32, 32])
    pos = torch.stack([torch.arange(T, device="cuda") // 10, torch.arange(T, device="cuda") % 10]).to(torch.int32)
    return {"x": _randn((nb, T, E), gen), "y": _randn((nb, T, E), gen, BF16), "gate": _randn((nb, E), gen), "scale": 0.1 * _randn((nb, E), gen),
            "shift": _randn((nb, E), gen), "W": W, "sW": sW, "b": _randn((2 * H * D,), gen), "pos": pos, "freq": freq, "axis": axis,
            "H": H, "D": D}


def test_a_block_together(scg, oracle_mod):
    _note("a block together")
    s = _block_state(scg, _gen(9))
    r = _block(scg, s)
    h32 = scg.residual_norm(s["x"], s["y"], gate=s["gate"], pre_weight=s["scale"], pre_bias=s["shift"], pre_offset=1.0)[1]
    hr, shr = R.fp8_quantize32(h32.cpu(), E4, 1)
    assert torch.equal(r["sh"].cpu(), shr)
    _same_bytes(r["h"].cpu(), hr)
    ref, mag = R.fp8_gemm(r["h"], r["sh"], 1, s["W"], s["sW"], 128, s["b"])
    _within(r["qk"].flatten(2), ref, R.gemm_tolerance(mag, 384, BF16, ref), "qk")
    turned, mag = R.rope(r["qk"], s["pos"][None], s["freq"], s["axis"], False, False)
    deq = torch.cat([(r[k].double() * r[n].double()[..., None]).transpose(1, 2) for k, n in (("Q", "sq"), ("K", "sk"))], 2)
    step = torch.cat([r["sq"], r["sk"]], 1).double().transpose(1, 2)[..., None]
    _within(deq, turned, 0.5 * step * (1 + 1e-5) + 16 * R.U * mag, "int8 heads")
    for i in (0, 5):
        c, _ = oracle_mod.sc_gemm(*(r[k].flatten(0, 1)[i].cpu().numpy() for k in ("Q", "K", "sq", "sk")), np.full(50, 32, np.int32), 32, 0, 3)
        assert np.array_equal(r["counts"][i].cpu().numpy(), c)


def _grads(scg, s):
    return scg.residual_norm_backward(s["x"], s["y"], dxo=s["x"], dh=s["y"], gate=s["gate"], pre_weight=s["scale"], pre_bias=s["shift"],
                                      pre_offset=1.0)


def test_another_stream_and_two_at_once(scg):
    _note("streams")
    s1, s2 = _block_state(scg, _gen(10)), _block_state(scg, _gen(11))
    want = [{**_block(scg, s), **_grads(scg, s)} for s in (s1, s2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(3):
        for k, s in enumerate((s1, s2)):
            with torch.cuda.stream(streams[k]):
                got[k].append({**_block(scg, s), **_grads(scg, s)})
    torch.cuda.synchronize()
    for k in range(2):
        for r in got[k]:
            for n in want[k]:
                assert torch.equal(r[n].view(torch.uint8), want[k][n].view(torch.uint8)), n
    # the stream given by name, from the default one
    out = scg.fp8_gemm(want[0]["h"], want[0]["sh"], s1["W"], s1["sW"], bias=s1["b"], stream=streams[0])
    g = scg.residual_norm_backward(s1["x"], s1["y"], dxo=s1["x"], dh=s1["y"], gate=s1["gate"], stream=streams[0])
    streams[0].synchronize()
    assert torch.equal(out.view_as(want[0]["qk"]), want[0]["qk"]) and torch.isfinite(g["x"]).all()


def _long_work():
    """Some 20 ms of products on the current stream."""
    a = torch.ones((8192, 8192), dtype=BF16, device="cuda")
    for _ in range(30):
        a = torch.mm(a, a.clone())
    return a


def _calls(scg, gen):
    """A call of each operator that makes tensors, as functions of the stream, with results of more than a megabyte."""
    x, y = _randn((1100, 1152), gen), _randn((1100, 1152), gen)
    A, sA = _operand((600, 8192), gen, E4, 1)
    B, sB = _operand((700, 8192), gen, E4, 128)
    A2, sA2 = _operand((128, 8192), gen, E4, 1)
    B2, sB2 = _operand((128, 8192), gen, E4, 128)
    f, ax = scg.rope_table([64])
    pos = torch.arange(1100, dtype=torch.int32, device="cuda")[None]
    heads = x.view(1100, 18, 64)
    w = _randn((1152,), gen)
    return [
        lambda s: scg.fp8_quantize(x, stream=s),
        lambda s: (scg.fp8_gemm(A, sA, B, sB, out_dtype=F32, stream=s),),
        lambda s: (scg.fp8_gemm(A2, sA2, B2, sB2, stream=s),),                      # sums of blocks in a workspace
        lambda s: scg.residual_norm(x, y, out_dtype=torch.int8, want_rowmax=True, stream=s),
        lambda s: tuple(scg.residual_norm_backward(x, y, dxo=y, dh=x, gate=w, pre_weight=w, stream=s).values()),
        lambda s: (scg.rope(heads, pos, f, ax, stream=s),),
        lambda s: scg.rope_quantize(heads, pos, f, ax, want_rowmax=True, stream=s),
    ]


def test_memory_of_a_given_stream(scg):
    # what a call makes for another stream must not lie where work that waits on the current one still writes
    _note("memory of a given stream")
    side = torch.cuda.Stream()
    for call in _calls(scg, _gen(30)):
        want = [t for t in call(None) if t is not None]
        torch.cuda.synchronize()
        old = [torch.empty_like(t) for t in want] + [torch.empty(4 << 20, dtype=torch.uint8, device="cuda") for _ in range(4)]
        work = _long_work()
        for t in old:
            t.view(torch.uint8).fill_(0x3C)              # (behind that work, when `side` has long been done)
        left = {t.data_ptr() for t in old}
        del old, t
        got = [t for t in call(side) if t is not None]
        assert not left & {t.data_ptr() for t in got}
        torch.cuda.synchronize()
        assert len(got) == len(want) and all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, want))
        del work


def test_stream_of_another_device(scg):
    _note("stream of another device")
    there = types.SimpleNamespace(device=torch.device("cuda", torch.cuda.device_count()), cuda_stream=0)
    for call in _calls(scg, _gen(32)):
        with pytest.raises(ValueError):
            call(there)


def test_workspace_of_another_stream(scg):
    # a workspace that was made on one stream and is used and grown on another is not given away before that one is done
    _note("workspace of another stream")
    gen = _gen(31)
    A, sA = _operand((100, 8192), gen, E4, 1)
    B, sB = _operand((128, 8192), gen, E4, 128)
    A2, sA2 = _operand((128, 16384), gen, E4, 1)
    B2, sB2 = _operand((256, 16384), gen, E4, 128)
    want = scg.fp8_gemm(A, sA, B, sB), scg.fp8_gemm(A2, sA2, B2, sB2)
    side = torch.cuda.Stream()
    for given in (False, True):
        ws = scg.Workspace(2 << 20)
        for k in range(2):
            torch.cuda.synchronize()
            first = ws._buf.data_ptr(), ws._buf.numel()
            with torch.cuda.stream(side):
                work = _long_work()
                one = None if given else scg.fp8_gemm(A, sA, B, sB, workspace=ws)
            if given:
                one = scg.fp8_gemm(A, sA, B, sB, workspace=ws, stream=side)
            assert ws._buf.data_ptr() == first[0]
            if k == 0:
                with torch.cuda.stream(side):
                    two = scg.fp8_gemm(A2, sA2, B2, sB2, workspace=ws)
                assert ws._buf.data_ptr() != first[0]
            else:
                two = want[1]
                ws = None
            t = torch.empty(first[1], dtype=torch.uint8, device="cuda")
            assert t.data_ptr() != first[0] or side.query()          # (once all is done there it may be given away)
            t.fill_(0x3C)
            torch.cuda.synchronize()
            assert torch.equal(one, want[0]) and torch.equal(two, want[1])
            del t, work


def test_writes_over_saved_tensors_are_seen(scg):
    # a tensor that autograd has saved and that a call writes over: the backward pass raises, and uses no changed value
    _note("writes over saved tensors")
    gen = _gen(33)
    A, sA = _operand((64, 128), gen, E4, 1)
    freq, axis = scg.rope_table([64])
    pos = torch.arange(64, dtype=torch.int32, device="cuda")[None]
    calls = [lambda t: scg.residual_norm(t, t.clone(), inplace=True), lambda t: scg.fp8_gemm(A, sA, A, sA, out=t),
             lambda t: scg.rope(t.view(64, 1, 64), pos, freq, axis, out=t.view(64, 1, 64))]
    for call in calls:
        w, t = torch.ones(64, 64, device="cuda", requires_grad=True), _randn((64, 64), gen)
        loss = (w * t).sum()
        call(t)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
        with torch.inference_mode():
            call(torch.zeros(64, 64, device="cuda"))
    # parameters without recording, and their gradients asked for by name
    w = torch.ones(64, device="cuda", requires_grad=True)
    with torch.no_grad():
        xo, h, _, _ = scg.residual_norm(t, pre_weight=w)
    assert not h.requires_grad and set(scg.residual_norm_backward(xo, dh=h, pre_weight=w)) == {"x", "pre_weight"}


def test_graph_replays(scg):
    _note("graphs")
    s = _block_state(scg, _gen(12))
    fresh = [_block_state(scg, _gen(20 + k)) for k in range(3)]
    big = {"A": None}
    A, sA = _operand((300, 1100), _gen(13), E4, 1)
    B, sB = _operand((200, 1100), _gen(14), E4, 128)
    big.update(A=A, B=B)

    def work():
        return {**_block(scg, s), **_grads(scg, s), "odd": scg.fp8_gemm(A, sA, B, sB), "turned": scg.fp8_quantize(s["x"][0], block=2)[0]}

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = work()
    for f in fresh:
        for k in ("x", "y", "gate", "scale", "shift", "b"):
            s[k].copy_(f[k])
        graph.replay()
        torch.cuda.synchronize()
        eager = work()
        torch.cuda.synchronize()
        for n in eager:
            assert torch.equal(held[n].view(torch.uint8), eager[n].view(torch.uint8)), n


def test_a_given_stream_in_a_graph(scg):
    _note("a given stream in a graph")
    gen = _gen(36)
    A, sA = _operand((128, 8192), gen, E4, 1)
    B, sB = _operand((128, 8192), gen, E4, 128)
    x = _randn((500, 1152), gen)
    want = scg.fp8_gemm(A, sA, B, sB), scg.residual_norm(x, x)[1]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        a, b = scg.fp8_gemm(A, sA, B, sB, stream=side), scg.residual_norm(x, x, stream=side)[1]
        torch.cuda.current_stream().wait_stream(side)
        c = a * 2
    for _ in range(3):
        for t in (a, b, c):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        eager = scg.fp8_gemm(A, sA, B, sB)
        assert torch.equal(a, eager) and torch.equal(a, want[0]) and torch.equal(b, want[1]) and torch.equal(c, want[0] * 2)


def test_refusals_of_tensors(scg):
    _note("refusals")
    z = lambda *s, t=F32: torch.zeros(s, device="cuda").to(t)  # noqa: E731
    for bad in (lambda: scg.fp8_quantize(z(4, 64, t=torch.float64)), lambda: scg.fp8_quantize(z(4, 64), dtype=torch.int8),
                lambda: scg.fp8_gemm(z(4, 64), z(4, 1), z(4, 64, t=E4), z(4, 1)),
                lambda: scg.fp8_gemm(z(4, 64, t=E4), z(4, 1, t=BF16), z(4, 64, t=E4), z(4, 1)),
                lambda: scg.residual_norm(z(4, 64), z(4, 64), gate=z(64), pre_weight=z(64, t=BF16)),
                lambda: scg.residual_norm_backward(z(4, 64), dxo=z(4, 64, t=BF16)),
                lambda: scg.rope(z(4, 2, 64), z(1, 4), z(32), z(32))):
        with pytest.raises(TypeError):
            bad()
    i32, f64 = torch.int32, torch.float64
    for bad in (lambda: scg.fp8_quantize(z(64, 4).t()), lambda: scg.fp8_quantize(torch.zeros(4, 64)), lambda: scg.fp8_quantize(z(64)),
                lambda: scg.fp8_gemm(z(4, 64, t=E4), z(4, 1), z(4, 65, t=E4), z(4, 1)),
                lambda: scg.fp8_gemm(z(4, 64, t=E4), z(4, 2), z(4, 64, t=E4), z(4, 1)),
                lambda: scg.fp8_gemm(z(4, 64, t=E4), z(4, 1), z(4, 64, t=E4), z(4, 1), out=z(4, 5)),
                lambda: scg.fp8_gemm(z(4, 64, t=E4), z(4, 1), z(2, 4, 64, t=E4), z(2, 4, 1)),
                lambda: scg.residual_norm(z(4, 64), z(4, 65)), lambda: scg.residual_norm(z(4, 64), gate=z(4, 64)),
                lambda: scg.residual_norm(z(4, 64), want_rowmax=True), lambda: scg.residual_norm(z(4, 64), want_x=False, inplace=True),
                lambda: scg.residual_norm_backward(z(4, 64), dh=z(4, 64), gate=z(64)),
                lambda: scg.rope(z(4, 2, 64), z(1, 5, t=i32), z(32, t=f64), z(32, t=i32)),
                lambda: scg.rope(z(4, 2, 64), z(1, 4, t=i32), z(32, t=f64), z(31, t=i32)), lambda: scg.rope_table([3])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: scg.rope(z(4, 2, 64), z(1, 4, t=i32), z(33, t=f64), z(33, t=i32)),
                lambda: scg.rope(z(4, 2, 300), z(1, 4, t=i32), z(32, t=f64), z(32, t=i32)),
                lambda: scg.residual_norm(z(2, 16385)), lambda: scg.residual_norm(z(4, 64), pre=3),
                lambda: scg.residual_norm(z(4, 64), z(4, 64), post_weight=z(64)),
                lambda: scg.residual_norm(z(4, 64), pre_eps=0.0), lambda: scg.fp8_quantize(z(4, 64), block=3),
                lambda: scg.rope(z(4, 2, 64), z(1, 4, t=i32), z(32, t=f64), z(32, t=i32), out=z(1, 2, 64).expand(4, 2, 64))):
        with pytest.raises(scg.ScError):
            bad()
