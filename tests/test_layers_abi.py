"""The layer operators' descriptors and argument checks, through the C ABI on the CPU: nothing here launches a kernel."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 40                          # never dereferenced: every call returns early


@pytest.fixture(scope="module")
def lib():
    import paper_2609_32922_amd._lib as L
    if not os.path.exists(L.LIB_PATH):
        from paper_2609_32922_amd import build
        build.build()
    return L


@pytest.mark.parametrize("struct,mirror", [("sc_fp8_gemm_desc", "ScFp8GemmDesc"), ("sc_norm_desc", "ScNormDesc"), ("sc_rope_desc", "ScRopeDesc")])
def test_descriptors_match_the_header(lib, struct, mirror, tmp_path):
    D = getattr(lib, mirror)
    fields = "\n".join('printf("%s %%zu\\n", offsetof(%s, %s));' % (n, struct, n) for n, _ in D._fields_)
    src = tmp_path / "d.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "scgemm.h"\nint main(void) {\nprintf("size %%zu\\n", sizeof(%s));\n%s\nreturn 0;\n}\n'
                   % (struct, fields))
    exe = tmp_path / "d"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = dict(ln.split() for ln in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines())
    assert int(got["size"]) == ctypes.sizeof(D)
    for n, _ in D._fields_:
        assert int(got[n]) == getattr(D, n).offset, n


def test_numbers_match_the_header(lib, tmp_path):
    names = [n for n in dir(lib) if n.startswith("SC_") and isinstance(getattr(lib, n), int)]
    src = tmp_path / "n.c"
    src.write_text('#include <stdio.h>\n#include "scgemm.h"\nint main(void) {\n%s\nreturn 0;\n}\n'
                   % "\n".join('printf("%s %%lld\\n", (long long)%s);' % (n, n) for n in names))
    exe = tmp_path / "n"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = dict(ln.split() for ln in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines())
    assert {n: int(v) for n, v in got.items()} == {n: getattr(lib, n) for n in names}
    assert lib.strerror(lib.SC_ERR_TYPE).startswith("SC_ERR_TYPE")


# batch, rows, K, typeX, X, ldx, strideX, typeQ, block, Q, ldq, strideQ, scale, lds, strideS
QUANT = dict(batch=2, rows=200, K=300, typeX=0, X=FAKE, ldx=300, strideX=60000, typeQ=3, block=0, Q=FAKE, ldq=300, strideQ=60000,
             scale=FAKE, lds=3, strideS=600)


@pytest.mark.parametrize("change,code", [
    (dict(batch=-1), "SHAPE"), (dict(rows=-1), "SHAPE"), (dict(K=-1), "SHAPE"), (dict(K=(1 << 20) + 1, ldx=1 << 21, ldq=1 << 21), "SHAPE"),
    (dict(typeX=3), "TYPE"), (dict(typeX=-1), "TYPE"), (dict(typeQ=0), "TYPE"), (dict(typeQ=5), "TYPE"), (dict(block=3), "TYPE"), (dict(block=-1), "TYPE"),
    (dict(ldx=299), "STRIDE"), (dict(ldq=299), "STRIDE"), (dict(lds=2), "STRIDE"), (dict(strideX=-1), "STRIDE"), (dict(strideQ=59999), "STRIDE"),
    (dict(strideS=599), "STRIDE"), (dict(block=2), "STRIDE"), (dict(X=0), "NULL"), (dict(Q=0), "NULL"), (dict(scale=0), "NULL"),
    (dict(X=FAKE + 2), "STRIDE"), (dict(scale=FAKE + 2), "STRIDE"), (dict(typeX=1, X=FAKE + 1), "STRIDE"),
    (dict(batch=0, X=0), "OK"), (dict(rows=0, X=0), "OK"), (dict(K=0, X=0), "OK"),
])
def test_fp8_quantize_refuses(lib, change, code):
    a = {**QUANT, **change}
    assert lib.sc_fp8_quantize(*a.values(), 0) == getattr(lib, "SC_OK" if code == "OK" else "SC_ERR_" + code)


def _gemm(lib, **kw):
    d = lib.ScFp8GemmDesc()
    base = dict(batch=2, M=64, N=48, K=300, lda=300, ldb=300, ldo=48, strideA=64 * 300, strideB=0, strideO=64 * 48, ldsA=3, ldsB=3,
                strideSA=192, strideSB=0, typeA=3, typeB=4, rowsA=1, rowsB=128, typeO=1)
    for k, v in {**base, **kw}.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("change,code", [
    (dict(M=-1), "SHAPE"), (dict(batch=-1), "SHAPE"), (dict(N=-2), "SHAPE"), (dict(K=-1), "SHAPE"), (dict(K=(1 << 20) + 1, lda=1 << 21, ldb=1 << 21), "SHAPE"),
    (dict(M=2 ** 31 - 1, N=2 ** 31 - 1, ldo=2 ** 31, strideO=2 ** 62), "SHAPE"),
    (dict(typeA=0), "TYPE"), (dict(typeB=5), "TYPE"), (dict(typeO=3), "TYPE"), (dict(rowsA=64), "TYPE"), (dict(rowsB=0), "TYPE"),
    (dict(lda=299), "STRIDE"), (dict(ldb=1), "STRIDE"), (dict(ldo=47), "STRIDE"), (dict(ldsA=2), "STRIDE"), (dict(ldsB=2), "STRIDE"),
    (dict(strideA=-1), "STRIDE"), (dict(strideO=64 * 48 - 1), "STRIDE"), (dict(strideO=0), "STRIDE"), (dict(strideBias=-1), "STRIDE"),
    (dict(reserved=1), "RESERVED"),
])
def test_fp8_gemm_refuses(lib, change, code):
    so, n = lib.load(), ctypes.c_size_t(0)
    d = _gemm(lib, **change)
    assert so.sc_fp8_gemm_workspace_size(ctypes.byref(d), ctypes.byref(n)) == getattr(lib, "SC_ERR_" + code)
    assert lib.sc_fp8_gemm(d, *[FAKE] * 7, 1 << 40, 0) == getattr(lib, "SC_ERR_" + code)


def test_fp8_gemm_refuses_pointers(lib):
    d = _gemm(lib)
    ok = [FAKE] * 6
    for k in (0, 1, 2, 3, 5):
        a = list(ok)
        a[k] = 0
        assert lib.sc_fp8_gemm(d, *a, 0, 0, 0) == lib.SC_ERR_NULL
    for k in (1, 3, 4, 5):
        a = list(ok)
        a[k] = FAKE + 1
        assert lib.sc_fp8_gemm(d, *a, FAKE, 1 << 40, 0) == lib.SC_ERR_STRIDE
    # sums of blocks that share a tile, and operands laid out anew, lie in the workspace
    for more in (dict(K=8192, lda=8192, ldb=8192, ldsA=64, ldsB=64), dict(M=4096, N=4096, lda=301, ldo=4096, strideO=1 << 24, strideA=1 << 21)):
        d = _gemm(lib, **more)
        need = lib.sc_fp8_gemm_workspace_size(d)
        assert need > 0
        for ws, n in ((0, need), (FAKE, need - 1), (FAKE + 16, need)):
            assert lib.sc_fp8_gemm(d, *ok, ws, n, 0) == lib.SC_ERR_WORKSPACE
    so = lib.load()
    assert so.sc_fp8_gemm_workspace_size(None, ctypes.byref(ctypes.c_size_t())) == lib.SC_ERR_NULL
    assert so.sc_fp8_gemm_workspace_size(ctypes.byref(d), None) == lib.SC_ERR_NULL
    for empty in (dict(M=0), dict(N=0), dict(batch=0)):
        assert lib.sc_fp8_gemm(_gemm(lib, **empty), *[0] * 7, 0, 0) == lib.SC_OK


def _norm(lib, **kw):
    d = lib.ScNormDesc()
    base = dict(batch=2, rows=5, D=256, post=1, pre=2, typeX=0, typeY=1, typeP=1, typeH=1, eps_post=1e-6, eps_pre=1e-6, scale_res=1.0,
                ldx=256, strideX=1280, ldy=256, strideY=1280, ldxo=256, strideXO=1280, ldh=256, strideH=1280, lds=2, strideS=10,
                lddxo=256, strideDXO=1280, lddy=256, strideDY=1280)
    for k, v in {**base, **kw}.items():
        setattr(d, k, v)
    return d


COMMON = [
    (dict(batch=-1), "SHAPE"), (dict(rows=-1), "SHAPE"), (dict(D=16385, ldx=20000, ldy=20000, ldxo=20000, ldh=20000), "SHAPE"),
    (dict(post=3), "TYPE"), (dict(pre=-1), "TYPE"), (dict(typeX=3), "TYPE"), (dict(typeY=5), "TYPE"), (dict(typeP=4), "TYPE"),
    (dict(typeH=6), "TYPE"), (dict(typeH=-1), "TYPE"), (dict(eps_pre=0.0), "SHAPE"), (dict(eps_post=-1.0), "SHAPE"),
    (dict(eps_pre=float("nan")), "SHAPE"), (dict(ldx=255), "STRIDE"), (dict(ldy=255), "STRIDE"), (dict(ldxo=1), "STRIDE"), (dict(ldh=0), "STRIDE"),
    (dict(stride_gate=-1), "STRIDE"), (dict(strideY=-4), "STRIDE"), (dict(reserved=2), "RESERVED"),
]


@pytest.mark.parametrize("change,code", COMMON + [
    (dict(strideXO=1279), "STRIDE"), (dict(strideH=0), "STRIDE"), (dict(typeH=3, lds=1), "STRIDE"), (dict(typeH=3, strideS=9), "STRIDE"),
    (dict(typeH=5, strideS=4), "STRIDE"), (dict(typeH=1), "TYPE"),           # rowmax without int8
])
def test_residual_norm_refuses(lib, change, code):
    assert lib.sc_residual_norm(_norm(lib, **change), *[FAKE] * 11, 0) == getattr(lib, "SC_ERR_" + code)


def test_residual_norm_refuses_pointers(lib):
    names = ["x", "y", "post_w", "post_b", "gate", "pre_w", "pre_b", "xo", "h", "scale", "rowmax"]

    def call(d, **kw):
        return lib.sc_residual_norm(d, *[{**dict.fromkeys(names, FAKE), "rowmax": 0, **kw}[n] for n in names], 0)

    d = _norm(lib)
    assert call(d, x=0) == lib.SC_ERR_NULL
    assert call(_norm(lib, typeH=5), scale=0) == call(_norm(lib, typeH=3), scale=0) == lib.SC_ERR_NULL
    # parameters of what is not there
    assert call(d, y=0) == lib.SC_ERR_TYPE
    assert call(_norm(lib, post=0)) == call(_norm(lib, pre=0), post_w=FAKE) == lib.SC_ERR_TYPE
    for n in ("x", "y", "gate", "pre_b", "xo", "h", "scale"):
        assert call(d, **{n: FAKE + 1}) == lib.SC_ERR_STRIDE
    assert call(_norm(lib, rows=0), x=0) == call(_norm(lib, batch=0), x=0) == lib.SC_OK
    assert call(d, xo=0, h=0) == lib.SC_OK


@pytest.mark.parametrize("change,code", COMMON + [
    (dict(typeH=3), "TYPE"), (dict(typeH=5), "TYPE"), (dict(lddxo=255), "STRIDE"), (dict(lddy=255), "STRIDE"),
    (dict(strideX=1279), "STRIDE"), (dict(strideDY=0), "STRIDE"),
])
def test_residual_norm_backward_refuses(lib, change, code):
    assert lib.sc_residual_norm_backward(_norm(lib, **change), *[FAKE] * 16, 1 << 40, 0) == getattr(lib, "SC_ERR_" + code)


def test_residual_norm_backward_refuses_pointers(lib):
    names = ["xo", "y", "post_w", "post_b", "gate", "pre_w", "dxo", "dh", "dx", "dy", "dpost_w", "dpost_b", "dgate", "dpre_w", "dpre_b",
             "workspace"]

    def call(d, nbytes=1 << 40, **kw):
        return lib.sc_residual_norm_backward(d, *[{**dict.fromkeys(names, FAKE), **kw}[n] for n in names], nbytes, 0)

    d = _norm(lib)
    need = lib.sc_residual_norm_backward_workspace_size(d)
    assert need > 0
    assert call(d, xo=0) == call(d, y=0) == lib.SC_ERR_NULL
    assert call(d, workspace=0) == call(d, nbytes=need - 1) == call(d, workspace=FAKE + 16) == lib.SC_ERR_WORKSPACE
    assert call(_norm(lib, post=0)) == call(_norm(lib, pre=0)) == lib.SC_ERR_TYPE
    for n in ("xo", "dxo", "dy", "dgate", "gate"):
        assert call(d, **{n: FAKE + 1}) == lib.SC_ERR_STRIDE
    assert call(d, **dict.fromkeys(names[8:15], 0)) == lib.SC_OK


def _rope(lib, **kw):
    d = lib.ScRopeDesc()
    base = dict(batch=2, tokens=10, heads=3, D=64, pairs=32, axes=3, strideXB=1920, strideXT=192, strideXH=64, strideOB=1920, strideOT=192,
                strideOH=64, strideSB=30, strideST=1, strideSH=10, stridePA=10)
    for k, v in {**base, **kw}.items():
        if k == "reserved":
            d.reserved[v] = 1
        else:
            setattr(d, k, v)
    return d


@pytest.mark.parametrize("change,code", [
    (dict(batch=-1), "SHAPE"), (dict(tokens=-1), "SHAPE"), (dict(heads=-1), "SHAPE"), (dict(heads=(1 << 30) + 1), "SHAPE"), (dict(D=258), "SHAPE"), (dict(pairs=33), "SHAPE"), (dict(pairs=-1), "SHAPE"),
    (dict(axes=0), "SHAPE"), (dict(axes=9), "SHAPE"), (dict(typeX=5), "TYPE"), (dict(typeO=3), "TYPE"), (dict(pairing=2), "TYPE"),
    (dict(inverse=2), "TYPE"), (dict(reserved=0), "RESERVED"), (dict(reserved=1), "RESERVED"), (dict(strideXT=-1), "STRIDE"),
    (dict(strideOH=63), "STRIDE"), (dict(strideOT=100), "STRIDE"), (dict(strideOB=0), "STRIDE"), (dict(typeO=5, strideSH=9), "STRIDE"),
    (dict(typeO=5, strideST=0), "STRIDE"), (dict(), "TYPE"),                  # rowmax without int8
])
def test_rope_refuses(lib, change, code):
    assert lib.sc_rope(_rope(lib, **change), *[FAKE] * 7, 0) == getattr(lib, "SC_ERR_" + code)


def test_rope_refuses_pointers(lib):
    ok = [FAKE] * 5 + [0, 0]
    for k in range(5):
        a = list(ok)
        a[k] = 0
        assert lib.sc_rope(_rope(lib), *a, 0) == lib.SC_ERR_NULL
        a[k] = FAKE + 1
        assert lib.sc_rope(_rope(lib), *a, 0) == lib.SC_ERR_STRIDE
    assert lib.sc_rope(_rope(lib, typeO=5), *ok, 0) == lib.SC_ERR_NULL
    for empty in (dict(batch=0), dict(tokens=0), dict(heads=0)):
        assert lib.sc_rope(_rope(lib, **empty), *[0] * 7, 0) == lib.SC_OK
    assert lib.load().sc_rope(None, *[None] * 8) == lib.SC_ERR_NULL


def test_workspace_of_another_device(lib):
    import torch
    import paper_2609_32922_amd as scg
    with pytest.raises(ValueError):
        scg.Workspace(64, device="cpu")
    # (one that lies there already, as a call finds it)
    ws = scg.Workspace.__new__(scg.Workspace)
    ws.nbytes, ws._buf, ws._made_on = 64, torch.empty(320, dtype=torch.uint8), 0
    with pytest.raises(ValueError):
        ws.ensure(0).use(torch.device("cuda", 0))


@pytest.mark.parametrize("stride,ld,apart", [(48, 96, True), (47, 96, False), (48, 95, False), (64 * 48, 48, True), (64 * 48 - 1, 48, False),
                                             (1 << 40, 48, True), (48, 1 << 40, True), (0, 96, False)])
def test_rows_of_entries_may_alternate(lib, stride, ld, apart):
    # the result [2, 64, 48] of strides (stride, ld)
    so, n, d = lib.load(), ctypes.c_size_t(0), _gemm(lib, ldo=ld, strideO=stride)
    assert so.sc_fp8_gemm_workspace_size(ctypes.byref(d), ctypes.byref(n)) == (lib.SC_OK if apart else lib.SC_ERR_STRIDE)
    if not apart:
        norm = dict(rows=64, D=48, ldx=ld, strideX=stride, ldy=ld, ldxo=ld, strideXO=stride, ldh=ld, strideH=stride, lddxo=ld, lddy=ld,
                    strideDY=stride)
        assert lib.sc_residual_norm(_norm(lib, **norm), *[FAKE] * 10, 0, 0) == lib.SC_ERR_STRIDE
        assert lib.sc_residual_norm_backward(_norm(lib, **norm), *[FAKE] * 16, 1 << 40, 0) == lib.SC_ERR_STRIDE
        quant = dict(QUANT, rows=64, K=48, ldx=48, ldq=ld, strideQ=stride)
        assert lib.sc_fp8_quantize(*quant.values(), 0) == lib.SC_ERR_STRIDE


def test_tensors_that_require_gradients_are_refused(lib):
    # (before anything else is looked at; without recording the call goes on, here to its refusal of tensors on the CPU)
    import torch
    import paper_2609_32922_amd as scg
    z = torch.zeros
    E4 = torch.float8_e4m3fn
    g = lambda *shape: z(*shape, requires_grad=True)  # noqa: E731
    pos, freq, axis = z(1, 4, dtype=torch.int32), z(32, dtype=torch.float64), z(32, dtype=torch.int32)
    a, s = z(4, 64).to(E4), z(4, 1)
    calls = [lambda: scg.fp8_quantize(g(4, 64)), lambda: scg.fp8_gemm(a, s, a, s, bias=g(4)), lambda: scg.fp8_gemm(a, g(4, 1), a, s),
             lambda: scg.fp8_gemm(a, s, a, s, out=g(4, 4)), lambda: scg.residual_norm(g(4, 64)), lambda: scg.residual_norm(z(4, 64), g(4, 64)),
             lambda: scg.residual_norm(z(4, 64), pre_weight=g(64)), lambda: scg.residual_norm(z(4, 64), z(4, 64), gate=g(64)),
             lambda: scg.rope(g(4, 2, 64), pos, freq, axis), lambda: scg.rope(z(4, 2, 64), pos, freq, axis, out=g(4, 2, 64)),
             lambda: scg.rope_quantize(g(4, 2, 64), pos, freq, axis)]
    for call in calls:
        with pytest.raises(ValueError, match="autograd"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="GPU"):
            call()
