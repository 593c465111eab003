"""Refusals of the language-model operators, on the CPU: the C entries check
their arguments before anything is enqueued, the helpers before any entry."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def iseg():
    from paper_2011_14504_amd import iseg
    iseg.lib()
    return iseg


ONE = C.c_void_p(1 << 20)
BIG = 1 << 60


def test_layernorm_entries(iseg):
    L = iseg.lib()

    def geom(M=4, C_=8, x_ld=8, y_ld=8, dx_ld=8, xd=iseg.ISEG_F32, pd=iseg.ISEG_F32, eps=1e-5):
        return iseg.LayernormGeom(M, C_, x_ld, y_ld, dx_ld, xd, pd, eps, 0)

    def fwd(g, x=ONE, y=ONE):
        return L.iseg_layernorm_fwd(x, ONE, ONE, C.byref(g), y, ONE, ONE, None, None)

    def bwd(g, ws=ONE, n=BIG, dy=ONE, mean=ONE):
        return L.iseg_layernorm_bwd(dy, ONE, ONE, mean, ONE, C.byref(g), ONE, ONE, ONE, ws, n, None)

    assert L.iseg_layernorm_fwd(ONE, None, None, None, ONE, None, None, None, None) == iseg.ISEG_ERR_ARG
    for bad in (dict(xd=iseg.ISEG_I8), dict(pd=iseg.ISEG_I32), dict(xd=9), dict(xd=-1)):
        assert fwd(geom(**bad)) == iseg.ISEG_ERR_ARG and bwd(geom(**bad)) == iseg.ISEG_ERR_ARG
        assert L.iseg_layernorm_bwd_ws(C.byref(geom(**bad))) == 0
    for bad in (dict(M=-1), dict(C_=0), dict(x_ld=7), dict(y_ld=7), dict(C_=1 << 31, x_ld=1 << 31, y_ld=1 << 31)):
        assert fwd(geom(**bad)) == iseg.ISEG_ERR_SHAPE and bwd(geom(**bad)) == iseg.ISEG_ERR_SHAPE
    assert bwd(geom(dx_ld=7)) == iseg.ISEG_ERR_SHAPE
    n = (1 << 27) + 1
    assert fwd(geom(C_=n, x_ld=n, y_ld=n)) == iseg.ISEG_ERR_UNSUPPORTED
    r = geom()
    r.reserved = 1
    assert fwd(r) == iseg.ISEG_ERR_ARG and bwd(r) == iseg.ISEG_ERR_ARG
    for eps in (0.0, -1.0, float("inf"), float("nan")):
        assert fwd(geom(eps=eps)) == iseg.ISEG_ERR_ARG
    assert fwd(geom(), x=None) == iseg.ISEG_ERR_ARG and fwd(geom(), y=None) == iseg.ISEG_ERR_ARG
    assert bwd(geom(), dy=None) == iseg.ISEG_ERR_ARG and bwd(geom(), mean=None) == iseg.ISEG_ERR_ARG
    assert bwd(geom(), ws=None) == iseg.ISEG_ERR_WORKSPACE
    assert bwd(geom(), n=L.iseg_layernorm_bwd_ws(C.byref(geom())) - 1) == iseg.ISEG_ERR_WORKSPACE
    assert fwd(geom(M=0), x=None, y=None) == iseg.ISEG_OK


def test_quantizer_entries(iseg):
    L = iseg.lib()

    def rows(t=iseg.ISEG_F32, M=4, C_=8, x_ld=8, bits=8, mode=0, c_ld=8, x=ONE, codes=ONE, scale=ONE):
        return L.iseg_quantize_rows(x, t, M, C_, x_ld, None, bits, mode, codes, c_ld, scale, None, None)

    def cols(t=iseg.ISEG_F32, M=4, C_=8, x_ld=8, bits=8, mode=0, c_ld=8, x=ONE, codes=ONE, scale=ONE, ws=ONE, n=BIG):
        return L.iseg_quantize_cols(x, t, M, C_, x_ld, None, bits, mode, codes, c_ld, scale, None, ws, n, None, None)

    for f in (rows, cols):
        for bad in (dict(t=iseg.ISEG_I8), dict(bits=1), dict(bits=9), dict(mode=2), dict(mode=-1), dict(x=None),
                    dict(codes=None), dict(scale=None)):
            assert f(**bad) == iseg.ISEG_ERR_ARG, bad
        for bad in (dict(M=-1), dict(C_=-1), dict(x_ld=7), dict(C_=1 << 31, x_ld=1 << 31, c_ld=1 << 31)):
            assert f(**bad) == iseg.ISEG_ERR_SHAPE, bad
    assert rows(c_ld=7) == iseg.ISEG_ERR_SHAPE and cols(c_ld=3) == iseg.ISEG_ERR_SHAPE
    assert rows(M=0, x=None, codes=None, scale=None) == iseg.ISEG_OK
    assert cols(C_=0, x=None, codes=None, scale=None) == iseg.ISEG_OK
    assert cols(ws=None) == iseg.ISEG_ERR_WORKSPACE and cols(n=16) == iseg.ISEG_ERR_WORKSPACE
    assert L.iseg_quantize_cols_ws(-1, 4) == 0
    n = (1 << 28) + 1
    assert cols(C_=n, x_ld=n) == iseg.ISEG_ERR_UNSUPPORTED and L.iseg_transpose_i8(ONE, 4, n, n, ONE, 4, None) == iseg.ISEG_ERR_UNSUPPORTED
    assert L.iseg_transpose_i8(ONE, 4, 8, 7, ONE, 4, None) == iseg.ISEG_ERR_SHAPE
    assert L.iseg_transpose_i8(ONE, 4, 8, 8, ONE, 3, None) == iseg.ISEG_ERR_SHAPE
    assert L.iseg_transpose_i8(None, 4, 8, 8, ONE, 4, None) == iseg.ISEG_ERR_ARG
    assert L.iseg_transpose_i8(None, 0, 8, 8, None, 4, None) == iseg.ISEG_OK


def test_matmul_entry(iseg):
    L = iseg.lib()

    def mm(M=4, N=4, K=16, lda=16, ldb=16, ldc=4, t=iseg.ISEG_F32, a=ONE, out=ONE, ws=ONE, n=BIG, un=0):
        g = iseg.MatmulGeom(M, N, K, lda, ldb, ldc, t, un)
        return L.iseg_matmul_i8(a, None, ONE, None, None, C.byref(g), out, ws, n, None)

    assert mm(t=iseg.ISEG_I32) == iseg.ISEG_ERR_ARG
    for bad in (dict(M=-1), dict(N=-1), dict(K=-1), dict(lda=15), dict(ldb=15), dict(ldc=3), dict(M=1 << 31)):
        assert mm(**bad) == iseg.ISEG_ERR_SHAPE, bad
    assert mm(K=131072, lda=131072, ldb=131072) == iseg.ISEG_ERR_UNSUPPORTED
    n, m = 1 << 28, (1 << 31) - 1                            # more blocks than a launch holds
    assert mm(N=n, ldc=n) == iseg.ISEG_ERR_UNSUPPORTED and mm(M=m, N=1) == iseg.ISEG_ERR_UNSUPPORTED
    assert mm(M=0, N=n, ldc=n, a=None, out=None) == iseg.ISEG_OK
    off = C.c_void_p(ONE.value + 8)
    assert mm(a=off) == iseg.ISEG_ERR_ARG and mm(a=off, un=1, n=0) == iseg.ISEG_ERR_WORKSPACE
    need = [L.iseg_matmul_i8_ws(C.byref(iseg.MatmulGeom(100, 200, 70, ld, 80, 200, iseg.ISEG_F32, un))) for ld, un in ((80, 0), (80, 1), (70, 0))]
    assert need[0] == 256 and need[1] >= 300 * 128 and need[1] > need[2] >= 100 * 128
    assert mm(a=None) == iseg.ISEG_ERR_ARG and mm(out=None) == iseg.ISEG_ERR_ARG
    assert mm(ws=None) == iseg.ISEG_ERR_WORKSPACE and mm(n=1) == iseg.ISEG_ERR_WORKSPACE
    assert mm(M=0, a=None, out=None) == iseg.ISEG_OK and mm(N=0, ldc=0) == iseg.ISEG_OK


def test_linear_entry(iseg):
    L = iseg.lib()

    def lin(M=4, N=4, K=16, x_ld=16, w_ld=16, c_ld=16, y_ld=4, xd=iseg.ISEG_BF16, yd=iseg.ISEG_F32, bits=8, mode=0, un=0, x=ONE, w=ONE,
            codes=ONE, scale=ONE, y=ONE, ws=ONE, n=BIG):
        g = iseg.LinearGeom(M, N, K, x_ld, w_ld, c_ld, y_ld, xd, yd, bits, mode, un, 0)
        return L.iseg_linear_i8_fwd(x, w, None, None, C.byref(g), codes, scale, y, ws, n, None, None)

    off = C.c_void_p(ONE.value + 4)
    for bad in (dict(xd=iseg.ISEG_I8), dict(yd=iseg.ISEG_I32), dict(bits=1), dict(bits=9), dict(mode=3), dict(x=None), dict(w=None), dict(codes=None),
                dict(scale=None), dict(y=None), dict(w=off), dict(codes=off)):
        assert lin(**bad) == iseg.ISEG_ERR_ARG, bad
    for bad in (dict(M=-1), dict(N=-1), dict(K=-1), dict(x_ld=15), dict(w_ld=15), dict(c_ld=15), dict(c_ld=24), dict(y_ld=3), dict(N=1 << 31, y_ld=1 << 31)):
        assert lin(**bad) == iseg.ISEG_ERR_SHAPE, bad
    assert lin(K=131072, x_ld=131072, w_ld=131072, c_ld=131072) == iseg.ISEG_ERR_UNSUPPORTED
    n = 1 << 28
    assert lin(N=n, y_ld=n) == iseg.ISEG_ERR_UNSUPPORTED and lin(M=1, N=n, y_ld=n) == iseg.ISEG_ERR_UNSUPPORTED
    assert lin(ws=None) == iseg.ISEG_ERR_WORKSPACE and lin(n=1) == iseg.ISEG_ERR_WORKSPACE
    assert lin(M=0, x=None, codes=None, scale=None, y=None) == iseg.ISEG_OK


def test_linear_backward_entry(iseg):
    L = iseg.lib()

    def bwd(M=4, N=32, K=16, dy_ld=32, a_ld=16, w_ld=16, wt_ld=0, dx_ld=16, dw_ld=16, dd=iseg.ISEG_BF16, od=iseg.ISEG_F32, bits=8, mode=0, un=0,
            dy=ONE, a=ONE, w=ONE, w_t=None, dx=ONE, dw=ONE, db=ONE, ws=ONE, n=BIG):
        g = iseg.LinearBwdGeom(M, N, K, dy_ld, a_ld, w_ld, wt_ld, dx_ld, dw_ld, dd, od, bits, mode, un, 0)
        return L.iseg_linear_i8_bwd(dy, a, None, w, None, w_t, C.byref(g), dx, dw, db, ws, n, None, None)

    off = C.c_void_p(ONE.value + 4)
    for bad in (dict(dd=iseg.ISEG_I8), dict(od=iseg.ISEG_I32), dict(bits=1), dict(bits=9), dict(mode=3), dict(dy=None), dict(w=None), dict(a=None),
                dict(wt_ld=32, w_t=None), dict(wt_ld=32, w_t=off)):
        assert bwd(**bad) == iseg.ISEG_ERR_ARG, bad
    for bad in (dict(M=-1), dict(N=-1), dict(K=-1), dict(dy_ld=31), dict(a_ld=15), dict(w_ld=15), dict(wt_ld=31, w_t=ONE), dict(dx_ld=15), dict(dw_ld=15),
                dict(K=1 << 31, a_ld=1 << 31, w_ld=1 << 31, dx_ld=1 << 31, dw_ld=1 << 31)):
        assert bwd(**bad) == iseg.ISEG_ERR_SHAPE, bad
    assert bwd(N=131072, dy_ld=131072, dw=None, db=None) == iseg.ISEG_ERR_UNSUPPORTED
    assert bwd(M=131072, dx=None) == iseg.ISEG_ERR_UNSUPPORTED
    n = (1 << 28) + 1                                        # columns beyond one launch, found before any work
    wide = dict(M=40, N=2, K=n, a_ld=n, w_ld=n, dx_ld=n, dw_ld=n)
    assert bwd(**wide) == bwd(**wide, dx=None, db=None) == bwd(**wide, dw=None, db=None) == iseg.ISEG_ERR_UNSUPPORTED
    assert bwd(N=n, dy_ld=n, dx=None, dw=None) == iseg.ISEG_ERR_UNSUPPORTED
    assert bwd(ws=None) == iseg.ISEG_ERR_WORKSPACE and bwd(n=1) == iseg.ISEG_ERR_WORKSPACE
    assert bwd(dx=None, dw=None, db=None, dy=None, a=None, w=None) == iseg.ISEG_OK
    assert bwd(M=0, N=0, dy=None, a=None, w=None) == iseg.ISEG_OK


def test_logprob_entries(iseg):
    L = iseg.lib()

    def geom(M=4, V=100, ld=100, out_ld=100, t=iseg.ISEG_BF16, tt=iseg.ISEG_I64, k=5):
        return iseg.LogprobGeom(M, V, ld, out_ld, t, tt, k, 0)

    def fwd(g, x=ONE, lp=ONE, ids=ONE, ws=ONE, n=BIG):
        return L.iseg_logprob_fwd(x, ONE, C.byref(g), lp, ONE, ONE, ids, ONE, ws, n, None, None)

    def bwd(g, glp=ONE, gh=ONE, ent=ONE, lse=ONE):
        return L.iseg_logprob_bwd(ONE, ONE, lse, ent, glp, gh, C.byref(g), ONE, None, None)

    for bad in (dict(t=iseg.ISEG_I8), dict(tt=iseg.ISEG_I8), dict(k=-1), dict(k=65), dict(V=4, ld=4, out_ld=4, k=5)):
        assert fwd(geom(**bad)) == iseg.ISEG_ERR_ARG and bwd(geom(**bad)) == iseg.ISEG_ERR_ARG
        assert L.iseg_logprob_fwd_ws(C.byref(geom(**bad))) == 0
    for bad in (dict(M=-1), dict(V=0), dict(ld=99), dict(V=1 << 31, ld=1 << 31, out_ld=1 << 31)):
        assert fwd(geom(**bad)) == iseg.ISEG_ERR_SHAPE and bwd(geom(**bad)) == iseg.ISEG_ERR_SHAPE
    assert bwd(geom(out_ld=99)) == iseg.ISEG_ERR_SHAPE
    assert fwd(geom(), x=None) == iseg.ISEG_ERR_ARG and fwd(geom(), lp=None) == iseg.ISEG_ERR_ARG
    assert fwd(geom(), ids=None) == iseg.ISEG_ERR_ARG
    assert fwd(geom(), ws=None) == iseg.ISEG_ERR_WORKSPACE and fwd(geom(), n=1) == iseg.ISEG_ERR_WORKSPACE
    assert bwd(geom(), glp=None, gh=None) == iseg.ISEG_ERR_ARG and bwd(geom(), ent=None) == iseg.ISEG_ERR_ARG
    assert bwd(geom(), lse=None) == iseg.ISEG_ERR_ARG
    assert fwd(geom(M=0), x=None, ws=None) == iseg.ISEG_OK and bwd(geom(M=0), lse=None) == iseg.ISEG_OK


def test_a_workspace_of_256_bytes_is_untouched(iseg):
    """The least size stands for calls that use no workspace (one buffer serves
    all of them); the smallest calls that use one ask for more."""
    L, B = iseg.lib(), C.byref
    ln = lambda M, n: L.iseg_layernorm_bwd_ws(B(iseg.LayernormGeom(M, n, n, n, n, iseg.ISEG_F32, iseg.ISEG_F32, 1.0, 0)))
    assert ln(8, 4) == ln(0, 64) == 256 and ln(9, 4) > 256 and ln(1, 3) > 256 and ln(2, 1) > 256
    assert L.iseg_quantize_cols_ws(1, 1) > 256 and L.iseg_quantize_cols_ws(0, 1) > 256
    lp = lambda M, V, k: L.iseg_logprob_fwd_ws(B(iseg.LogprobGeom(M, V, V, V, iseg.ISEG_F32, iseg.ISEG_I64, k, 0)))
    assert lp(1, 4092, 0) == 256 and lp(1, 4093, 0) > 256 and lp(1, 1 << 20, 5) > 256
    mm = lambda M, N, K, lda: L.iseg_matmul_i8_ws(B(iseg.MatmulGeom(M, N, K, lda, K, N, iseg.ISEG_F32, 0)))
    assert mm(32, 5, 16, 17) == 256 and mm(33, 1, 16, 16) == 256 and mm(33, 1, 16, 17) > 256 and mm(40, 40, 8192, 8192) > 256
    lb = iseg.LinearBwdGeom(1, 1, 1, 1, 1, 1, 0, 1, 1, iseg.ISEG_F32, iseg.ISEG_F32, 8, 0, 0, 0)
    assert L.iseg_linear_i8_bwd_ws(B(lb)) > 256


def test_helpers(iseg):
    x, i8 = torch.zeros(4, 32), torch.zeros(4, 32, dtype=torch.int8)
    v, tok = torch.zeros(4), torch.zeros(4, dtype=torch.int64)
    calls = [
        lambda: iseg.layernorm_fwd(x.double()), lambda: iseg.layernorm_fwd(torch.zeros(())),
        lambda: iseg.layernorm_fwd(x, torch.zeros(31)), lambda: iseg.layernorm_fwd(x, torch.zeros(32).half(), torch.zeros(32)),
        lambda: iseg.layernorm_fwd(x, eps=0.0), lambda: iseg.layernorm_fwd(torch.zeros(4, 0)), lambda: iseg.layernorm_fwd(x),
        lambda: iseg.layernorm_fwd(x, eps=float("nan")),
        lambda: iseg.layernorm_bwd(x.half(), x, None, v, v), lambda: iseg.layernorm_bwd(x[:3], x, None, v, v),
        lambda: iseg.layernorm_bwd(x, x, None, v.double(), v), lambda: iseg.layernorm_bwd(x, x, None, v[:3], v),
        lambda: iseg.layernorm_bwd(x, x, None, v, v),
        lambda: iseg.quantize_rows(i8), lambda: iseg.quantize_rows(x, 9), lambda: iseg.quantize_rows(x, 8, 2),
        lambda: iseg.quantize_rows(x, mul=v), lambda: iseg.quantize_rows(x), lambda: iseg.quantize_cols(x, mul=torch.zeros(32)),
        lambda: iseg.quantize_cols(x, 1), lambda: iseg.quantize_cols(x),
        lambda: iseg.transpose_i8(x), lambda: iseg.transpose_i8(i8[0]), lambda: iseg.transpose_i8(i8),
        lambda: iseg.matmul_i8(i8, x), lambda: iseg.matmul_i8(i8, i8[:, :31]), lambda: iseg.matmul_i8(i8, i8, v[:3]),
        lambda: iseg.matmul_i8(i8, i8, v, v.double()), lambda: iseg.matmul_i8(i8, i8, out_dtype=torch.int32),
        lambda: iseg.matmul_i8(i8, i8), lambda: iseg.matmul_i8(torch.zeros(1, 131072, dtype=torch.int8), torch.zeros(1, 131072, dtype=torch.int8)),
        lambda: iseg.linear_i8_fwd(x, i8[:, :31]), lambda: iseg.linear_i8_fwd(x, i8, v[:3]), lambda: iseg.linear_i8_fwd(x, i8, v, v.half()),
        lambda: iseg.linear_i8_fwd(x, x), lambda: iseg.linear_i8_fwd(x, i8, bits=1), lambda: iseg.linear_i8_fwd(x, i8, out_dtype=torch.int8), lambda: iseg.linear_i8_fwd(x, i8),
        lambda: iseg.linear_i8_bwd(x, i8, v, i8), lambda: iseg.linear_i8_bwd(x[:, :4], i8, v, i8, w_t=i8),
        lambda: iseg.linear_i8_bwd(x[:3, :4], i8, v, i8),
        lambda: iseg.logprob_fwd(x, tok[:3]), lambda: iseg.logprob_fwd(x, tok.float()), lambda: iseg.logprob_fwd(x, tok, top_k=33),
        lambda: iseg.logprob_fwd(x, tok, top_k=-1), lambda: iseg.logprob_fwd(torch.zeros(2, 100), tok[:2], top_k=65),
        lambda: iseg.logprob_fwd(torch.zeros(4, 0), tok), lambda: iseg.logprob_fwd(x, tok),
        lambda: iseg.logprob_bwd(x, tok, v, v), lambda: iseg.logprob_bwd(x, tok, v, None, v, v),
        lambda: iseg.logprob_bwd(x, tok, v[:3], v, v), lambda: iseg.logprob_bwd(x, tok, None, v, v), lambda: iseg.logprob_bwd(x, tok, v, v, v),
    ]
    for i, f in enumerate(calls):
        with pytest.raises(ValueError):
            f()
            print("accepted:", i)


def test_tape_knows_the_operators(iseg):
    L = iseg.lib()
    for n in ("iseg_layernorm_fwd", "iseg_layernorm_bwd", "iseg_quantize_rows", "iseg_quantize_cols", "iseg_transpose_i8",
              "iseg_matmul_i8", "iseg_linear_i8_fwd", "iseg_linear_i8_bwd", "iseg_logprob_fwd", "iseg_logprob_bwd"):
        e = L.iseg_tape_entry(n.encode())
        assert e >= 0 and L.iseg_tape_entry_nargs(e) == len(iseg._SIGS[n][0])
