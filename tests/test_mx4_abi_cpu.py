"""Host-side refusals of the 4-bit entry points (nothing is launched, no GPU needed)."""

import ctypes as C

import pytest

from paper_2111_05188_amd import tp

X = 0x100000


def _refused(rc, text, code=tp.TP_EINVAL):
    assert rc == code and text in tp.last_error(), (rc, tp.last_error())


def test_bytes():
    # whole tiles of 32 rows and 256 elements
    assert tp.mx4_bytes(1, 1) == 32 * 256 * 17 // 32
    assert tp.mx4_bytes(32, 256) == 32 * 256 * 17 // 32
    assert tp.mx4_bytes(33, 257) == 4 * 32 * 256 * 17 // 32
    assert tp.mx4_bytes(512, 1024) == 512 * 1024 * 17 // 32
    L = tp.load()
    for rows, K in ((0, 4), (4, 0), (-1, 4), (1 << 30, 4), (4, 1 << 30)):
        assert L.tp_mx4_bytes(rows, K) == 0 and "rows of" in tp.last_error()
        assert L.tp_mx4_workspace_bytes(rows, 4, K) == 0
    assert L.tp_mx4_workspace_bytes(4, 0, 4) == 0
    assert L.tp_mx4_bytes(1 << 27, 1 << 27) == 0 and "grid" in tp.last_error()
    with pytest.raises(tp.TPError):
        tp.mx4_bytes(0, 1)
    assert L.tp_mx4_workspace_bytes(64, 100, 1001) >= tp.mx4_bytes(64, 1001)


def test_quantize_refuses():
    L = tp.load()
    m = C.byref(tp.Mx4(X, 4, 64))
    q = L.tp_mx4_quantize
    _refused(q(None, tp.TP_F32, 64, 1, m, None), "NULL")
    _refused(q(X, 5, 64, 1, m, None), "dtype")
    _refused(q(X + 2, tp.TP_F32, 64, 1, m, None), "misaligned")
    _refused(q(X, tp.TP_F32, -64, 1, m, None), "stride")
    _refused(q(X, tp.TP_F32, 128, 2, m, None), "one of them", tp.TP_EUNSUPPORTED)
    _refused(q(X, tp.TP_F32, 64, 1, None, None), "NULL")
    _refused(q(X, tp.TP_F32, 64, 1, C.byref(tp.Mx4(None, 4, 64)), None), "NULL")
    _refused(q(X, tp.TP_F32, 64, 1, C.byref(tp.Mx4(X + 16, 4, 64)), None), "256-byte")
    _refused(q(X, tp.TP_F32, 64, 1, C.byref(tp.Mx4(X, 0, 64)), None), "rows of")
    _refused(L.tp_mx4_dequantize(m, X, tp.TP_BF16, 63, None), "pitch")
    _refused(L.tp_mx4_dequantize(m, None, tp.TP_BF16, 64, None), "NULL")


def test_products_refuse():
    L = tp.load()
    a, w = C.byref(tp.Mx4(X, 4, 64)), C.byref(tp.Mx4(X, 5, 64))
    ok = dict(a=a, w=w, bias=None, act=0, y=X, dtype=tp.TP_F32, ldy=5, work=X, nb=1 << 30, s=None)

    def mm(**kw):
        return L.tp_mx4_matmul(*{**ok, **kw}.values())

    _refused(mm(a=None), "NULL")
    _refused(mm(w=C.byref(tp.Mx4(X, 5, 65))), "elements a row")
    _refused(mm(bias=X + 2), "bias")
    _refused(mm(act=2), "activation")
    _refused(mm(y=None), "y is NULL")
    _refused(mm(ldy=4), "pitch")
    _refused(mm(dtype=3), "dtype")
    _refused(mm(work=None), "workspace")
    _refused(mm(work=X + 64), "workspace")
    _refused(mm(nb=0), "needed")
    big = C.byref(tp.Mx4(X, 1 << 27, 64))
    _refused(mm(a=big, w=big, ldy=1 << 27), "grid", tp.TP_EUNSUPPORTED)
    lin = dict(x=X, xd=tp.TP_BF16, M=4, ldx=64, w=w, bias=None, act=0, y=X, dtype=tp.TP_F32, ldy=5,
               work=X, nb=1 << 30, s=None)

    def linear(**kw):
        return L.tp_mx4_linear(*{**lin, **kw}.values())

    _refused(linear(x=None), "x is NULL")
    _refused(linear(M=0), "rows of")
    _refused(linear(ldx=63), "pitch")
    _refused(linear(x=X + 1), "misaligned")
    _refused(linear(w=None), "NULL")
    _refused(linear(nb=5), "needed")
