"""The 8-bit integer layer and the linear cross entropy of include/pvconv_train.h:
invalid arguments are rejected on the host before anything is enqueued. No GPU: every
call here fails validation or has nothing to do."""
import pytest
import torch

from paper_1907_03739_amd import binding as b
from test_abi_train import BE, C, DB, DG, DY, EINVAL, EWS, G, L, LO, LS, ODD, OK, Q, S, ST, T, WS, X, Y


def _call(fn, a, kw):
    a.update(kw)
    return fn(*a.values())


def _quant(**kw):
    return _call(L.pvconv_int8_quantize, dict(x=X, xd=0, xl=0, R=20, K=40, q=Q, sc=S, s=None), kw)


@pytest.mark.parametrize("kw,status", [
    (dict(R=-1), EINVAL), (dict(R=(1 << 30) + 1), EINVAL), (dict(K=0), EINVAL),
    (dict(K=65537), EINVAL), (dict(xd=2), EINVAL), (dict(xl=39), EINVAL), (dict(x=None), EINVAL),
    (dict(q=None), EINVAL), (dict(sc=None), EINVAL), (dict(x=ODD), EINVAL), (dict(q=Q + 8), EINVAL),
    (dict(sc=ODD), EINVAL), (dict(q=X), EINVAL), (dict(sc=X + 4), EINVAL), (dict(sc=Q + 128), EINVAL),
    (dict(R=0), OK), (dict(R=0, K=0), EINVAL),
])
def test_int8_quantize_rejects(kw, status):
    assert _quant(**kw) == status


def _lin(**kw):
    return _call(L.pvconv_int8_linear, dict(
        x=X, xd=0, xl=0, M=300, K=40, N=70, w=Q, sc=S, bias=BE, act=1, sl=0.0, y=Y, yd=1, yl=0,
        rows=None, rs=None, ws=WS, wsb=1 << 30, s=None), kw)


LIN_BAD = [dict(M=-1), dict(K=0), dict(N=0), dict(K=70000), dict(N=70000), dict(yd=5), dict(act=3),
           dict(yl=69), dict(w=None), dict(sc=None), dict(y=None), dict(w=Q + 8), dict(sc=ODD),
           dict(bias=ODD), dict(y=ODD), dict(y=Q), dict(y=S), dict(y=BE),
           dict(M=1 << 30, K=60000, N=60000)]


@pytest.mark.parametrize("kw,status", [(k, EINVAL) for k in LIN_BAD] + [
    (dict(xd=5), EINVAL), (dict(xl=39), EINVAL), (dict(x=None), EINVAL), (dict(x=ODD), EINVAL),
    (dict(y=X), EINVAL), (dict(rows=T), EINVAL), (dict(rs=C), EINVAL), (dict(rows=T + 4, rs=C), EINVAL),
    (dict(rows=X, rs=C), EINVAL), (dict(rows=T, rs=Y), EINVAL), (dict(rows=T, rs=T), EINVAL),
    (dict(rows=T, rs=ODD), EINVAL), (dict(rows=Q, rs=C), EINVAL), (dict(M=0), OK),
    (dict(M=5000, N=2048, ws=None), EWS), (dict(M=5000, N=2048, wsb=256), EWS),
    (dict(M=5000, N=2048, ws=WS + 128), EWS),
])
def test_int8_linear_rejects(kw, status):
    if status == EWS:
        kw = dict(kw, x=1 << 40, y=1 << 42)
    assert _lin(**kw) == status


def _lrows(**kw):
    return _call(L.pvconv_int8_linear_rows, dict(
        rows=T, rs=C, M=300, K=40, N=70, w=Q, sc=S, bias=BE, act=1, sl=0.0, y=Y, yd=1, yl=0, ws=WS,
        wsb=1 << 30, s=None), kw)


@pytest.mark.parametrize("kw,status", [(k, EINVAL) for k in LIN_BAD] + [
    (dict(rows=None), EINVAL), (dict(rs=None), EINVAL), (dict(rows=T + 1), EINVAL),
    (dict(rs=ODD), EINVAL), (dict(y=T), EINVAL), (dict(y=C), EINVAL), (dict(M=0), OK),
    (dict(K=60000, ws=None), EWS),
])
def test_int8_linear_rows_rejects(kw, status):
    if status == EWS:
        kw = dict(kw, rows=1 << 40, w=1 << 42)
    assert _lrows(**kw) == status


def _linb(**kw):
    return _call(L.pvconv_int8_linear_backward, dict(
        dy=DY, dd=0, dl=0, rows=T, rs=C, M=100, K=40, N=20, w=Q, sc=S, dx=Y, od=0, ol=0, dw=DG,
        db=DB, ws=WS, wsb=1 << 30, s=None), kw)


@pytest.mark.parametrize("kw,status", [
    (dict(dx=None, dw=None, db=None), EINVAL), (dict(dy=None), EINVAL), (dict(rows=None), EINVAL),
    (dict(rs=None), EINVAL), (dict(w=None), EINVAL), (dict(sc=None), EINVAL), (dict(w=Q + 4), EINVAL),
    (dict(rows=T + 8), EINVAL), (dict(dw=DB), EINVAL), (dict(dx=DY), EINVAL), (dict(dw=DY), EINVAL),
    (dict(db=DY), EINVAL), (dict(dx=Q), EINVAL), (dict(dw=T), EINVAL), (dict(dl=19), EINVAL),
    (dict(ol=39), EINVAL), (dict(dd=2), EINVAL), (dict(od=2), EINVAL), (dict(ws=None), EWS),
    (dict(wsb=1), EWS), (dict(M=0, dw=None, db=None), OK), (dict(M=-1), EINVAL),
])
def test_int8_linear_backward_rejects(kw, status):
    assert _linb(**kw) == status


CE_BAD = [dict(M=-1), dict(M=(1 << 24) + 1), dict(K=0), dict(K=65537), dict(V=0),
          dict(V=(1 << 24) + 1), dict(xd=2), dict(wd=2), dict(od=2), dict(gd=2), dict(xl=39),
          dict(wl=39), dict(ol=39), dict(x=None), dict(w=None), dict(lab=None), dict(x=ODD),
          dict(w=ODD), dict(bias=ODD), dict(lab=ODD), dict(dx=ODD), dict(dw=ODD), dict(db=ODD),
          dict(dx=X), dict(dx=Q), dict(dx=BE), dict(dx=T), dict(dw=X), dict(dw=Y), dict(dw=Q),
          dict(db=DG), dict(db=X), dict(rw=ODD)]


def _ce(**kw):
    return _call(L.pvconv_linear_cross_entropy, dict(
        x=X, xd=0, xl=0, w=Q, wd=0, wl=0, M=100, K=40, V=70, bias=BE, lab=T, rw=None, loss=LO,
        lse=LS, dx=Y, od=0, ol=0, dw=DG, gd=0, db=DB, ws=WS, wsb=1 << 30, s=None), kw)


def _ceb(**kw):
    kw = dict(kw)
    if "rw" in kw:
        kw["dl"] = kw.pop("rw")
    return _call(L.pvconv_linear_cross_entropy_backward, dict(
        x=X, xd=0, xl=0, w=Q, wd=0, wl=0, M=100, K=40, V=70, bias=BE, lab=T, lse=LS, dl=None, dx=Y,
        od=0, ol=0, dw=DG, gd=0, db=DB, ws=WS, wsb=1 << 30, s=None), kw)


@pytest.mark.parametrize("kw,status", [(k, EINVAL) for k in CE_BAD] + [
    (dict(loss=None), EINVAL), (dict(loss=ODD), EINVAL), (dict(lse=ODD), EINVAL),
    (dict(loss=X), EINVAL), (dict(lse=LO), EINVAL), (dict(loss=Y), EINVAL), (dict(loss=T), EINVAL),
    (dict(ws=None), EWS), (dict(wsb=64), EWS), (dict(ws=WS + 64), EWS),
    (dict(M=0, dw=None, db=None), OK),
])
def test_linear_cross_entropy_rejects(kw, status):
    assert _ce(**kw) == status


@pytest.mark.parametrize("kw,status", [(k, EINVAL) for k in CE_BAD] + [
    (dict(lse=None), EINVAL), (dict(lse=ODD), EINVAL), (dict(dx=LS), EINVAL), (dict(dw=LS), EINVAL),
    (dict(dx=None, dw=None, db=None), EINVAL), (dict(ws=None), EWS), (dict(wsb=64), EWS),
    (dict(M=0, dw=None, db=None), OK),
])
def test_linear_cross_entropy_backward_rejects(kw, status):
    assert _ceb(**kw) == status


def test_workspace_queries():
    f = L.pvconv_int8_linear_workspace_size
    assert f(5000, 4928, 2048) >= 5000 * (39 * 128 + 4) and f(1, 2048, 256) == 0
    assert f(-1, 5, 5) == 0 and f(5, 0, 5) == 0 and f(5, 5, 70000) == 0
    assert L.pvconv_int8_linear_rows_workspace_size(-1, 5, 5) == 0
    f = L.pvconv_int8_linear_backward_workspace_size
    for M in (1, 127, 5000):
        assert f(M, 300, 50) > 0
    f = L.pvconv_linear_cross_entropy_workspace_size
    assert f(100, 40, 0, 0, 0, 0, 0, 1) == 0 and f(100, 40, 70, 2, 0, 0, 0, 1) == 0
    # far less than the logits of a long vocabulary
    assert 0 < f(65536, 512, 50000, 1, 1, 1, 1, 0) < 65536 * 50000 // 4
    assert f(65536, 512, 50000, 1, 1, 1, 1, 1) < 65536 * 50000
    for M in (0, 1, 63, 4097):
        for V in (1, 64, 65, 2049, 100003):
            # one for every gradient serves any of them
            assert f(M, 77, V, 0, 1, 1, 0, 1) >= f(M, 77, V, 0, 1, 1, 0, 0) >= 0


def test_binding_refuses_before_the_library():
    x, v = torch.zeros(2, 5, 8), torch.zeros(8)
    i8, i32 = torch.zeros(4, 128, dtype=torch.int8), torch.zeros(10, dtype=torch.int32)
    s, w = torch.zeros(4), torch.zeros(6, 8)
    apart = x.transpose(1, 2)
    for bad in (lambda: b.pvconv_int8_quantize(apart),
                lambda: b.pvconv_int8_linear(x, i8.to(torch.uint8), s),
                lambda: b.pvconv_int8_linear(x, i8[:, :64], s),
                lambda: b.pvconv_int8_linear(x, i8, v),
                lambda: b.pvconv_int8_linear(x, i8, s.double()),
                lambda: b.pvconv_int8_linear(x, i8, s, bias=v),
                lambda: b.pvconv_int8_linear(x, i8, s, out=x),
                lambda: b.pvconv_int8_linear(apart, i8, s),
                lambda: b.pvconv_int8_linear_rows(i8, v, i8, s),
                lambda: b.pvconv_int8_linear_rows(i8[:, :64], s, i8, s),
                lambda: b.pvconv_int8_linear_rows(i8, s, i8, s, out=w),
                lambda: b.pvconv_int8_linear_backward(x[0, :, :4], None, None, None, None, 8),
                lambda: b.pvconv_int8_linear_backward(x[0, :4, :4], i8, s, i8, s, 129),
                lambda: b.pvconv_int8_linear_backward(x[0, :, :4], i8, s, i8, s, 8),
                lambda: b.pvconv_int8_linear_backward(x[0, :4, :5], i8, s, i8, s, 8),
                lambda: b.pvconv_int8_linear_backward(x, i8, s, i8, s, 8, False, False, False),
                lambda: b.pvconv_linear_cross_entropy(v, w, i32),
                lambda: b.pvconv_linear_cross_entropy(x, w[:, :7], i32),
                lambda: b.pvconv_linear_cross_entropy(x, w, i32[:9]),
                lambda: b.pvconv_linear_cross_entropy(x, w, i32.long()),
                lambda: b.pvconv_linear_cross_entropy(x, w, i32, bias=v),
                lambda: b.pvconv_linear_cross_entropy(x, w, i32, row_weight=v),
                lambda: b.pvconv_linear_cross_entropy(apart, torch.zeros(6, 5), i32),
                lambda: b.pvconv_linear_cross_entropy(x, w, None),
                lambda: b.pvconv_linear_cross_entropy(x, w, i32, None, None, True, False, False,
                                                      False),
                lambda: b.pvconv_linear_cross_entropy_backward(x, w, i32, None),
                lambda: b.pvconv_linear_cross_entropy_backward(x, w, i32, v)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: b.pvconv_int8_quantize(x.half()),
                lambda: b.pvconv_linear_cross_entropy(x.half(), w, i32),
                lambda: b.pvconv_linear_cross_entropy(x, w, i32, out_dtype=torch.float16)):
        with pytest.raises(TypeError):
            bad()


def test_binding_refuses_sizes_beyond_a_c_int():
    rows = torch.empty(((1 << 32) + 5, 1), dtype=torch.bfloat16, device="meta")
    for bad in (lambda: b.pvconv_int8_quantize(rows),
                lambda: b.pvconv_linear_cross_entropy(rows, rows[:5], None),
                lambda: b.pvconv_linear_cross_entropy(rows[:5], rows, None)):
        with pytest.raises(ValueError, match="2\\^31"):
            bad()
