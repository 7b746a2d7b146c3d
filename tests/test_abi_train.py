"""include/pvconv_train.h: every declared symbol is exported and bound, and invalid
arguments are rejected on the host before anything is enqueued. No GPU: every call
here fails validation or has nothing to do."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

from paper_1907_03739_amd import binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "pvconv_train.h")
L = b._lib
OK, EINVAL, EWS = 0, 1, 3
ODD = 0x100001
X, Y, G, BE, ST, WS, DY, Q, S, DG, DB, T, C, LO, LS = (0x10000000 * i for i in range(1, 16))


def test_every_declared_symbol_is_exported_and_bound():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(pvconv_\w+)\s*\(", text)))
    out = subprocess.run(["nm", "-D", "--defined-only", b.LIB_PATH], capture_output=True,
                         text=True, check=True).stdout
    assert set(names) <= set(re.findall(r"\bT (pvconv_\w+)", out))
    assert set(names) == set(b.EXPORTED_TRAIN) and not set(names) & set(b.EXPORTED)


def test_workspace_queries():
    f = L.pvconv_group_norm_act_workspace_size
    assert f(16, 32768, 128, 8) > 0 and f(0, 5, 8, 2) == 0
    assert f(2, 5, 8, 3) == 0 and f(-1, 5, 8, 2) == 0 and f(1, 5, 0, 1) == 0
    f = L.pvconv_fp8_linear_workspace_size
    # rows apart from their product: bytes and scales of every block
    assert f(4096, 4928, 2048) >= 4096 * 39 * 128 + 4096 * 39
    assert f(1, 2048, 256) == 0 and f(-1, 5, 5) == 0 and f(5, 0, 5) == 0 and f(5, 70000, 5) == 0
    f = L.pvconv_fp8_linear_backward_workspace_size
    assert f(1000, 300, 50) >= 8 * 128 * (300 + 50) and f(1000, 300, 0) == 0
    for M in (0, 1, 127, 128, 129, 5000):  # every size of plan is computed
        assert f(M, 9, 7) >= 0


def _gn(**kw):
    a = dict(x=X, xd=0, xl=0, B=2, N=10, C=8, g=2, len=None, ga=G, be=BE, eps=1e-5, act=3, sl=0.1,
             y=Y, yd=0, yl=0, st=ST, ws=WS, wsb=1 << 30, s=None)
    a.update(kw)
    return L.pvconv_group_norm_act(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(B=-1), EINVAL), (dict(N=-1), EINVAL), (dict(C=0), EINVAL), (dict(C=20000, g=2), EINVAL),
    (dict(g=3), EINVAL), (dict(g=0), EINVAL), (dict(xd=2), EINVAL), (dict(yd=-1), EINVAL),
    (dict(act=4), EINVAL), (dict(act=-1), EINVAL), (dict(eps=-1.0), EINVAL),
    (dict(eps=float("nan")), EINVAL), (dict(xl=7), EINVAL), (dict(yl=7), EINVAL),
    (dict(x=None), EINVAL), (dict(y=None), EINVAL), (dict(ga=None), EINVAL), (dict(be=None), EINVAL),
    (dict(x=ODD), EINVAL), (dict(ga=ODD), EINVAL), (dict(st=ODD), EINVAL), (dict(len=ODD), EINVAL),
    (dict(y=X), EINVAL), (dict(y=X + 64), EINVAL), (dict(st=Y), EINVAL),
    (dict(B=1 << 20, N=1 << 11), EINVAL), (dict(B=64, N=1 << 20, C=64, g=8, ws=None), EWS),
    (dict(B=64, N=1 << 20, C=64, g=8, ws=WS + 128), EWS),
    (dict(B=64, N=1 << 20, C=64, g=8, wsb=64), EWS), (dict(B=0), OK), (dict(N=0, st=None), OK),
])
def test_group_norm_rejects(kw, status):
    if status == EWS:  # buffers of this size, apart from one another
        kw = dict(kw, x=1 << 40, y=1 << 42)
    assert _gn(**kw) == status


def _gnb(**kw):
    a = dict(dy=DY, dd=0, dl=0, x=X, xd=0, xl=0, B=2, N=10, C=8, g=2, len=None, st=ST, ga=G, be=BE,
             act=3, sl=0.1, dx=Y, od=0, ol=0, dg=DG, db=DB, ws=WS, wsb=1 << 30, s=None)
    a.update(kw)
    return L.pvconv_group_norm_act_backward(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(g=5), EINVAL), (dict(dy=None), EINVAL), (dict(x=None), EINVAL), (dict(st=None), EINVAL),
    (dict(dx=None), EINVAL), (dict(ga=None), EINVAL), (dict(dx=X), EINVAL), (dict(dx=DY), EINVAL),
    (dict(dg=Y), EINVAL), (dict(dg=DB), EINVAL), (dict(dg=G), EINVAL), (dict(dd=3), EINVAL),
    (dict(ol=4), EINVAL), (dict(act=9), EINVAL), (dict(dy=ODD), EINVAL), (dict(ws=None), EWS),
    (dict(wsb=8), EWS), (dict(B=0, dg=None, db=None), OK),
])
def test_group_norm_backward_rejects(kw, status):
    assert _gnb(**kw) == status


def _lin(**kw):
    a = dict(x=X, xd=0, xl=0, M=100, K=40, N=20, q=Q, sc=S, bias=BE, act=1, sl=0.0, y=Y, yd=1, yl=0,
             ws=WS, wsb=1 << 30, s=None)
    a.update(kw)
    return L.pvconv_fp8_linear(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(M=-1), EINVAL), (dict(K=0), EINVAL), (dict(N=0), EINVAL), (dict(K=70000), EINVAL),
    (dict(xd=5), EINVAL), (dict(yd=5), EINVAL), (dict(act=3), EINVAL), (dict(xl=39), EINVAL),
    (dict(yl=19), EINVAL), (dict(x=None), EINVAL), (dict(q=None), EINVAL), (dict(sc=None), EINVAL),
    (dict(y=None), EINVAL), (dict(q=Q + 8), EINVAL), (dict(bias=ODD), EINVAL), (dict(x=ODD), EINVAL),
    (dict(y=X), EINVAL), (dict(y=Q), EINVAL), (dict(y=BE), EINVAL), (dict(M=0), OK),
    (dict(M=5000, K=4928, N=2048, ws=None), EWS), (dict(M=5000, K=4928, N=2048, wsb=256), EWS),
    (dict(M=1 << 30, K=60000, N=60000), EINVAL),
])
def test_fp8_linear_rejects(kw, status):
    if status == EWS:
        kw = dict(kw, x=1 << 40, y=1 << 42)
    assert _lin(**kw) == status


def _linb(**kw):
    a = dict(dy=DY, dd=0, dl=0, x=X, xd=0, xl=0, M=100, K=40, N=20, q=Q, sc=S, dx=Y, od=0, ol=0,
             dw=DG, db=DB, ws=WS, wsb=1 << 30, s=None)
    a.update(kw)
    return L.pvconv_fp8_linear_backward(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(dx=None, dw=None, db=None), EINVAL), (dict(dy=None), EINVAL), (dict(x=None), EINVAL),
    (dict(q=None), EINVAL), (dict(sc=None), EINVAL), (dict(q=Q + 4), EINVAL), (dict(dw=DB), EINVAL),
    (dict(dx=DY), EINVAL), (dict(dx=X), EINVAL), (dict(dw=X), EINVAL), (dict(db=DY), EINVAL),
    (dict(dl=19), EINVAL), (dict(xl=39), EINVAL), (dict(ol=39), EINVAL), (dict(ws=None), EWS),
    (dict(wsb=1), EWS), (dict(M=0, dw=None, db=None), OK),
])
def test_fp8_linear_backward_rejects(kw, status):
    assert _linb(**kw) == status


def _qw(**kw):
    a = dict(w=X, wd=0, wl=0, N=20, K=40, q=Q, sc=S, qt=Y, st=ST, s=None)
    a.update(kw)
    return L.pvconv_fp8_quantize_weight(*a.values())


@pytest.mark.parametrize("kw", [
    dict(N=0), dict(K=0), dict(wd=3), dict(wl=39), dict(w=None), dict(q=None), dict(sc=None),
    dict(qt=None), dict(st=None), dict(q=Q + 8), dict(qt=Y + 1), dict(w=ODD), dict(q=X),
    dict(qt=Q), dict(sc=Q), dict(st=S),
])
def test_fp8_quantize_weight_rejects(kw):
    assert _qw(**kw) == EINVAL


def _dis(**kw):
    a = dict(z=X, zd=0, zl=0, M=10, V=50, tv=T, tc=C, top=4, lab=None, temp=2.0, al=0.5, rw=None,
             loss=LO, lse=LS, dz=Y, dd=0, dl=0, ws=None, wsb=0, s=None)
    a.update(kw)
    return L.pvconv_distill_topk(*a.values())


BAD_DISTILL = [
    dict(M=-1), dict(V=0), dict(V=(1 << 24) + 1), dict(top=0), dict(top=257), dict(zd=2),
    dict(zl=49), dict(temp=0.0), dict(temp=-1.0), dict(temp=float("nan")), dict(temp=float("inf")),
    dict(al=-0.1), dict(al=1.5), dict(al=float("nan")), dict(z=None), dict(tv=None), dict(tc=None),
    dict(z=ODD), dict(tc=ODD), dict(lab=ODD), dict(dd=7), dict(dl=49), dict(dz=X), dict(dz=T),
    dict(dz=ODD),
]


@pytest.mark.parametrize("kw", BAD_DISTILL + [dict(loss=None), dict(loss=X), dict(lse=LO),
                                              dict(loss=Y), dict(rw=ODD), dict(lse=ODD)])
def test_distill_rejects(kw):
    assert _dis(**kw) == EINVAL


def test_distill_nothing_to_do():
    assert _dis(M=0) == OK


@pytest.mark.parametrize("kw", BAD_DISTILL + [dict(lse=None), dict(dl_=ODD), dict(dz=LS)])
def test_distill_backward_rejects(kw):
    a = dict(z=X, zd=0, zl=0, M=10, V=50, tv=T, tc=C, top=4, lab=None, temp=2.0, al=0.5, lse=LS,
             dl_=None, dz=Y, dd=0, dl=0, s=None)
    a.update(kw)
    assert L.pvconv_distill_topk_backward(*a.values()) == EINVAL


def test_binding_refuses_before_the_library():
    x, v = torch.zeros(2, 5, 8), torch.zeros(8)
    i32 = torch.zeros(2, dtype=torch.int32)
    for bad in (lambda: b.pvconv_group_norm_act(x[0], 2, v, v),
                lambda: b.pvconv_group_norm_act(x, 3, v, v),
                lambda: b.pvconv_group_norm_act(x, 2, v[:4], v),
                lambda: b.pvconv_group_norm_act(x, 2, v.double(), v),
                lambda: b.pvconv_group_norm_act(x, 2, v, v, lengths=i32.long()),
                lambda: b.pvconv_group_norm_act(x.transpose(1, 2), 5, v[:5], v[:5]),
                lambda: b.pvconv_group_norm_act(x[:, :1].expand(2, 5, 8), 2, v, v),
                lambda: b.pvconv_group_norm_act(x, 2, v, v, out=x[:1]),
                lambda: b.pvconv_group_norm_act_backward(x, x[:1], v, 2, v, v),
                lambda: b.pvconv_group_norm_act_backward(x, x, v, 2, v, v),
                lambda: b.pvconv_fp8_quantize_weight(v),
                lambda: b.pvconv_fp8_linear(x, torch.zeros(4, 8, dtype=torch.uint8), i32),
                lambda: b.pvconv_fp8_linear(x, torch.zeros(4, 128, dtype=torch.uint8), i32),
                lambda: b.pvconv_fp8_linear(x, torch.zeros(4, 128, dtype=torch.uint8),
                                            torch.zeros(1, 1, dtype=torch.uint8), bias=v),
                lambda: b.pvconv_fp8_linear_backward(x, None, None, None),
                lambda: b.pvconv_fp8_linear_backward(x, x[:1], None, None, want_dx=False),
                lambda: b.pvconv_fp8_linear_backward(x, x, None, None, False, False, False),
                lambda: b.pvconv_distill_topk(x, v, v),
                lambda: b.pvconv_distill_topk(x[0], torch.zeros(5, 2), torch.zeros(5, 2)),
                lambda: b.pvconv_distill_topk(x[0], torch.zeros(4, 2), i32.view(1, 2).expand(4, 2)),
                lambda: b.pvconv_distill_topk(x[0], torch.zeros(5, 2),
                                              torch.zeros(5, 2, dtype=torch.int32), labels=i32)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        b._dt(x.half())


@pytest.mark.parametrize("temp", [1e-45, 2.0 ** -128])
def test_distill_rejects_a_temperature_without_an_inverse(temp):
    assert _dis(temp=temp) == EINVAL and _dis(temp=temp, M=0) == EINVAL


def test_binding_refuses_a_workspace_that_is_not_whole():
    # many elements that are one byte of memory
    x, v = torch.zeros(2, 5, 8), torch.zeros(8)
    ws = torch.zeros(1, dtype=torch.uint8).expand(1 << 20)
    with pytest.raises(ValueError):
        b.pvconv_group_norm_act(x, 2, v, v, workspace=ws)
    with pytest.raises(ValueError):
        b.pvconv_fp8_linear_backward(x, x, None, None, want_dx=False, workspace=ws)


def test_binding_refuses_sizes_beyond_a_c_int():
    # ctypes would pass their low 32 bits: 2^32 + 5 rows as 5
    v, one = torch.zeros(8), torch.zeros(1)
    bf = dict(dtype=torch.bfloat16, device="meta")
    rows = torch.empty(((1 << 32) + 5, 1), **bf)
    apart = torch.empty_strided((2, 3, 8), (3 * ((1 << 32) + 8), (1 << 32) + 8, 1), **bf)
    q, s = torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(1, 1, dtype=torch.uint8)
    for bad in (lambda: b.pvconv_group_norm_act(rows.view(-1, 1, 1), 1, one, one),
                lambda: b.pvconv_group_norm_act(apart, 2, v, v),
                lambda: b.pvconv_fp8_linear(rows, q.to("meta"), s.to("meta")),
                lambda: b.pvconv_fp8_linear(apart, q.to("meta"), s.to("meta")),
                lambda: b.pvconv_fp8_linear_backward(rows, None, None, None, False, False),
                lambda: b.pvconv_fp8_quantize_weight(rows),
                lambda: b.pvconv_distill_topk(rows, rows.float(), rows.int())):
        with pytest.raises(ValueError, match="2\\^31"):
            bad()
