"""The linear layer in 8-bit integers, its gradients from the kept rows, on the GPU,
against the plain 64-bit forms (_more_ref).

Tolerances, from the arithmetic (u = 2^-24; bf16 rounds by 2^-9 of a value's power of
two, 2^-8 of the value at most):
* bytes and scales: equal.
* y: the sum of products is exact, then one rounding each for its float, the scale
  (the scales' product has 16 bits), the bias and the activation: 4 u (|sum| + |bias|);
  a bf16 output 2^-8 of the value besides.
* dx, dw, fp32: dy's parts hold 24 bits of dy s (dy s itself: one rounding), products
  of bf16 are exact, n terms are summed in 32 bits, in any order: (n + 4) u of the sum
  of magnitudes, sqrt(n) of which would do for random signs: 4 (sqrt(n) + 4) u.
* dx, bf16: dy s is rounded to bf16 before (2^-8 of each term at most: 2^-8 of the sum
  of magnitudes), the result once more.
* dbias: 64-bit sums of up to 256 rows, rounded, 64-bit sums of those: 3 u of the sum
  of magnitudes.
"""
import numpy as np
import pytest
import torch

import _more_ref as ref
from paper_1907_03739_amd import binding as pv
from _helpers import host
from test_gpu_train_ops import check, put

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TD = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(autouse=True)
def _gpu_case(request):
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    print(f"\n[gpu case] {request.node.nodeid}", flush=True)
    yield
    torch.cuda.synchronize()


def step(dt):
    return 2.0 ** -8 if dt == "bf16" else 0.0


def rows_of(M, K, seed):
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(M, K)) * np.exp(rng.normal(size=(M, 1)))
    return np.where(rng.random((M, K)) < 0.3, 0.0, x), rng


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,pad,lead", [
    (1, 1, 0, 0), (3, 7, 0, 0), (5, 8, 3, 1), (67, 127, 0, 0), (130, 128, 8, 0), (33, 129, 1, 2),
    (9, 512, 0, 0), (4, 513, 0, 0), (300, 2048, 0, 0), (5, 2049, 1, 0), (3, 8192, 0, 0),
    (2, 9001, 7, 5), (2, 65536, 0, 0),
])
def test_quantised_rows_are_the_definition_bit_for_bit(M, K, pad, lead, dt):
    x, _ = rows_of(M, K, M + K)
    t = put(x, dt, pad, lead)
    q, s = pv.pvconv_int8_quantize(t)
    wq, ws = ref.int8_rows(host(t))
    assert q.shape == (M, -(-K // 128) * 128)
    np.testing.assert_array_equal(host(s), ws)
    np.testing.assert_array_equal(q.cpu().numpy()[:, :K], wq)
    assert not q.cpu().numpy()[:, K:].any()


def test_borders_scales_and_rows_that_are_not_finite():
    big, tiny = float(np.finfo(np.float32).max), 2.0 ** -149
    rows = np.zeros((14, 260), np.float32)
    rows[0, :] = 0
    rows[1, :255] = (np.arange(255) - 127) * 0.5       # scale 0.5: whole numbers
    rows[2, 0], rows[2, 1:255] = 127, np.arange(254) * 0.5 - 63.5  # scale 1: halves, ties to even
    rows[3, 0], rows[3, 1:255] = 127, np.nextafter(np.float32(np.arange(254) * 0.5 - 63.5),
                                                   np.float32(1e9))
    rows[4, 0], rows[4, 1:255] = 127, np.nextafter(np.float32(np.arange(254) * 0.5 - 63.5),
                                                   np.float32(-1e9))
    rows[5, 0], rows[5, 1] = big, -big
    rows[6, 0], rows[6, 1] = tiny, -5 * tiny
    rows[7, 259] = np.nan
    rows[8, 3] = np.inf
    rows[9, 4] = -np.inf
    rows[10, 0] = 127 * 1.0078125                      # 127 times a scale exactly
    rows[11, 0] = np.nextafter(np.float32(127 * 1.0078125), np.float32(1e9))
    rows[12, 0], rows[12, 1:200] = 127 * 2.0 ** -126, 2.0 ** -127 * np.arange(199)
    rows[13, :] = 2.0 ** -130
    for pad in (0, 3):
        t = put(rows, "f32", pad)
        q, s = pv.pvconv_int8_quantize(t)
        wq, ws = ref.int8_rows(rows)
        np.testing.assert_array_equal(host(s), ws)
        np.testing.assert_array_equal(q.cpu().numpy()[:, :260], wq)


LIN = [
    # M, K, N, x, y, act, bias, pad, lead
    (1, 1, 1, "f32", "f32", "none", True, 0, 0),
    (1, 4928, 256, "f32", "f32", "none", True, 0, 0),
    (1, 64, 4096, "bf16", "bf16", "relu", False, 0, 0),
    (16, 323, 50, "bf16", "f32", "leaky", True, 5, 0),
    (17, 128, 33, "f32", "bf16", "none", False, 0, 3),
    (257, 256, 256, "bf16", "bf16", "relu", True, 0, 0),   # tiles
    (999, 323, 77, "f32", "f32", "leaky", True, 5, 1),
    (1000, 1030, 130, "bf16", "f32", "none", True, 2, 0),
    (4100, 512, 64, "bf16", "bf16", "relu", True, 0, 0),   # few columns
    (2000, 5000, 40, "f32", "f32", "none", True, 0, 0),    # splits
    (700, 9000, 200, "bf16", "bf16", "leaky", True, 0, 0),
    (33000, 512, 1024, "bf16", "bf16", "relu", True, 0, 0),
]


def linear_want(x, w, bias, act):
    q, s = ref.int8_rows(x)
    wq, ws = ref.int8_rows(w)
    total = (q * s[:, None]) @ (wq * ws[:, None]).T
    return ref.activate(total + bias, act), np.abs(total) + np.abs(bias)


@pytest.mark.parametrize("M,K,N,xd,yd,act,has_bias,pad,lead", LIN)
def test_linear(M, K, N, xd, yd, act, has_bias, pad, lead):
    x, rng = rows_of(M, K, 3 * M + K + N)
    xt = put(x, xd, pad, lead)
    wt = put(rng.normal(size=(N, K)) * np.exp(0.5 * rng.normal(size=(N, 1))), xd)
    bias = put(rng.normal(size=N), "f32") if has_bias else None
    wq, ws = pv.pvconv_int8_quantize(wt)
    out = put(np.zeros((M, N)), yd, pad, lead)
    kw = dict(bias=bias, act=act, slope=0.1)
    got = pv.pvconv_int8_linear(xt, wq, ws, out=out, **kw)
    want, mag = linear_want(host(xt), host(wt), host(bias) if has_bias else np.zeros(N), act)
    check(host(got), want, 4 * U * mag + step(yd) * np.abs(want) + 1e-38, "y")
    # the rows kept, and the layer of them: the same bits
    y, rows, scale = pv.pvconv_int8_linear(xt, wq, ws, out_dtype=TD[yd], want_rows=True, **kw)
    again = pv.pvconv_int8_linear_rows(rows, scale, wq, ws, out_dtype=TD[yd], **kw)
    assert torch.equal(y, got) and torch.equal(again, got)
    q, s = pv.pvconv_int8_quantize(xt)
    assert torch.equal(rows, q) and torch.equal(scale, s)


def test_linear_scales_beyond_the_range_of_their_product():
    # s_m s_n leaves the 32-bit range, the result does not
    x = np.ones((300, 96)) * np.where(np.arange(300) % 2, 1e36, 1e-36)[:, None]
    w = np.ones((70, 96)) * np.where(np.arange(70) % 2, 1e-30, 1e30)[:, None]
    xt, wt = put(x, "f32"), put(w, "f32")
    wq, ws = pv.pvconv_int8_quantize(wt)
    want, mag = linear_want(host(xt), host(wt), np.zeros(70), "none")
    with np.errstate(over="ignore"):
        want, mag = want.astype(np.float32).astype(np.float64), mag
    for rows in (xt, xt[:5]):
        got = host(pv.pvconv_int8_linear(rows, wq, ws))
        n = len(got)
        inf = np.isinf(want[:n])
        assert (np.isinf(got) == inf).all()
        check(np.where(inf, 0, got), np.where(inf, 0, want[:n]),
              np.where(inf, 0, 4 * U * mag[:n]) + 2.0 ** -149, "y")


def test_linear_rows_and_channels_that_are_not_finite():
    x, rng = rows_of(200, 300, 5)
    w = rng.normal(size=(90, 300))
    x[3, 5], x[130, 299], w[7, 0] = np.nan, np.inf, -np.inf
    for rows in (x, x[:6]):
        got = host(pv.pvconv_int8_linear(put(rows, "f32"), *pv.pvconv_int8_quantize(put(w, "f32")),
                                         act="relu"))
        bad = ~np.isfinite(rows).all(1)[:, None] | (np.arange(90) == 7)[None]
        np.testing.assert_array_equal(np.isnan(got), bad)


def test_linear_of_clouds_and_of_nothing():
    x, rng = rows_of(6 * 50, 40, 9)
    w = pv.pvconv_int8_quantize(put(rng.normal(size=(24, 40)), "f32"))
    flat = pv.pvconv_int8_linear(put(x, "bf16"), *w)
    cloud = pv.pvconv_int8_linear(put(x, "bf16").view(6, 50, 40), *w)
    assert cloud.shape == (6, 50, 24) and torch.equal(cloud.view(300, 24), flat)
    empty = torch.empty((0, 40), device="cuda")
    assert pv.pvconv_int8_linear(empty, *w).shape == (0, 24)
    y, rows, scale = pv.pvconv_int8_linear(empty, *w, want_rows=True)
    assert rows.shape == (0, 128) and scale.shape == (0,)
    dx, dw, db = pv.pvconv_int8_linear_backward(torch.empty((0, 24), device="cuda"), rows, scale,
                                                *w, 40)
    assert dx.shape == (0, 40) and not dw.any() and not db.any()


BWD = [
    # M, K, N, dy, dx, pad, lead
    (1, 1, 1, "f32", "f32", 0, 0),
    (1, 256, 64, "bf16", "bf16", 0, 0),
    (130, 256, 128, "bf16", "bf16", 0, 0),
    (777, 203, 99, "f32", "f32", 7, 1),
    (777, 203, 99, "bf16", "f32", 0, 0),
    (500, 64, 300, "f32", "bf16", 3, 0),
    (5000, 130, 40, "bf16", "bf16", 0, 5),
    (64, 2304, 512, "bf16", "f32", 0, 0),
    (20000, 70, 24, "f32", "f32", 0, 0),     # long sums, splits
]


def sum_tol(n):
    return 4 * (np.sqrt(n) + 4) * U


@pytest.mark.parametrize("M,K,N,yd,xd,pad,lead", BWD)
def test_backward_from_kept_rows(M, K, N, yd, xd, pad, lead):
    x, rng = rows_of(M, K, 7 * M + K + N)
    w = put(rng.normal(size=(N, K)) * np.exp(0.5 * rng.normal(size=(N, 1))), "f32")
    xt = put(x, "f32")
    dyt = put(1e-3 * rng.normal(size=(M, N)), yd, pad, lead)
    wq, ws = pv.pvconv_int8_quantize(w)
    rows, scale = pv.pvconv_int8_quantize(xt)
    dx, dw, db = pv.pvconv_int8_linear_backward(dyt, rows, scale, wq, ws, K, out_dtype=TD[xd])
    dy = host(dyt)
    q, s = ref.int8_rows(host(xt))
    v, t = ref.int8_rows(host(w))
    xq, wv = q * s[:, None], v * t[:, None]
    want, mag = dy @ wv, np.abs(dy) @ np.abs(wv)
    check(host(dx), want, (sum_tol(N) + step(xd)) * mag + step(xd) * np.abs(want) + 1e-40, "dx")
    want, mag = dy.T @ xq, np.abs(dy).T @ np.abs(xq)
    check(host(dw), want, sum_tol(M) * mag + 1e-40, "dw")
    check(host(db), dy.sum(0), 3 * U * np.abs(dy).sum(0) + 1e-40, "dbias")
    # one at a time: the same bits
    kw = dict(want_dx=False, want_dw=False, want_dbias=False)
    one = pv.pvconv_int8_linear_backward(dyt, None, None, wq, ws, K, out_dtype=TD[xd],
                                         **dict(kw, want_dx=True))
    assert torch.equal(one[0], dx) and one[1] is None and one[2] is None
    one = pv.pvconv_int8_linear_backward(dyt, rows, scale, None, None, K, **dict(kw, want_dw=True))
    assert torch.equal(one[1], dw)
    one = pv.pvconv_int8_linear_backward(dyt, None, None, None, None, K, **dict(kw, want_dbias=True))
    assert torch.equal(one[2], db)


def test_backward_against_differences():
    # of the layer at its quantised values: linear in W's values, x's values and bias
    M, K, N = 40, 24, 10
    x, rng = rows_of(M, K, 77)
    q, s = pv.pvconv_int8_quantize(put(x, "f32"))
    wq, ws = pv.pvconv_int8_quantize(put(rng.normal(size=(N, K)), "f32"))
    dy = put(rng.normal(size=(M, N)), "f32")
    dx, dw, db = pv.pvconv_int8_linear_backward(dy, q, s, wq, ws, K)

    def total(q, wq):
        y = pv.pvconv_int8_linear_rows(q, s, wq, ws, out_dtype=torch.float32)
        return (host(y) * host(dy)).sum()
    for i, k in ((0, 0), (13, 5), (39, 23)):
        a, b = q.clone(), q.clone()
        a[i, k], b[i, k] = 100, -100
        want = (total(a, wq) - total(b, wq)) / (200 * float(s[i]))
        assert abs(float(dx[i, k]) - want) <= 1e-4 * (1 + abs(want))
    for n, k in ((0, 0), (9, 23)):
        a, b = wq.clone(), wq.clone()
        a[n, k], b[n, k] = 100, -100
        want = (total(q, a) - total(q, b)) / (200 * float(ws[n]))
        assert abs(float(dw[n, k]) - want) <= 1e-4 * (1 + abs(want))
