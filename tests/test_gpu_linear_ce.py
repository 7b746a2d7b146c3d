"""The cross entropy of a linear layer without its logits, on the GPU, against the
plain 64-bit form (_more_ref), forward and gradients.

Tolerances, from the arithmetic (u = 2^-24; a bf16 rounding is 2^-8 of the value at
most):
* a logit: products are exact (bf16) or good to 2^-24, K of them are summed in 32
  bits: Z = (4 (sqrt(K) + 4)) u sum |x w| + 4 u |z|, of the row's largest.
* lse and loss: 2 Z, exponentials of differences (|d| + 4 u relative, weighed by the
  exponential itself: 4 u), logarithm and sums: 16 u (1 + |lse| + |z_label|).
* dz: weight times (p (2 Z + 64 u) + u [class = label]): an exponential's argument
  is off by 2 Z and by (|d| + 4) u, |d| < 60 here.
* dx, dw: dz's error, its rounding and the other factor's (2^-8 each for a bf16
  output, u for fp32), n terms summed in 32 bits (4 (sqrt(n) + 4) u of the sum of
  magnitudes), the output's rounding. dbias: dz's error and 32-bit sums of up to 128
  rows: 64 u of the sum of magnitudes.
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
    return 2.0 ** -8 if dt == "bf16" else U


def sum_tol(n):
    return 4 * (np.sqrt(n) + 4) * U


def inputs(M, K, V, xd, wd, seed, pad=0, lead=0, scale=2.0):
    rng = np.random.default_rng(seed)
    x = put(rng.normal(size=(M, K)) * np.exp(0.3 * rng.normal(size=(M, 1))), xd, pad, lead)
    w = put(rng.normal(size=(V, K)) * scale / np.sqrt(K), wd, pad, lead)
    b = put(0.3 * rng.normal(size=V), "f32")
    label = rng.integers(0, V, M)
    label[rng.random(M) < 0.1] = -1
    weight = rng.random(M)
    weight[rng.random(M) < 0.1] = 0
    return (x, w, b, torch.tensor(label, dtype=torch.int32, device="cuda"), put(weight, "f32"))


def tolerances(r, x, w, weight, xd, wd, dxd, dwd):
    M, K = x.shape
    V = w.shape[0]
    zz = np.where(np.isneginf(r["z"]), 0.0, r["z"])
    Z = (sum_tol(K) * (np.abs(x) @ np.abs(w).T).max(1) + 4 * U * np.abs(zz).max(1))
    g = np.abs(weight)
    live = np.abs(r["dz"]).sum(1) > 0
    onehot = (r["dz"] * np.sign(weight)[:, None] < 0) & live[:, None]
    p = np.where(live[:, None], np.abs(r["dz"]) / np.where(g == 0, 1, g)[:, None], 0)
    p = np.where(onehot, 1 - p, p)
    edz = g[:, None] * (p * (2 * Z + 64 * U)[:, None] + onehot * U)
    mag = g[:, None] * (p + onehot)
    tdx = (edz + np.abs(r["dz"]) * (2 * step(dxd))) @ np.abs(w) + sum_tol(V) * (mag @ np.abs(w)) \
        + step(dxd) * np.abs(r["dx"]) + 1e-37
    tdw = (edz + np.abs(r["dz"]) * (2 * step(dwd))).T @ np.abs(x) + \
        sum_tol(M) * (mag.T @ np.abs(x)) + step(dwd) * np.abs(r["dw"]) + 1e-37
    tdb = edz.sum(0) + 64 * U * mag.sum(0) + 1e-37
    tl = 2 * Z + 16 * U * (1 + np.abs(r["lse"]) + np.abs(zz).max(1))
    return tl, tdx, tdw, tdb


CASES = [
    # M, K, V, x, w, dx, dw, bias, pad, lead
    (1, 1, 1, "f32", "f32", "f32", "f32", True, 0, 0),
    (1, 512, 2003, "bf16", "bf16", "bf16", "bf16", True, 0, 0),
    (3, 7, 5, "f32", "bf16", "f32", "bf16", False, 2, 1),
    (300, 128, 50, "bf16", "f32", "bf16", "f32", True, 0, 0),     # whole rows in a wave
    (129, 64, 64, "bf16", "bf16", "f32", "f32", True, 0, 0),
    (129, 64, 65, "bf16", "bf16", "bf16", "bf16", True, 8, 0),
    (1000, 256, 13, "bf16", "bf16", "bf16", "bf16", False, 0, 0),
    (64, 130, 128, "f32", "f32", "bf16", "f32", True, 0, 3),
    (257, 323, 1003, "f32", "f32", "f32", "f32", True, 5, 0),
    (500, 200, 777, "bf16", "f32", "f32", "bf16", True, 1, 0),
    (130, 192, 5000, "bf16", "bf16", "bf16", "bf16", True, 64, 8),  # rows that are read in place
    (2000, 64, 129, "f32", "bf16", "bf16", "f32", True, 0, 0),
    (5000, 40, 300, "bf16", "bf16", "bf16", "f32", True, 0, 0),     # splits
]


@pytest.mark.parametrize("M,K,V,xd,wd,dxd,dwd,has_bias,pad,lead", CASES)
def test_loss_and_gradients(M, K, V, xd, wd, dxd, dwd, has_bias, pad, lead):
    x, w, b, label, weight = inputs(M, K, V, xd, wd, M + K + V, pad, lead)
    if V > 8 and has_bias:
        b[-(V // 8):] = -float("inf")  # a vocabulary's padding
        label[label >= V - V // 8] = 0
    bias = b if has_bias else None
    kw = dict(bias=bias)
    dt = dict(out_dtype=TD[dxd], dw_dtype=TD[dwd])
    loss, lse = pv.pvconv_linear_cross_entropy(x, w, label, **kw)
    hx, hw, hg = host(x), host(w), host(weight)
    with np.errstate(invalid="ignore"):
        r = ref.linear_ce(hx, hw, host(b) if has_bias else None, label.cpu().numpy(), hg)
    tl, tdx, tdw, tdb = tolerances(r, hx, hw, hg, xd, wd, dxd, dwd)
    check(host(lse), r["lse"], tl, "lse")
    check(host(loss), r["loss"], tl, "loss")
    got = pv.pvconv_linear_cross_entropy(x, w, label, row_weight=weight, want_grad=True, **kw, **dt)
    check(host(got[0]), r["loss"], tl, "loss, one call")
    check(host(got[1]), r["lse"], tl, "lse, one call")
    split = pv.pvconv_linear_cross_entropy_backward(x, w, label, lse, weight, **kw, **dt)
    for name, a in (("one call", got[2:]), ("two calls", split)):
        check(host(a[0]), r["dx"], tdx, f"dx, {name}")
        check(host(a[1]), r["dw"], tdw, f"dw, {name}")
        check(host(a[2]), r["db"], tdb, f"dbias, {name}")
        assert a[0].dtype == TD[dxd] and a[1].dtype == TD[dwd]
    assert not host(got[2])[hg == 0].any() or (hg != 0).all()
    again = pv.pvconv_linear_cross_entropy(x, w, label, row_weight=weight, want_grad=True, **kw,
                                           **dt)
    for a, c in zip(got, again):
        assert torch.equal(a, c)  # the same bits on every run
    # one gradient at a time: the same bits
    for i, want in enumerate(("want_dx", "want_dw", "want_dbias")):
        off = {k: k == want for k in ("want_dx", "want_dw", "want_dbias")}
        one = pv.pvconv_linear_cross_entropy_backward(x, w, label, lse, weight, **kw, **dt, **off)
        assert torch.equal(one[i], split[i])
        assert [t is None for t in one] == [j != i for j in range(3)]


def test_pieces_of_the_vocabulary():
    # six parts of 20032 rows: a piece of the backward holds 2048 classes
    M, K, V = 20000, 9, 2305
    x, w, b, label, weight = inputs(M, K, V, "f32", "f32", 5)
    r = ref.linear_ce(host(x), host(w), host(b), label.cpu().numpy(), host(weight))
    tl, tdx, tdw, tdb = tolerances(r, host(x), host(w), host(weight), "f32", "f32", "f32", "f32")
    loss, lse, dx, dw, db = pv.pvconv_linear_cross_entropy(x, w, label, bias=b, row_weight=weight,
                                                           want_grad=True)
    check(host(loss), r["loss"], tl, "loss")
    check(host(dx), r["dx"], tdx, "dx")
    check(host(dw), r["dw"], tdw, "dw")
    check(host(db), r["db"], tdb, "dbias")


def test_pieces_of_the_forward():
    # statistics of 140000 rows: a piece of the forward holds 4096 classes
    M, K, V = 140000, 16, 4200
    x, w, b, label, _ = inputs(M, K, V, "bf16", "bf16", 6)
    loss, lse = pv.pvconv_linear_cross_entropy(x, w, label, bias=b)
    at = np.concatenate([np.arange(0, M, 977), np.arange(M - 130, M)])
    hx, hw = host(x)[at], host(w)
    r = ref.linear_ce(hx, hw, host(b), label.cpu().numpy()[at])
    tl = tolerances(r, hx, hw, np.ones(len(at)), "bf16", "bf16", "bf16", "bf16")[0]
    check(host(lse)[at], r["lse"], tl, "lse")
    check(host(loss)[at], r["loss"], tl, "loss")


@pytest.mark.parametrize("V", [50, 200, 2500])
def test_rows_that_nothing_is_left_of(V):
    M, K = 140, 48
    x, w, b, label, weight = inputs(M, K, V, "f32", "f32", V)
    weight += 1
    # every class masked: lse -inf, no loss, no gradient
    none = torch.full_like(b, -float("inf"))
    loss, lse, dx, dw, db = pv.pvconv_linear_cross_entropy(x, w, label, bias=none,
                                                           row_weight=weight, want_grad=True)
    assert torch.isneginf(lse).all()
    for t in (loss, dx, dw, db):
        assert not t.any()
    # masked by the type's lowest value: the logits differ by nothing
    low = torch.full_like(b, torch.finfo(torch.float32).min)
    loss, lse, dx, dw, db = pv.pvconv_linear_cross_entropy(x, w, label, bias=low,
                                                           row_weight=weight, want_grad=True)
    assert all(torch.isfinite(t).all() for t in (loss, lse, dx, dw, db))
    # no row has a label
    nobody = torch.full_like(label, V)
    loss, lse, dx, dw, db = pv.pvconv_linear_cross_entropy(x, w, nobody, bias=b,
                                                           row_weight=weight, want_grad=True)
    assert torch.isfinite(lse).all()
    for t in (loss, dx, dw, db):
        assert not t.any()
    # extreme labels, a label whose class is masked
    odd = label.clone()
    odd[0], odd[1], odd[2] = -2 ** 31, 2 ** 31 - 1, 1
    mask = b.clone()
    mask[1] = -float("inf")
    odd[3:] = torch.where(odd[3:] == 1, 0, odd[3:])
    loss, lse = pv.pvconv_linear_cross_entropy(x, w, odd, bias=mask)
    assert loss[0] == 0 and loss[1] == 0 and torch.isposinf(loss[2])
    assert torch.isfinite(loss[3:]).all()


@pytest.mark.parametrize("V", [50, 200])
def test_values_that_are_not_finite(V):
    M, K = 70, 64
    for xd in ("f32", "bf16"):
        x, w, b, label, weight = inputs(M, K, V, xd, "f32", 3 * V)
        label[label < 0] = 0
        x[5, 3], x[64, 0] = float("nan"), float("nan")
        loss, lse, dx, dw, db = pv.pvconv_linear_cross_entropy(x, w, label, bias=b,
                                                               row_weight=weight + 1,
                                                               want_grad=True)
        bad = np.isin(np.arange(M), (5, 64))
        np.testing.assert_array_equal(np.isnan(host(loss)), bad)
        np.testing.assert_array_equal(np.isnan(host(lse)), bad)
        np.testing.assert_array_equal(np.isnan(host(dx)).all(1), bad)
        np.testing.assert_array_equal(np.isnan(host(dx)).any(1), bad)
        up = b.clone()
        up[7] = float("inf")
        loss, lse = pv.pvconv_linear_cross_entropy(x[10:20], w, label[10:20], bias=up)
        assert torch.isnan(loss).all() and torch.isnan(lse).all()


def test_no_rows_and_clouds_of_rows():
    x, w, b, label, weight = inputs(6 * 40, 32, 50, "bf16", "bf16", 1)
    flat = pv.pvconv_linear_cross_entropy(x, w, label, bias=b, row_weight=weight, want_grad=True)
    cloud = pv.pvconv_linear_cross_entropy(x.view(6, 40, 32), w, label, bias=b, row_weight=weight,
                                           want_grad=True)
    assert cloud[2].shape == (6, 40, 32)
    for a, c in zip(flat, cloud):
        assert torch.equal(a, c.view(a.shape))
    for V in (50, 100):
        loss, lse, dx, dw, db = pv.pvconv_linear_cross_entropy(
            x[:0], put(np.ones((V, 32)), "f32"), label[:0], want_grad=True)
        assert loss.shape == (0,) and dx.shape == (0, 32) and not dw.any() and not db.any()


def test_gradients_against_differences():
    M, K, V = 30, 20, 90
    x, w, b, label, weight = inputs(M, K, V, "f32", "f32", 8)
    dx, dw, db = pv.pvconv_linear_cross_entropy(x, w, label, bias=b, row_weight=weight,
                                                want_grad=True)[2:]

    def total(x, w, b):
        return (host(pv.pvconv_linear_cross_entropy(x, w, label, bias=b)[0]) * host(weight)).sum()
    rng, e = np.random.default_rng(0), 2.0 ** -6
    for t, grad in ((x, dx), (w, dw), (b, db)):
        d = put(rng.normal(size=tuple(t.shape)), "f32")
        args = [dict(zip("xwb", (x, w, b))), dict(zip("xwb", (x, w, b)))]
        key = "x" if t is x else "w" if t is w else "b"
        args[0][key], args[1][key] = t + e * d, t - e * d
        num = (total(**args[0]) - total(**args[1])) / (2 * e)
        want = (host(grad) * host(d)).sum()
        # e^2 / 6 of a third derivative of a sum over 30 rows, losses good to 1e-6 each
        assert abs(num - want) <= 2e-2 * (1 + abs(want)), key
