"""bf16 gradients of the 8-bit integer layer and of the linear cross entropy hold 16 bits of
every factor inside, whatever the sizes: what is left of their error is the rounding of
the result.

Tolerances, from the arithmetic (u = 2^-24; half a step of bf16 is 2^-8 of a value at most,
so that two parts of a value leave 2^-8 of 2^-8 of it, 2^-16):
* dx of the layer, bf16 dy: the scaled weight (15 bits) is two parts exactly, products are
  exact, n terms are summed in 32 bits: 4 (sqrt(n) + 4) u of the sum of magnitudes, then
  the result's rounding, 2^-8 of it. fp32 dy: dy times its scale leaves u + 2^-16 of each
  term besides.
* dx and dw of the loss: dz in two parts, 2^-16 of each term; the other factor the same
  where it is fp32, and the product of both second parts, which is left out, the same
  again (bf16 ones are exact); dz's own error and the sums as in test_gpu_linear_ce.
"""
import numpy as np
import pytest
import torch

import _more_ref as ref
from paper_1907_03739_amd import binding as pv
from _helpers import host
from test_gpu_int8 import rows_of
from test_gpu_linear_ce import TD, U, inputs, sum_tol, tolerances
from test_gpu_train_ops import check, put

pytestmark = pytest.mark.gpu
HALF, TWO = 2.0 ** -8, 2.0 ** -16


@pytest.fixture(autouse=True)
def _gpu_case(request):
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    print(f"\n[gpu case] {request.node.nodeid}", flush=True)
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("yd", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N", [
    (1, 512, 130), (256, 700, 130), (257, 700, 130), (257, 20, 9), (600, 101, 120),
    (4100, 512, 300), (9000, 300, 64),
])
def test_dx_of_the_8_bit_layer(M, K, N, yd):
    _, rng = rows_of(1, 1, M + K + N)
    w = put(rng.normal(size=(N, K)) * np.exp(0.5 * rng.normal(size=(N, 1))), "f32")
    dyt = put(1e-3 * rng.normal(size=(M, N)) * np.exp(rng.normal(size=(M, 1))), yd)
    wq, ws = pv.pvconv_int8_quantize(w)
    kw = dict(want_dw=False, want_dbias=False, out_dtype=torch.bfloat16)
    dx = pv.pvconv_int8_linear_backward(dyt, None, None, wq, ws, K, **kw)[0]
    v, t = ref.int8_rows(host(w))
    dy, wv = host(dyt), v * t[:, None]
    want, mag = dy @ wv, np.abs(dy) @ np.abs(wv)
    inside = (0.0 if yd == "bf16" else TWO + U) + sum_tol(N)
    check(host(dx), want, inside * (1 + HALF) * mag + HALF * np.abs(want) + 1e-38, "dx")


def _sharp(r, x, w, weight, xd, wd):
    """The tolerances of bf16 gradients whose factors keep 16 bits."""
    f = "f32"  # (the form of an fp32 result: dz's error, 2 u for the factors, the sums)
    _, tdx, tdw, tdb = tolerances(r, x, w, weight, xd, wd, f, f)
    dz = np.abs(r["dz"])
    tdx = tdx + (1 if wd == "bf16" else 3) * TWO * (dz @ np.abs(w))
    tdw = tdw + (1 if xd == "bf16" else 3) * TWO * (dz.T @ np.abs(x))
    return (tdx * (1 + HALF) + HALF * np.abs(r["dx"]), tdw * (1 + HALF) + HALF * np.abs(r["dw"]),
            tdb)


SIZES = [
    # M, K, V, x, w
    (1, 40, 65, "bf16", "bf16"), (256, 40, 300, "bf16", "bf16"), (257, 40, 300, "bf16", "bf16"),
    (257, 64, 64, "bf16", "f32"), (257, 64, 65, "bf16", "f32"), (700, 130, 65, "f32", "bf16"),
    (1000, 100, 777, "f32", "f32"), (5000, 72, 200, "bf16", "bf16"),
]


def _check_loss_gradients(x, w, b, label, weight, xd, wd):
    kw = dict(bias=b, out_dtype=torch.bfloat16, dw_dtype=torch.bfloat16)
    loss, lse, *fused = pv.pvconv_linear_cross_entropy(x, w, label, row_weight=weight,
                                                       want_grad=True, **kw)
    split = pv.pvconv_linear_cross_entropy_backward(x, w, label, lse, weight, **kw)
    hx, hw, hg = host(x), host(w), host(weight)
    r = ref.linear_ce(hx, hw, host(b), label.cpu().numpy(), hg)
    tols = _sharp(r, hx, hw, hg, xd, wd)
    for got in (fused, split):
        for name, a, tol in zip(("dx", "dw", "db"), got, tols):
            check(host(a), r[name], tol, name)


@pytest.mark.parametrize("M,K,V,xd,wd", SIZES)
def test_gradients_of_the_loss(M, K, V, xd, wd):
    _check_loss_gradients(*inputs(M, K, V, xd, wd, M + K + V), xd, wd)


@pytest.mark.parametrize("M", [257, 5000])
def test_the_mean_over_rows_of_an_unsure_layer(M):
    # every row has the weight 1 / M and probabilities near 1 / V: each label's dz is nearly
    # the same number, whose rounding to fewer bits nothing would average
    x, w, b, label, _ = inputs(M, 48, 300, "bf16", "bf16", M, scale=0.05)
    label[label < 0] = 0
    b *= 0
    weight = torch.full((M,), 1.0 / M, device="cuda")
    _check_loss_gradients(x, w, b, label, weight, "bf16", "bf16")
    kw = dict(bias=b, row_weight=weight, want_grad=True)
    got = pv.pvconv_linear_cross_entropy(x, w, label, **kw)[2:4]
    want = pv.pvconv_linear_cross_entropy(x, w, label, out_dtype=torch.float32,
                                          dw_dtype=torch.float32, **kw)[2:4]
    for a, e in zip(got, want):
        # no common factor: a result's roundings have either sign. Of n of them, each within
        # 2^-8, the weighed mean is within 6 / sqrt(n) of that, and 2^-16 of what is inside
        # times the sum of magnitudes over the result's (at most 2^6 here)
        a, e = host(a).ravel(), host(e).ravel()
        bound = HALF * 6 * np.sqrt((e ** 4).sum()) / (e * e).sum() + TWO * 64
        assert abs((a * e).sum() / (e * e).sum() - 1) <= bound
