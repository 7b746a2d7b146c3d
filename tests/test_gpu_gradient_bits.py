"""bf16 gradients of the 8-bit integer layer hold 16 bits of every factor inside, whatever
the sizes: what is left of their error is the rounding of the result.

Tolerances, from the arithmetic (u = 2^-24; half a step of bf16 is 2^-8 of a value at most,
so that two parts of a value leave 2^-8 of 2^-8 of it, 2^-16):
* dx of the layer, bf16 dy: the scaled weight (15 bits) is two parts exactly, products are
  exact, n terms are summed in 32 bits: 4 (sqrt(n) + 4) u of the sum of magnitudes, then
  the result's rounding, 2^-8 of it. fp32 dy: dy times its scale leaves u + 2^-16 of each
  term besides.
"""
import numpy as np
import pytest
import torch

import _more_ref as ref
from paper_1907_03739_amd import binding as pv
from _helpers import host
from test_gpu_int8 import U, rows_of, sum_tol
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
