"""The training and 8-bit operators where few digits or little range are left
(statistics of far means, huge and tiny spreads, masks of the lowest value), beside
values that are not finite, and on both sides of the rules that choose a kernel. The
tolerances are those of test_gpu_train_ops.py unless a test derives its own."""
import numpy as np
import pytest
import torch

import _train_ref as ref
from paper_1907_03739_amd import binding as pv
from _helpers import host

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TD = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(autouse=True)
def _gpu_case(request):
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    print(f"\n[gpu case] {request.node.nodeid}", flush=True)
    yield
    torch.cuda.synchronize()


def put(a, dt="f32"):
    return torch.as_tensor(np.asarray(a, np.float32)).cuda().to(TD[dt])


# 16 channels in 2 groups: vectors of 8 (bf16) or 4; 21 in 3: single elements across
# groups of 7
@pytest.mark.parametrize("N", [5, 200, 3000, 20000])
@pytest.mark.parametrize("C,G", [(16, 2), (21, 3)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [2.0 ** 63, 2.0 ** -83])
def test_group_norm_statistics_keep_their_range(N, C, G, dt, scale):
    # squares of these are beyond, or below, what 32 bits hold
    rng = np.random.default_rng(N + C)
    xt = put(rng.normal(size=(2, N, C)) * scale, dt)
    x = host(xt)
    one, zero = put(np.ones(C)), put(np.zeros(C))
    y, st = pv.pvconv_group_norm_act(xt, G, one, zero, eps=0.0, act="none", want_stats=True,
                                     out_dtype=torch.float32)
    ry, rs = ref.group_norm(x, G, np.ones(C), np.zeros(C), 0.0, "none", 0.0)
    assert (np.abs(host(st)[..., 1] - rs[..., 1]) <= 1e-6 * rs[..., 1]).all()
    mag = np.abs(x) * np.repeat(rs[..., 1], C // G, 1)[:, None] + 1
    assert (np.abs(host(y) - ry) <= 16 * U * mag).all()


@pytest.mark.parametrize("N", [5, 200, 3000, 20000])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_group_norm_means_of_terms_that_cancel(N, dt):
    # 2^33 and its negative beside small whole numbers: the mean, of 64-bit sums
    # that lose nothing here, rounds once
    rng = np.random.default_rng(N)
    x = rng.integers(1, 9, (2, N, 16)).astype(np.float64)
    x[..., 1::8], x[..., 6::8] = 2.0 ** 33, -(2.0 ** 33)
    st = pv.pvconv_group_norm_act(put(x, dt), 2, put(np.ones(16)), put(np.zeros(16)),
                                  want_stats=True)[1]
    rs = ref.group_norm(x, 2, np.ones(16), np.zeros(16), 1e-5, "none", 0.0)[1]
    assert (np.abs(host(st)[..., 0] - rs[..., 0]) <= 4 * U * np.abs(rs[..., 0])).all()


@pytest.mark.parametrize("N", [5, 200, 3000, 20000])
@pytest.mark.parametrize("C,G", [(16, 2), (21, 3), (40, 40)])
@pytest.mark.parametrize("first", [0, 1])
def test_group_norm_spread_beside_a_very_far_mean(N, C, G, first):
    # values of 2^22 + 0 .. 7.5: E[x^2] - mean^2 in 64 bits has 9 binary digits left.
    # first = 1: an empty cloud, and rows past a cloud's length that are NaN, beside it
    rng = np.random.default_rng(N)
    x = 2.0 ** 22 + rng.integers(0, 16, (2, N, C)) / 2
    lengths, xt = None, put(x)
    if first:
        lengths = [0, N - N // 3]
        xt[0], xt[1, lengths[1]:] = float("nan"), float("nan")
    lt = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    y, st = pv.pvconv_group_norm_act(xt, G, put(np.ones(C)), put(np.zeros(C)), lengths=lt,
                                     want_stats=True)
    rs = ref.group_norm(x, G, np.ones(C), np.zeros(C), 1e-5, "none", 0.0, lengths)[1]
    assert (np.abs(host(st)[..., 0] - rs[..., 0]) <= 4 * U * np.abs(rs[..., 0])).all()
    assert (np.abs(host(st)[..., 1] - rs[..., 1]) <= 1e-6 * rs[..., 1]).all()
    if first:
        assert (y[0] == 0).all() and (y[1, lengths[1]:] == 0).all()
    assert torch.isfinite(y).all()


# both sides of each rule that chooses between a group in a workgroup's registers and
# the sums in chunks, forward or gradient
@pytest.mark.parametrize("B,N,C,G,dt,lengths", [
    (512, 1, 128, 8, "bf16", None), (513, 1, 128, 8, "bf16", None),   # 4096 groups
    (4096, 3, 64, 2, "f32", None),
    (64, 3, 128, 8, "bf16", None), (65, 3, 128, 8, "bf16", None),     # 8192 channels
    (2, 5, 264, 8, "f32", None), (2, 5, 256, 8, "f32", None),         # 33 and 32 a group
    (64, 256, 256, 32, "f32", None), (65, 191, 256, 32, "f32", None),  # full workgroups
    (64, 512, 128, 8, "bf16", None), (65, 512, 128, 8, "bf16", None),  # 512 groups
    (11, 4096, 64, 8, "bf16", None), (1, 4097, 64, 8, "bf16", [4000]),  # 32768 values a group
    (12, 2048, 128, 8, "bf16", None), (24, 2048, 128, 8, "bf16", None),
    (23, 2048, 128, 8, "bf16", None), (2, 1024, 128, 8, "bf16", [1024, 3]),
    (32, 900, 96, 32, "f32", None), (24, 700, 96, 32, "bf16", None),  # single elements
    (300, 2, 459, 3, "f32", None), (2, 6, 1088, 8, "bf16", [6, 1]),  # a thread a channel
])
def test_group_norm_on_both_sides_of_its_rules(B, N, C, G, dt, lengths):
    import test_gpu_train_ops as ops
    ops.test_group_norm_forward_and_gradients(B, N, C, G, dt, dt, "silu", lengths, 0, 0)


# the type's lowest value as a mask of whole rows, where 1 / T > 1 takes it beyond the
# type: rows of lanes, and of a workgroup
@pytest.mark.parametrize("V", [13, 700, 5000])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("alpha", [1.0, 0.5])
def test_distill_lowest_values_at_a_low_temperature(V, dt, alpha):
    rng = np.random.default_rng(V)
    M, top, T = 6, 4, 0.5
    zt = put(rng.normal(size=(M, V)), dt)
    lowest = torch.finfo(zt.dtype).min
    zt[1] = lowest                              # nothing left over T: 0, no gradient
    zt[2, 3:] = lowest
    val = rng.normal(size=(M, top)).astype(np.float32)
    val[3] = np.finfo(np.float32).min           # a teacher of it: uniform
    val[4, 1:] = np.finfo(np.float32).min
    cls = np.tile(np.arange(top, dtype=np.int32), (M, 1))
    cls[2] = [0, 1, 2, -1]
    labels = np.zeros(M, np.int32)
    tv, tc, lt = (torch.as_tensor(a).cuda() for a in (val, cls, labels))
    kw = dict(labels=lt, temperature=T, alpha=alpha)
    loss, _, dz = pv.pvconv_distill_topk(zt, tv, tc, want_grad=True, **kw)
    loss2, lse = pv.pvconv_distill_topk(zt, tv, tc, **kw)
    dz2 = pv.pvconv_distill_topk_backward(zt, tv, tc, lse, **kw)
    # (equal entries, given to the oracle as zeros: at their own size even 64 bits would
    # not hold log 4 beside them)
    tval = np.where(np.arange(M)[:, None] == 3, 0.0, val.astype(np.float64))
    rl, rg = ref.distill(host(zt), tval, cls, labels, T, alpha)
    rl[1], rg[1] = 0, 0
    step = 2.0 ** -8 if dt == "bf16" else 0.0
    for l, g in ((loss, dz), (loss2, dz2)):
        assert (np.abs(host(l) - rl) <= 2e-5 * (1 + 4 * T * T + np.abs(rl))).all()
        assert (np.abs(host(g) - rg) <= 2e-5 * (1 + T) + step * np.abs(rg)).all()


# Gradients whose vectors run across groups, without a rectifier's jumps (none, SiLU):
# the bound of dx is then that of the rounding alone, 64 u of the terms. Groups of 3 and
# of 10 channels in vectors of 4, and of 25 and 15 in vectors of 8 (bf16).
@pytest.mark.parametrize("B,N,C,G,dt", [(1, 30000, 96, 32, "f32"), (2, 9000, 60, 6, "f32"),
                                        (2, 9000, 200, 8, "bf16"), (2, 30000, 120, 8, "bf16")])
@pytest.mark.parametrize("act", ["none", "silu"])
def test_group_norm_gradients_across_groups(B, N, C, G, dt, act):
    import test_gpu_train_ops as ops
    lengths = None if B == 1 else [N, N // 2 + 1]
    ops.test_group_norm_forward_and_gradients(B, N, C, G, dt, dt, act, lengths, 0, 0)


# A rectifier's derivative jumps where v is 0, and an element within the rounding of v
# may take either side. That changes its own dx by r |gamma dy| (1 - slope), and the
# others of its group by r (|gamma dy| + |xh| |gamma dy xh|) / n only, through the means.
@pytest.mark.parametrize("B,N,C,G,dt,act,lengths", [
    (1, 30000, 96, 32, "f32", "relu", None), (2, 9000, 60, 6, "f32", "leaky", [9000, 777]),
    (3, 577, 60, 6, "f32", "leaky", None), (2, 9000, 200, 8, "bf16", "relu", None),
    (4, 2048, 128, 8, "bf16", "relu", [2048, 1, 0, 2047])])
def test_group_norm_rectifier_gradients(B, N, C, G, dt, act, lengths):
    import test_gpu_train_ops as ops
    x, gamma, beta, rng = ops.gn_inputs(B, N, C, 300 + N + C)
    xt, dyt = put(x, dt), put(rng.normal(size=x.shape), dt)
    x, dy = host(xt), host(dyt)
    lt = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    kw = dict(act=act, slope=0.1, lengths=lt)
    _, st = pv.pvconv_group_norm_act(xt, G, put(gamma), put(beta), want_stats=True, **kw)
    dx, dg, db = pv.pvconv_group_norm_act_backward(dyt, xt, st, G, put(gamma), put(beta), **kw)
    st = host(st)
    rdx, rdg, rdb, mg, mb = ref.group_norm_backward(dy, x, G, gamma, beta, 1e-5, act, 0.1, lengths, st)
    W = C // G
    mean, r = (np.repeat(st[:, :, i], W, 1)[:, None] for i in (0, 1))
    xh = (x - mean) * r
    n = np.array(lengths or [N] * B)[:, None, None]
    live = np.arange(N)[None, :, None] < n
    mag = (np.abs(x) + np.abs(mean)) * r * np.abs(gamma) + np.abs(beta)
    jump = np.abs(dy) * ((np.abs(xh * gamma + beta) <= 16 * U * mag) & live)
    group = lambda a: np.repeat(a.reshape(B, N, G, W).sum((1, 3)), W, 1)[:, None] / np.maximum(n * W, 1)
    own = np.abs(gamma) * jump
    shift = group(own) + np.abs(xh) * group(own * np.abs(xh))
    size = r * np.abs(gamma * dy)
    top = np.repeat(np.where(live, size, 0).reshape(B, N, G, W).max((1, 3)), W, 1)[:, None]
    tol = 64 * U * (size + top * (1 + np.abs(xh))) + r * (own + shift)
    step = 2.0 ** -8 if dt == "bf16" else 0.0
    ops.check(host(dx), rdx, tol + step * np.abs(rdx), "dx")
    # the bound is one that a wrong dx does not meet
    assert (np.abs(rdx) > 100 * tol).mean() > 0.4 * live.mean()
    ops.check(host(dg), rdg, 64 * U * mg + (jump * np.abs(xh)).sum((0, 1)) + 1e-30, "dgamma")
    ops.check(host(db), rdb, 64 * U * mb + jump.sum((0, 1)) + 1e-30, "dbeta")


# A value that is not finite becomes NaN in its own place and does not count for its
# block's largest: seen in the scale and the other values of a quantised weight.
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("N,K", [(130, 257), (5, 3), (128, 128)])
@pytest.mark.parametrize("transposed", [False, True])
def test_fp8_weights_that_are_not_finite(dt, N, K, transposed):
    rng = np.random.default_rng(N)
    w = rng.normal(size=(N, K))
    bad = [(0, 0, np.inf), (N - 1, K - 1, np.nan), (N // 2, K // 2, -np.inf)]
    for i, j, v in bad:
        w[i, j] = v
    wt = put(w, dt)
    w = host(wt)
    v, e = ref.quantise_weight(w)
    out = pv.pvconv_fp8_quantize_weight(wt, transposed=transposed)
    for q, s, want, es, rows, cols in ((out[0], out[1], v, e, N, K),) + (
            ((out[2], out[3], v.T, e.T, K, N),) if transposed else ()):
        assert (s.cpu().numpy().astype(int) - 127 == es).all()
        scale = 2.0 ** np.repeat(np.repeat(es, 128, 0)[:rows], 128, 1)[:, :cols]
        got = q.float().cpu().numpy().astype(np.float64)[:, :cols] * scale
        assert (np.isnan(got) == np.isnan(want)).all() and np.isnan(want).sum() == len(bad)
        assert (got[np.isfinite(want)] == want[np.isfinite(want)]).all()


# The same of the weight's gradient, whose blocks run along the rows of dy and x: the
# channel of a value that is not finite is NaN, every other one is whole.
@pytest.mark.parametrize("M,K,N", [(300, 40, 24), (5000, 300, 130), (40, 5, 3)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_fp8_gradients_that_are_not_finite(M, K, N, dt):
    rng = np.random.default_rng(M)
    x, dy, w = rng.normal(size=(M, K)), rng.normal(size=(M, N)), rng.normal(size=(N, K))
    x[M // 2, K - 1], dy[7, 0] = np.inf, np.nan
    xt, dyt = put(x, dt), put(dy, dt)
    x, dy = host(xt), host(dyt)
    _, _, qt, st = pv.pvconv_fp8_quantize_weight(put(w), transposed=True)
    dx, dw, db = (host(t) for t in pv.pvconv_fp8_linear_backward(dyt, xt, qt, st,
                                                                out_dtype=torch.float32))
    assert np.isnan(dw[0]).all() and np.isnan(dw[:, K - 1]).all()
    qc, xc = ref.quantise(dy, 0)[0][:, 1:], ref.quantise(x, 0)[0][:, :K - 1]
    want, mag = qc.T @ xc, np.abs(qc).T @ np.abs(xc)
    assert (np.abs(dw[1:, :K - 1] - want) <= (4 * np.sqrt(M) + 8) * U * mag).all()
    assert np.isnan(db[0]) and np.isfinite(db[1:]).all()
    assert np.isnan(dx[7]).all() and np.isfinite(np.delete(dx, 7, 0)).all()


# A row that holds a value that is not finite is NaN whole, also where the weight that
# meets it is 0; every other row is whole.
@pytest.mark.parametrize("M", [1, 70, 5000])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_fp8_rows_beside_values_that_are_not_finite(M, dt):
    rng = np.random.default_rng(M)
    x = rng.normal(size=(M, 256))
    x[0, 3] = np.inf
    xt = put(x, dt)
    w = np.zeros((128, 256))
    w[np.arange(128), 128 + np.arange(128)] = 1.0
    q, s = pv.pvconv_fp8_quantize_weight(put(w))
    y = host(pv.pvconv_fp8_linear(xt, q, s, out_dtype=torch.float32))
    assert np.isnan(y[0]).all()
    assert (y[1:] == ref.quantise(host(xt), 1)[0][1:, 128:]).all()
