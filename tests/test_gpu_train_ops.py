"""Group norm, the 8-bit linear layer and the distillation loss on the GPU,
against their plain 64-bit forms (_train_ref), forward and gradients, at the
sizes, masks and layouts where they can go wrong.

Tolerances, from the arithmetic (u = 2^-24, the fp32 unit; bf16 rounds by
2^-9 relative):
* group norm, fp32: the statistics are exact sums rounded once; x - mean,
  * rstd, * gamma, + beta and the activation round five times, relative to
  operands of at most |x| rstd |gamma| + |mean| rstd |gamma| + |beta|, and the
  exponential's error of a few u enters SiLU: 16 u of that magnitude.
* its dx: three terms, each a product of at most six rounded factors, and
  means of at most n terms summed in 64 bits of fp32 partial sums of up to
  some hundred terms: 64 u of the sum of the terms' magnitudes, floored by the
  cloud's largest; dgamma, dbeta: fp32 partial sums of some hundred terms:
  64 u of the sum of magnitudes.
* 8-bit product with an fp32 output: exact operands, fp32 sums of K terms:
  4 sqrt(K) u + 8 u of sum |q_x q_w|; with a bf16 output the instruction adds a block's
  products on a grid of the largest: 2^-12 of that sum, and bf16's 2^-8.
* distillation: exponentials of differences rounded at their magnitude (at most
  |z - max| u each, z here within 40): loss 1e-5 of (1 + its terms), dz 2e-5 of
  the row's largest softmax value 1.
"""
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


def put(a, dt, pad=0, lead=0):
    """The array on the GPU as rows of a wider buffer (a column slice)."""
    t = torch.as_tensor(np.asarray(a, np.float32)).cuda().to(TD[dt])
    if pad == 0 and lead == 0:
        return t.contiguous()
    wide = torch.full(t.shape[:-1] + (t.shape[-1] + pad + lead,), float("nan"), dtype=t.dtype,
                      device="cuda")
    wide[..., lead:lead + t.shape[-1]] = t
    return wide[..., lead:lead + t.shape[-1]]


def check(got, want, tol, what):
    d = np.abs(got - want)
    bad = ~(d <= tol)
    if bad.any():
        i = np.unravel_index(np.argmax(np.where(bad, d - tol, -np.inf)), d.shape)
        raise AssertionError(f"{what}: {bad.sum()} of {d.size} outside tolerance; worst at {i}: "
                             f"got {got[i]:.6g}, want {want[i]:.6g}, tol {np.broadcast_to(tol, d.shape)[i]:.3g}")


def bf16_step(dt):
    return 2.0 ** -8 if dt == "bf16" else 0.0


# ----------------------------------------------------------------------------
# group norm
# ----------------------------------------------------------------------------
GN = [
    # B, N, C, groups, x, y, act, lengths, pad, lead
    (1, 1, 32, 4, "f32", "f32", "silu", None, 0, 0),
    (1, 1, 2048, 32, "bf16", "bf16", "silu", None, 0, 0),
    (2, 7, 6, 6, "f32", "f32", "relu", None, 0, 0),          # a channel a group
    (2, 1, 3, 3, "f32", "f32", "none", None, 0, 0),          # an element a group: xh = 0
    (3, 577, 60, 6, "f32", "f32", "leaky", None, 36, 0),     # a slice, 10 channels a group
    (3, 577, 60, 6, "bf16", "f32", "leaky", [577, 0, 33], 5, 3),
    (4, 2048, 128, 8, "bf16", "bf16", "silu", [2048, 1, 0, 2047], 0, 0),
    (2, 4097, 64, 8, "f32", "bf16", "silu", [9999, -5], 0, 0),  # lengths are clamped
    (1, 300, 1030, 1, "f32", "f32", "silu", None, 0, 0),     # one group, wider than a workgroup
    (2, 130, 4104, 3, "bf16", "bf16", "none", [130, 65], 0, 0),
    (70, 3, 24, 2, "f32", "f32", "silu", None, 0, 0),        # many small clouds
    (1, 40000, 16, 2, "bf16", "bf16", "relu", None, 8, 0),   # a long cloud
    (2, 33, 35, 5, "bf16", "bf16", "silu", None, 2, 1),      # odd rows: no vectors
    (1, 30000, 96, 32, "f32", "f32", "relu", None, 0, 0),    # vectors across groups of 3
    (2, 21000, 72, 24, "bf16", "bf16", "silu", [21000, 50], 0, 0),
    (1, 20000, 30, 2, "bf16", "f32", "leaky", None, 2, 0),   # 15 channels a group
    (2, 9000, 200, 8, "bf16", "bf16", "silu", None, 8, 8),   # 25 channels a group
    (1, 70000, 132, 3, "f32", "f32", "none", [65537], 0, 0),
]


def gn_inputs(B, N, C, seed, mean=0.0):
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(B, N, C)) * np.exp(0.5 * rng.normal(size=C)) + rng.normal(size=C) + mean
    return (x, rng.uniform(0.5, 1.5, C).astype(np.float32).astype(np.float64),
            (0.5 * rng.normal(size=C)).astype(np.float32).astype(np.float64), rng)


@pytest.mark.parametrize("B,N,C,G,xd,yd,act,lengths,pad,lead", GN)
def test_group_norm_forward_and_gradients(B, N, C, G, xd, yd, act, lengths, pad, lead):
    x, gamma, beta, rng = gn_inputs(B, N, C, 100 + N + C)
    dx_t = put(x, xd, pad, lead)
    x = host(dx_t)
    dy_t = put(rng.normal(size=x.shape), yd, pad, lead)
    dy = host(dy_t)
    lt = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    ga, be = put(gamma, "f32"), put(beta, "f32")
    kw = dict(act=act, slope=0.1, lengths=lt)
    y, stats = pv.pvconv_group_norm_act(dx_t, G, ga, be, eps=1e-5, want_stats=True,
                                        out_dtype=TD[yd], **kw)
    ry, rs = ref.group_norm(x, G, gamma, beta, 1e-5, act, 0.1, lengths)
    W = C // G
    r, mean = (np.repeat(rs[:, :, i], W, 1)[:, None] for i in (1, 0))
    mag = (np.abs(x) + np.abs(mean)) * r * np.abs(gamma) + np.abs(beta)
    check(host(stats)[..., 0], rs[..., 0], 4 * U * (np.abs(rs[..., 0]) + 1e-3), "mean")
    check(host(stats)[..., 1], rs[..., 1], 1e-6 * rs[..., 1], "rstd")
    check(host(y), ry, 16 * U * mag + bf16_step(yd) * np.abs(ry), "y")

    dx, dg, db = pv.pvconv_group_norm_act_backward(dy_t, dx_t, stats, G, ga, be, **kw)
    rdx, rdg, rdb, mg, mb = ref.group_norm_backward(dy, x, G, gamma, beta, 1e-5, act, 0.1, lengths,
                                                     host(stats))
    # a rectifier's derivative jumps where v is 0: elements within the rounding
    # of v may take either side, in their own dx and in their sums
    v = (x - mean) * r * gamma + beta
    n = np.array([N if lengths is None else min(max(l, 0), N) for l in
                  (lengths or [N] * B)])[:, None, None]
    near = (np.abs(v) <= 16 * U * mag) & (np.arange(N)[None, :, None] < n)
    jump = near * np.abs(dy) if act in ("relu", "leaky") else np.zeros_like(x)
    terms = r * np.abs(gamma * dy) * 1.1
    cloud = terms.max((1, 2), keepdims=True)
    floor = 64 * U * (terms + cloud * (1 + np.abs((x - mean) * r)))
    floor = floor + r * np.abs(gamma) * jump + 4 * cloud * (jump > 0).any((1, 2), keepdims=True)
    check(host(dx), rdx, floor + bf16_step(xd) * np.abs(rdx), "dx")
    xh = np.abs((x - mean) * r)
    check(host(dg), rdg, 64 * U * mg + (jump * xh).sum((0, 1)) + 1e-30, "dgamma")
    check(host(db), rdb, 64 * U * mb + jump.sum((0, 1)) + 1e-30, "dbeta")


def test_group_norm_keeps_digits_of_a_far_mean():
    # mean 4096 spreads of 1: the variance of sums of squares in 32 bits would
    # have no digits left
    x, gamma, beta, _ = gn_inputs(2, 5000, 16, 5, mean=4096.0)
    x = x.astype(np.float32).astype(np.float64)
    y, stats = pv.pvconv_group_norm_act(put(x, "f32"), 2, put(gamma, "f32"), put(beta, "f32"),
                                        act="none", want_stats=True)
    ry, rs = ref.group_norm(x, 2, gamma, beta, 1e-5, "none", 0.0)
    check(host(stats)[..., 1], rs[..., 1], 1e-6 * rs[..., 1], "rstd")
    # the mean itself is kept in 32 bits: half an ulp of 4096 of x - mean
    check(host(y), ry, (2.0 ** -12 + 16 * U * 5) * np.repeat(rs[..., 1], 8, 1)[:, None] * gamma
          + 16 * U * np.abs(beta), "y")


def test_group_norm_gradients_against_differences():
    rng = np.random.default_rng(3)
    x, gamma, beta, _ = gn_inputs(2, 9, 12, 3)
    w = rng.normal(size=x.shape)
    dx, dg, db, _, _ = ref.group_norm_backward(w, x, 3, gamma, beta, 1e-5, "silu", 0.0, [9, 4])
    f = lambda x, g, b: (w * ref.group_norm(x, 3, g, b, 1e-5, "silu", 0.0, [9, 4])[0]).sum()
    for _ in range(4):
        vx, vg, vb = rng.normal(size=x.shape), rng.normal(size=12), rng.normal(size=12)
        h = 1e-6
        num = (f(x + h * vx, gamma + h * vg, beta + h * vb) -
               f(x - h * vx, gamma - h * vg, beta - h * vb)) / (2 * h)
        assert abs(num - ((dx * vx).sum() + dg @ vg + db @ vb)) <= 1e-6 * (1 + abs(num))


@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_group_norm_keeps_a_bad_value_to_its_group(bad):
    x, gamma, beta, _ = gn_inputs(2, 50, 16, 9)
    x[1, 20, 3] = bad                       # cloud 1, group 0 of 2
    y = host(pv.pvconv_group_norm_act(put(x, "f32"), 2, put(gamma, "f32"), put(beta, "f32")))
    assert np.isnan(y[1, :, :8]).all()
    assert np.isfinite(y[0]).all() and np.isfinite(y[1, :, 8:]).all()
    # past a cloud's length nothing is read
    lt = torch.tensor([50, 20], dtype=torch.int32, device="cuda")
    y = host(pv.pvconv_group_norm_act(put(x, "f32"), 2, put(gamma, "f32"), put(beta, "f32"),
                                      lengths=lt))
    assert np.isfinite(y).all() and (y[1, 20:] == 0).all()


def test_group_norm_empty():
    g = put(np.ones(8), "f32")
    y, st = pv.pvconv_group_norm_act(torch.empty((2, 0, 8), device="cuda"), 2, g, g,
                                     want_stats=True)
    assert y.shape == (2, 0, 8) and (host(st) == 0).all()
    dx, dg, db = pv.pvconv_group_norm_act_backward(y, y, st, 2, g, g)
    assert (host(dg) == 0).all() and (host(db) == 0).all()
    assert pv.pvconv_group_norm_act(torch.empty((0, 5, 8), device="cuda"), 2, g, g).shape == (0, 5, 8)


# ----------------------------------------------------------------------------
# 8-bit linear layer
# ----------------------------------------------------------------------------
def fp8_inputs(M, K, N, seed):
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(M, K)) * np.exp(rng.normal(size=K)) * np.exp(rng.normal(size=(M, 1)))
    x[rng.random(x.shape) < 0.3] = 0
    w = rng.normal(size=(N, K)) * np.exp(0.5 * rng.normal(size=(N, 1))) / np.sqrt(K)
    return x, w, rng


def as_values(q, s, cols):
    v = q.float().cpu().numpy().astype(np.float64)
    e = s.cpu().numpy().astype(int) - 127
    e = np.repeat(np.repeat(e, 128, 0)[:v.shape[0]], 128, 1)
    assert (v[:, cols:] == 0).all()
    return (v * 2.0 ** e)[:, :cols]


@pytest.mark.parametrize("N,K,dt,pad", [(1, 1, "f32", 0), (50, 323, "f32", 5), (128, 128, "bf16", 0),
                                        (129, 257, "bf16", 8), (300, 640, "f32", 0),
                                        (13, 2304, "bf16", 1)])
def test_fp8_quantised_weight_is_exact(N, K, dt, pad):
    _, w, _ = fp8_inputs(1, K, N, N + K)
    wt = put(w, dt, pad)
    w = host(wt)
    q, s, qt, st = pv.pvconv_fp8_quantize_weight(wt, transposed=True)
    v, e = ref.quantise_weight(w)
    assert (s.cpu().numpy().astype(int) - 127 == e).all()
    assert (as_values(q, s, K) == v).all()
    assert (as_values(qt, st, N) == v.T).all()
    q2, s2 = pv.pvconv_fp8_quantize_weight(wt)
    assert torch.equal(q2.view(torch.uint8), q.view(torch.uint8)) and torch.equal(s, s2)


def test_fp8_quantises_the_edges_of_the_range():
    # ties, the largest value, blocks of zeros, of tiny and of huge values; a
    # product with the identity returns Q(x)
    K = 128
    rows = [np.zeros(K), np.full(K, 448.0), np.full(K, 448.0 * 1.0000001), np.full(K, 1e-40),
            np.full(K, 3e38), np.linspace(-448, 448, K), 2.0 ** np.linspace(-30, 8, K),
            np.where(np.arange(K) % 2, 17.0, 448), np.where(np.arange(K) % 2, 1.0625, 448),
            np.where(np.arange(K) == 5, -2.0 ** -10, 256), np.full(K, -1.75 * 2 ** 20)]
    x = np.array(rows).astype(np.float32).astype(np.float64)
    q, s = pv.pvconv_fp8_quantize_weight(put(np.eye(K), "f32"))
    assert (s.cpu().numpy() == 127 - 8).all()
    for M in (len(rows), 1):
        y = host(pv.pvconv_fp8_linear(put(x[:M], "f32"), q, s))
        assert (y == ref.quantise(x[:M], 1)[0]).all()
    big = np.concatenate([x] * 20)
    assert (host(pv.pvconv_fp8_linear(put(big, "f32"), q, s)) == ref.quantise(big, 1)[0]).all()


@pytest.mark.parametrize("M", [1, 3, 200])
def test_fp8_values_that_are_not_finite(M):
    rng = np.random.default_rng(M)
    x = rng.normal(size=(M, 300))
    x[0, 130], x[M - 1, 5] = np.inf, np.nan
    w = rng.normal(size=(20, 300))
    q, s = pv.pvconv_fp8_quantize_weight(put(w, "f32"))
    for dt in ("f32", "bf16"):
        y = host(pv.pvconv_fp8_linear(put(x, "f32"), q, s, out_dtype=TD[dt]))
        rows = np.isnan(y).all(1)
        assert rows[0] and rows[M - 1] and np.isfinite(y[1:M - 1]).all()
    # they do not count for the block's largest
    xc = x.astype(np.float32).astype(np.float64)
    xc[0, 130] = xc[M - 1, 5] = 0
    if M == 200:
        w2 = w.copy()
        w2[:, :] = 0
        w2[0, 131] = 1.0
        assert (ref.quantise(x, 1)[1] == ref.quantise(xc, 1)[1]).all()


PRODUCT = [
    # M, K, N, x, y, act, bias, pad, lead
    (1, 1, 1, "f32", "f32", "none", True, 0, 0),
    (1, 2048, 256, "f32", "f32", "none", True, 0, 0),
    (1, 4928, 50, "bf16", "bf16", "relu", True, 0, 0),
    (5, 130, 13, "bf16", "f32", "leaky", False, 3, 1),
    (16, 512, 128, "bf16", "bf16", "none", True, 0, 0),
    (17, 127, 129, "f32", "f32", "none", True, 1, 0),
    (33, 257, 100, "f32", "bf16", "relu", True, 0, 0),
    (64, 640, 48, "bf16", "f32", "none", False, 0, 0),
    (128, 128, 128, "bf16", "bf16", "none", False, 0, 0),
    (999, 323, 50, "f32", "f32", "none", True, 5, 0),
    (1000, 1100, 300, "bf16", "bf16", "leaky", True, 8, 8),
    (2048, 512, 520, "bf16", "f32", "relu", True, 0, 0),
    (4099, 384, 256, "bf16", "bf16", "relu", True, 0, 0),
    (300, 4928, 256, "bf16", "f32", "none", True, 0, 0),
    (40000, 64, 13, "f32", "f32", "none", True, 0, 0),
    (2500, 1024, 700, "bf16", "bf16", "relu", True, 0, 0),   # rows of 8 blocks that stay in LDS
    (700, 1000, 2500, "f32", "bf16", "none", True, 3, 0),    # more columns than one share
    (3000, 512, 2304, "bf16", "bf16", "leaky", False, 0, 8),
    (600, 1100, 1030, "bf16", "bf16", "none", True, 0, 0),   # quantiser and product apart
    (5000, 7, 300, "f32", "f32", "relu", True, 2, 0),        # fewer channels than a vector
    (40, 4, 9, "bf16", "bf16", "none", True, 0, 0),
    (600, 2900, 100, "bf16", "bf16", "none", True, 1, 1),    # odd strides, a ragged last block
    (33001, 200, 70, "bf16", "bf16", "relu", True, 0, 0),    # tiles of 128 rows
    (33001, 141, 200, "bf16", "f32", "none", True, 3, 1),
    (8300, 1100, 1000, "bf16", "bf16", "leaky", False, 0, 0),
]


@pytest.mark.parametrize("M,K,N,xd,yd,act,bias,pad,lead", PRODUCT)
def test_fp8_linear(M, K, N, xd, yd, act, bias, pad, lead):
    x, w, rng = fp8_inputs(M, K, N, M + K + N)
    xt, wt = put(x, xd, pad, lead), put(w, xd)
    x, w = host(xt), host(wt)
    b = 0.1 * rng.normal(size=N).astype(np.float32).astype(np.float64)
    q, s = pv.pvconv_fp8_quantize_weight(wt)
    y = pv.pvconv_fp8_linear(xt, q, s, bias=put(b, "f32") if bias else None, act=act, slope=0.1,
                             out_dtype=TD[yd])
    qx, qw = ref.quantise(x, 1)[0], ref.quantise_weight(w)[0]
    want = ref.act(qx @ qw.T + (b if bias else 0), act, 0.1)
    mag = np.abs(qx) @ np.abs(qw).T + (np.abs(b) if bias else 0)
    tol = (4 * np.sqrt(K) + 8) * U * mag
    if yd == "bf16":
        tol = 2.0 ** -12 * mag + 2.0 ** -8 * np.abs(want)
    check(host(y), want, tol, "y")


@pytest.mark.parametrize("M,K,N,xd,dd,pad", [(1, 9, 5, "f32", "f32", 0), (999, 323, 50, "f32", "f32", 5),
                                             (130, 257, 129, "bf16", "bf16", 3),
                                             (4096, 512, 256, "bf16", "bf16", 0),
                                             (2500, 130, 384, "bf16", "f32", 0)])
def test_fp8_gradients(M, K, N, xd, dd, pad):
    x, w, rng = fp8_inputs(M, K, N, M + K + N)
    dy = 1e-3 * rng.normal(size=(M, N)) * np.exp(rng.normal(size=(M, 1)))
    xt, wt, dt_ = put(x, xd, pad), put(w, xd), put(dy, dd, pad)
    x, w, dy = host(xt), host(wt), host(dt_)
    _, _, qt, st = pv.pvconv_fp8_quantize_weight(wt, transposed=True)
    dx, dw, db = pv.pvconv_fp8_linear_backward(dt_, xt, qt, st)
    qw = ref.quantise_weight(w)[0]
    qr, qc, xc = ref.quantise(dy, 1)[0], ref.quantise(dy, 0)[0], ref.quantise(x, 0)[0]
    want, mag = qr @ qw, np.abs(qr) @ np.abs(qw)
    tol = (4 * np.sqrt(N) + 8) * U * mag if dd == "f32" else \
        2.0 ** -12 * mag + 2.0 ** -8 * np.abs(want)
    check(host(dx), want, tol, "dx")
    check(host(dw), qc.T @ xc, (4 * np.sqrt(M) + 8) * U * (np.abs(qc).T @ np.abs(xc)) + 1e-30, "dw")
    check(host(db), dy.sum(0), (4 * np.sqrt(M) + 8) * U * np.abs(dy).sum(0) + 1e-30, "db")
    # each alone gives the same bits
    only = dict(want_dx=False, want_dw=False, want_dbias=False)
    assert torch.equal(pv.pvconv_fp8_linear_backward(dt_, None, qt, st, **{**only, "want_dx": True})[0], dx)
    assert torch.equal(pv.pvconv_fp8_linear_backward(dt_, xt, None, None, **{**only, "want_dw": True})[1], dw)
    assert torch.equal(pv.pvconv_fp8_linear_backward(dt_, None, None, None, **{**only, "want_dbias": True})[2], db)


def test_fp8_no_rows():
    q, s, qt, st = pv.pvconv_fp8_quantize_weight(put(np.ones((6, 40)), "f32"), transposed=True)
    x = torch.empty((0, 40), device="cuda")
    assert pv.pvconv_fp8_linear(x, q, s).shape == (0, 6)
    dx, dw, db = pv.pvconv_fp8_linear_backward(torch.empty((0, 6), device="cuda"), x, qt, st)
    assert dx.shape == (0, 40) and (host(dw) == 0).all() and (host(db) == 0).all()


# ----------------------------------------------------------------------------
# distillation
# ----------------------------------------------------------------------------
def distill_inputs(M, V, top, seed, dt, pad=0, lead=0):
    rng = np.random.default_rng(seed)
    zt = put(3 * rng.normal(size=(M, V)), dt, pad, lead)
    z = host(zt)
    t = z + rng.normal(size=z.shape)
    cls = np.argsort(-t, 1)[:, :top].astype(np.int32)
    val = np.take_along_axis(t, cls.astype(int), 1).astype(np.float32)
    few = rng.random((M, 1)) < 0.3
    cls[few & (np.arange(top) >= (top + 1) // 2)[None]] = -1
    if M > 4:
        cls[M // 2] = -1
        cls[M // 3, 0] = V  # outside: absent
    labels = rng.integers(0, V, M).astype(np.int32)
    labels[rng.random(M) < 0.2] = -1
    if M > 4:
        labels[M // 2], labels[1] = -1, V + 3
    return zt, z, val, cls, labels, rng


def run_distill(zt, z, val, cls, labels, T, alpha, weight, out_dtype=None):
    tv, tc = torch.as_tensor(val).cuda(), torch.as_tensor(cls).cuda()
    lt = None if labels is None else torch.as_tensor(labels).cuda()
    wt = None if weight is None else torch.as_tensor(weight.astype(np.float32)).cuda()
    kw = dict(labels=lt, temperature=T, alpha=alpha)
    loss, lse, dz = pv.pvconv_distill_topk(zt, tv, tc, row_weight=wt, want_grad=True,
                                           out_dtype=out_dtype, **kw)
    loss2, lse2 = pv.pvconv_distill_topk(zt, tv, tc, **kw)
    dz2 = pv.pvconv_distill_topk_backward(zt, tv, tc, lse2, wt, out_dtype=out_dtype, **kw)
    return [host(a) for a in (loss, dz, loss2, dz2)]


DISTILL = [
    # M, V, top, dtype, T, alpha, labels, pad, lead
    (1, 1, 1, "f32", 1.0, 1.0, False, 0, 0),
    (1, 3, 3, "f32", 2.0, 0.5, True, 0, 0),
    (40, 13, 4, "f32", 2.0, 0.7, True, 0, 0),
    (300, 50, 8, "f32", 4.0, 0.9, True, 1, 0),
    (300, 50, 8, "bf16", 1.0, 1.0, False, 0, 0),
    (77, 50, 50, "bf16", 1.5, 0.0, True, 3, 1),
    (65, 64, 5, "f32", 1.0, 0.5, True, 0, 0),
    (33, 257, 100, "f32", 2.0, 0.5, True, 0, 0),
    (20, 1000, 16, "bf16", 2.0, 0.5, True, 0, 0),
    (9, 1025, 16, "f32", 3.0, 1.0, False, 7, 2),
    (5, 4097, 256, "bf16", 2.0, 0.5, True, 1, 0),
    (3, 32001, 32, "bf16", 1.0, 1.0, False, 0, 0),
    (2, 70001, 64, "f32", 1.5, 0.5, True, 0, 0),
    (37, 16, 16, "f32", 2.0, 0.5, True, 0, 0),       # the widths between two kinds of team
    (37, 17, 9, "bf16", 2.0, 0.5, True, 1, 0),
    (33, 128, 70, "f32", 1.0, 0.5, True, 0, 3),
    (33, 129, 5, "f32", 2.0, 0.5, True, 0, 0),
    (9, 512, 200, "bf16", 2.0, 0.5, True, 0, 0),
    (9, 513, 7, "f32", 2.0, 0.5, True, 3, 0),
    (5, 2048, 64, "f32", 2.0, 0.5, True, 0, 0),
    (5, 2049, 255, "bf16", 2.0, 0.5, True, 5, 1),
    (6, 3000, 256, "f32", 2.0, 0.5, True, 0, 0),     # an entry a thread, and one for the label
    (300, 9001, 16, "bf16", 1.5, 0.5, True, 0, 1),
]


@pytest.mark.parametrize("M,V,top,dt,T,alpha,lab,pad,lead", DISTILL)
def test_distill(M, V, top, dt, T, alpha, lab, pad, lead):
    zt, z, val, cls, labels, rng = distill_inputs(M, V, top, M + V, dt, pad, lead)
    labels = labels if lab else None
    weight = rng.random(M).astype(np.float32).astype(np.float64)
    if M > 2:
        weight[2] = 0
    loss, dz, loss2, dz2 = run_distill(zt, z, val, cls, labels, T, alpha, weight)
    rl, rg = ref.distill(z, val.astype(np.float64), cls, labels, T, alpha, weight)
    check(loss, rl, 1e-5 * (1 + T * T * 4 + np.abs(rl)), "loss")
    big = (alpha * T + 1 - alpha) * weight[:, None]
    check(dz, rg, 2e-5 * big * (np.abs(rg).max() / big.max() + 1e-3) + bf16_step(dt) * np.abs(rg),
          "dz")
    check(loss2, rl, 1e-5 * (1 + T * T * 4 + np.abs(rl)), "loss alone")
    check(dz2, rg, 2e-5 * big * (np.abs(rg).max() / big.max() + 1e-3) + bf16_step(dt) * np.abs(rg),
          "gradient alone")


@pytest.mark.parametrize("V", [5, 50, 700, 5000, 40000])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_distill_masks_and_repeated_classes(V, dt):
    rng = np.random.default_rng(V)
    M, top = 12, 6
    zt = put(3 * rng.normal(size=(M, V)), dt)
    zt[0] = -float("inf")                       # nothing left: loss 0, no gradient
    zt[1, : V // 2] = -float("inf")             # half masked
    zt[2] = -float("inf")
    zt[2, V - 1] = 1.0                          # one class left
    lowest = torch.finfo(zt.dtype).min
    zt[3, 1:] = lowest                          # the type's lowest value as a mask
    zt[4] = lowest                              # a row of it: uniform
    z = host(zt)
    val = rng.normal(size=(M, top)).astype(np.float32)
    cls = rng.integers(0, V, (M, top)).astype(np.int32)
    cls[1] = rng.integers(V // 2, V, top)
    cls[2], cls[3] = V - 1, 0
    cls[5, 1:] = cls[5, 0]                      # one class, six entries
    val[6, 2:] = -np.inf                        # entries without weight
    val[7] = -np.inf                            # none with weight
    cls[8] = -7
    labels = rng.integers(0, V, M).astype(np.int32)
    labels[1], labels[2], labels[3] = V - 1, V - 1, 0
    labels[5] = cls[5, 0]
    labels[9] = -1
    with np.errstate(over="ignore"):
        for T, alpha in ((1.0, 0.5), (2.0, 0.7), (2.0, 1.0), (1.0, 0.0)):
            loss, dz, loss2, dz2 = run_distill(zt, z, val, cls, labels, T, alpha, None)
            rl, rg = ref.distill(z, val.astype(np.float64), cls, labels, T, alpha)
            tol = 2e-5 * (1 + T * T * 4 + np.abs(rl))
            for l in (loss, loss2):
                check(l, rl, tol, "loss")
            for g in (dz, dz2):
                check(g, rg, 2e-5 * (1 + T) + bf16_step(dt) * np.abs(rg), "dz")
                assert (g[0] == 0).all() and (g[1, : V // 2] == 0).all()


@pytest.mark.parametrize("V", [50, 5000])
def test_distill_bad_logits_stay_in_their_row(V):
    rng = np.random.default_rng(1)
    zt = put(rng.normal(size=(6, V)), "f32")
    zt[1, 3], zt[2, 4] = float("nan"), float("inf")
    val = rng.normal(size=(6, 3)).astype(np.float32)
    val[4, 1] = np.nan
    cls = np.tile(np.arange(3, dtype=np.int32), (6, 1))
    loss, dz, loss2, dz2 = run_distill(zt, host(zt), val, cls, None, 2.0, 1.0, None)
    for l, g in ((loss, dz), (loss2, dz2)):
        assert (np.isnan(l) == [False, True, True, False, True, False]).all()
        assert np.isnan(g[1]).all() and np.isnan(g[2]).any() and np.isfinite(g[[0, 3, 5]]).all()


def test_distill_mixed_types_and_differences():
    zt, z, val, cls, labels, rng = distill_inputs(30, 21, 5, 8, "bf16")
    _, dz, _, dz2 = run_distill(zt, z, val, cls, labels, 2.0, 0.6, None, out_dtype=torch.float32)
    rg = ref.distill(z, val.astype(np.float64), cls, labels, 2.0, 0.6)[1]
    check(dz, rg, 5e-5, "dz")
    check(dz2, rg, 5e-5, "dz alone")
    for _ in range(3):
        d, h = rng.normal(size=z.shape), 1e-6
        f = lambda a: ref.distill(a, val.astype(np.float64), cls, labels, 2.0, 0.6)[0].sum()
        num = (f(z + h * d) - f(z - h * d)) / (2 * h)
        assert abs(num - (rg * d).sum()) <= 1e-6 * (1 + abs(num))


def test_distill_no_rows():
    z = torch.empty((0, 9), device="cuda")
    t, c = torch.empty((0, 2), device="cuda"), torch.empty((0, 2), dtype=torch.int32, device="cuda")
    loss, lse, dz = pv.pvconv_distill_topk(z, t, c, want_grad=True)
    assert loss.shape == (0,) and lse.shape == (0, 2) and dz.shape == (0, 9)


# ----------------------------------------------------------------------------
# streams, graphs, repeats
# ----------------------------------------------------------------------------
def _chain(x, w, gamma, beta, tv, tc):
    q, s, qt, st = pv.pvconv_fp8_quantize_weight(w, transposed=True)
    h = pv.pvconv_fp8_linear(x, q, s, out_dtype=torch.bfloat16)
    y, stats = pv.pvconv_group_norm_act(h.view(4, -1, h.shape[1]), 8, gamma, beta, want_stats=True)
    loss, _, dz = pv.pvconv_distill_topk(y.view(h.shape), tv, tc, want_grad=True)
    dh, dg, db = pv.pvconv_group_norm_act_backward(dz.view(y.shape), h.view(y.shape), stats, 8,
                                                   gamma, beta)
    dx, dw, dbias = pv.pvconv_fp8_linear_backward(dh.view(h.shape), x, qt, st)
    return [loss, dg, db, dx, dw, dbias]


def _chain_inputs(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)
    tv, tc = torch.topk(r(1200, 64), 5)
    return (r(1200, 300).bfloat16(), 0.1 * r(64, 300), 1 + 0.1 * r(64), 0.1 * r(64), tv,
            tc.int())


def test_same_bits_on_every_run_and_on_another_stream():
    a = _chain_inputs(1)
    want = _chain(*a)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = _chain(*a)
    side.synchronize()
    for u, v in zip(want, got):
        assert torch.equal(u, v)


def test_graph_replays_give_the_eager_results():
    a = _chain_inputs(2)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        _chain(*a)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = _chain(*a)
    for seed in (3, 4, 5):
        b = _chain_inputs(seed)
        for dst, src in zip(a, b):
            dst.copy_(src)
        want = [t.clone() for t in _chain(*b)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for u, v in zip(want, outs):
            assert torch.equal(u, v)
