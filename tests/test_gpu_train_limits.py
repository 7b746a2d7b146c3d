"""The training and 8-bit operators at sizes whose launches come near what HIP
takes (fewer than 2^32 threads): every declared size runs."""
import numpy as np
import pytest
import torch

import _train_ref as ref
from paper_1907_03739_amd import binding as pv
from _helpers import host

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(autouse=True)
def _gpu_case(request):
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    print(f"\n[gpu case] {request.node.nodeid}", flush=True)
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def randn(*shape, seed, dtype=torch.bfloat16, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, device="cuda", generator=g, dtype=dtype).mul_(scale)


# 2^24 groups of two channels (256 threads each would be 2^32), 2^22 groups of 513
# rows (1024 threads each)
@pytest.mark.parametrize("B,N,C,G", [(1 << 20, 1, 32, 16), (1 << 20, 513, 4, 4)])
def test_group_norm_of_very_many_groups(B, N, C, G):
    x, dy = randn(B, N, C, seed=1), randn(B, N, C, seed=2)
    ga, be = 1 + 0.1 * randn(C, seed=3, dtype=torch.float32), 0.5 * randn(C, seed=4, dtype=torch.float32)
    y, st = pv.pvconv_group_norm_act(x, G, ga, be, want_stats=True)
    dx, dg, db = pv.pvconv_group_norm_act_backward(dy, x, st, G, ga, be)
    sums, sizes = np.zeros((2, C)), np.zeros((2, C))
    step = max(1, (1 << 22) // (N * C))
    # whole clouds at both ends and in between; every cloud where they are short
    runs = range(0, B, step) if N == 1 else (0, B // 2 + 3, B - step)
    gd, bd = host(ga), host(be)
    for b in runs:
        xs, ds = host(x[b:b + step]), host(dy[b:b + step])
        n, W = xs.shape[0], C // G
        u = xs.reshape(n, N, G, W)
        mean = u.mean((1, 3), keepdims=True)
        r = 1 / np.sqrt(((u - mean) ** 2).mean((1, 3), keepdims=True) + 1e-5)
        xh = ((u - mean) * r).reshape(n, N, C)
        v = xh * gd + bd
        want = ref.act(v, "silu", 0.0)
        rr = np.broadcast_to(r, u.shape).reshape(n, N, C)
        mag = (np.abs(xs) + np.abs(np.broadcast_to(mean, u.shape).reshape(n, N, C))) * rr * np.abs(gd) \
            + np.abs(bd)
        got = host(y[b:b + step])
        assert (np.abs(got - want) <= 16 * U * mag + 2.0 ** -8 * np.abs(want)).all()
        dv = ds * ref.dact(v, "silu", 0.0)
        sums += [(dv * xh).sum((0, 1)), dv.sum((0, 1))]
        size = np.abs(ds) * ref.dact_magnitude(v, "silu", 0.0)
        sizes += [(size * np.abs(xh)).sum((0, 1)), size.sum((0, 1))]
        h = (gd * dv).reshape(u.shape)
        xg = xh.reshape(u.shape)
        m1, m2 = h.mean((1, 3), keepdims=True), (h * xg).mean((1, 3), keepdims=True)
        want = (r * (h - m1 - xg * m2)).reshape(n, N, C)
        # as the other tests of this gradient: 64 u of the terms' largest of the cloud,
        # and what an error of x - mean and rstd leaves in xh, by which dv is evaluated
        size = rr * np.abs(gd * ds) * 1.1
        cloud = size.max((1, 2), keepdims=True)
        floor = 64 * U * (size + cloud * (1 + mag))
        got = host(dx[b:b + step])
        assert (np.abs(got - want) <= floor + 2.0 ** -8 * np.abs(want)).all()
    if N == 1:
        assert (np.abs(host(dg) - sums[0]) <= 64 * U * sizes[0]).all()
        assert (np.abs(host(db) - sums[1]) <= 64 * U * sizes[1]).all()


def test_fp8_linear_of_very_many_rows():
    # 2^23 tiles of 64 rows, 512 threads each: 2^32
    M, K, N = 1 << 29, 8, 3
    x = randn(M, K, seed=1, dtype=torch.float32)
    w = randn(N, K, seed=2, dtype=torch.float32)
    q, s = pv.pvconv_fp8_quantize_weight(w)
    qw = ref.quantise_weight(host(w))[0]
    y = pv.pvconv_fp8_linear(x, q, s, out_dtype=torch.bfloat16)
    for m in (0, M // 4 - 500, M // 2 - 500, M - 1000):
        qx = ref.quantise(host(x[m:m + 1000]), 1)[0]
        want, mag = qx @ qw.T, np.abs(qx) @ np.abs(qw).T
        got = host(y[m:m + 1000])
        assert (np.abs(got - want) <= 2.0 ** -12 * mag + 2.0 ** -8 * np.abs(want)).all()


def test_fp8_gradients_of_very_many_rows():
    # 2^24 tiles of 128 rows of dy and x, 256 threads each: 2^32
    M = 1 << 30
    dy = torch.zeros(M, 1, device="cuda", dtype=torch.bfloat16)
    at = [0, 1, 127, 128, M // 2 - 1, M // 2, M // 4 * 3, M - 129, M - 1]
    dy[at] = torch.arange(1.0, len(at) + 1, device="cuda", dtype=torch.bfloat16)[:, None]
    x = torch.full((M, 1), 0.5, device="cuda", dtype=torch.bfloat16)
    total = len(at) * (len(at) + 1) / 2
    _, _, qt, st = pv.pvconv_fp8_quantize_weight(torch.full((1, 1), 1.5, device="cuda"),
                                                 transposed=True)
    # every value here is one of e4m3's, and every sum exact
    dx, dw, db = pv.pvconv_fp8_linear_backward(dy, x, qt, st)
    assert dw.item() == 0.5 * total and db.item() == total
    assert torch.equal(dx, dy * 1.5)
    del dx
    db = pv.pvconv_fp8_linear_backward(dy, None, None, None, want_dx=False, want_dw=False)[2]
    assert db.item() == total


# x (and dy) of 256 MiB and more, which are read past the caches' order: every cloud as
# it comes out alone, where they are not, in fp32
@pytest.mark.parametrize("B,N,C,G,dt", [(40, 32768, 128, 8, torch.bfloat16),
                                        (12, 65536, 96, 32, torch.float32)])
def test_group_norm_of_more_than_the_caches_hold(B, N, C, G, dt):
    x, dy = randn(B, N, C, seed=5, dtype=dt), randn(B, N, C, seed=6, dtype=dt)
    assert x.numel() * x.element_size() >= 1 << 28
    ga, be = 1 + 0.1 * randn(C, seed=7, dtype=torch.float32), 0.5 * randn(C, seed=8, dtype=torch.float32)
    y, st = pv.pvconv_group_norm_act(x, G, ga, be, want_stats=True)
    dx, dg, db = pv.pvconv_group_norm_act_backward(dy, x, st, G, ga, be)
    f32 = torch.float32
    step = 2.0 ** -8 if dt == torch.bfloat16 else 0.0
    sums, sizes = torch.zeros(2, C, dtype=torch.float64, device="cuda"), torch.zeros(2, C, device="cuda")
    for b in range(B):
        xb, db_ = x[b:b + 1], dy[b:b + 1]
        y1, st1 = pv.pvconv_group_norm_act(xb, G, ga, be, want_stats=True, out_dtype=f32)
        # one rounding of 64-bit sums whose order may differ
        assert torch.allclose(st1, st[b:b + 1], rtol=4 * U, atol=4 * U)
        dx1, dg1, db1 = pv.pvconv_group_norm_act_backward(db_, xb, st1, G, ga, be, out_dtype=f32)
        mean, r = (st1[0, :, i].repeat_interleave(C // G) for i in (0, 1))
        xs = xb[0].float().abs()
        mag = (xs + mean.abs()) * r * ga.abs() + be.abs()
        # each side is within the bounds that the tests against the oracle hold it to
        assert ((y1 - y[b]).float().abs() <= 32 * U * mag + step * y1.float().abs()).all()
        size = r * (ga * db_[0].float()).abs() * 1.1
        floor = 128 * U * (size + size.max() * (1 + (xs + mean.abs()) * r))
        assert ((dx1 - dx[b]).float().abs() <= floor + step * dx1.float().abs()).all()
        sums += torch.stack([dg1, db1]).double()
        dv = db_[0].float().abs() * 1.1
        sizes += torch.stack([(dv * (xs + mean.abs()) * r).sum(0), dv.sum(0)])
    assert ((sums - torch.stack([dg, db])).abs() <= 128 * U * sizes).all()


def test_distill_of_more_logits_than_the_caches_hold():
    # 256 MiB and more, which the loss alone reads past the caches' order: the loss that
    # comes with a gradient reads them in order
    M, V, top = 2700, 50001, 8
    z = randn(M, V, seed=9, scale=3.0)
    assert z.numel() * 2 >= 1 << 28
    tv, tc = torch.topk(z.float(), top)
    kw = dict(labels=tc[:, 3].int().contiguous(), temperature=2.0, alpha=0.5)
    loss, lse = pv.pvconv_distill_topk(z, tv, tc.int(), **kw)
    loss2, lse2, _ = pv.pvconv_distill_topk(z, tv, tc.int(), want_grad=True, **kw)
    assert torch.equal(loss, loss2) and torch.equal(lse, lse2)
    for m in (0, M // 2, M - 1):
        want = ref.distill(host(z[m:m + 1]), host(tv[m:m + 1]), tc[m:m + 1].cpu().numpy(),
                           kw["labels"][m:m + 1].cpu().numpy(), 2.0, 0.5)[0][0]
        assert abs(loss[m].item() - want) <= 1e-5 * (1 + 4 * 4 + abs(want))
