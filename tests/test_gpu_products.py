"""The products behind the 8-bit integer layer and the linear cross entropy in every tile
that they take, split and not, over one tile a workgroup and several, and the loss over
several pieces of its classes, on the GPU, against plain 64-bit forms (_wide_ref, which says
where the tolerances come from). test_plan checks that the sizes reach what they are for."""
import pytest
import torch

from _steps import LAYER_STEPS, LOSS_STEPS, PIECES
from _wide_ref import U, HALF, layer_gradients, loss, near
from paper_1907_03739_amd import binding as pv

pytestmark = pytest.mark.gpu
TD = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(autouse=True)
def _gpu_case(request):
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    print(f"\n[gpu case] {request.node.nodeid}", flush=True)
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def _new(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return dict(device="cuda", generator=g)


@pytest.mark.parametrize("M,K,N,yd,xd", LAYER_STEPS)
def test_layer(M, K, N, yd, xd):
    new = _new(M + K + N)
    x = torch.randn(M, K, **new) * torch.exp(torch.randn(M, 1, **new))
    w = torch.randn(N, K, **new) * torch.exp(0.5 * torch.randn(N, 1, **new))
    b = torch.randn(N, **new)
    dy = (1e-3 * torch.randn(M, N, **new) * torch.exp(torch.randn(M, 1, **new))).to(TD[yd])
    v, t = pv.pvconv_int8_quantize(w)
    y, rows, s = pv.pvconv_int8_linear(x, v, t, bias=b, out_dtype=TD[yd], want_rows=True)
    # the sum is exact, then a rounding each for its float, the scales and the bias
    total = (rows.double() @ v.double().t().contiguous()) * s.double()[:, None] * t.double()
    want = total + b.double()
    tol = 4 * U * (total.abs() + b.double().abs())
    near(y, want, tol + HALF * want.abs() if yd == "bf16" else tol, "y")
    # rows that are not kept lie block by block: the same bits
    assert torch.equal(pv.pvconv_int8_linear(x, v, t, bias=b, out_dtype=TD[yd]), y)
    got = pv.pvconv_int8_linear_backward(dy, rows, s, v, t, K, out_dtype=TD[xd])
    want, tol = layer_gradients(dy, rows[:, :K], s, v[:, :K], t, TD[xd])
    for name, a, e, d in zip(("dx", "dw", "dbias"), got, want, tol):
        near(a, e, d, name)
    again = pv.pvconv_int8_linear_backward(dy, rows, s, v, t, K, out_dtype=TD[xd])
    for a, c in zip(got, again):
        assert torch.equal(a, c)


def _loss_inputs(M, K, V, xd, wd):
    new = _new(M + K + V)
    x = (torch.randn(M, K, **new) * torch.exp(0.3 * torch.randn(M, 1, **new))).to(TD[xd])
    w = (2 / K ** 0.5 * torch.randn(V, K, **new)).to(TD[wd])
    b = 0.3 * torch.randn(V, **new)
    b[3::11] = -float("inf")  # classes that take no part
    label = torch.randint(0, V, (M,), **new).int()
    label = torch.where(label % 11 == 3, 0, label)
    label[torch.rand(M, **new) < 0.1] = -1
    weight = torch.rand(M, **new)
    weight[torch.rand(M, **new) < 0.1] = 0
    return x, w, b, label, weight


def _check_loss(M, K, V, xd, wd, dxd, dwd):
    x, w, b, label, weight = _loss_inputs(M, K, V, xd, wd)
    want, tol = loss(x, w, b, label, weight, TD[dxd], TD[dwd])
    dt = dict(bias=b, out_dtype=TD[dxd], dw_dtype=TD[dwd])
    need = pv._lib.pvconv_linear_cross_entropy_workspace_size(
        M, K, V, *[int(d == "bf16") for d in (xd, wd, dxd, dwd)], 1)
    guard = 1 << 16
    buf = torch.full((need + 2 * guard,), 0xAB, dtype=torch.uint8, device="cuda")
    kw = dict(dt, workspace=buf[guard:guard + need])
    got = pv.pvconv_linear_cross_entropy(x, w, label, row_weight=weight, want_grad=True, **kw)
    names = ("loss", "lse", "dx", "dw", "dbias")
    for name, a, e, d in zip(names, got, want, tol):
        near(a, e, d, name)
    del want, tol
    split = pv.pvconv_linear_cross_entropy_backward(x, w, label, got[1], weight, **kw)
    for a, c in zip(split, got[2:]):  # (the same lse: the same bits)
        assert torch.equal(a, c)
    for i, one in enumerate(("want_dx", "want_dw", "want_dbias")):
        only = {k: k == one for k in ("want_dx", "want_dw", "want_dbias")}
        a = pv.pvconv_linear_cross_entropy_backward(x, w, label, got[1], weight, **only, **kw)[i]
        assert torch.equal(a, got[2 + i])
    assert (buf[:guard] == 0xAB).all() and (buf[guard + need:] == 0xAB).all()


@pytest.mark.parametrize("M,K,V,xd,wd,dxd,dwd", LOSS_STEPS)
def test_loss(M, K, V, xd, wd, dxd, dwd):
    _check_loss(M, K, V, xd, wd, dxd, dwd)


@pytest.mark.parametrize("M,K,V,xd,wd,dxd,dwd,pieces", PIECES)
def test_pieces_of_the_classes(M, K, V, xd, wd, dxd, dwd, pieces):
    _check_loss(M, K, V, xd, wd, dxd, dwd)
