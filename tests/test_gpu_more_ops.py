"""The 8-bit integer layer and the linear cross entropy as a program runs them: captured
in a graph and replayed, on other streams, two at once, into slices of larger buffers,
and together in a training step."""
import numpy as np
import pytest
import torch

from paper_1907_03739_amd import binding as pv
from test_gpu_int8 import test_backward_from_kept_rows as _backward_from_kept_rows
from test_gpu_linear_ce import test_loss_and_gradients as _loss_and_gradients
from test_gpu_train_ops import put

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu_case(request):
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    print(f"\n[gpu case] {request.node.nodeid}", flush=True)
    yield
    torch.cuda.synchronize()


def _tensors(M, K, N, seed, dt=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    new = dict(device="cuda", generator=g)
    return (torch.randn(M, K, **new).to(dt), (torch.randn(N, K, **new) / K ** 0.5).to(dt),
            torch.randn(N, **new), torch.randint(-1, N, (M,), **new).int(),
            torch.randn(M, N, **new).to(dt))


def _step(x, w, b, label, dy):
    """A training step of an 8-bit layer, and the cross entropy on its input."""
    wq, ws = pv.pvconv_int8_quantize(w)
    y, rows, scale = pv.pvconv_int8_linear(x, wq, ws, bias=b, want_rows=True)
    again = pv.pvconv_int8_linear_rows(rows, scale, wq, ws, bias=b, out_dtype=x.dtype)
    grads = pv.pvconv_int8_linear_backward(dy, rows, scale, wq, ws, x.shape[1])
    loss, lse, *lg = pv.pvconv_linear_cross_entropy(x, w, label, bias=b, want_grad=True)
    sg = pv.pvconv_linear_cross_entropy_backward(x, w, label, lse, bias=b)
    return [y, again, rows, scale, *grads, loss, lse, *lg, *sg]


SIZES = [(1, 256, 64), (300, 200, 50), (2000, 512, 700), (4000, 128, 5000), (64, 2304, 2048)]


@pytest.mark.parametrize("M,K,N", SIZES)
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_captured_and_replayed(M, K, N, dt):
    t = _tensors(M, K, N, 1, dt)
    want = _step(*t)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        _step(*t)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _step(*t)
    for i in range(4):
        new = _tensors(M, K, N, 10 + i, dt)
        for a, b in zip(t, new):
            a.copy_(b)
        graph.replay()
        eager = _step(*new)  # the program's own work beside the graph's
        torch.cuda.synchronize()
        for a, b in zip(got, eager):
            assert torch.equal(a, b)
    t0 = _tensors(M, K, N, 1, dt)
    for a, b in zip(t, t0):
        a.copy_(b)
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_two_graphs_that_share_a_workspace_run_in_turn():
    x, w, b, label, dy = _tensors(1000, 256, 900, 2)
    need = pv._lib.pvconv_linear_cross_entropy_workspace_size(1000, 256, 900, 1, 1, 1, 1, 1)
    ws = torch.empty(max(need, pv._lib.pvconv_int8_linear_backward_workspace_size(1000, 256, 900)),
                     dtype=torch.uint8, device="cuda")
    wq, wsc = pv.pvconv_int8_quantize(w)
    rows, scale = pv.pvconv_int8_quantize(x)
    calls = (lambda: pv.pvconv_linear_cross_entropy(x, w, label, bias=b, want_grad=True, workspace=ws),
             lambda: pv.pvconv_int8_linear_backward(dy, rows, scale, wq, wsc, 256, workspace=ws))
    want = [c() for c in calls]
    graphs, outs = [], []
    for c in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(c())
        graphs.append(g)
    for i in (0, 1, 1, 0, 1):
        graphs[i].replay()
        torch.cuda.synchronize()
        ws.fill_(0xff)  # nothing is kept in it between calls
        for a, e in zip(outs[i], want[i]):
            assert torch.equal(a, e)


def test_two_streams_at_once():
    sets = [_tensors(3000, 256, 700, 20 + i) for i in range(2)]
    want = [_step(*t) for t in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(_step(*sets[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for run in got[i]:
            for a, b in zip(run, want[i]):
                assert torch.equal(a, b)


@pytest.mark.parametrize("M,N", [(1, 7), (37, 70), (300, 130), (5000, 64)])
def test_nothing_is_written_beside_an_output(M, N):
    x, w, b, _, _ = _tensors(M, 96, N, 4)
    wq, ws = pv.pvconv_int8_quantize(w)
    want = pv.pvconv_int8_linear(x, wq, ws, bias=b, out_dtype=torch.float32)
    for dt in (torch.float32, torch.bfloat16):
        wide = torch.full((M + 2, N + 11), 7.0, dtype=dt, device="cuda")
        out = wide[1:-1, 5:5 + N]
        pv.pvconv_int8_linear(x, wq, ws, bias=b, out=out)
        assert torch.equal(out, want.to(dt))
        wide[1:-1, 5:5 + N] = 7.0
        assert (wide == 7).all()


def test_gradients_of_a_column_slice_and_of_shared_rows():
    # x and dy are columns of one buffer; labels and weights that many rows share
    buf = torch.randn(500, 300, device="cuda").bfloat16()
    x, dy = buf[:, 8:136], buf[:, 136:200]
    w = torch.randn(64, 128, device="cuda") / 11
    wq, ws = pv.pvconv_int8_quantize(w)
    rows, scale = pv.pvconv_int8_quantize(x)
    a = pv.pvconv_int8_linear_backward(dy, rows, scale, wq, ws, 128)
    b = pv.pvconv_int8_linear_backward(dy.contiguous(), rows, scale, wq, ws, 128)
    for p, q in zip(a, b):
        assert torch.equal(p, q)
    label = torch.randint(0, 64, (500,), device="cuda").int()
    a = pv.pvconv_linear_cross_entropy(x, w, label, want_grad=True)
    b = pv.pvconv_linear_cross_entropy(x.contiguous(), w.clone(), label, want_grad=True)
    for p, q in zip(a, b):
        assert torch.equal(p, q)
    same = torch.full_like(label, 5)
    loss, _, dx, dw, db = pv.pvconv_linear_cross_entropy(x, w, same, want_grad=True)
    z = x.double() @ w.double().t()
    p = torch.softmax(z, 1)
    p[:, 5] -= 1
    # fp32 sums of 500 rows, dz to 24 bits
    tol = 64 * 2.0 ** -24 * (p.abs().t() @ x.double().abs() + 1)
    assert ((dw - p.t() @ x.double()).abs() <= tol).all()


def test_a_long_run_of_rows_past_32_bits():
    # offsets of bytes beyond 2^32: rows of a buffer of 5 GB
    M, K, N = 1 << 18, 64, 48
    wide = torch.empty((M, 5 * 1024 * 2), dtype=torch.bfloat16, device="cuda")
    x = wide[:, :K]
    x.copy_(torch.randn(M, K, device="cuda"))
    w = (torch.randn(N, K, device="cuda") / 8).bfloat16()
    dense = x.contiguous()
    wq, ws = pv.pvconv_int8_quantize(w)
    assert torch.equal(pv.pvconv_int8_linear(x, wq, ws), pv.pvconv_int8_linear(dense, wq, ws))
    label = torch.randint(0, N, (M,), device="cuda").int()
    a = pv.pvconv_linear_cross_entropy(x, w, label, want_grad=True)
    b = pv.pvconv_linear_cross_entropy(dense, w, label, want_grad=True)
    for p, q in zip(a, b):
        assert torch.equal(p, q)


@pytest.mark.parametrize("M,K,N", [(1, 9, 3), (65, 130, 64), (257, 64, 65), (700, 300, 2100),
                                   (3000, 70, 50), (64, 2000, 9000), (9000, 128, 300)])
def test_the_workspace_that_is_asked_for_is_all_that_is_used(M, K, N):
    guard = 1 << 16

    def fenced(need):
        buf = torch.full((need + 2 * guard,), 0xAB, dtype=torch.uint8, device="cuda")
        return buf, buf[guard:guard + need]

    def whole(buf, need):
        return (buf[:guard] == 0xAB).all() and (buf[guard + need:] == 0xAB).all()
    for xd in (torch.bfloat16, torch.float32):
        for wd in (torch.bfloat16, torch.float32):
            x, _, b, label, dy = _tensors(M, K, N, 5, xd)
            w = _tensors(M, K, N, 6, wd)[1]
            q = [int(t is torch.bfloat16) for t in (xd, wd)]
            for grad in (False, True):
                need = pv._lib.pvconv_linear_cross_entropy_workspace_size(M, K, N, *q, *q, grad)
                buf, ws = fenced(need)
                got = pv.pvconv_linear_cross_entropy(x, w, label, bias=b, want_grad=grad,
                                                     workspace=ws if need else None)
                assert whole(buf, need)
            for off in ("want_dx", "want_dw", "want_dbias"):
                one = pv.pvconv_linear_cross_entropy_backward(x, w, label, got[1], bias=b,
                                                              workspace=ws, **{off: False})
                assert whole(buf, need) and sum(t is not None for t in one) == 2
        wq, wsc = pv.pvconv_int8_quantize(w)
        need = pv._lib.pvconv_int8_linear_workspace_size(M, K, N)
        buf, ws = fenced(need)
        y = pv.pvconv_int8_linear(x, wq, wsc, workspace=ws if need else None)
        assert whole(buf, need)
        need = pv._lib.pvconv_int8_linear_rows_workspace_size(M, K, N)
        buf, ws = fenced(need)
        z, rows, scale = pv.pvconv_int8_linear(x, wq, wsc, want_rows=True,
                                               workspace=ws if need else None)
        assert whole(buf, need) and torch.equal(y, z)
        need = pv._lib.pvconv_int8_linear_backward_workspace_size(M, K, N)
        buf, ws = fenced(need)
        for od in (torch.bfloat16, torch.float32):
            pv.pvconv_int8_linear_backward(dy, rows, scale, wq, wsc, K, out_dtype=od, workspace=ws)
            assert whole(buf, need)


# products of dx and dw that are one launch and, beside them, ones that are two: single rows
# and columns, tiles that fill the chip's workgroups or just do not, column sums of one run
# and of several, of few columns and of many
SMALL_STEPS = [(1, 1, 1), (64, 64, 64), (65, 65, 65), (999, 323, 1003), (1025, 323, 1003),
               (1100, 48, 4200), (2000, 100, 300), (2300, 700, 130), (6000, 64, 64)]


@pytest.mark.parametrize("yd,xd", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16")])
@pytest.mark.parametrize("M,K,N", SMALL_STEPS)
def test_gradients_of_small_steps_from_kept_rows(M, K, N, yd, xd):
    _backward_from_kept_rows(M, K, N, yd, xd, 0, 0)


@pytest.mark.parametrize("xd,wd", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16")])
@pytest.mark.parametrize("M,K,V", SMALL_STEPS)
def test_gradients_of_small_steps_of_the_loss(M, K, V, xd, wd):
    _loss_and_gradients(M, K, V, xd, wd, xd, wd, True, 0, 0)
