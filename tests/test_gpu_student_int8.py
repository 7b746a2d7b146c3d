"""The student head with layers in 8-bit integers, and its steps against labels: a step
is the calls of its layers in order, and what it trained is served."""
import pytest
import torch

from paper_1907_03739_amd import binding as pv
from paper_1907_03739_amd.student import DeviceStudent
from test_gpu_student import _inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu_case(request):
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    print(f"\n[gpu case] {request.node.nodeid}", flush=True)
    yield
    torch.cuda.synchronize()


def test_int8_step_is_its_layers_calls():
    x, tv, tc, labels = _inputs()
    st = DeviceStudent([40, 32, 24, 13], groups=4, seed=1, layers="int8")
    lengths = torch.tensor([300, 111], dtype=torch.int32, device="cuda")
    weight = torch.full((600,), 1 / 411, device="cuda")
    weight[300 + 111:] = 0
    loss, grads, dx = st.step(x, tv, tc, labels=labels, alpha=0.7, row_weight=weight,
                              lengths=lengths, want_dx=True)
    q = [pv.pvconv_int8_quantize(w) for w in st.weights]
    bf = torch.bfloat16
    rows, hs, zs, stats = [], [x], [], []
    for i in range(2):
        z, r, s = pv.pvconv_int8_linear(hs[-1], *q[i], out_dtype=bf, want_rows=True)
        h, t = pv.pvconv_group_norm_act(z, 4, st.gamma[i], st.beta[i], lengths=lengths,
                                        want_stats=True)
        rows.append((r, s)), zs.append(z), stats.append(t), hs.append(h)
    z2, r, s = pv.pvconv_int8_linear(hs[-1], *q[2], bias=st.bias, out_dtype=torch.float32,
                                     want_rows=True)
    rows.append((r, s))
    l, _, dz = pv.pvconv_distill_topk(z2.view(600, 13), tv, tc, labels=labels, temperature=2.0,
                                      alpha=0.7, row_weight=weight, want_grad=True, out_dtype=bf)
    dy, dws, dgs, dbs = dz.view(2, 300, 13), [None] * 3, [None] * 2, [None] * 2
    dy, dws[2], dbias = pv.pvconv_int8_linear_backward(dy, *rows[2], *q[2], 24)
    for i in (1, 0):
        # what the step multiplies again has the forward's bits
        again = pv.pvconv_int8_linear_rows(*rows[i], *q[i], out_dtype=bf)
        assert torch.equal(again.view(zs[i].shape), zs[i])
        dy, dgs[i], dbs[i] = pv.pvconv_group_norm_act_backward(
            dy, zs[i], stats[i], 4, st.gamma[i], st.beta[i], lengths=lengths)
        dy, dws[i], _ = pv.pvconv_int8_linear_backward(dy, *rows[i], *q[i], [40, 32][i],
                                                       want_dbias=False)
    assert torch.equal(loss, l) and torch.equal(dx, dy)
    for a, b, p in zip(grads, [*dws, dbias, *dgs, *dbs], st.parameters()):
        assert torch.equal(a, b) and a.shape == p.shape
    assert (dx[1, 111:] == 0).all() and (dx[1, :111] != 0).any()


@pytest.mark.parametrize("layers", ["fp8", "int8"])
def test_step_labels_is_the_cross_entropy_of_the_last_layer(layers):
    x, _, _, labels = _inputs()
    st = DeviceStudent([40, 32, 13], groups=4, seed=2, layers=layers)
    weight = torch.rand(600, device="cuda") / 600
    labels[::7] = -1
    loss, grads, dx = st.step_labels(x, labels, row_weight=weight, want_dx=True)
    saved = []
    model = st._train_model(1)
    h = st._hidden(x, model, None, saved)
    l, _, dh, dw, db = pv.pvconv_linear_cross_entropy(h, st.weights[-1], labels, bias=st.bias,
                                                      row_weight=weight, want_grad=True)
    assert torch.equal(loss, l) and torch.equal(grads[1], dw) and torch.equal(grads[2], db)
    assert dw.dtype == torch.float32 and dh.dtype == torch.bfloat16
    assert not loss[::7].any() and len(grads) == len(st.parameters())
    for g, p in zip(grads, st.parameters()):
        assert g.shape == p.shape and torch.isfinite(g).all()
    assert dx.shape == x.shape and torch.isfinite(dx).all()
    # no hidden layers: the loss of x itself
    one = DeviceStudent([40, 13], groups=4, seed=3, layers=layers)
    loss, grads, dx = one.step_labels(x, labels, want_dx=True)
    want = pv.pvconv_linear_cross_entropy(x, one.weights[0], labels, bias=one.bias, want_grad=True)
    assert torch.equal(loss, want[0]) and torch.equal(dx, want[2])
    assert torch.equal(grads[0], want[3]) and torch.equal(grads[1], want[4])
    assert one.step_labels(x, labels)[2] is None


@pytest.mark.parametrize("layers", ["fp8", "int8"])
def test_what_steps_trained_is_served(layers):
    x, _, _, labels = _inputs(B=2, N=400)
    st = DeviceStudent([40, 64, 13], groups=8, seed=4, layers=layers)
    weight = torch.full((800,), 1 / 800, device="cuda")
    for _ in range(3):
        _, grads, _ = st.step_labels(x, labels, row_weight=weight)
        for p, g in zip(st.parameters(), grads):
            assert torch.isfinite(g).all() and g.any()
            p -= 0.1 * g
    st.freeze()
    z = st.logits(x)
    assert z.shape == (2, 400, 13) and torch.isfinite(z).all()
    assert torch.equal(z, st._forward(x, st._model(), None, None))
    one = st.logits(x[:, :1])  # one point
    assert one.shape == (2, 1, 13) and torch.isfinite(one).all()
    with pytest.raises(ValueError):
        DeviceStudent([4, 4], layers="int4")
