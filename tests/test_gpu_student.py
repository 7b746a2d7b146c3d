"""The student head: a training step is the calls of its layers in order, learns
its teacher, and serves what it trained."""
import numpy as np
import pytest
import torch

import synth
from paper_1907_03739_amd import binding as pv
from paper_1907_03739_amd.network import DeviceNetwork
from paper_1907_03739_amd.student import DeviceStudent

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu_case(request):
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    print(f"\n[gpu case] {request.node.nodeid}", flush=True)
    yield
    torch.cuda.synchronize()


def _inputs(B=2, N=300, C=40, classes=13, top=4, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(B, N, C, device="cuda", generator=g).bfloat16()
    w = torch.randn(classes, C, device="cuda", generator=g) * (3 / C ** 0.5)
    tv, tc = torch.topk(x.float().view(-1, C) @ w.t(), top)
    labels = tc[:, 0].int().contiguous()
    return x, tv.contiguous(), tc.int().contiguous(), labels


def test_step_is_its_layers_calls():
    x, tv, tc, labels = _inputs()
    st = DeviceStudent([40, 32, 24, 13], groups=4, seed=1)
    lengths = torch.tensor([300, 111], dtype=torch.int32, device="cuda")
    weight = torch.full((600,), 1 / 411, device="cuda")
    weight[300 + 111:] = 0
    loss, grads, dx = st.step(x, tv, tc, labels=labels, alpha=0.7, row_weight=weight,
                              lengths=lengths, want_dx=True)
    q = [pv.pvconv_fp8_quantize_weight(w, transposed=True) for w in st.weights]
    bf = torch.bfloat16
    z0 = pv.pvconv_fp8_linear(x, q[0][0], q[0][1], out_dtype=bf)
    h0, s0 = pv.pvconv_group_norm_act(z0, 4, st.gamma[0], st.beta[0], lengths=lengths, want_stats=True)
    z1 = pv.pvconv_fp8_linear(h0, q[1][0], q[1][1], out_dtype=bf)
    h1, s1 = pv.pvconv_group_norm_act(z1, 4, st.gamma[1], st.beta[1], lengths=lengths, want_stats=True)
    z2 = pv.pvconv_fp8_linear(h1, q[2][0], q[2][1], bias=st.bias, out_dtype=torch.float32)
    l, _, dz = pv.pvconv_distill_topk(z2.view(600, 13), tv, tc, labels=labels, temperature=2.0,
                                      alpha=0.7, row_weight=weight, want_grad=True, out_dtype=bf)
    d2, dw2, db2 = pv.pvconv_fp8_linear_backward(dz.view(2, 300, 13), h1, q[2][2], q[2][3])
    d1, dg1, dbe1 = pv.pvconv_group_norm_act_backward(d2, z1, s1, 4, st.gamma[1], st.beta[1],
                                                      lengths=lengths)
    e1, dw1, _ = pv.pvconv_fp8_linear_backward(d1, h0, q[1][2], q[1][3], want_dbias=False)
    d0, dg0, dbe0 = pv.pvconv_group_norm_act_backward(e1, z0, s0, 4, st.gamma[0], st.beta[0],
                                                      lengths=lengths)
    e0, dw0, _ = pv.pvconv_fp8_linear_backward(d0, x, q[0][2], q[0][3], want_dbias=False)
    assert torch.equal(loss, l) and torch.equal(dx, e0)
    want = [dw0, dw1, dw2, db2, dg0, dg1, dbe0, dbe1]
    assert len(grads) == len(want) == len(st.parameters())
    for a, b, p in zip(grads, want, st.parameters()):
        assert torch.equal(a, b) and a.shape == p.shape
    # points past a cloud's length get nothing
    assert (dx[1, 111:] == 0).all() and (dx[1, :111] != 0).any()


def test_student_learns_its_teacher_and_serves_it():
    wl = synth.make_workload(3, B=2, N=512)
    net = DeviceNetwork(wl.layers, wl.mlps, wl.head, 2, 512)
    logits = net.forward(torch.as_tensor(wl.coords).cuda(), torch.as_tensor(wl.feats).cuda())
    tv, tc = torch.topk(logits.view(1024, -1), 8)
    tv, tc = tv.contiguous(), tc.int().contiguous()
    x = net.stage_view(1)  # a column slice of the concatenation buffer
    st = DeviceStudent([x.shape[-1], 64, logits.shape[-1]], seed=2)
    w = torch.full((1024,), 1 / 1024, device="cuda")
    params = st.parameters()
    m, v = [torch.zeros_like(p) for p in params], [torch.zeros_like(p) for p in params]
    first = last = None
    for i in range(1, 61):
        loss, grads, _ = st.step(x, tv, tc, row_weight=w)
        last = loss.mean().item()
        first = last if first is None else first
        for p, g, a, b in zip(params, grads, m, v):
            a.mul_(0.9).add_(g, alpha=0.1)
            b.mul_(0.99).addcmul_(g, g, value=0.01)
            p.sub_(1e-2 * (a / (1 - 0.9 ** i)) / ((b / (1 - 0.99 ** i)).sqrt() + 1e-8))
    print(f"loss {first:.3f} -> {last:.3f}")
    assert np.isfinite(last) and last < 0.6 * first
    st.freeze()
    served = st.logits(x)
    assert served.shape == (2, 512, logits.shape[-1])
    loss = pv.pvconv_distill_topk(served.view(1024, -1), tv, tc, temperature=2.0)[0]
    assert loss.mean().item() < 0.6 * first
    # a cloud served alone gives its own rows
    alone = st.logits(x[1:2])
    assert torch.allclose(alone[0], served[1], rtol=2e-2, atol=2e-2)


def test_served_model_is_one_model():
    # training goes on in place between two answers: the kept model answers as before,
    # in every parameter, until it is kept anew
    x, tv, tc, labels = _inputs(seed=4)
    st = DeviceStudent([40, 32, 24, 13], groups=4, seed=3)
    first = st.logits(x)
    st.freeze()
    kept = st.logits(x)
    assert torch.equal(kept, first)
    g = torch.Generator(device="cuda").manual_seed(5)
    for p in st.parameters():
        p.add_(torch.randn(p.shape, device="cuda", generator=g), alpha=0.3)
    assert torch.equal(st.logits(x), kept)
    st.freeze()
    changed = st.logits(x)
    assert not torch.equal(changed, kept)
    # what the present parameters give without freeze()
    live = DeviceStudent([40, 32, 24, 13], groups=4, seed=9)
    for a, b in zip(live.parameters(), st.parameters()):
        a.copy_(b)
    assert torch.equal(live.logits(x), changed)
    for p in live.parameters():
        p.mul_(0.5)
    assert not torch.equal(live.logits(x), changed)
