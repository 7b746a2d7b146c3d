"""A student head: a narrow shared MLP on per-point features, trained against a
segmentation network's top logits or against labels, and served in 8 bits.

Each hidden layer is an 8-bit linear layer, then group norm over a cloud's points
with an activation; the last is an 8-bit linear layer with a bias. The linear
layers are in 8-bit floating point (a power-of-two scale for each block of 128)
or in 8-bit integers (a scale for each point and each output channel). A training
step is the forward, a loss, and the backward of every layer. The loss is that of
the logits against the stored top entries of a teacher, mixed with the labels'
cross-entropy (step), or the labels' cross-entropy alone, which takes the last
layer with it and never stores a logit (step_labels). Weights are fp32 masters,
quantised once a step, and once for serving; activations and their gradients are
bf16, logits and parameter gradients fp32.

Between forward and backward a layer in 8-bit floating point keeps its input and
its output before the norm, in bf16: 2 (C_in + C_out) bytes a point. A layer in 8-bit
integers keeps the quantised rows of its input, 4 bytes and C_in rounded up to 128s:
a quarter where both widths are alike and wide, more where C_in is small (64 to 64:
132 for 256; 32 to 24: 132 for 112). The backward multiplies them again for the
output, which has the forward's bits, and takes the weight's gradient from them.

Every arithmetic step runs in libpvconv through the calls of the binding; this
module only lays out device buffers and orders the calls.
"""
from __future__ import annotations

from typing import Optional, Sequence

import torch

from . import binding as pv


class DeviceStudent:
    """widths: input channels, the hidden layers' channels, classes. groups divides
    every hidden width. weights [C_out][C_in] and the last layer's bias, gamma and
    beta are the tensors that a training program updates in place. layers: "fp8" or
    "int8"."""

    def __init__(self, widths: Sequence[int], groups: int = 8, act: str = "silu",
                 eps: float = 1e-5, slope: float = 0.1, seed: int = 0, device="cuda",
                 layers: str = "fp8"):
        if layers not in ("fp8", "int8"):
            raise ValueError('layers must be "fp8" or "int8"')
        self.layers = layers
        if len(widths) < 2:
            raise ValueError("a student needs its input width and its classes")
        if any(w % groups for w in widths[1:-1]):
            raise ValueError("groups must divide every hidden width")
        self.widths, self.groups, self.act, self.eps, self.slope = \
            list(widths), groups, act, eps, slope
        gen = torch.Generator().manual_seed(seed)
        f32 = dict(dtype=torch.float32)
        self.weights = [(torch.randn((o, i), generator=gen, **f32) * (2.0 / i) ** 0.5).to(device)
                        for i, o in zip(widths[:-1], widths[1:])]
        self.bias = torch.zeros(widths[-1], device=device, **f32)
        self.gamma = [torch.ones(w, device=device, **f32) for w in widths[1:-1]]
        self.beta = [torch.zeros(w, device=device, **f32) for w in widths[1:-1]]
        self._served = None

    def parameters(self):
        """Every trained tensor, in the order of step()'s gradients."""
        return [*self.weights, self.bias, *self.gamma, *self.beta]

    # -- serving --
    def _quantize(self, w):
        return pv.pvconv_int8_quantize(w) if self.layers == "int8" else \
            pv.pvconv_fp8_quantize_weight(w)

    def _model(self):
        return ([self._quantize(w) for w in self.weights], self.bias, self.gamma, self.beta)

    def freeze(self):
        """Keeps the model as it is now for logits(): the weights quantised once,
        and a copy of every other parameter. Again after training has changed it."""
        quantised, bias, gamma, beta = self._model()
        self._served = (quantised, bias.clone(), [t.clone() for t in gamma],
                        [t.clone() for t in beta])

    def logits(self, x: torch.Tensor, lengths: Optional[torch.Tensor] = None) -> torch.Tensor:
        """x [B][N][C_in] (rows evenly strided; one point is N = 1) -> logits
        [B][N][classes] f32 of the model as the last freeze() kept it. Before any,
        of the parameters as they are now, the weights quantised on every call."""
        return self._forward(x, self._served or self._model(), lengths, None)

    def _linear(self, h, q, saved, **kw):
        """A linear layer of h; with saved, what its backward needs is appended."""
        if self.layers == "fp8":
            if saved is not None:
                saved.append((h,))
            return pv.pvconv_fp8_linear(h, q[0], q[1], **kw)
        if saved is None:
            return pv.pvconv_int8_linear(h, q[0], q[1], **kw)
        z, rows, scale = pv.pvconv_int8_linear(h, q[0], q[1], want_rows=True, **kw)
        saved.append((rows, scale))
        return z

    def _hidden(self, x, model, lengths, saved):
        quantised, _, gamma, beta = model
        h = x
        for i, q in enumerate(quantised[:len(gamma)]):
            z = self._linear(h, q, saved, out_dtype=torch.bfloat16)
            kw = dict(eps=self.eps, act=self.act, slope=self.slope, lengths=lengths)
            if saved is None:
                y = pv.pvconv_group_norm_act(z, self.groups, gamma[i], beta[i], **kw)
            else:
                y, stats = pv.pvconv_group_norm_act(z, self.groups, gamma[i], beta[i],
                                                    want_stats=True, **kw)
                saved[i] += (stats,) if self.layers == "int8" else (z, stats)
            h = y
        return h

    def _forward(self, x, model, lengths, saved):
        h = self._hidden(x, model, lengths, saved)
        return self._linear(h, model[0][-1], saved, bias=model[1], out_dtype=torch.float32)

    # -- training --
    def _train_model(self, count):
        """The first `count` weights quantised, with what their gradients take."""
        q = [pv.pvconv_int8_quantize(w) if self.layers == "int8" else
             pv.pvconv_fp8_quantize_weight(w, transposed=True) for w in self.weights[:count]]
        return q, self.bias, self.gamma, self.beta

    def _linear_backward(self, i, dy, q, saved, **kw):
        if self.layers == "fp8":
            return pv.pvconv_fp8_linear_backward(dy, saved[i][0], q[i][2], q[i][3], **kw)
        return pv.pvconv_int8_linear_backward(dy, saved[i][0], saved[i][1], q[i][0], q[i][1],
                                              self.widths[i], **kw)

    def _hidden_backward(self, dy, q, saved, lengths, dws, want_dx):
        """From dy, the gradient of the hidden layers' output: fills dws, returns
        (dgammas, dbetas, dx)."""
        n = len(self.gamma)
        dgammas, dbetas = [None] * n, [None] * n
        for i in reversed(range(n)):
            stats = saved[i][-1]
            if self.layers == "int8":  # the output before the norm again, bit for bit
                z = pv.pvconv_int8_linear_rows(saved[i][0], saved[i][1], q[i][0], q[i][1],
                                               out_dtype=torch.bfloat16).view(dy.shape)
            else:
                z = saved[i][1]
            dy, dgammas[i], dbetas[i] = pv.pvconv_group_norm_act_backward(
                dy, z, stats, self.groups, self.gamma[i], self.beta[i], act=self.act,
                slope=self.slope, lengths=lengths)
            dy, dws[i], _ = self._linear_backward(i, dy, q, saved, want_dx=i > 0 or want_dx,
                                                  want_dbias=False)
        return dgammas, dbetas, dy

    def step(self, x: torch.Tensor, t_val: torch.Tensor, t_class: torch.Tensor,
             labels: Optional[torch.Tensor] = None, temperature: float = 2.0,
             alpha: float = 1.0, row_weight: Optional[torch.Tensor] = None,
             lengths: Optional[torch.Tensor] = None, want_dx: bool = False):
        """Forward and backward of sum(row_weight * loss): x [B][N][C_in], the
        teacher's t_val, t_class [B*N][top], labels [B*N] int32 -> (loss [B*N],
        gradients in the order of parameters(), dx [B][N][C_in] or None). Give the
        points past a cloud's length the weight 0, and finite x: the first weight's
        gradient multiplies their rows of x by 0."""
        B, N, _ = x.shape
        model = self._train_model(len(self.weights))
        saved = []
        z = self._forward(x, model, lengths, saved)
        loss, _, dz = pv.pvconv_distill_topk(
            z.view(B * N, -1), t_val, t_class, labels=labels, temperature=temperature,
            alpha=alpha, row_weight=row_weight, want_grad=True, out_dtype=torch.bfloat16)
        n = len(self.weights)
        dws = [None] * n
        dy, dws[-1], dbias = self._linear_backward(n - 1, dz.view(B, N, -1), model[0], saved,
                                                   want_dx=n > 1 or want_dx, want_dbias=True)
        dgammas, dbetas, dx = self._hidden_backward(dy, model[0], saved, lengths, dws, want_dx)
        return loss, [*dws, dbias, *dgammas, *dbetas], dx

    def step_labels(self, x: torch.Tensor, labels: torch.Tensor,
                    row_weight: Optional[torch.Tensor] = None,
                    lengths: Optional[torch.Tensor] = None, want_dx: bool = False):
        """Forward and backward of sum(row_weight * cross-entropy of the labels):
        labels [B*N] int32, outside the classes: no loss, no gradient -> what step()
        returns. The last layer multiplies its fp32 weight and the bf16 features as
        they are (step() trains it as logits() serves it, in 8 bits), and its logits are
        never stored. The points past a cloud's length as for step()."""
        model = self._train_model(len(self.gamma))
        saved = []
        h = self._hidden(x, model, lengths, saved)
        loss, _, dy, dw, dbias = pv.pvconv_linear_cross_entropy(
            h, self.weights[-1], labels, bias=self.bias, row_weight=row_weight, want_grad=True,
            want_dx=len(self.gamma) > 0 or want_dx)
        dws = [None] * len(self.gamma) + [dw]
        dgammas, dbetas, dx = self._hidden_backward(dy, model[0], saved, lengths, dws, want_dx)
        return loss, [*dws, dbias, *dgammas, *dbetas], dx
