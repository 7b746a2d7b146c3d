"""A student head: a narrow shared MLP on per-point features, trained against a
segmentation network's top logits and served in 8-bit floating point.

Each hidden layer is an 8-bit linear layer (a power-of-two scale for each block
of 128), then group norm over a cloud's points with an activation; the last is
an 8-bit linear layer with a bias. A training step is the forward, the
distillation loss of the logits against the stored top entries of the teacher,
mixed with the labels' cross-entropy, and the backward of every layer. Weights
are fp32 masters, quantised once a step, and once for serving; activations and
their gradients are bf16, logits and parameter gradients fp32.

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
    beta are the tensors that a training program updates in place."""

    def __init__(self, widths: Sequence[int], groups: int = 8, act: str = "silu",
                 eps: float = 1e-5, slope: float = 0.1, seed: int = 0, device="cuda"):
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
    def _model(self):
        return ([pv.pvconv_fp8_quantize_weight(w) for w in self.weights], self.bias, self.gamma,
                self.beta)

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

    def _forward(self, x, model, lengths, saved):
        quantised, bias, gamma, beta = model
        h = x
        for i, (w, s) in enumerate(quantised[:-1]):
            z = pv.pvconv_fp8_linear(h, w, s, out_dtype=torch.bfloat16)
            kw = dict(eps=self.eps, act=self.act, slope=self.slope, lengths=lengths)
            if saved is None:
                y = pv.pvconv_group_norm_act(z, self.groups, gamma[i], beta[i], **kw)
            else:
                y, stats = pv.pvconv_group_norm_act(z, self.groups, gamma[i], beta[i],
                                                    want_stats=True, **kw)
                saved.append((h, z, stats))
            h = y
        w, s = quantised[-1]
        if saved is not None:
            saved.append((h,))
        return pv.pvconv_fp8_linear(h, w, s, bias=bias, out_dtype=torch.float32)

    # -- training --
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
        q = [pv.pvconv_fp8_quantize_weight(w, transposed=True) for w in self.weights]
        saved = []
        z = self._forward(x, ([(w, s) for w, s, _, _ in q], self.bias, self.gamma, self.beta),
                          lengths, saved)
        loss, _, dz = pv.pvconv_distill_topk(
            z.view(B * N, -1), t_val, t_class, labels=labels, temperature=temperature,
            alpha=alpha, row_weight=row_weight, want_grad=True, out_dtype=torch.bfloat16)
        n = len(self.weights)
        dws, dgammas, dbetas = [None] * n, [None] * (n - 1), [None] * (n - 1)
        dy, dbias = dz.view(B, N, -1), None
        for i in reversed(range(n)):
            if i < n - 1:
                _, pre, stats = saved[i]
                dy, dgammas[i], dbetas[i] = pv.pvconv_group_norm_act_backward(
                    dy, pre, stats, self.groups, self.gamma[i], self.beta[i], act=self.act,
                    slope=self.slope, lengths=lengths)
            last = i == n - 1
            dx, dws[i], db = pv.pvconv_fp8_linear_backward(
                dy, saved[i][0], q[i][2], q[i][3], want_dx=i > 0 or want_dx, want_dbias=last)
            dbias = db if last else dbias
            dy = dx
        return loss, [*dws, dbias, *dgammas, *dbetas], dy
