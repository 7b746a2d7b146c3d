"""Plain 64-bit forms on the GPU, for sizes that take too long on the CPU: the definitions
of the 8-bit layer's gradients and of the linear cross entropy, a run of rows at a time,
with the tolerances that test_gpu_int8, test_gpu_linear_ce and test_gpu_gradient_bits
derive."""
import math

import torch

U, HALF, TWO = 2.0 ** -24, 2.0 ** -8, 2.0 ** -16
ROWS_AT_A_TIME = 1 << 24  # values


def sum_tol(n):
    return 4 * (math.sqrt(n) + 4) * U


def near(got, want, tol, what):
    d = (got.double() - want).abs()
    bad = ~(d <= tol)
    if bad.any():
        over = torch.where(bad, d - tol, torch.full_like(d, -math.inf))
        at = int(over.argmax())
        raise AssertionError(
            f"{what}: {int(bad.sum())} of {d.numel()} outside tolerance; worst at {at} of "
            f"{tuple(d.shape)}: got {got.flatten()[at].item():.6g}, want "
            f"{want.flatten()[at].item():.6g}, tol {tol.expand_as(d).flatten()[at].item():.3g}")


def _result(inside, want, dt):
    return inside * (1 + HALF) + HALF * want.abs() if dt is torch.bfloat16 else inside


def layer_gradients(dy, q, s, v, t, dx_dt):
    """(dx, dw, dbias, their tolerances) of rows s q by a weight t v."""
    x, w, d = q.double() * s.double()[:, None], v.double() * t.double()[:, None], dy.double()
    rounded = U if dy.dtype is torch.float32 else 0.0
    if dx_dt is torch.bfloat16 and dy.dtype is torch.float32:
        rounded += TWO
    dx, dt = d @ w, d.t().contiguous()
    tdx = (sum_tol(d.shape[1]) + rounded) * (d.abs() @ w.abs()) + 1e-38
    dw = dt @ x
    tdw = sum_tol(d.shape[0]) * (dt.abs() @ x.abs()) + 1e-38
    tdb = 3 * U * d.abs().sum(0) + 1e-38
    return (dx, dw, d.sum(0)), (_result(tdx, dx, dx_dt), tdw, tdb)


def loss(x, w, b, label, weight, dx_dt, dw_dt):
    """(loss, lse, dx, dw, dbias), their tolerances. Labels outside [0, V): none."""
    V, K = w.shape
    M = x.shape[0]
    W, wt = w.double(), w.double().t().contiguous()
    parts = lambda out, f: TWO * (1 if f.dtype is torch.bfloat16 else 3) \
        if out is torch.bfloat16 else 0.0  # noqa: E731
    fx, fw = 2 * U + parts(dx_dt, w), 2 * U + parts(dw_dt, x)
    out = [[], [], [], 0.0, 0.0]
    tol = [[], [], [], 0.0, 0.0]
    run = max(1, ROWS_AT_A_TIME // V)
    for i in range(0, M, run):
        xs, l = x[i:i + run].double(), label[i:i + run].long()
        z = torch.addmm(b.double(), xs, wt)
        size = torch.where(z.isneginf(), 0.0, z).abs().max(1).values
        Z = sum_tol(K) * (xs.abs() @ wt.abs()).max(1).values + 4 * U * size
        lse = torch.logsumexp(z, 1)
        known = (l >= 0) & (l < V)
        at = torch.where(known, l, 0)[:, None]
        out[0].append(torch.where(known, lse - z.gather(1, at)[:, 0], 0.0))
        out[1].append(lse)
        t = 2 * Z + 16 * U * (1 + lse.abs() + size)
        tol[0].append(t), tol[1].append(t)
        g = (weight[i:i + run].double() * known)[:, None]
        p = torch.exp(z - lse[:, None])
        one = torch.zeros_like(p).scatter_(1, at, 1.0)
        dz = g * (p - one)
        mag = g.abs() * (p + one)
        edz = g.abs() * (p * (2 * Z + 64 * U)[:, None] + one * U)
        dx, dzt = dz @ W, dz.t().contiguous()
        out[2].append(dx)
        tol[2].append(_result((edz + fx * dz.abs() + sum_tol(V) * mag) @ W.abs(), dx, dx_dt))
        out[3] = out[3] + dzt @ xs
        tol[3] = tol[3] + (edz + fw * dz.abs() + sum_tol(M) * mag).t().contiguous() @ xs.abs()
        out[4] = out[4] + dz.sum(0)
        tol[4] = tol[4] + (edz + 64 * U * mag).sum(0)
    tol[3] = _result(tol[3], out[3], dw_dt)
    cat = [[torch.cat(a) if isinstance(a, list) else a for a in v] for v in (out, tol)]
    return cat[0], [t + 1e-37 for t in cat[1]]
