"""Plain 64-bit forms of the operators of include/pvconv_train.h (numpy), from
their definitions: the oracle of their GPU tests."""
from __future__ import annotations

import numpy as np

BLOCK = 128


def act(v, kind, slope):
    if kind == "silu":
        with np.errstate(over="ignore"):
            return v / (1 + np.exp(-v))
    return v if kind == "none" else np.where(v >= 0, v, v * (slope if kind == "leaky" else 0.0))


def dact(v, kind, slope):
    if kind == "none":
        return np.ones_like(v)
    if kind == "silu":
        with np.errstate(over="ignore"):
            s = 1 / (1 + np.exp(-v))
        return s * (1 + v * (1 - s))
    return np.where(v > 0, 1.0, slope if kind == "leaky" else 0.0)


def dact_magnitude(v, kind, slope):
    """dact's expression on absolute values: what its rounding is relative to."""
    if kind != "silu":
        return dact(v, kind, slope)
    with np.errstate(over="ignore"):
        s = 1 / (1 + np.exp(-v))
    return s * (1 + np.abs(v) * (1 - s))


def group_norm(x, groups, gamma, beta, eps, kind, slope, lengths=None):
    """-> (y, stats [B][groups][2])."""
    B, N, C = x.shape
    W = C // groups
    y, stats = np.zeros_like(x), np.zeros((B, groups, 2))
    for b in range(B):
        n = N if lengths is None else int(np.clip(lengths[b], 0, N))
        if n == 0:
            continue
        u = x[b, :n].reshape(n, groups, W)
        mean = u.mean((0, 2))
        var = ((u - mean[None, :, None]) ** 2).mean((0, 2))
        r = 1 / np.sqrt(var + eps)
        stats[b, :, 0], stats[b, :, 1] = mean, r
        v = ((u - mean[None, :, None]) * r[None, :, None]).reshape(n, C) * gamma + beta
        y[b, :n] = act(v, kind, slope)
    return y, stats


def group_norm_backward(dy, x, groups, gamma, beta, eps, kind, slope, lengths=None, stats=None):
    """-> (dx, dgamma, dbeta), and the sums of magnitudes that bound the rounding
    of dgamma and dbeta. stats: the statistics that the call was given (the
    forward's, in 32 bits), else exact ones."""
    B, N, C = x.shape
    W = C // groups
    dx, dg, db = np.zeros_like(x), np.zeros(C), np.zeros(C)
    mg, mb = np.zeros(C), np.zeros(C)
    if stats is None:
        stats = group_norm(x, groups, gamma, beta, eps, kind, slope, lengths)[1]
    for b in range(B):
        n = N if lengths is None else int(np.clip(lengths[b], 0, N))
        if n == 0:
            continue
        mean, r = (np.repeat(stats[b, :, i], W) for i in (0, 1))
        xh = (x[b, :n] - mean) * r
        dv = dy[b, :n] * dact(gamma * xh + beta, kind, slope)
        dg += (dv * xh).sum(0)
        db += dv.sum(0)
        size = np.abs(dy[b, :n]) * dact_magnitude(gamma * xh + beta, kind, slope)
        mg += (size * np.abs(xh)).sum(0)
        mb += size.sum(0)
        h = gamma * dv
        m1 = np.repeat(h.reshape(n, groups, W).mean((0, 2)), W)
        m2 = np.repeat((h * xh).reshape(n, groups, W).mean((0, 2)), W)
        dx[b, :n] = r * (h - m1 - xh * m2)
    return dx, dg, db, mg, mb


def e4m3(v):
    """Nearest e4m3 value (ties to even) of |v| <= 448; NaN where v is not finite."""
    a = np.abs(v)
    with np.errstate(divide="ignore", invalid="ignore"):
        step = 2.0 ** (np.floor(np.log2(np.maximum(a, 2.0 ** -6))) - 3)
        a = np.where(np.isfinite(v), a, 0)
    return np.where(np.isfinite(v), np.sign(v) * np.round(a / step) * step, np.nan)


def exponent(top):
    """The smallest e >= -126 with top <= 448 * 2^e; 0 for 0."""
    if top == 0:
        return 0
    e = -126
    m, x = np.frexp(top)  # top = m 2^x
    return max(e, int(x) - 9 + (1 if m > 0.875 else 0))


def quantise(x, axis):
    """(values that x stands for in blocks of 128 along `axis`, exponents)."""
    x = np.moveaxis(np.asarray(x, np.float64), axis, -1)
    out, es = np.empty_like(x), np.zeros(x.shape[:-1] + (-(-x.shape[-1] // BLOCK),), int)
    for b in range(es.shape[-1]):
        part = x[..., b * BLOCK:(b + 1) * BLOCK]
        tops = np.where(np.isfinite(part), np.abs(part), 0).max(-1)
        es[..., b] = np.vectorize(exponent)(tops)
        f = 2.0 ** es[..., b][..., None]
        out[..., b * BLOCK:(b + 1) * BLOCK] = e4m3(part / f) * f
    return np.moveaxis(out, -1, axis), np.moveaxis(es, -1, axis)


def quantise_weight(w):
    """(values, exponents [N/128][K/128]) in blocks of 128 x 128."""
    N, K = w.shape
    out = np.empty((N, K))
    es = np.zeros((-(-N // BLOCK), -(-K // BLOCK)), int)
    for i in range(es.shape[0]):
        for j in range(es.shape[1]):
            at = (slice(i * BLOCK, (i + 1) * BLOCK), slice(j * BLOCK, (j + 1) * BLOCK))
            es[i, j] = exponent(np.where(np.isfinite(w[at]), np.abs(w[at]), 0).max())
            out[at] = e4m3(w[at] / 2.0 ** es[i, j]) * 2.0 ** es[i, j]
    return out, es


def distill(z, t_val, t_class, labels, T, alpha, weight=None):
    """-> (loss [M], dz [M][V])."""
    M, V = z.shape
    loss, dz = np.zeros(M), np.zeros((M, V))
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        for m in range(M):
            w = 1.0 if weight is None else weight[m]
            top = np.max(z[m])
            if top == -np.inf:
                continue
            lse = lambda a: np.max(a) + np.log(np.exp(a - np.max(a)).sum())
            g = np.zeros(V)
            have = [(float(v) / T, int(c)) for v, c in zip(t_val[m], t_class[m]) if 0 <= c < V]
            tv = np.array([v for v, _ in have])
            if alpha > 0 and have and not np.max(tv) == -np.inf:
                lq = z[m] / T - lse(z[m] / T)
                lp = tv - lse(tv)
                p = np.exp(lp)
                for (_, c), pj, lpj in zip(have, p, lp):
                    if pj != 0:
                        loss[m] += alpha * T * T * pj * (lpj - lq[c])
                g += alpha * T * np.exp(lq)
                for (_, c), pj in zip(have, p):
                    g[c] -= alpha * T * pj
            if labels is not None and alpha < 1 and 0 <= labels[m] < V:
                l1 = z[m] - lse(z[m])
                loss[m] += (1 - alpha) * -l1[labels[m]]
                g += (1 - alpha) * np.exp(l1)
                g[labels[m]] -= 1 - alpha
            if w != 0:
                dz[m] = w * g
    return loss, dz
