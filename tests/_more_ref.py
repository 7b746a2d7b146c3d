"""Plain 64-bit forms of the 8-bit integer linear layer and of the cross entropy of a
linear layer, from their definitions; they share nothing with the kernels."""
import numpy as np


def int8_scale(top):
    """The smallest number of eight significant bits >= 2^-126 with 127 s >= top."""
    t = np.maximum(np.asarray(top, np.float64) / 127, 2.0 ** -126)
    step = 2.0 ** (np.floor(np.log2(t)) - 7)
    s = np.ceil(t / step) * step
    s = np.where((127 * (s - step) >= top) & (s - step >= 2.0 ** -126), s - step, s)
    return np.where(127 * s < top, s + step, s)


def int8_rows(x):
    """(whole numbers, scales) of rows; NaN and 0 for a row that is not finite."""
    x = np.asarray(x, np.float64)
    bad = ~np.isfinite(x).all(1)
    x = np.where(bad[:, None], 0.0, x)
    s = int8_scale(np.abs(x).max(1, initial=0.0))
    return np.round(x / s[:, None]), np.where(bad, np.nan, s)


def activate(v, act, slope=0.1):
    return v if act == "none" else np.where(v < 0, v * (slope if act == "leaky" else 0.0), v)


def linear_ce(x, w, b, label, weight=None):
    """(loss, lse, dx, dw, db, parts): parts are the sums of magnitudes behind dx, dw, db."""
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    M, V = x.shape[0], w.shape[0]
    z = x @ w.T + (0 if b is None else b)
    top = z.max(1, keepdims=True)
    with np.errstate(all="ignore"):
        e = np.exp(z - np.where(np.isneginf(top), 0.0, top))
        lse = np.log(e.sum(1)) + np.where(np.isneginf(top), 0.0, top)[:, 0]
    known = (label >= 0) & (label < V) & ~np.isneginf(lse)
    at = np.where(known, label, 0)
    loss = np.where(known, lse - z[np.arange(M), at], 0.0)
    p = np.where(known[:, None], np.exp(z - np.where(known, lse, 0.0)[:, None]), 0.0)
    one = np.zeros_like(p)
    one[np.arange(M)[known], at[known]] = 1.0
    g = np.ones(M) if weight is None else np.asarray(weight, np.float64)
    dz = np.where(g[:, None] == 0, 0.0, (p - one) * g[:, None])
    mag = (p + one) * np.abs(g)[:, None]
    return dict(loss=loss, lse=lse, z=z, dz=dz, dx=dz @ w, dw=dz.T @ x, db=dz.sum(0),
                dx_mag=mag @ np.abs(w), dw_mag=mag.T @ np.abs(x), db_mag=mag.sum(0))
