"""Performance cases of a linear layer in 8-bit integers, of its training step from
8-bit rows kept for the backward, and of the softmax cross entropy of a linear
layer without its logits, through the public entry points of paper_1907_03739_amd.

Kinds of case:

  int8   a linear layer on rows in 8-bit integers, a scale for each row of x and
         each row (output channel) of the weight: serving, with a weight that was
         quantised once
  rows   a training step of that layer. The forward quantises the weight and the
         rows of x and keeps those bytes in the place of x; the backward takes the
         gradients of x, the weight and the bias from them
  lce    the cross entropy of a label with the softmax of x W^T + bias over many
         classes. mode "loss": the loss; "fused": the loss and the gradients of x,
         W and bias of known row weights in one call; "split": the loss, then the
         gradients from the saved statistics

Quantising: a row's scale is the smallest number s of 8 significant bits (a
bfloat16), s >= 2^-126, with 127 s >= the row's largest magnitude; a value becomes
the whole number nearest to value / s, ties to even.

Where `own` is false the operators are computed in elementary torch operations.
"""
import math
from types import SimpleNamespace

import torch

own = False

DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
SLOPE = 0.1
BLOCK = 128  # quantised rows are padded with zeros to a multiple of this


# --------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------
def _int8(name, M, K, N, dt, out, act, pad=0):
    c = dict(kind="int8", M=M, K=K, N=N, dt=dt, out=out, act=act, pad=pad)
    return dict(c, name=name) if name else c


def _rows(name, M, K, N, dt, pad=0):
    c = dict(kind="rows", M=M, K=K, N=N, dt=dt, pad=pad)
    return dict(c, name=name) if name else c


def _lce(name, M, K, V, dt, wdt, mode, masked=False, pad=0):
    c = dict(kind="lce", M=M, K=K, V=V, dt=dt, wdt=wdt, mode=mode, masked=masked, pad=pad)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the part-segmentation head's first layer on one feature row: latency alone
        _int8("int8 one row", 1, 4928, 256, "f32", "f32", "none"),
        # that layer on the points of 16 clouds
        _int8("int8 head", 32768, 4928, 256, "bf16", "bf16", "relu"),
        # the widest shared MLP of the part-segmentation network
        _int8("int8 mlp", 32768, 512, 2048, "bf16", "bf16", "relu"),
        # a column slice of a concatenation buffer, odd in every size, fp32
        _int8("int8 odd slice", 999, 323, 77, "f32", "f32", "leaky", pad=5),
        # a student's hidden layer on a small batch of points, a training step
        _rows("rows small train", 130, 256, 128, "bf16"),
        # the scene-segmentation head's first layer, a training step
        _rows("rows scene train", 32768, 2304, 512, "bf16"),
        # odd in every size, fp32, from a wider buffer
        _rows("rows odd train", 777, 203, 99, "f32", pad=36),
        # one row over a long vocabulary, the loss alone: latency and W's bytes
        _lce("lce one row", 1, 512, 32001, "bf16", "bf16", "loss"),
        # the part-segmentation classes of every point, fp32 master weights
        _lce("lce parts train", 32768, 128, 50, "bf16", "f32", "fused"),
        # odd in every size, fp32, from a wider buffer
        _lce("lce odd train", 999, 323, 1003, "f32", "f32", "fused", pad=5),
        # a batch of tokens over a long vocabulary whose end is padding, loss and
        # gradients apart
        _lce("lce vocabulary train", 4096, 512, 49999, "bf16", "bf16", "split", masked=True),
        # wide features, a shorter vocabulary, one call
        _lce("lce wide train", 8192, 2048, 5003, "bf16", "bf16", "fused"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    kind = rng.choice(("int8", "rows", "lce"))
    most = max(_cost(c) for c in listed() if c["kind"] == kind)
    while True:
        pad = rng.choice((0, 0, 0, 8, 3))
        if kind == "int8":
            c = _int8(None, _log(rng, 1, 65536), _log(rng, 9, 5000), _log(rng, 5, 2048),
                      rng.choice(("bf16", "bf16", "f32")), rng.choice(("bf16", "f32")),
                      rng.choice(("none", "relu", "leaky")), pad=pad)
        elif kind == "rows":
            c = _rows(None, _log(rng, 1, 65536), _log(rng, 9, 5000), _log(rng, 5, 2048),
                      rng.choice(("bf16", "bf16", "f32")), pad=pad)
        else:
            c = _lce(None, _log(rng, 1, 65536), _log(rng, 9, 2048), _log(rng, 3, 60000),
                     rng.choice(("bf16", "bf16", "f32")), rng.choice(("bf16", "bf16", "f32")),
                     rng.choice(("loss", "fused", "split")), masked=rng.random() < 0.3, pad=pad)
            if c["M"] * c["V"] > 1 << 28:  # the plain form holds the logits
                continue
        if _cost(c) <= most:
            return c


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------
def _slice(t, pad):
    """The same values as the first columns of a wider row-major buffer."""
    if not pad:
        return t.contiguous()
    wide = torch.zeros(t.shape[:-1] + (t.shape[-1] + pad,), dtype=t.dtype, device=t.device)
    wide[..., :t.shape[-1]] = t
    return wide[..., :t.shape[-1]]


def prepare(case, seed):
    s = SimpleNamespace(**{k: v for k, v in case.items() if k != "name"})
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * {"int8": 11, "rows": 12, "lce": 13}[s.kind] + int(seed))
    f32 = dict(device=DEV, dtype=torch.float32, generator=g)
    if s.kind in ("int8", "rows"):
        # rectified features of uneven scale, weights of uneven channels
        x = torch.relu(torch.randn(s.M, s.K, **f32)) * torch.exp(0.5 * torch.randn(s.K, **f32))
        s.x = _slice((x * torch.exp(torch.randn(s.M, 1, **f32))).to(DT[s.dt]), s.pad)
        w = torch.randn(s.N, s.K, **f32) * math.sqrt(2 / s.K)
        w = (w * torch.exp(0.5 * torch.randn(s.N, 1, **f32))).to(DT[s.dt])
        s.bias = 0.1 * torch.randn(s.N, **f32)
        if s.kind == "rows":
            s.w = w
            dy = 1e-3 * torch.randn(s.M, s.N, **f32) * torch.exp(torch.randn(s.M, 1, **f32))
            s.dy = _slice(dy.to(DT[s.dt]), s.pad)
        else:  # a serving program keeps the quantised weight alone, rows padded by zeros
            q, s.ws = _quantize(w)
            s.wq = torch.nn.functional.pad(q, (0, -s.K % BLOCK)).to(torch.int8).contiguous()
    else:
        x = torch.randn(s.M, s.K, **f32) * torch.exp(0.3 * torch.randn(s.M, 1, **f32))
        s.x = _slice(x.to(DT[s.dt]), s.pad)
        s.w = (torch.randn(s.V, s.K, **f32) * (2 / math.sqrt(s.K))).to(DT[s.wdt])
        s.bias = 0.3 * torch.randn(s.V, **f32)
        known = s.V
        if s.masked and s.V > 4:  # the vocabulary's padding takes no part
            known = s.V - max(1, s.V // 50)
            s.bias[known:] = -math.inf
        s.label = torch.randint(0, known, (s.M,), device=DEV, generator=g).int()
        if s.M > 1:  # rows without a label
            s.label[torch.rand(s.M, **f32) < 0.05] = -1
        s.weight = torch.rand(s.M, **f32) / s.M
    return s


# --------------------------------------------------------------------------
# the plain forms: 32 bits, rounded once at the end
# --------------------------------------------------------------------------
def _quantize(x):
    """(whole numbers in 32 bits, scales [rows])."""
    top = x.float().abs().amax(1)
    # the bits of top / 127 up to eight significant ones, then the next such
    # number where that is too small; 127 times eight bits is exact
    s = ((top / 127).clamp(min=2.0 ** -126).view(torch.int32) & -65536).view(torch.float32)
    s = torch.where(127 * s < top, (s.view(torch.int32) + 65536).view(torch.float32), s)
    # quotients next to a half need more than 32 bits
    return torch.round(x.double() / s.double()[:, None]).float(), s


def _act(v, act):
    return v if act == "none" else torch.where(v >= 0, v, v * (SLOPE if act == "leaky" else 0.0))


def _plain_int8(s):
    q, scale = _quantize(s.x)
    y = (q @ s.wq[:, :s.K].float().t()) * (scale[:, None] * s.ws) + s.bias
    return {"y": _act(y, s.act).to(DT[s.out])}


def _plain_rows(s):
    wq, ws = _quantize(s.w)
    q, scale = _quantize(s.x)
    y = (q @ wq.t()) * (scale[:, None] * ws) + s.bias
    dy = s.dy.float()
    dx = (dy * ws) @ wq
    dw = (dy * scale[:, None]).t() @ q
    return {"y": y.to(DT[s.dt]), "dx": dx.to(DT[s.dt]), "dw": dw, "db": dy.sum(0)}


def _plain_lce(s):
    x, w = s.x.float(), s.w.float()
    z = x @ w.t() + s.bias
    top = z.amax(1, keepdim=True)
    lse = top[:, 0] + torch.log(torch.exp(z - top).sum(1))
    known, lab = s.label >= 0, s.label.long().clamp(min=0)[:, None]
    out = {"loss": torch.where(known, lse - z.gather(1, lab)[:, 0], 0.0), "lse": lse}
    if s.mode == "loss":
        return out
    k = (s.weight * known)[:, None]
    dz = torch.exp(z - lse[:, None]) * k
    dz.scatter_add_(1, lab, -k)
    return dict(out, dx=(dz @ w).to(s.x.dtype), dw=(dz.t() @ x).to(s.w.dtype), db=dz.sum(0))


# --------------------------------------------------------------------------
# the framework's entry points
# --------------------------------------------------------------------------
def _own_int8(s):
    from paper_1907_03739_amd import binding as pv
    return {"y": pv.pvconv_int8_linear(s.x, s.wq, s.ws, bias=s.bias, act=s.act, slope=SLOPE,
                                       out_dtype=DT[s.out])}


def _own_rows(s):
    from paper_1907_03739_amd import binding as pv
    wq, ws = pv.pvconv_int8_quantize(s.w)
    y, rows, scale = pv.pvconv_int8_linear(s.x, wq, ws, bias=s.bias, want_rows=True)
    dx, dw, db = pv.pvconv_int8_linear_backward(s.dy, rows, scale, wq, ws, s.K)
    return {"y": y, "dx": dx, "dw": dw, "db": db}


def _own_lce(s):
    from paper_1907_03739_amd import binding as pv
    if s.mode == "fused":
        loss, lse, dx, dw, db = pv.pvconv_linear_cross_entropy(
            s.x, s.w, s.label, bias=s.bias, row_weight=s.weight, want_grad=True)
        return {"loss": loss, "lse": lse, "dx": dx, "dw": dw, "db": db}
    loss, lse = pv.pvconv_linear_cross_entropy(s.x, s.w, s.label, bias=s.bias)
    out = {"loss": loss, "lse": lse}
    if s.mode == "loss":
        return out
    dx, dw, db = pv.pvconv_linear_cross_entropy_backward(s.x, s.w, s.label, lse, s.weight,
                                                         bias=s.bias)
    return dict(out, dx=dx, dw=dw, db=db)


def run(state):
    if own:
        return {"int8": _own_int8, "rows": _own_rows, "lce": _own_lce}[state.kind](state)
    return {"int8": _plain_int8, "rows": _plain_rows, "lce": _plain_lce}[state.kind](state)


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------
def work(case):
    c = SimpleNamespace(**case)
    size = {"bf16": 2, "f32": 4}
    s = size[c.dt]
    if c.kind == "int8":
        return {"bytes": c.M * c.K * s + c.N * (c.K + 8) + c.M * c.N * size[c.out],
                "flops": 2 * c.M * c.N * c.K}
    if c.kind == "rows":  # x, w, bias, dy read; y, dx, dw, db written
        return {"bytes": 2 * c.M * (c.K + c.N) * s + c.N * c.K * (s + 4) + 8 * c.N,
                "flops": 6 * c.M * c.N * c.K}
    ws = size[c.wdt]
    byt = c.M * (c.K * s + 12) + c.V * (c.K * ws + 4)
    if c.mode == "loss":
        return {"bytes": byt, "flops": 2 * c.M * c.V * c.K + 3 * c.M * c.V}
    return {"bytes": byt + c.M * (c.K * s + 4) + c.V * (c.K * ws + 4),
            "flops": 6 * c.M * c.V * c.K + 6 * c.M * c.V}


# --------------------------------------------------------------------------
# the definition in 64 bits
# --------------------------------------------------------------------------
def _exact_quantize(x):
    x = x.double()
    top = x.abs().max(dim=1).values
    t = (top / 127).clamp(min=2.0 ** -126)
    step = torch.exp2(torch.floor(torch.log2(t)) - 7)
    s = torch.ceil(t / step) * step
    s = torch.where(127 * (s - step) >= top, s - step, s).clamp(min=2.0 ** -126)
    s = torch.where(127 * s < top, s + step, s)
    u = x / s[:, None]
    low = torch.floor(u)
    up = (u - low > 0.5) | ((u - low == 0.5) & (low % 2 == 1))
    return low + up, s


def _exact_linear(s):
    q, scale = _exact_quantize(s.x)
    if s.kind == "int8":
        wq, ws, act = s.wq[:, :s.K].double(), s.ws.double(), s.act
    else:
        (wq, ws), act = _exact_quantize(s.w), "none"
    x, w = q * scale[:, None], wq * ws[:, None]
    v = torch.addmm(s.bias.double(), x, w.t())
    neg = {"none": 1.0, "relu": 0.0, "leaky": SLOPE}[act]
    out = {"y": v.clamp(min=0) + neg * v.clamp(max=0)}
    if s.kind == "rows":
        dy = s.dy.double()
        out.update(dx=dy @ w, dw=dy.t().contiguous() @ x, db=dy.sum(0))
    return out


def _exact_lce(s):
    w = s.w.double()
    wt = w.t().contiguous()
    out = {"loss": [], "lse": [], "dx": []}
    dw = torch.zeros_like(w)
    db = torch.zeros(s.V, dtype=torch.float64, device=DEV)
    rows = max(1, (1 << 26) // s.V)
    for i in range(0, s.M, rows):
        x = s.x[i:i + rows].double()
        z = torch.addmm(s.bias.double(), x, wt)
        lse = torch.logsumexp(z, 1)
        lab = s.label[i:i + rows].long()
        has = (lab >= 0).nonzero()[:, 0]
        loss = torch.zeros_like(lse)
        loss[has] = lse[has] - z[has, lab[has]]
        out["loss"].append(loss)
        out["lse"].append(lse)
        if s.mode == "loss":
            continue
        p = torch.softmax(z, 1)
        p[has, lab[has]] -= 1
        p *= (s.weight[i:i + rows].double() * (lab >= 0))[:, None]
        out["dx"].append(p @ w)
        dw += p.t().contiguous() @ x
        db += p.sum(0)
    if s.mode == "loss":
        return {"loss": torch.cat(out["loss"]), "lse": torch.cat(out["lse"])}
    return dict({k: torch.cat(v) for k, v in out.items()}, dw=dw, db=db)


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_lce(s) if s.kind == "lce" else _exact_linear(s)
