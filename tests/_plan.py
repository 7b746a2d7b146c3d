"""The rules by which products take a tile and are split (csrc/pv_product.h) and the loss
its pieces (csrc/linear_ce.hip), again, so that tests can choose sizes that reach each of
them and notice when they no longer do."""
import numpy as np

F = np.float32
# rows, columns, workgroups that the chip holds, us a slice, us beside them
COSTS = {"L": (256, 256, 256, 1.4, 6.0), "G": (256, 128, 256, 0.82, 4.5),
         "M": (128, 128, 256, 0.62, 3.5), "S": (64, 64, 512, 0.42, 3.0)}
WAVE_ROWS = {"L": 128, "G": 64, "M": 64, "S": 32, "P": 16}
PIECE_BYTES, LEAST_CLASSES, STATS_BYTES = 1 << 29, 2048, 1 << 26


def up(n, per):
    return -(-n // per)


def pairs(a, b):
    """Products of parts that a product of operands in a and b parts takes."""
    orders = 2 if a < 3 and b < 3 else 3
    return sum(1 for i in range(a) for j in range(b) if i + j < orders)


def _costs(parts, sizes):
    costs = [(k, *v) for k, v in COSTS.items() if k in sizes]
    if "P" in sizes and parts in ((3, 3), (3, 1), (1, 3)):
        costs.append(("P", 64, 64, 256, 0.18 if pairs(*parts) > 3 else 0.22, 3.0))
    return costs


def plan(rows, cols, depth, per=64, parts=(1, 1), may_split=True, sizes="LGMSP"):
    """(tile, splits, slices of a split, tiles, us) of a product over `depth`, `per` a slice."""
    n_pairs, chosen = pairs(*parts), None
    total = up(depth, per) * n_pairs
    for name, tm, tn, slots, a_slice, rest in _costs(parts, sizes):
        tiles, n = up(rows, tm) * up(cols, tn), 1
        while n == 1 or (may_split and tiles * (n - 1) < slots and total // n >= 4):
            each = up(total, n)
            if name == "P":
                each = up(each, n_pairs) * n_pairs
            splits = up(total, each) if each else 1
            us = F(up(tiles * splits, slots)) * (F(each) * F(a_slice) + F(rest))
            if splits > 1:
                us = us + (F(4) + F(splits) * F(rows) * F(cols) * F(8 / 4e6))
            if chosen is None or us < chosen[4]:
                chosen = (name, splits, each, tiles, us)
            n += 1 if n < 8 else n // 4
    return chosen


def pair_tile(x, y):
    """The tile in which two products (rows, cols, depth, parts) are one launch, or None."""
    best = plan(*x[:3], parts=x[3])[4] + plan(*y[:3], parts=y[3])[4] + F(3)
    choices = _costs((1, 1), "S")
    if x[3][0] == 3 and y[3][0] == 3 and x[3][1] == y[3][1]:
        choices += _costs(x[3], "P")
    tile = None
    for name, tm, tn, slots, a_slice, rest in choices:
        blocks = 8 + sum(up(up(p[0], tm) * up(p[1], tn), 8) * 8 for p in (x, y))
        slices = max(up(p[2], 64) * pairs(*p[3]) for p in (x, y))
        us = F(slices) * F(a_slice) + F(rest)
        if blocks <= slots and us <= best:
            best, tile = us, name
    return tile


def factor_parts(dt, out="f32"):
    return 1 if dt == "bf16" else 2 if out == "bf16" else 3


def dz_parts(out):
    return 2 if out == "bf16" else 3


def piece(M, V, dxd, dwd):
    """The classes of a piece of the loss's gradients."""
    row = up(max(M, 1), 64) * 64 * 2 * max(dz_parts(dxd), dz_parts(dwd))
    return min(V, max(PIECE_BYTES // row // 256 * 256, LEAST_CLASSES))


def _key(what, chosen):
    tile, splits, each, tiles, _ = chosen
    # (several tiles a workgroup; a loop of several rounds of stages, or its short form)
    return (what, tile, splits > 1, tiles * splits > (512 if tile == "S" else 256), each > 6)


def layer_products(M, K, N, yd, xd):
    """What the 8-bit layer's product and its gradients run: (which, tile, split, several
    tiles a workgroup, deep)."""
    dx = (1, 2) if yd == "bf16" else (2 if xd == "bf16" else 3, 1)
    dw = (2 if yd == "bf16" else 3, 1)
    return {_key("8-bit", plan(M, N, K, 128, sizes="LGMS")), _key("dx", plan(M, K, N, parts=dx)),
            _key("dw", plan(N, K, M, parts=dw))}


def _gradients(M, K, V, xd, wd, dxd, dwd):
    return ((M, K, V, (dz_parts(dxd), factor_parts(wd, dxd))),
            (V, K, M, (dz_parts(dwd), factor_parts(xd, dwd))))


def loss_products(M, K, V, xd, wd, dxd, dwd):
    """The same of the loss and its gradients (more than 64 classes, one piece of them)."""
    z = dict(parts=(factor_parts(xd), factor_parts(wd)), may_split=False)
    dx, dw = _gradients(M, K, V, xd, wd, dxd, dwd)
    return {_key("loss", plan(M, V, K, **z)), _key("dz", plan(M, V, K, sizes="GMSP", **z)),
            _key("dx", plan(*dx[:3], parts=dx[3])), _key("dw", plan(*dw[:3], parts=dw[3]))}


def loss_workspace(M, K, V, xd, wd, dxd, dwd):
    """Bytes that the loss with all of its gradients asks for."""
    def a256(n):
        return up(n, 256) * 256

    def panel(rows, pitch, parts):
        return a256(rows * pitch) * parts

    def wide(n):
        return up(n, 64) * 128
    total = panel(M, wide(K), factor_parts(xd)) + panel(V, wide(K), factor_parts(wd))
    if V > 64:
        most = STATS_BYTES // 8 // max(M, 1) * 64
        classes = V if most >= V else min(V, max(4096, most // 128 * 128))
        total += a256(M * up(classes, 64) * 8) + a256(M * 8) + a256(M * 4)
    total += a256(M * 4)
    n = piece(M, V, dxd, dwd)
    pitch = wide(n)
    if pitch % 4096 == 0:
        pitch += 128
    total += panel(up(M, 64) * 64, pitch, max(dz_parts(dxd), dz_parts(dwd)))
    if n < V:
        total += a256(M * K * 4)  # the sums of dx over the pieces
    partial, sums = 0, 0
    for classes in (n, V % n):
        if classes == 0:
            continue
        dx, dw = _gradients(M, K, classes, xd, wd, dxd, dwd)
        alone = n < V or pair_tile(dx, dw) is None
        for p in (dx, dw):
            splits = plan(*p[:3], parts=p[3])[1] if alone else 1
            partial = max(partial, splits * p[0] * p[1] * 4 if splits > 1 else 0)
        z = plan(M, classes, K, parts=(factor_parts(xd), factor_parts(wd)), may_split=False,
                 sizes="SP" if V <= 64 else "GMSP")[0]
        rows = {"G": 256, "M": 128}.get(z, 64)
        sums = max(sums, up(M, rows) * rows // WAVE_ROWS[z] * classes * 4)
    return total + a256(partial) + a256(sums)
