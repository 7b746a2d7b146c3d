"""The rules by which the products of the 8-bit layer and of the linear cross entropy are
planned, seen through the sizes of their workspaces, and that the steps of test_gpu_products
reach every tile. No GPU."""
import random

import pytest

import _plan as p
from _steps import LAYER_STEPS, LOSS_STEPS, PIECES
from paper_1907_03739_amd import binding as pv


def loss_size(M, K, V, *dt):
    return pv._lib.pvconv_linear_cross_entropy_workspace_size(
        M, K, V, *[int(d == "bf16") for d in dt], 1)


def test_the_rules_are_those_of_the_library():
    rng = random.Random(3)

    def size(most):
        return int(most ** rng.random())
    for _ in range(1500):
        M, K, V = size(1 << 17), size(6000), size(1 << 16)
        dt = [rng.choice(("f32", "bf16")) for _ in range(4)]
        assert loss_size(M, K, V, *dt) == p.loss_workspace(M, K, V, *dt), (M, K, V, dt)
        splits = p.plan(M, V, K, 128, sizes="LGMS")[1]
        want = p.up(splits * M * V * 4, 256) * 256 if splits > 1 else 0
        assert pv._lib.pvconv_int8_linear_rows_workspace_size(M, K, V) == want, (M, K, V)


def test_the_steps_reach_every_tile():
    reached = set()
    for step in LAYER_STEPS:
        reached |= p.layer_products(*step)
    for step in LOSS_STEPS:
        assert loss_size(*step) == p.loss_workspace(*step)
        assert p.piece(step[0], step[2], *step[5:]) == step[2]
        reached |= p.loss_products(*step)
    # (deep enough for several rounds of the stages, all of them)
    deep = {k[:4] for k in reached if k[4]}
    want = {(w, t, s, False) for w in ("dx", "dw") for t in "LGMSP" for s in (False, True)}
    want |= {(w, t, False, True) for w in ("dx", "dw") for t in "LGMP"}
    want |= {("8-bit", t, False, False) for t in "LGMS"}
    want |= {("8-bit", t, True, False) for t in "GMS"}
    want |= {("8-bit", t, False, True) for t in "GM"}
    want |= {("loss", t, False, False) for t in "LGMSP"} | {("dz", t, False, False) for t in "GMSP"}
    want |= {("loss", t, False, True) for t in "LGMP"} | {("dz", t, False, True) for t in "GMP"}
    assert want <= deep, sorted(want - deep)


@pytest.mark.parametrize("M,K,V,xd,wd,dxd,dwd,pieces", PIECES)
def test_pieces_of_the_classes(M, K, V, xd, wd, dxd, dwd, pieces):
    n = p.piece(M, V, dxd, dwd)
    assert p.up(V, n) == pieces and V % n
    # (dz of a piece, the sums of dx over the pieces, what a whole and the last one take)
    assert loss_size(M, K, V, xd, wd, dxd, dwd) == p.loss_workspace(M, K, V, xd, wd, dxd, dwd)
    if M <= 100:  # dx split, in the first piece and the last
        for classes in (n, V % n):
            assert p.plan(M, K, classes, parts=(p.dz_parts(dxd), p.factor_parts(wd, dxd)))[1] > 1
