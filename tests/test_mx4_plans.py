"""Which kernel a product of microscaled 4-bit matrices goes to, asked on the host: the shapes that the GPU tests run are still of the
kernels that they are meant for, and there is one for every kernel that a product can go to."""
import ctypes
import math
import random

import pytest

from mx4_plans import INSIDE, PLANS
from paper_2510_19482_amd import binding as B

F16, F32, BF16, MX4 = B.HLQ_F16, B.HLQ_F32, B.HLQ_BF16, B.HLQ_MX4


def plan(R, N, K, E, gated, xtype=MX4):
    p = B.mx4_plan_query(N, K, R, E, R, xtype, gated)
    return (p.kernel, p.tile_rows, p.tile_cols, p.k_parts, gated), bool(p.quantizes), p.workspace_bytes


def kind(key, experts, inside):
    """What a kernel is compiled or branches for."""
    kernel, rows, cols, parts, gated = key
    return kernel, rows, cols, parts > 1, gated, experts, inside


@pytest.mark.parametrize("key", list(PLANS), ids=str)
def test_shapes_are_of_the_plan_that_they_stand_for(key):
    for R, N, K, E in PLANS[key]:
        assert plan(R, N, K, E, key[4])[:2] == (key, False)
        if not plan(R, N, K, E, key[4], F32)[1]:
            assert plan(R, N, K, E, key[4], F32)[0] == key


@pytest.mark.parametrize("parts,gated", list(INSIDE))
def test_shapes_are_quantized_where_they_stand_for_it(parts, gated):
    for R, N, K, E in INSIDE[parts, gated]:
        for xtype in (F16, BF16, F32):
            assert plan(R, N, K, E, gated, xtype)[:2] == ((1, 16, 16, parts, gated), True)


def draw(rng):
    def log(lo, hi):
        return int(math.exp(rng.uniform(math.log(lo), math.log(hi))))
    E = rng.choice([1, 1, rng.randint(2, 64), log(2, 1024)])
    N, K, R = log(1, 60000), log(1, rng.choice([16000, 16000, 1 << 21])), log(1, 30000)
    gated = rng.random() < 0.5
    return R, N + (N % 2 if gated else 0), K, E, gated


def test_every_kernel_has_a_shape():
    have = {kind(key, E > 1, False) for key, shapes in PLANS.items() for _, _, _, E in shapes}
    have |= {kind((1, 16, 16, parts, gated), E > 1, True) for (parts, gated), shapes in INSIDE.items() for _, _, _, E in shapes}
    parts = {key[:4] for key in PLANS}
    rng = random.Random(7)
    for _ in range(60000):
        R, N, K, E, gated = draw(rng)
        if E * N > 1 << 31:
            continue
        for xtype in (F32, MX4):
            key, inside, _ = plan(R, N, K, E, gated, xtype)
            assert kind(key, E > 1, inside) in have, (R, N, K, E, gated, xtype)
            assert key[:4] in parts, (R, N, K, E, gated)


def test_a_call_fits_the_workspace_that_is_asked_for():
    rng = random.Random(8)
    for _ in range(30000):
        R, N, K, E, gated = draw(rng)
        if E * N > 1 << 31:
            continue
        x_rows = rng.choice([R, max(1, R // 8)])
        room = B.mx4_workspace_bytes(N, K, E, x_rows, R)
        for rows in {R, max(1, R // 2), max(1, R // 7), 1}:      # fewer rows never need more
            assert B.mx4_plan_query(N, K, rows, E, min(x_rows, rows), F32, gated).workspace_bytes <= room


@pytest.mark.parametrize("R,N", [(17, 100), (128, 128), (300, 700)])
def test_room_for_partial_sums_wherever_k_may_be_cut(R, N):
    # a share of K has four panels of 128 at least, the first of two of seven panels has four; whether the estimate takes it or not
    def partial(panels):
        return B.mx4_workspace_bytes(N, 128 * panels, 1, R, R) - 131072 - (R * panels * 68 + 255) // 256 * 256
    assert partial(6) == 0
    for panels in (7, 8, 9, 100):
        assert partial(panels) >= 2 * 4 * R * N


def test_refusals():
    out = B.Mx4PlanInfo()
    q = B.lib.hlq_mx4_plan_query
    assert q(64, 96, 1, 4, 4, 0, 0, None) == 1
    assert q(0, 96, 1, 4, 4, 0, 0, ctypes.byref(out)) == 2 and q(64, 0, 1, 4, 4, 0, 0, ctypes.byref(out)) == 2 and q(64, 96, 0, 4, 4, 0, 0, ctypes.byref(out)) == 2
    assert q(64, 96, 1, 4, 0, 0, 0, ctypes.byref(out)) == 2 and q(63, 96, 1, 4, 4, 0, 1, ctypes.byref(out)) == 2 and q(64, 96, 1, -1, 4, 0, 0, ctypes.byref(out)) == 2
    assert q(64, 96, 1025, 4, 4, 0, 0, ctypes.byref(out)) == 3 and q(64, 96, 1, 4, 4, 4, 0, ctypes.byref(out)) == 3 and q(64, 96, 1, 4, 4, 0, 2, ctypes.byref(out)) == 3
    assert q(64, 96, 1, 4, 1 << 31, 0, 0, ctypes.byref(out)) == 3 and q((1 << 20) + 1, 96, 1, 4, 4, 0, 0, ctypes.byref(out)) == 3
    assert q(64, (1 << 21) + 1, 1, 4, 4, 0, 0, ctypes.byref(out)) == 3
