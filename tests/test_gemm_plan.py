"""The choice of tiles of a GEMM launch (csrc/gemm_plan.cuh), on the CPU: every tile of every length is computed by somebody."""
import ctypes as C
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROWS, PAIR, SPLIT = 72, 8, 16
ALL, GATED = 0x7f, 0x55


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("plan") / "gemm_plan.so")
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-x", "c++", os.path.join(ROOT, "tests", "gemm_plan_lib.cpp"),
                           "-I", os.path.join(ROOT, "paper_2607_14647_b200", "csrc"), "-o", so])
    return C.CDLL(so)


def plan(lib, N, K, T_cap, gated=False, may_split=True, short_k_alone=True, sm=148, clusters=74, pair_mode=True, force=-1, mask=ALL):
    by_m, grid = (C.c_ubyte * ROWS)(), C.c_int(0)
    lib.gemm_plan(N, -(-K // 64) * 64, T_cap, int(gated), int(may_split and not gated), int(short_k_alone), sm, clusters, int(pair_mode), force,
                  mask & (GATED if gated else ALL), by_m, C.byref(grid))
    return list(by_m), grid.value


def tiles(N, p, gated):
    width = 256 - 32 * (p & 7)
    return -(-N // (width // 2 if gated else width))


def check(by_m, grid, N, T_cap, gated, mask=ALL, clusters=74):
    m_cap = -(-T_cap // 128)
    for m in sorted({*range(1, min(m_cap, 2 * ROWS) + 1), m_cap}):       # row blocks, as the kernel looks them up
        p = by_m[min(m, ROWS) - 1]
        assert p & 7 < 7 and p < SPLIT + 8 and ((mask & (GATED if gated else ALL)) | 1) >> (p & 7) & 1
        if p >= SPLIT:                                                    # a pair takes one tile
            assert not gated and m * tiles(N, p, gated) <= grid // 2, (m, p, grid)
        if p >= PAIR:
            assert clusters > 0 and grid % 2 == 0


@pytest.mark.parametrize("gated", [False, True])
def test_a_pair_for_every_tile_of_a_split(lib, gated):
    rng = random.Random(int(gated))
    for _ in range(4000):
        N, K, T_cap = (int(2 ** rng.uniform(0, b)) for b in (16, 13, 21))
        clusters = rng.choice([74, 74, 72, 1, 0])
        by_m, grid = plan(lib, N, K, T_cap, gated, clusters=clusters, force=rng.choice([-1, -1, *range(24)]), mask=rng.choice([ALL, 1, 0x11]))
        check(by_m, grid, N, T_cap, gated, clusters=clusters)


@pytest.mark.parametrize("N", [1, 64, 200, 256])
@pytest.mark.parametrize("blocks", [72, 73, 74, 75, 100, 16384])
def test_few_columns_and_very_many_rows(lib, N, blocks):
    by_m, grid = plan(lib, N, 1000, 128 * blocks)
    check(by_m, grid, N, 128 * blocks, False)


@pytest.mark.parametrize("force", [*range(7), *range(8, 15), *range(16, 23)])
def test_a_forced_plan_is_taken_where_it_can_be(lib, force):
    shapes = [(9, 331, 584), (300, 331, 600), (9, 336, 584), (300, 336, 600)]            # test_gpu_linear.py runs these
    for T, N, K, gated in [(*s, g) for s in shapes for g in (False, True)] + [(200, 777, 520, False)]:
        p = plan(lib, N, K, T, gated, force=force)[0][-(-T // 128) - 1]
        can = (not gated or GATED >> (force & 7) & 1) and not (gated and force >= SPLIT)
        assert (p == force) == bool(can), (T, N, K, gated, p)
    assert all(p < PAIR for p in plan(lib, 331, 512, 300, force=force)[0])          # few k-blocks: one SM per tile


def test_plans_that_cannot_be_forced_fall_back_to_the_rule(lib):
    rule = plan(lib, 6144, 4096, 1088)
    assert plan(lib, 6144, 4096, 1088, force=7) == rule and plan(lib, 6144, 4096, 1088, force=23) == rule
    assert plan(lib, 6144, 4096, 1088, force=16)[0][8] == rule[0][8] != 16          # 9 x 24 tiles, 74 pairs
    assert plan(lib, 6144, 4096, 1088, force=8, pair_mode=False) == plan(lib, 6144, 4096, 1088, pair_mode=False)
