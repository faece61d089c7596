"""The work partition of the shared-prefix attention, walked on the CPU: every key block exactly once, pieces and merges
agree, segments are even."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("plan") / "walk.so")
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-x", "c++", os.path.join(ROOT, "tests", "prefix_plan_walk.cpp"),
                           "-I", os.path.join(ROOT, "paper_2607_14647_b200", "csrc"), "-o", so])
    return C.CDLL(so)


def walk(lib, tokens, lens, group_size, n_kv_heads, n_seg):
    t, p = np.ascontiguousarray(tokens, np.int32), np.ascontiguousarray(lens, np.int32)
    most, least = C.c_longlong(0), C.c_longlong(0)
    rc = lib.walk(len(t), t.ctypes.data_as(C.c_void_p), p.ctypes.data_as(C.c_void_p), group_size, n_kv_heads, n_seg, C.byref(most), C.byref(least))
    assert rc == 0, (rc, tokens, lens, group_size, n_kv_heads, n_seg)
    return most.value, least.value


@pytest.mark.parametrize("n_seg", [1, 2, 148, 256])
@pytest.mark.parametrize("group_size", [1, 3, 4, 5, 8, 16])
def test_single_group(lib, n_seg, group_size):
    for tokens in (1, 7, 8, 31, 32, 33, 64, 65, 603, 4352):
        for length in (0, 1, 127, 128, 129, 2048, 4099, 131072):
            for kv in (1, 2, 8):
                walk(lib, [tokens], [length], group_size, kv, n_seg)


def test_random_groups(lib):
    rng = np.random.default_rng(0)
    for _ in range(3000):
        G = int(rng.integers(1, 9))
        tokens = rng.integers(0, 200, G) * (rng.random(G) < 0.8)
        lens = np.exp(rng.uniform(0, 10, G)).astype(int) * (rng.random(G) < 0.7)
        walk(lib, tokens, lens, int(rng.choice([1, 2, 3, 4, 6, 8, 9, 16])), int(rng.choice([1, 2, 4, 8, 16])), int(rng.choice([1, 2, 3, 7, 148, 160, 256])))


def test_many_groups(lib):
    rng = np.random.default_rng(1)
    walk(lib, rng.integers(0, 18, 4096), rng.integers(0, 3000, 4096), 4, 8, 148)


def test_segments_are_even_where_there_is_enough_work(lib):
    most, least = walk(lib, [603], [4099], 4, 8, 148)
    assert most <= 1.25 * least                               # one item's overhead more or less, of about four items' worth
