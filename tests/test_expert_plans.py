"""Which tile the shapes of the GPU tests take: the library's own choice (csrc/expert_mm_plan.hpp, compiled by the system's C++
compiler) for 256 compute units.  All tiles report one path, so a line that moves would take the coverage with it unseen."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import test_gpu_expert_tiles as big
import test_gpu_experts as small

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CUS = 256


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("plans") / "expert_plans.so")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_1802_04730_amd", "csrc"),
                    "-o", lib, os.path.join(ROOT, "tests", "expert_plans_host.cpp")], check=True)
    L = ctypes.CDLL(lib)
    i, q = ctypes.c_int, ctypes.c_int64
    L.rows_side.argtypes, L.weights_side.argtypes, L.weights_parts.argtypes = [i, i, q, q, q], [i, i, q, q, q], [i, i, q, q, q, q, i]
    L.row_tiles.argtypes, L.row_tiles.restype = [q, q, q], q
    return L


def test_the_large_tiles_are_taken(plans):
    for T, R, E, N, K in big.FORWARD:
        assert R // E >= 64  # (else the kernel for few rows)
        assert plans.rows_side(256 if K % 8 == 0 else 128, CUS, R, E, N) == (256 if K % 8 == 0 else 128)
    for R, E, N, K in big.BACK_X:
        assert plans.rows_side(128, CUS, R, E, K) == 128
    for T, R, E, N, K in big.BACK_W:
        assert plans.weights_side(128, CUS, E, N, K) == 128
    for R, E, N, K in big.PARTS:
        assert plans.weights_parts(0, CUS, R, E, N, K, plans.weights_side(128 if min(N, K) >= 8 else 64, CUS, E, N, K)) > 1
        assert plans.weights_parts(1, CUS, R, E, N, K, 64) > 1


def test_small_shapes_take_every_small_kernel(plans):
    kinds = set()
    for T, R, E, N, K in small.MM_SHAPES + big.SOME_ROWS:
        kinds.add("few" if R // E < 16 else "some" if R // E < 64 else "tile of %d" % plans.rows_side(256, CUS, R, E, N))
        kinds.add("weights by %d" % plans.weights_side(128, CUS, E, N, K))
        kinds.add("rows' gradient by %d" % plans.rows_side(128, CUS, R, E, K))
    assert {"few", "some", "tile of 64", "weights by 64", "rows' gradient by 64"} <= kinds


def test_row_tiles_bound_every_share_of_the_experts(plans):
    rng = np.random.default_rng(1)
    for _ in range(2000):
        R, E, bm = int(rng.integers(1, 3000)), int(rng.integers(1, 80)), int(rng.choice([16, 64, 128, 256]))
        shape = rng.integers(0, 4)
        if shape == 0:  # single rows as far as they go
            cuts = np.minimum(np.arange(1, E + 1), R)
        elif shape == 1:  # one row into a new tile
            cuts = np.minimum(np.cumsum(np.full(E, bm + 1)), R)
        else:
            cuts = np.sort(rng.integers(0, R + 1, E))
        counts = np.diff(np.concatenate([[0], cuts, [R]]))  # (the last: rows of no expert)
        assert (-(-counts // bm)).sum() <= plans.row_tiles(R, E, bm)


def test_the_chosen_tile_is_never_larger_than_asked_for(plans):
    rng = np.random.default_rng(2)
    for _ in range(2000):
        R, E, N = (int(2 ** rng.uniform(0, 20)) for _ in range(3))
        for most in (64, 128, 256):
            assert plans.rows_side(most, CUS, R, E, N) in (64, 128, 256)
            assert plans.rows_side(most, CUS, R, E, N) <= most


def test_offsets_that_decrease_are_tried_on_every_large_kernel(plans):
    (R, E, N, K), (R2, E2, N2, K2), (R3, E3, N3, K3) = big.DECREASING
    assert plans.rows_side(256, CUS, R, E, N) == 256
    assert plans.rows_side(128, CUS, R2, E2, K2) == 128
    assert plans.weights_parts(0, CUS, R3, E3, N3, K3, plans.weights_side(128, CUS, E3, N3, K3)) > 1
