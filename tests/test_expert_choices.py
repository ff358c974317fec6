"""The library's choices between kernels of the products grouped by expert (csrc/expert_mm_plan.hpp, compiled by the system's C++
compiler, for 256 compute units) against times measured on an MI355X: the kernel that is chosen is never far from the better one."""
import ctypes
import os
import subprocess

import pytest

import test_gpu_expert_few as few
import test_gpu_expert_parts as parts
import test_gpu_expert_tiles as big

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CUS = 256


@pytest.fixture(scope="module")
def choices(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("choices") / "expert_choices.so")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_1802_04730_amd", "csrc"),
                    "-o", lib, os.path.join(ROOT, "tests", "expert_choices_host.cpp")], check=True)
    L = ctypes.CDLL(lib)
    i, q = ctypes.c_int, ctypes.c_int64
    L.few_rows.argtypes = [i, i, i, q, q, q]
    L.weights_parts.argtypes, L.weights_side.argtypes, L.rows_side.argtypes = [i, i, q, q, q, q, i], [i, i, q, q, q], [i, i, q, q, q]
    return L


# fp32, R, E, N, K, us by the kernel for few rows, us by tiles: uneven shares, weights from memory
FEW_OR_TILES = [
    (0, 32, 8, 4096, 2048, 30.2, 34.6), (0, 64, 8, 4096, 2048, 31.6, 34.7), (0, 192, 8, 4096, 2048, 51.2, 35.0), (0, 256, 8, 4096, 2048, 61.3, 35.2),
    (0, 384, 8, 4096, 2048, 80.7, 36.5), (0, 504, 8, 4096, 2048, 103.0, 40.1), (0, 384, 32, 2048, 1024, 35.3, 26.9), (0, 1024, 32, 2048, 1024, 60.1, 36.5),
    (0, 2016, 32, 2048, 1024, 99.7, 40.6), (0, 2048, 64, 1024, 2048, 117.1, 83.3), (0, 4032, 64, 1024, 2048, 198.2, 91.2), (0, 128, 8, 4099, 2047, 112.9, 56.7),
    (0, 504, 8, 4099, 2047, 333.5, 70.8), (0, 700, 12, 130, 1000, 7.4, 10.2), (0, 250, 5, 64, 512, 4.3, 5.4), (0, 1, 1, 64, 512, 3.7, 4.9),
    (0, 96, 4, 2048, 8192, 51.1, 90.0), (0, 504, 8, 512, 1024, 11.0, 10.3), (1, 32, 8, 2048, 1024, 13.3, 24.5), (1, 128, 8, 2048, 1024, 19.2, 24.8),
    (1, 504, 8, 2048, 1024, 49.9, 38.4), (1, 384, 16, 2047, 1001, 69.5, 47.6), (1, 6144, 128, 130, 1000, 56.3, 43.2), (1, 253, 128, 973, 459, 68.2, 95.7),
]


@pytest.mark.parametrize("f32,R,E,N,K,us_few,us_tiles", FEW_OR_TILES)
def test_few_rows_or_tiles(choices, f32, R, E, N, K, us_few, us_tiles):
    chosen = us_few if choices.few_rows(f32, K % (4 if f32 else 8) == 0, CUS, R, E, N) else us_tiles
    assert chosen <= 1.25 * min(us_few, us_tiles)


def test_shapes_of_the_gpu_tests(choices):
    for f32 in (0, 1):
        whole = lambda K: K % (4 if f32 else 8) == 0  # noqa: E731
        for T, R, E, N, K in big.SOME_ROWS + few.FEW:
            assert choices.few_rows(f32, whole(K), CUS, R, E, N)
        for T, R, E, N, K in few.TILES:
            assert R // E < 64 and not choices.few_rows(f32, whole(K), CUS, R, E, N)
        for R, E in ((64, 1), (128, 2), (100000, 3)):  # from 64 rows an expert on: tiles
            assert not choices.few_rows(f32, 1, CUS, R, E, 16)


# fp32, R, E, N, K, us with the rows in 1, 2, 4, 8, 16 parts: uneven shares
PARTS = [
    (0, 65536, 4, 256, 256, (161.3, 91.3, 50.7, 36.7, 41.6)), (0, 8192, 1, 512, 512, (58.5, 35.7, 22.1, 18.3, 21.6)), (0, 3000, 2, 64, 64, (11.4, 10.5, 8.0, 7.5, 7.2)),
    (0, 131072, 4, 1024, 1024, (634.0, 449.4, 403.0, 397.0, 424.8)), (0, 16384, 16, 256, 512, (22.9, 25.1, 28.2, 36.7, 54.1)), (0, 20000, 3, 130, 120, (86.7, 49.6, 27.8, 19.0, 18.0)),
    (0, 8059, 4, 704, 184, (24.2, 18.6, 17.3, 19.4, 24.1)), (0, 8418, 1, 712, 845, (91.2, 57.9, 42.8, 47.3, 57.0)), (0, 5263, 4, 816, 72, (16.8, 13.6, 12.1, 13.2, 16.0)),
    (0, 8192, 8, 1024, 512, (26.2, 31.4, 39.0, 55.9, 106.9)), (0, 16384, 32, 128, 256, (13.4, 15.6, 16.5, 19.7, 28.9)), (1, 65536, 4, 256, 256, (512.2, 261.3, 135.8, 114.4, 112.8)),
    (1, 8192, 1, 512, 512, (178.2, 96.7, 52.8, 47.7, 47.8)), (1, 3000, 2, 64, 64, (40.9, 24.5, 14.6, 10.2, 9.1)), (1, 37945, 2, 332, 240, (484.8, 247.2, 129.1, 108.3, 77.1)),
    (1, 2000, 1, 1024, 1024, (47.7, 45.4, 46.7, 49.3, 56.7)), (1, 8192, 8, 1024, 512, (92.8, 102.5, 101.5, 114.2, 168.3)), (1, 131072, 4, 1024, 1024, (2300.1, 2404.7, 2408.7, 2362.3, 2361.0)),
]


@pytest.mark.parametrize("f32,R,E,N,K,us", PARTS)
def test_parts_of_the_rows(choices, f32, R, E, N, K, us):
    side = choices.weights_side(64 if f32 else 128, CUS, E, N, K)
    parts = choices.weights_parts(f32, CUS, R, E, N, K, side)
    assert us[parts.bit_length() - 1] <= 1.25 * min(us)


# what, R, E, N, K, us by tiles of 256 (forward), 128, 64: bfloat16, uneven shares (one expert: dense)
SIDES = [
    ("fwd", 8192, 1, 8192, 8192, (774.2, 974.8, 1468.1)), ("fwd", 16384, 8, 4096, 4096, (507.8, 603.0, 910.1)), ("fwd", 8192, 16, 4096, 2048, (181.3, 175.5, 248.9)),
    ("fwd", 16384, 32, 2048, 4096, (349.3, 351.8, 492.7)), ("fwd", 2048, 16, 2048, 2048, (45.6, 30.5, 40.1)), ("fwd", 2000, 4, 512, 512, (15.6, 7.5, 6.2)),
    ("fwd", 4096, 8, 1024, 1024, (25.3, 17.0, 22.0)), ("fwd", 16384, 64, 1024, 2048, (128.0, 119.0, 154.9)), ("fwd", 1000, 2, 2048, 8192, (150.7, 82.3, 65.6)),
    ("dX", 8192, 1, 8192, 8192, (None, 985.2, 2177.4)), ("dX", 16384, 32, 2048, 4096, (None, 345.1, 496.2)), ("dX", 2000, 4, 512, 512, (None, 7.8, 6.4)),
    ("dX", 1200, 4, 8192, 1024, (None, 79.5, 61.0)), ("dX", 2048, 16, 2048, 2048, (None, 31.8, 40.8)), ("dX", 1000, 2, 2048, 8192, (None, 52.1, 59.7)),
    ("dW", 16384, 32, 2048, 4096, (None, 346.9, 489.9)), ("dW", 2000, 4, 512, 512, (None, 10.3, 6.9)), ("dW", 2048, 16, 2048, 2048, (None, 43.1, 55.2)),
]


@pytest.mark.parametrize("what,R,E,N,K,us", SIDES)
def test_sides_of_tiles(choices, what, R, E, N, K, us):
    if what == "dW":
        side = choices.weights_side(128, CUS, E, N, K)
    else:
        side = choices.rows_side(256 if what == "fwd" else 128, CUS, R, E, N if what == "fwd" else K)
    assert us[{256: 0, 128: 1, 64: 2}[side]] <= 1.15 * min(u for u in us if u)


def test_shapes_of_the_gpu_tests_of_parts(choices):
    for N, K in parts.SMALL:
        for f32 in (0, 1):
            per = 4 if f32 else 8
            side = choices.weights_side(64 if f32 or min(N, K) < per else 128, CUS, parts.E, N, K)
            assert side == 64 and choices.weights_parts(f32, CUS, parts.R, parts.E, N, K, side) > 1
    for R, E, N, K in parts.LARGE:
        assert choices.weights_side(128, CUS, E, N, K) == 128 and choices.weights_parts(0, CUS, R, E, N, K, 128) > 1
