"""The library's choices between kernels of the products grouped by expert (csrc/expert_mm_plan.hpp, compiled by the system's C++
compiler, for 256 compute units) against times measured on an MI355X: the kernel that is chosen is never far from the better one."""
import ctypes
import os
import subprocess

import pytest

import test_gpu_expert_few as few
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
