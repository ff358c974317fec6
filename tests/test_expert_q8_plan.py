"""Which kernel and tile the shapes of the GPU tests of products with 8-bit weights take, and how far the choice is from the better one by measured times: the library's own
choice (csrc/expert_mm_q8_plan.hpp, compiled by the system's C++ compiler) for 256 compute units."""
import ctypes
import os
import subprocess

import pytest

import test_gpu_even as small
import test_gpu_even_tiles as big

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CUS = 256


@pytest.fixture(scope="module")
def kernel(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("plans") / "expert_q8_plan.so")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_1802_04730_amd", "csrc"),
                    "-o", lib, os.path.join(ROOT, "tests", "expert_q8_plan_host.cpp")], check=True)
    L = ctypes.CDLL(lib)
    i, q = ctypes.c_int, ctypes.c_int64
    L.q8_side.argtypes, L.q8_few.argtypes = [i, i, q, q, q, q], [i, i, q, q, q]
    return lambda f32, R, E, N, K: 0 if L.q8_few(f32, CUS, R, E, N) else L.q8_side(f32, CUS, R, E, N, -(-K // 128))


def test_every_kernel_is_tested(kernel):
    for side, f32, T, R, E, N, K in big.SHAPES:
        assert kernel(f32, R, E, N, K) == side
    assert {kernel(0, *shape) for shape in big.SHORT} == {256}
    taken = {kernel(f32, R, E, N, K) for T, R, E, N, K in small.MM_SHAPES for f32 in (0, 1)}
    assert {0, 64} <= taken


def test_float_never_takes_the_largest_tile(kernel):
    for n in (100, 3000, 100000):
        assert kernel(1, n, 1, n, 8192) <= 128


# f32, R, E, N, K, us by the kernel for few rows (None: not measured), by tiles of 64, 128, 256: operands in 8 bits, uneven shares
TIMES = [
    (0, 16384, 32, 2048, 4096, None, 290.8, 224.9, 223.9), (0, 16384, 32, 4096, 2048, None, 331.3, 239.3, 234.9), (0, 4096, 1, 8192, 4096, None, 203.9, 132.6, 124.5),
    (0, 4096, 1, 8192, 1024, None, 63.3, 44.4, 48.5), (0, 2048, 16, 2048, 2048, None, 25.6, 19.1, 31.1), (0, 8192, 8, 1024, 4096, None, 70.9, 58.2, 59.9),
    (0, 512, 1, 4096, 4096, None, 20.5, 28.3, 53.6), (0, 300, 1, 1000, 4000, None, 13.4, 19.6, 52.2), (0, 4096, 64, 1024, 1024, None, 19.9, 16.5, 24.7),
    (0, 2000, 4, 512, 512, None, 5.3, 7.0, 14.3), (0, 32, 8, 4096, 2048, 14.3, 14.0, 17.8, 31.9), (0, 128, 8, 4096, 2048, 22.0, 14.0, 18.1, 32.8),
    (0, 512, 8, 4096, 2048, 60.0, 17.5, 18.7, 33.3), (0, 512, 32, 2048, 1024, 35.4, 13.6, 15.2, 22.6), (0, 1, 1, 8192, 4096, 7.5, 17.8, 23.3, 49.4),
    (0, 16, 1, 8192, 4096, 9.9, 18.7, 24.2, 49.5), (0, 63, 1, 8192, 4096, 27.3, 19.7, 24.9, 50.6), (0, 2048, 64, 1024, 2048, 66.4, 24.2, 25.7, 38.6),
    (0, 32, 1, 2048, 8192, 15.5, 23.0, 33.5, None), (0, 100, 1, 512, 4096, 9.0, 12.7, 18.8, None), (0, 8, 8, 1024, 4096, 8.0, 13.3, 19.3, None),
    (0, 58, 12, 130, 1000, 5.7, 6.0, 8.0, None), (1, 2100, 12, 1001, 517, 52.2, 12.4, 17.2, None), (1, 4096, 1, 4096, 4096, 788.0, 215.9, 182.7, None),
    (1, 8192, 32, 2048, 2048, 421.5, 146.1, 128.3, None), (1, 2048, 16, 2048, 2048, 108.4, 39.4, 46.6, None), (1, 16, 1, 8192, 4096, 10.9, 26.0, 49.2, None),
    (1, 32, 8, 4096, 2048, 15.5, 20.5, 31.4, None), (1, 256, 8, 4096, 2048, 35.2, 21.0, 32.4, None),
]


# the same with sets of operands in turn, so that they come from memory
TIMES += [
    (0, 2000, 4, 512, 512, None, 6.0, 8.0, 15.8), (0, 2048, 32, 2048, 1024, None, 24.3, 26.9, 27.6), (0, 512, 1, 4096, 4096, None, 21.1, 26.7, 54.6),
    (0, 2048, 8, 2048, 2048, None, 33.4, 25.0, 36.4), (0, 8192, 16, 1024, 1024, None, 29.1, 25.7, 23.7), (0, 8192, 128, 1024, 1024, None, 45.1, 47.7, 58.0),
    (0, 700, 1, 3000, 1000, None, 9.1, 11.0, 21.4), (0, 4096, 4, 1024, 4096, None, 50.0, 37.5, 60.7), (0, 8192, 32, 1024, 2048, None, 51.4, 43.7, 38.3),
    (0, 2048, 1, 2048, 2048, None, 16.0, 16.9, 32.4), (0, 8192, 1, 1024, 4096, None, 63.1, 41.9, 60.7), (0, 16384, 32, 2048, 4096, None, 276.8, 195.0, 194.7),
    (0, 16384, 32, 4096, 2048, None, 293.7, 211.2, 184.0), (0, 32768, 32, 2048, 4096, None, 501.3, 349.6, 312.9), (0, 65536, 32, 2048, 4096, None, 936.4, 651.7, 560.8),
    (0, 16384, 16, 2048, 4096, None, 259.4, 190.7, 185.8), (0, 16384, 8, 2048, 4096, None, 241.3, 174.2, 178.7), (0, 8192, 4, 4096, 4096, None, 239.1, 174.2, 178.4),
    (0, 8192, 16, 4096, 2048, None, 151.4, 111.2, 106.8), (0, 16384, 64, 2048, 2048, None, 173.3, 134.6, 113.7), (0, 8192, 8, 1024, 4096, None, 79.8, 65.2, 62.4),
    (0, 4096, 1, 8192, 4096, None, 242.1, 165.9, 132.2), (0, 8192, 1, 8192, 8192, None, 847.5, 591.9, 460.9), (0, 4096, 1, 8192, 1024, None, 66.2, 48.7, 49.5),
    (0, 4096, 64, 1024, 1024, None, 26.4, 29.4, 29.2), (0, 4096, 16, 2048, 2048, None, 51.3, 43.5, 38.0), (0, 2048, 16, 2048, 2048, None, 35.3, 26.2, 37.0),
    (0, 16384, 128, 2048, 1024, None, 133.2, 102.9, 123.9), (0, 32768, 128, 1024, 2048, None, 184.7, 135.5, 119.7), (0, 1024, 1, 4096, 4096, None, 27.1, 28.0, 54.7),
    (0, 4096, 8, 4096, 4096, None, 151.5, 116.2, 122.8), (0, 2048, 1, 4096, 4096, None, 63.5, 41.5, 60.9), (0, 1500, 1, 8192, 4096, None, 86.1, 74.8, 63.0),
    (0, 3000, 1, 4096, 8192, None, 156.6, 120.3, 110.4), (0, 65536, 64, 1024, 2048, None, 292.2, 204.5, 182.7),
]


@pytest.mark.parametrize("f32,R,E,N,K,few,t64,t128,t256", TIMES)
def test_the_choice_is_near_the_best(kernel, f32, R, E, N, K, few, t64, t128, t256):
    us = {0: few, 64: t64, 128: t128, 256: t256}
    assert us[kernel(f32, R, E, N, K)] <= 1.16 * min(t for t in us.values() if t is not None)
