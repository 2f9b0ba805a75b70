"""The prices by which 4-bit products pick tiles, on the host (mx4_tile_rules_host.cpp; 256 compute units)."""
import os
import subprocess

import pytest

from paper_2605_17889_amd import build as hip_build
from mx4_sizes import GATEUP, PLAIN

HERE = os.path.dirname(os.path.abspath(__file__))
FEW, FEW_WIDE, T16X64, T32X64_DEEP, T32X64, T64X64, T64X128, T128X128, T128X128_PAIR, LARGE = range(10)
GATE_FEW, GATE32, GATE64, GATE128, GATE_LARGE = range(5)


@pytest.fixture(scope="module")
def tile(tmp_path_factory):
    out = tmp_path_factory.mktemp("host") / "mx4_tile_rules_host"
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wno-unused-function", "-I", hip_build.CSRC,
                    os.path.join(HERE, "mx4_tile_rules_host.cpp"), "-o", str(out)], check=True)
    return lambda *args: int(subprocess.run([str(out), *map(str, args)], capture_output=True, text=True, timeout=60,
                                            check=True).stdout)


@pytest.mark.parametrize("R,E,N,K,want", [
    (1, 1, 4096, 14336, FEW),                  # us: 9.0, 32 columns 13.8, 16 x 64 tiles 17.6
    (16, 1, 6144, 16384, FEW_WIDE),            # 17.4, 16 columns 20.4, 16 x 64 tiles 20.4
    (16, 1, 16384, 4096, T16X64),              # 7.9, 32 x 64 8.1, a few rows 11.7
    (128, 1, 4096, 14336, T32X64_DEEP),        # 17.7, 64 x 64 21.5, 128 x 128 45.6
    (256, 1, 4096, 14336, T64X64),             # 21.7, 64 x 128 32.2, 32 x 64 28.1
    (512, 1, 4096, 14336, T64X128),            # 32.7, 64 x 64 35.8, 128 x 128 45.2
    (1024, 1, 4096, 14336, T128X128),          # 46.9, large 58.0
    (2048, 1, 4096, 14336, LARGE),             # 65.0, 128 x 128 two at once 75.5
    (512, 128, 2048, 768, T32X64), (8000, 128, 2048, 768, T128X128_PAIR), (64000, 128, 2048, 768, LARGE)])
def test_products(tile, R, E, N, K, want):
    assert tile("plain", R, E, N, K) == want


@pytest.mark.parametrize("R,E,f,d,want", [
    (8, 128, 768, 2048, GATE_FEW),             # us of the whole FFN: 10.3, 64 columns 11.4
    (16, 128, 768, 2048, GATE32),              # 13.1, 32 columns 13.5
    (32, 8, 14336, 4096, GATE32),              # 129.4, 64 rows 129.0, 128 rows 156
    (256, 8, 14336, 4096, GATE64),             # 123.5, 32 rows 140.9, 128 rows 156.0
    (800, 8, 14336, 4096, GATE128),            # 162.8, large 166.1, 64 rows 192.3
    (1024, 8, 14336, 4096, GATE_LARGE),        # 181.2, 128 rows 210.5
    (16000, 128, 768, 2048, GATE_LARGE), (2048, 128, 768, 2048, GATE32), (4096, 128, 768, 2048, GATE64)])
def test_gate_and_up(tile, R, E, f, d, want):
    assert tile("gateup", R, E, f, d) == want


def test_sizes_of_the_numerical_tests_take_every_tile(tile):
    assert {tile("plain", R, E, N, K) for R, E, N, K in PLAIN} == set(range(10))
    assert {tile("gateup", R, E, f, d) for R, E, f, d in GATEUP} == set(range(5))


# rows, columns, threads of a workgroup
SIZES = {FEW: (16, 16, 512), FEW_WIDE: (16, 32, 512), T16X64: (16, 64, 256), T32X64_DEEP: (32, 64, 256), T32X64: (32, 64, 256),
         T64X64: (64, 64, 256), T64X128: (64, 128, 256), T128X128: (128, 128, 256), T128X128_PAIR: (128, 128, 256)}


def test_launches_hold_fewer_than_2_32_threads(tile):
    """A workgroup per possible tile: with many groups and columns the smaller tiles would be too many."""
    for R in (1, 16, 100, 256, 1000, 4000, 16384):
        for E in (1, 64, 256):
            for N in (1 << 20, (1 << 21) + 16, 3 << 20, 1 << 22):
                for K in (32, 128, 256):
                    t = tile("plain", R, E, N, K)
                    rows, columns, threads = SIZES[t]
                    assert (R // rows + min(R, E)) * -(-N // columns) * threads < 2**32, (R, E, N, K, t)


def test_large_tiles_only_where_they_fit(tile):
    for R in (1, 100, 5000, 100000):
        for N in (16, 128, 240):
            assert tile("plain", R, 1, N, 4096) != LARGE
        for K in (32, 128, 256):
            assert tile("plain", R, 1, 4096, K) != LARGE and tile("gateup", R, 1, 4096, K) != GATE_LARGE
