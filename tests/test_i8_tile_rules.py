"""The rules by which 8-bit products pick tiles, on the host (i8_tile_rules_host.cpp; 256 compute units). No tile changes a bit of an
output, so only their choice can be checked: each line is a size at which both sides were measured."""
import os
import subprocess

import pytest

from paper_2605_17889_amd import build as hip_build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def say(tmp_path_factory):
    out = tmp_path_factory.mktemp("host") / "i8_tile_rules_host"
    subprocess.run([hip_build.HIPCC, "-x", "hip", "--offload-host-only", "-O1", "-std=c++17", "-Wno-unused-function",
                    "-I", os.path.join(hip_build.ROOT, "include"), "-I", hip_build.CSRC,
                    os.path.join(HERE, "i8_tile_rules_host.cpp"), "-o", str(out)], check=True)
    return lambda *args: subprocess.run([str(out), *map(str, args)], capture_output=True, text=True, timeout=60, check=True).stdout.strip()


ROWS256, ROWS128, ROWS64, ROWS32, ROWS96 = 0, 1, 2, 3, 4


@pytest.mark.parametrize("E,N,K,mid_n_tiles,want", [
    (16, 4096, 4096, 16, ROWS128), (32, 4096, 4096, 16, ROWS128),
    # a group past 128 rows costs more there than the others gain: skewed ones 119 -> 153 us, 136 -> 144, drawn evenly 135 -> 165
    (8, 4096, 14336, 32, ROWS256), (8, 8192, 8192, 32, ROWS256), (16, 8192, 8192, 32, ROWS256), (32, 2048, 8192, 8, ROWS256),
    (32, 5120, 5120, 20, ROWS256), (32, 4096, 7168, 16, ROWS256),
    (8, 4096, 4096, 16, ROWS256),                        # half the compute units without a tile
])
def test_down_projections_of_groups_that_mostly_fit_128_rows(say, E, N, K, mid_n_tiles, want):
    assert int(say("product", ROWS256, 110 * E, E, N, K, mid_n_tiles)) == want
    assert int(say("product", ROWS256, 130 * E, E, N, K, mid_n_tiles)) == ROWS256


@pytest.mark.parametrize("E,d,f,want", [
    (8, 4096, 14336, ROWS128), (16, 4096, 4096, ROWS128), (32, 4096, 4096, ROWS128), (8, 8192, 8192, ROWS128), (16, 8192, 4096, ROWS128),
    # rows that are no multiple of 4 KB apart: skewed groups 193 -> 225 us, 197 -> 207; a longer reduction: 331 -> 354
    (8, 5120, 10240, ROWS256), (8, 7168, 8192, ROWS256), (16, 6144, 6144, ROWS256), (8, 12288, 8192, ROWS256)])
def test_gateup_of_groups_that_mostly_fit_128_rows(say, E, d, f, want):
    assert int(say("gateup", ROWS256, 110 * E, E, f, d)) == want


@pytest.mark.parametrize("E,d,f,full", [(8, 6144, 16384, True), (8, 8192, 8192, True), (16, 6144, 6144, True), (16, 4096, 4096, True),
                                        (8, 4096, 14336, False), (8, 5120, 10240, False)])
def test_gateup_of_fewer_rows_takes_128_row_tiles_in_full_rounds_only(say, E, d, f, full):
    """Part of a round more costs even groups 7 to 10 % (154 -> 168, 154 -> 165 us at 46 rows)."""
    for rows, config in ((46, ROWS64), (58, ROWS96), (66, ROWS96)):
        assert int(say("gateup", config, rows * E, E, f, d)) == (ROWS128 if full else config)
    assert int(say("gateup", ROWS64, 45 * E, E, f, d)) == ROWS64 and int(say("gateup", ROWS32, 20 * E, E, f, d)) == ROWS32
    assert int(say("gateup", ROWS96, 70 * E, E, f, 2048)) == ROWS96          # shorter than 4096


def test_long_reductions_of_few_rows(say):
    for rows, config, want in ((20, ROWS32, ROWS96), (38, ROWS64, ROWS128), (52, ROWS96, ROWS128), (12, ROWS32, ROWS32)):
        assert int(say("product", config, 8 * rows, 8, 4096, 14336, 32)) == want
    assert int(say("product", ROWS32, 8 * 18, 8, 2048, 8192, 16)) == ROWS64      # half the compute units idle with 128 columns
    assert int(say("product", ROWS96, 64 * 72, 64, 2048, 1408, 16)) == ROWS96


@pytest.mark.parametrize("K,gateup,down,mid,one", [
    (512, 1, 0, 0, 1), (1024, 1, 0, 0, 1), (1536, 0, 0, 0, 0), (2048, 1, 0, 0, 1), (2560, 0, 0, 0, 0), (4096, 1, 1, 1, 1), (5120, 0, 0, 1, 0),
    (6144, 0, 0, 1, 0), (8192, 1, 1, 1, 1), (14336, 0, 0, 1, 0)])
def test_k_steps_in_turn_where_rows_fall_on_few_channels(say, K, gateup, down, mid, one):
    """Weight rows a multiple or a divisor of 4 KB apart, whichever; gate/up of divisors with 32 n-tiles and more."""
    assert say("turned", 0, 8192, K) == f"{gateup}{down}{mid}00"
    assert say("turned", 0, 1408, K)[0] == str(int(K % 4096 == 0))
    assert int(say("one", 37, 1, K)) == one and int(say("one", 65, 1, K)) == 0 and int(say("one", 37, 2, K)) == 0
