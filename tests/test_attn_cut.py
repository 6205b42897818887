"""How the windowed attention cuts packed clouds into tiles (csrc/sp_attn_cut.h), checked on the CPU with the header that the kernels
themselves use: starts that ascend give every row one tile, and starts that do not lead to no row outside of the arrays."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2012_13846_amd", "csrc")
HARNESS = r"""
#include "sp_attn_cut.h"
using namespace sp;
// the search of a wavefront of 64 lanes
static int cloud_of(const int32_t* starts, int clouds, int n, int64_t t, int per, int tile) {
    return last_cloud(clouds, [&](int lo, int step, int hi) {
        int k = 0;
        for (int lane = 0; lane < 64; ++lane) {
            const int at = lo + (lane + 1) * step;
            k += at <= hi && first_tile(starts, clouds, n, at, per, tile) <= t;
        }
        return k;
    });
}
// Every tile of n rows: how often a tile has each row ([n * per]); 1: a row outside of the array
extern "C" int tiles(const int32_t* starts, int clouds, int n, int per, int tile, int32_t* seen) {
    const int64_t count = tile_numbers(n, clouds, per, tile);
    for (int64_t t = 0; t < count; ++t) {
        const int c = cloud_of(starts, clouds, n, t, per, tile);
        const int64_t row = (t - first_tile(starts, clouds, n, c, per, tile)) * tile, rows = (int64_t)cloud_rows(starts, clouds, n, c) * per;
        if (!in_cloud(row, rows)) continue;
        for (int64_t r = row; r < row + tile && r < rows; ++r) {
            const int64_t at = (int64_t)cloud_begin(starts, clouds, n, c) * per + r;
            if (at < 0 || at >= (int64_t)n * per) return 1;
            ++seen[at];
        }
    }
    return 0;
}
// The sums of the first keys that the keys' tiles write: 1: outside of `clouds` parts
extern "C" int sums(const int32_t* starts, int clouds, int n, int tile, int kv_heads, int sinks, int dim) {
    const int64_t count = tile_numbers(n, clouds, 1, tile), bytes = sums_at(kv_heads, sinks, dim, clouds, 0, 0);
    for (int64_t t = 0; t < count; ++t) {
        const int c = cloud_of(starts, clouds, n, t, 1, tile);
        const int64_t row = (t - first_tile(starts, clouds, n, c, 1, tile)) * tile;
        const int rows = cloud_rows(starts, clouds, n, c);
        if (!in_cloud(row, rows) || c < 1 || c > clouds) continue;
        for (int64_t j = row; j < row + tile && j < rows; ++j)
            for (int kh = 0; j < sinks && kh < kv_heads; ++kh) {
                const int64_t at = sums_at(kv_heads, sinks, dim, c - 1, kh, (int)j);
                if (at < 0 || at + 2 * dim > bytes) return 1;
            }
    }
    return 0;
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("attn_cut")
    (d / "harness.cpp").write_text(HARNESS)
    so = str(d / "harness.so")
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(d / "harness.cpp"), "-o", so])
    return ctypes.CDLL(so)


def as_starts(values):
    return np.ascontiguousarray(values, np.int32)


def tiles(lib, starts, n, per, tile):
    starts, seen = as_starts(starts), np.zeros(max(1, n * per), np.int32)
    status = lib.tiles(starts.ctypes.data_as(ctypes.c_void_p), len(starts) - 1, n, per, tile, seen.ctypes.data_as(ctypes.c_void_p))
    return status, seen[:n * per]


def ascending(rng, clouds, n):
    return np.sort(rng.integers(0, n + 1, clouds + 1))


@pytest.mark.parametrize("per,tile", [(1, 32), (1, 128), (4, 128), (5, 32), (40, 128), (3, 1023)])
def test_every_row_of_ascending_starts_has_one_tile(lib, per, tile):
    rng = np.random.default_rng(per * tile)
    for clouds in (0, 1, 2, 7, 63, 64, 65, 200, 4100):
        for n in (0, 1, 31, 500, 3000):
            status, seen = tiles(lib, ascending(rng, clouds, n), n, per, tile)
            assert status == 0 and (seen == 1).all(), (clouds, n)


WRONG = [([2000, 0, 2000], 2000), ([0, 4000, 0, 4000], 4000), ([0, 250, 100], 100), ([-50, 30, 100], 100), ([60, 20, 90], 100), ([100, 0, 0], 100),
         ([2 ** 31 - 1, -2 ** 31, 5], 100), ([9000] * 70 + [0] * 70, 9000), ([0, 9000] * 50, 9000)]


def wrong_starts():
    yield from WRONG
    rng = np.random.default_rng(11)
    for _ in range(300):
        n = int(rng.integers(1, 6000))
        yield rng.integers(-n, 2 * n, int(rng.integers(1, 150))), n


def test_starts_that_do_not_ascend_lead_to_no_row_outside_of_the_array(lib):
    for starts, n in wrong_starts():
        for per, tile in ((1, 32), (1, 128), (4, 128)):
            assert tiles(lib, starts, n, per, tile)[0] == 0, (list(starts), n)


def test_starts_that_do_not_ascend_lead_to_no_sum_outside_of_its_memory(lib):
    for starts, n in wrong_starts():
        s = as_starts(starts)
        for tile in (32, 128):
            assert lib.sums(s.ctypes.data_as(ctypes.c_void_p), len(s) - 1, n, tile, 8, 4, 128) == 0, (list(starts), n)
