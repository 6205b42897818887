"""How the windowed attention cuts packed clouds into tiles (csrc/sp_attn_cut.h), checked on the CPU with the header that the kernels
themselves use: starts that ascend give every row one tile, and starts that do not lead to no row outside of the arrays."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2012_13846_amd", "csrc")
HARNESS = r"""
#include <functional>
#include <vector>

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
// The sums of the first keys that the keys' tiles write, 1: outside of their places, 2: two clouds at one place (starts that ascend)
extern "C" int sums(const int32_t* starts, int clouds, int n, int tile, int kv_heads, int sinks, int dim, int least, int ascending) {
    const LongClouds lc{starts, starts, n, n, clouds, 1, 128, least};
    const int64_t count = tile_numbers(n, clouds, 1, tile), end = sums_at(kv_heads, sinks, dim, lc.places(), 0, 0);
    std::vector<int> owner(lc.places(), -1);
    for (int64_t t = 0; t < count; ++t) {
        const int c = cloud_of(starts, clouds, n, t, 1, tile);
        const int64_t row = (t - first_tile(starts, clouds, n, c, 1, tile)) * tile;
        const int rows = cloud_rows(starts, clouds, n, c);
        if (!in_cloud(row, rows) || !lc.has(c)) continue;
        if (lc.place(c) < 0 || lc.place(c) >= lc.places()) return 1;
        if (ascending && owner[lc.place(c)] >= 0 && owner[lc.place(c)] != c) return 2;
        owner[lc.place(c)] = c;
        for (int64_t j = row; j < row + tile && j < rows; ++j)
            for (int kh = 0; j < sinks && kh < kv_heads; ++kh) {
                const int64_t at = sums_at(kv_heads, sinks, dim, lc.place(c), kh, (int)j);
                if (at < 0 || at + 2 * dim > end) return 1;
            }
    }
    return 0;
}
static int find(int clouds, int64_t t, const std::function<int64_t(int)>& first) {
    return last_cloud(clouds, [&](int lo, int step, int hi) {
        int k = 0;
        for (int lane = 0; lane < 64; ++lane) {
            const int at = lo + (lane + 1) * step;
            k += at <= hi && first(at) <= t;
        }
        return k;
    });
}
// Chunks that are written and joined.  1: a row outside of the array; 2: a chunk that is joined lies outside of their memory; starts that
// ascend: 3: a long cloud's row without a chunk, or one of several; 4: a place finds another cloud than its own; 5: a chunk is joined that another cloud wrote
extern "C" int chunks(const int32_t* qs, const int32_t* ks, int clouds, int n_q, int n_k, int per, int chunk, int least, int ascending) {
    const LongClouds lc{qs, ks, n_q, n_k, clouds, per, chunk, least};
    const int64_t count = lc.chunks();
    std::vector<int> seen((size_t)n_q * per), writer(count, -1);
    for (int64_t t = 0; t < count; ++t) {
        const int c = find(clouds, t, [&](int i) { return lc.first_chunk(i); });
        const int64_t row = (t - lc.first_chunk(c)) * chunk, rows = (int64_t)cloud_rows(qs, clouds, n_q, c) * per;
        if (!lc.has(c) || !in_cloud(row, rows)) continue;
        writer[t] = c;
        for (int64_t r = row; r < row + chunk && r < rows; ++r) {
            const int64_t at = (int64_t)cloud_begin(qs, clouds, n_q, c) * per + r;
            if (at < 0 || at >= (int64_t)n_q * per) return 1;
            ++seen[at];
        }
    }
    std::vector<int> joined(clouds + 2);
    for (int place = 0; place < lc.places(); ++place) {
        const int c = lc.by_number() ? place + 1 : find(clouds, place, [&](int i) { return lc.place(i); });
        if (!lc.has(c) || lc.place(c) != place) continue;
        ++joined[c];
        const int64_t rows = (int64_t)cloud_rows(qs, clouds, n_q, c) * per;
        for (int64_t u = 0; u < (rows + chunk - 1) / chunk; ++u) {
            const int64_t at = lc.first_chunk(c) + u;
            if (at < 0 || at >= count) return 2;
            if (ascending && writer[at] != c) return 5;
        }
    }
    for (int c = 1; ascending && c <= clouds; ++c) {
        if (joined[c] != lc.has(c)) return 4;
        for (int64_t r = (int64_t)cloud_begin(qs, clouds, n_q, c) * per; r < (int64_t)cloud_begin(qs, clouds, n_q, c + 1) * per; ++r)
            if (seen[r] != lc.has(c)) return 3;
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


def pointer(a):
    return a.ctypes.data_as(ctypes.c_void_p)


def test_starts_that_do_not_ascend_lead_to_no_sum_outside_of_its_memory(lib):
    for starts, n in wrong_starts():
        s = as_starts(starts)
        for tile, least in ((32, 1), (32, 650), (128, 1), (128, 1700)):
            assert lib.sums(pointer(s), len(s) - 1, n, tile, 8, 4, 128, least, 0) == 0, (list(starts), n)
            assert lib.chunks(pointer(s), pointer(s), len(s) - 1, n, n, 3, 129, least, 0) == 0, (list(starts), n)


def test_starts_of_queries_and_keys_that_do_not_belong_together_stay_inside(lib):
    rng = np.random.default_rng(12)
    for _ in range(200):
        n_q, n_k, clouds = int(rng.integers(1, 5000)), int(rng.integers(1, 5000)), int(rng.integers(1, 100))
        qs, ks = as_starts(rng.integers(-50, 2 * n_q, clouds + 1)), as_starts(rng.integers(-50, 2 * n_k, clouds + 1))
        assert lib.chunks(pointer(qs), pointer(ks), clouds, n_q, n_k, 2, 128, int(rng.integers(1, 900)), 0) == 0


@pytest.mark.parametrize("per,chunk", [(1, 128), (4, 128), (5, 130), (1, 1024)])
def test_every_long_cloud_has_a_place_and_chunks_of_its_own(lib, per, chunk):
    """Long clouds among many short and empty ones, more and fewer than there can be long ones; queries the last of a cloud's keys, or none."""
    rng = np.random.default_rng(per + chunk)
    for case in range(120):
        clouds = int(rng.choice([1, 3, 20, 300]))
        lens = np.where(rng.random(clouds) < 0.1, rng.integers(600, 3000, clouds), rng.integers(0, 30, clouds))
        if case % 3 == 0:
            lens = np.where(lens > 600, 641, lens)             # exactly the least
        asked = np.minimum(lens, rng.integers(0, 2000, clouds)) if case % 2 else lens
        gap = int(rng.integers(0, 700)) if case % 5 == 0 else 0
        ks, qs = as_starts(np.concatenate([[0], np.cumsum(lens)]) + gap), as_starts(np.concatenate([[0], np.cumsum(asked)]) + gap)
        n_k, n_q = int(ks[-1]) + gap, int(qs[-1]) + gap
        assert lib.sums(pointer(ks), clouds, n_k, 128, 2, 4, 8, 641, 1) == 0
        assert lib.chunks(pointer(qs), pointer(ks), clouds, n_q, n_k, per, chunk, 641, 1) == 0, case
