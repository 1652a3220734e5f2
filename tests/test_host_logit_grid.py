"""The border keys of sampling's grid (csrc/logit_grid.h), compiled for the host: each is the border, found in a bounded number of looks."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2306_17266_amd", "csrc")
SOURCE = '''
#include "logit_grid.h"
using namespace sushi;

struct Counting : Grid {  // gives up instead of looking on for minutes
    mutable long looks = 0;
    using Grid::Grid;
    double place(float z) const {
        if (++looks > 100000) throw 0;
        return Grid::place(z);
    }
};

// looks[i], keys[i]: of the border of interval b[i] for row maximum best[i] and temperature T[i]; looks -1: given up.
extern "C" void borders(int n, const float *best, const float *T, const int *b, int at_best, uint32_t *keys, long *looks) {
    for (int i = 0; i < n; ++i) {
        Counting grid(best[i], 1.0 / (double)T[i], at_best ? (double)best[i] : 0.0);
        grid.looks = 0;
        try {
            keys[i] = lowest_key(grid, b[i], best[i], (double)T[i] * (6.931471805599453094e-01 / BINS_PER_LOG2));
            looks[i] = grid.looks;
        } catch (int) {
            looks[i] = -1;
        }
    }
}
extern "C" uint32_t first(uint32_t guess, uint32_t lowest, uint32_t highest, uint32_t from, int *looks) {
    return first_key(guess, lowest, highest, [&](uint32_t k) { return ++*looks, k >= from; });
}
'''


@pytest.fixture(scope="module")
def grid(tmp_path_factory):
    at = tmp_path_factory.mktemp("grid")
    (at / "grid.cpp").write_text(SOURCE)
    # (no fused products: the device's place() has none either)
    subprocess.run(["g++", "-O2", "-std=c++17", "-ffp-contract=off", "-shared", "-fPIC", "-D__device__=", "-D__forceinline__=inline", "-I", CSRC,
                    str(at / "grid.cpp"), "-o", str(at / "grid.so")], check=True)
    return ctypes.CDLL(str(at / "grid.so"))


def value_of(key):
    """key_value() for an array."""
    key = np.asarray(key, dtype=np.uint32)
    return np.where(key & 0x80000000, key ^ np.uint32(0x80000000), ~key).astype(np.uint32).view(np.float32)


def key_of(z):
    u = (np.asarray(z, dtype=np.float32) + np.float32(0)).view(np.uint32)
    return np.where(u & 0x80000000, ~u, u | np.uint32(0x80000000)).astype(np.uint32)


def check(grid, best, T, b, at_best):
    """Every border is the lowest key that lies above interval b + 1; returns the looks that each took."""
    best, T, b = (np.ascontiguousarray(v, dtype=t) for v, t in ((best, np.float32), (T, np.float32), (b, np.int32)))
    n = len(best)
    keys, looks = np.zeros(n, dtype=np.uint32), np.zeros(n, dtype=np.int64)
    grid.borders(n, *(v.ctypes.data_as(ctypes.c_void_p) for v in (best, T, b)), int(at_best), *(v.ctypes.data_as(ctypes.c_void_p) for v in (keys, looks)))
    assert looks.min() >= 0, [(best[i], T[i], b[i]) for i in np.flatnonzero(looks < 0)[:5]]
    assert looks.max() <= 64
    scale = 1.0 / T.astype(np.float64) * (1.4426950408889634074 * 12.0)
    anchor = best.astype(np.float64) if at_best else np.zeros(n)
    place = lambda z: (anchor - z.astype(np.float64)) * scale
    x = np.floor(place(best)) + (b + 1.0)
    lowest, highest = np.uint32(0x00800000), key_of(best)
    inside = (keys >= lowest) & (keys <= highest)
    ok = (place(value_of(keys)) < x) | (keys == highest)
    below = (keys == lowest) | (place(value_of(keys - np.uint32(1))) >= x)
    bad = ~(inside & ok & below)
    assert not bad.any(), [(best[i], T[i], b[i], keys[i]) for i in np.flatnonzero(bad)[:5]]
    return looks


def test_borders_next_to_logit_zero(grid):
    """Maximum and temperature for which an interval's border nearly falls on logit 0: anchor - x / scale cancels to 1e-16 or 0."""
    looks = check(grid, [11.7255468, 11.7255468], [0.369084835, 3.98032665], [549, 50], True)
    assert looks.min() > 3  # (the guess is far off)
    rng = np.random.default_rng(1)
    best = np.float32(rng.uniform(0.1, 60.0, 200000))
    x = rng.integers(1, 1020, len(best))
    T = np.float32(best.astype(np.float64) * (1.4426950408889634074 * 12.0) / x)
    for step in (-1, 0, 1):
        check(grid, best, T, x - 1 + step, True)


@pytest.mark.parametrize("at_best", [True, False])
def test_borders_anywhere(grid, at_best):
    rng = np.random.default_rng(2)
    n = 200000
    best = np.float32(rng.standard_normal(n) * 10.0 ** rng.uniform(-38, 37, n))
    T = np.float32(10.0 ** rng.uniform(-44, 38, n))
    for best, T in ((best, T), (best, np.float32(np.clip(np.abs(best) * 10.0 ** rng.uniform(-3, 3, n), 1e-38, 3e38))),
                    (np.float32(rng.uniform(-40, 40, n)), np.float32(rng.uniform(0.05, 5.0, n)))):
        for b in (np.full(n, -1), np.zeros(n), rng.integers(-1, 1024, n)):
            inner = b < 1023  # (the last interval has no border: everything)
            looks = check(grid, best[inner], T[inner], b[inner], at_best)
    # ordinary rows: two looks, or three where the guess is a key off
    assert np.median(looks) <= 3


def test_first_key_against_all_keys(grid):
    for lowest, highest in ((5, 5), (5, 6), (5, 44), (0, 100), (0xFFFFFF00, 0xFFFFFFFF)):
        for start in range(lowest, highest + 2):
            for guess in {0, lowest, lowest + 1, (lowest + highest) // 2, highest, 0xFFFFFFFF} | set(range(lowest, highest + 1, 7)):
                looks = ctypes.c_int(0)
                grid.first.restype = ctypes.c_uint32
                got = grid.first(guess, lowest, highest, start, ctypes.byref(looks)) if start <= 0xFFFFFFFF else highest
                assert got == min(start, highest)
    rng = np.random.default_rng(3)
    for guess, start in rng.integers(0, 2 ** 32, (20000, 2)).tolist() + [(0, 2 ** 32 - 1), (2 ** 32 - 1, 0), (2 ** 32 - 1, 1), (0, 0)]:
        looks = ctypes.c_int(0)
        assert grid.first(guess, 0, 2 ** 32 - 1, start, ctypes.byref(looks)) == start
        assert looks.value <= 64
