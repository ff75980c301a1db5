"""How a launch of many new tokens over a cache of 8 bits is cut (csrc/kv8_cut.h, compiled here for the host), and that the two kernels that have to find the
same parts each for itself reach them by whole numbers alone."""
import ctypes
import os
import random
import re
import subprocess

import pytest

from test_kernel_code_cpu import _code

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = """
#include "kv8_cut.h"
using namespace lamps;
extern "C" {
uint64_t c_work(int stages, int tiles) { return cut8::work_of(stages, tiles); }
int c_size(uint64_t work, int heads, int log2_places) { return cut8::first_size(work, heads, log2_places); }
int c_least(int size, int later) { return cut8::least_cut(size, later != 0); }
int c_runs(int stages, int size, int worth) { return cut8::runs_of(stages, size, worth); }
int c_next(int size) { return cut8::next_size(size); }
int c_parts(int units, int runs, int *each) { const cut8::Parts p = cut8::parts_of(units, runs); *each = p.each; return p.count; }
int c_tiles_later(long long tiles, long long row, int window, int sinks, int tokens) { return cut8::tiles_later(tiles, cut8::most_seen(row, window, sinks, tokens)); }
int c_ranges_later(long long ranges, long long row, int window, int sinks) { return cut8::ranges_later(ranges, cut8::most_seen(row, window, sinks, 1)); }
int c_tries() { return cut8::kTries; }
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("cut")
    (d / "cut.cpp").write_text(SOURCE)
    so = str(d / "cut.so")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2410_18248_amd", "csrc"), str(d / "cut.cpp"), "-o", so])
    lib = ctypes.CDLL(so)
    lib.c_work.restype = ctypes.c_uint64
    lib.c_size.argtypes = [ctypes.c_uint64, ctypes.c_int, ctypes.c_int]
    lib.c_tiles_later.argtypes = [ctypes.c_longlong] * 2 + [ctypes.c_int] * 3
    lib.c_ranges_later.argtypes = [ctypes.c_longlong] * 2 + [ctypes.c_int] * 2
    lib.c_parts.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.POINTER(ctypes.c_int)]
    return lib


def _cut(lib, stages, tiles, heads, log2, later):
    """Parts of each request's tiles, as the kernels find them."""
    size = lib.c_size(sum(lib.c_work(s, t) for s, t in zip(stages, tiles)), heads, log2)
    least = lib.c_least(size, later)
    if not any(s > least for s in stages):
        return [1] * len(stages), size
    for tries in range(lib.c_tries() if later else 0, -1, -1):
        runs = [lib.c_runs(s, size, size if later else least) for s in stages]
        if tries == 0 or sum(t * n for t, n in zip(tiles, runs)) * heads <= 1 << log2:
            return runs, size
        size = lib.c_next(size)


def test_an_even_share_is_that_of_whole_numbers(lib):
    """To the last stage, also where the work is no number of 24 bits."""
    rng = random.Random(1)
    for _ in range(20000):
        n, heads, log2 = rng.randint(1, 256), rng.choice([1, 2, 8, 32, 40, 128]), rng.randint(0, 9)
        stages = [int(2 ** rng.uniform(0, 22)) for _ in range(min(n, 8))]
        tiles = [int(2 ** rng.uniform(0, 12)) for _ in stages]
        work = sum(a * b for a, b in zip(stages, tiles))
        assert lib.c_size(sum(lib.c_work(a, b) for a, b in zip(stages, tiles)), heads, log2) == max(8, min(1 << 26, work * heads // (1 << log2) + 1))
    assert 4 * lib.c_work(1 << 26, 1 << 30) <= 1 << 48                               # (of a lane: what the sum over a wave takes)
    assert lib.c_size(256 * lib.c_work(1 << 26, 1 << 30), 1 << 20, 9) == 1 << 26     # (nothing overflows)
    for stages, tiles in ((1, (1 << 20) + 1), (3000, 1 << 25)):                      # (more tiles than count: not cut)
        assert lib.c_size(lib.c_work(stages, tiles), 1, 9) > stages


@pytest.mark.parametrize("later", [0, 1])
def test_parts_are_fewer_than_twice_the_places(lib, later):
    """The room that there is for them, and workgroups: one for each part beyond a tile's first in addition to the tiles'."""
    rng = random.Random(2 + later)
    cuts = 0
    for _ in range(20000):
        n, heads, log2 = int(2 ** rng.uniform(0, 8)), rng.choice([1, 2, 4, 8, 16, 32, 40]), rng.choice([9, 9, 9, 5, 0])
        longest = 2 ** rng.uniform(1, 16)
        stages = [max(1, int(rng.random() ** rng.choice([1, 4]) * longest)) for _ in range(n)]
        tiles = [rng.choice([0, 1, 1, 2, int(2 ** rng.uniform(0, 6))]) for _ in range(n)]
        stages = [s if t else 0 for s, t in zip(stages, tiles)]
        runs, size = _cut(lib, stages, tiles, heads, log2, later)
        parts = sum(t * k for t, k in zip(tiles, runs) if k > 1) * heads
        beyond = sum(t * (k - 1) for t, k in zip(tiles, runs)) * heads
        assert parts < 2 << log2 and beyond <= 2 << log2
        assert all(k == 1 or s > size for s, k in zip(stages, runs))
        cuts += any(k > 1 for k in runs)
    assert cuts > 2000


def test_parts_of_a_tile_cover_it(lib):
    """A tile of earlier tokens may be shorter than the one that the parts are counted by."""
    each = ctypes.c_int()
    for units in list(range(1, 300)) + [1000, 12345, 1 << 26]:
        for runs in (1, 2, 3, 7, 64, 500, 1023):
            count = lib.c_parts(units, runs, ctypes.byref(each))
            assert 1 <= count <= runs and (count - 1) * each.value < units <= count * each.value
            assert count == 1 or each.value >= 4


def test_no_second_launch_where_a_window_leaves_nothing_to_cut(lib):
    """By what is seen, not by the table row alone; without a window by the row, as ever."""
    all_ = 1 << 30
    for row in (1024, 1040, 8192, 1 << 20):
        assert lib.c_ranges_later(8, row, all_, 0) == lib.c_ranges_later(8, row, all_, all_) == (row > 1024)
        assert lib.c_tiles_later(8, row, all_, all_, 32) == (row > 1024)
        for window, sinks in ((1, 0), (256, 4), (512, 16), (1000, 24)):
            assert not lib.c_ranges_later(8, row, window, sinks)
            assert not lib.c_tiles_later(8, row, window - 1 if window > 1 else 1, sinks, 1 if window < 2 else 2)
        assert lib.c_ranges_later(8, row, 1000, 25) == lib.c_tiles_later(8, row, 1000, 0, 26) == (row > 1024)
    assert not lib.c_ranges_later(128, 8192, all_, 0) and not lib.c_tiles_later(512, 8192, all_, 0, 32) and lib.c_tiles_later(511, 8192, all_, 0, 32)


def test_the_kernels_reach_the_cut_by_whole_numbers():
    """No sum of floats over the lanes of a wave, in the kernel of the tiles and in the one that adds their parts up."""
    code = {n: c for n, c in _code("kv8_").items() if re.search(r"kv8_(tiles|join)", n)}
    assert len(code) > 12
    for name, c in code.items():
        floats = [x for _, x in c if re.match(r"v_(add|fma|mac|fmac)_f32_dpp|v_add_f32.*row_(shr|bcast)", x)]
        assert not floats, (name, floats[:2])
