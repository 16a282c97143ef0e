"""Which units of the cache a tile of rows with windows looks up, and where shares of a list of units begin, on the host: the arithmetic that the
kernels use, compiled by itself."""
import ctypes as C
import itertools
import shutil
import subprocess

import numpy as np
import pytest

PROGRAM = """
#include "cache_span.h"
using namespace shplb;
extern "C" int span_units(int window, int n_sink, int first_row, int rows, int n, int group, int len, int room, int u1, int* out, int most) {
  const Span x = window_span(window, n_sink, first_row, rows, n, group, length_fits(len, room) ? len : 0);
  const int last = x.last(u1);
  for (int u = 0; u <= last && u < most; ++u) out[u] = x.unit(u);
  return x.count <= 0 ? -last - 1 : last + 1;
}
extern "C" int add_units(int x, int y, int most) { return UnitSums{most}(x, y); }
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory, repo_root):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    at = tmp_path_factory.mktemp("span")
    (at / "span.cpp").write_text(PROGRAM)
    lib = at / "libspan.so"
    subprocess.run(["g++", "-std=c++17", "-O2", "-fwrapv", "-shared", "-fPIC", "-I", repo_root + "/paper_2603_10353_amd/csrc", str(at / "span.cpp"), "-o", str(lib)],
                   check=True)
    return C.CDLL(str(lib))


@pytest.fixture(scope="module")
def units(program):
    call = program.span_units

    def of(window, n_sink, first_row, rows, n, group, length, room):
        """The units that are looked up, and whether there are any to attend to."""
        held = min(-(-length // 64), room // 64) if 0 <= length <= room else 0
        out = (C.c_int * (room // 64 + 2))()
        got = call(window, n_sink, first_row, rows, n, group, length, room, max(held, 1), out, len(out))
        return list(out[:abs(got)]), got > 0
    return of


@pytest.mark.parametrize("length", [-1, -5, -2 ** 20, -2 ** 30 - 3, -2 ** 31, 385, 1000, 10 ** 9, 2 ** 31 - 1])
def test_a_length_that_cannot_be_leads_to_the_first_unit(units, length):
    room = 384
    for window, n_sink, n, group, rows in itertools.product((1, 105, 1024, 2 ** 30), (0, 1, 4, 100, 2 ** 30), (1, 8, 100), (1, 4, 7), (16, 32)):
        for first_row in range(0, n * group, rows):
            got, _ = units(window, n_sink, first_row, rows, n, group, length, room)
            assert got == [0], (window, n_sink, n, group, first_row)


def test_units_are_those_that_some_row_sees(units):
    rng = np.random.default_rng(1)
    for _ in range(3000):
        room = int(rng.choice([64, 128, 640, 1280]))
        length, n, group = int(rng.integers(0, room + 1)), int(rng.integers(1, 60)), int(rng.integers(1, 9))
        window, n_sink = (int(rng.choice([1, 2, 63, 64, 65, 300, 2 ** 30, int(rng.integers(1, room + 1))])) for _ in range(2))
        n_sink -= int(rng.integers(0, 2))
        rows = int(rng.choice([16, 32]))
        first_row = rows * int(rng.integers(0, -(-n * group // rows)))
        seen = set()
        for j in range(first_row // group, (min(first_row + rows, n * group) - 1) // group + 1):
            p = length - n + j
            t = np.arange(max(0, p + 1))
            seen |= set((t[(t > p - window) | (t < n_sink)] // 64).tolist())
        got, some = units(window, n_sink, first_row, rows, n, group, length, room)
        assert all(0 <= u < room // 64 for u in got)
        assert seen <= set(got) and (not some or (min(got), max(got)) == (min(seen), max(seen))) and some == bool(seen)


def place(begin, runs, before, add):
    """Where unit `begin` of a list lies: the first of the consecutive addends whose sum passes it, and how far into it, as the kernels look for it."""
    total = before
    for i, mine in enumerate(runs):
        total = add(total, mine)
        left = begin - (total - mine)
        if 0 <= left < mine:
            return i, left
    return None, 0


@pytest.mark.parametrize("each", [300000000, 6552 * 8200, 2 ** 30 - 1])
def test_shares_of_groups_that_overlap(program, each):
    """The units of groups that overlap may pass 32 bits: every share begins in an addend, and the list goes on for as long as the sums do."""
    most = 2 ** 30 - 1
    add = lambda x, y: program.add_units(x, y, most)
    runs = [5, 0, 17] + [each, 3] * 40
    total = 0
    for x in runs:
        total = add(total, x)
    assert total == min(sum(runs), most)
    for worker in range(513):
        begin = min(worker * (total // 512), total - 1)
        i, left = place(begin, runs, 0, add)
        assert i is not None and sum(runs[i:]) - left >= total - begin
        for first in range(1, i):              # in two steps, as runs of several addends are looked through
            before = add(0, min(sum(runs[:first]), most))
            if before <= begin:
                assert place(begin, runs[first:], before, add) == (i - first, left)
