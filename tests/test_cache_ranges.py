"""Ranges that the paged cache's kernels take from lengths in device memory, on the CPU: the functions that the
kernels call, against integers without a limit."""
import ctypes
import subprocess

import pytest

from paper_2605_24793_amd import _build

LOW, HIGH = -(1 << 31), (1 << 31) - 1
SOURCE = """
#include "paged_ranges.h"
extern "C" void places(int64_t start, int64_t count, int64_t j, int log_page, int64_t *out) {
    const cospec::NewPlaces p = cospec::new_places(start, count, j, log_page);
    out[0] = p.base; out[1] = p.lo; out[2] = p.hi;
}
extern "C" void pieces(int kend, int part, int step, int least, int *out) {
    const cospec::Pieces p = cospec::pieces_of(kend, part, step, least);
    out[0] = p.chunk; out[1] = p.count;
}
"""


@pytest.fixture(scope="module")
def ranges(tmp_path_factory):
    folder = tmp_path_factory.mktemp("ranges")
    source, lib = folder / "ranges.cpp", folder / "ranges.so"
    source.write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-I", _build.CSRC, "-o", str(lib), str(source)],
                   check=True)
    return ctypes.CDLL(str(lib))


@pytest.mark.parametrize("log_page", [4, 5, 6, 7])
@pytest.mark.parametrize("n", [1, 2, 17, 500, HIGH // 2])
def test_new_places_of_a_page(ranges, log_page, n):
    P = 1 << log_page
    out = (ctypes.c_int64 * 3)()
    starts = [LOW, LOW + 1, LOW + P, -n - 1, -n, 1 - n, -P, -7, -1, 0, 1, P - 1, P, 5 * P + 3, HIGH - n, HIGH - 1, HIGH]
    for start in (s for s in starts if LOW <= s <= HIGH):
        for count in {0, 1, n // 2, n}:
            # the pages a call has workgroups for: from the first position's on, as many as n tokens can touch
            touched = (n + P - 2) // P + 1
            for i in {0, min(1, touched - 1), min(2, touched - 1), touched // 2, touched - 1}:
                j = max(start, 0) // P + i
                ranges.places(ctypes.c_int64(start), ctypes.c_int64(count), ctypes.c_int64(j), log_page, out)
                base, lo, hi = out
                assert base == j * P - start
                want = (max(j * P, start), min((j + 1) * P, start + count))      # positions
                if want[0] >= want[1]:
                    assert lo >= hi, (start, count, j)
                else:
                    assert (lo, hi) == (want[0] - j * P, want[1] - j * P), (start, count, j)
                    assert 0 <= lo + base and hi + base <= count


@pytest.mark.parametrize("least", [256, 512])
def test_pieces_hold_every_key(ranges, least):
    out = (ctypes.c_int * 2)()
    room = HIGH - 65536                                     # positions of a sequence, at most
    for splits in range(1, 65):
        ends = [0, 1, 63, 64, 65, least, least + 1, splits * least, splits * least + 1, 10 ** 6 + 7, 10 ** 9, 3 * 10 ** 8 * 5,
                1720000000, 2110000000, room - 127, room - 1, room]
        for kend in ends:
            ranges.pieces(kend, (kend + splits - 1) // splits, 64, least, out)
            chunk, count = out
            assert chunk % 64 == 0 and chunk >= least
            assert 1 <= count <= splits and (count - 1) * chunk < max(kend, 1) and count * chunk >= kend, (kend, splits)
            assert count * chunk <= HIGH                      # a piece's end, before it is cut to kend, fits
