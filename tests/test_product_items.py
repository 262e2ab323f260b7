"""The numbering of a products launch (csrc/product_items.h, compiled for the
host): items and scratch tiles do not overlap, the bytes cover every part, and a
phase that would need more arrival counters than there are is not split."""
import ctypes
import subprocess

import pytest

from paper_2108_00951_gb300 import build

SOURCE = r"""
#include "product_items.h"
struct Shape { uint32_t bn, tiles, batch, splits, join, item0, part0; };
struct Args {
  Shape shape[8];
  uint32_t phases, first[4], problems[4], items[4], entries, part_chunks;
};
extern "C" uint64_t number(Args* a, int pair, uint32_t counters) {
  return efs::number_items(*a, pair != 0, counters);
}
"""
u32 = ctypes.c_uint32


class Shape(ctypes.Structure):
    _fields_ = [(x, u32) for x in ("bn", "tiles", "batch", "splits", "join", "item0", "part0")]


class Args(ctypes.Structure):
    _fields_ = [("shape", Shape * 8), ("phases", u32), ("first", u32 * 4), ("problems", u32 * 4),
                ("items", u32 * 4), ("entries", u32), ("part_chunks", u32)]


@pytest.fixture(scope="module")
def number(tmp_path_factory):
    path = tmp_path_factory.mktemp("items")
    (path / "s.cpp").write_text(SOURCE)
    so = str(path / "s.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", build.CSRC,
                    str(path / "s.cpp"), "-o", so], check=True)
    fn = ctypes.CDLL(so).number
    fn.restype = ctypes.c_uint64

    def call(phases, pair, counters=65534):
        a = Args()
        a.phases = len(phases)
        at = 0
        for i, shapes in enumerate(phases):
            a.first[i], a.problems[i] = at, len(shapes)
            for s in shapes:  # bn, tiles, batch, splits, join
                a.shape[at] = Shape(*s, 99, 99)
                at += 1
        return a, fn(ctypes.byref(a), int(pair), counters)
    return call


PHASES = [
    [[(256, 10, 3, 4, 1), (128, 7, 1, 1, 1)], [(64, 5, 1, 16, 1)]],
    [[(256, 100, 100, 16, 1)]],                              # 160,000 parts
    [[(256, 1, 1, 16, 1)], [(128, 3000, 2, 8, 1), (256, 3000, 2, 8, 1)]],  # 96,000 in a phase
    [[(192, 65534, 1, 1, 1)], [(64, 4, 1, 32, 0)]],          # parts that are not joined
    [[(128, 65536, 1024, 16, 1)]],                           # 2^30: past 32 bits in pairs
]


@pytest.mark.parametrize("phases", PHASES)
@pytest.mark.parametrize("pair", [False, True])
def test_numbers_do_not_overlap(number, phases, pair):
    a, size = number(phases, pair)
    at = 0
    for i, shapes in enumerate(phases):
        items = parts = 0
        want = sum(s[1] * s[2] * s[3] * (2 if pair else 1) for s in shapes if s[3] > 1 and s[4])
        for s in shapes:
            got = a.shape[at]
            at += 1
            assert got.splits == (1 if s[4] and want > 65534 else s[3])
            assert got.item0 == items and got.part0 == parts
            items += s[1] * s[2] * got.splits
            if got.splits > 1 and s[4]:
                parts += s[1] * s[2] * got.splits * (2 if pair else 1)
                # every part's tile lies within the scratch
                assert parts * a.part_chunks * 32 * 128 * 4 <= size and got.bn <= a.part_chunks * 32
        assert a.items[i] == items and parts <= 65534
    assert a.entries == at
