"""The split of a rotation of dense rows into workgroups (csrc/rotate_plan.hpp), which is host code: compiled with the host
compiler behind a small C entry, over the sizes that nova_rotate accepts."""
import ctypes as C
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2509_21301_amd", "csrc")
SHIM = """
#include "rotate_plan.hpp"
extern "C" void split(int rows, int heads, int d, int rot, int inter, int cus, long* v) {
  const nova::RotateSplit s = nova::split_rotate(rows, heads, d, rot, inter != 0, cus);
  const long o[7] = {s.items, s.heads, s.rows, (long)s.per_item, (long)s.per_row, (long)s.row_groups, (long)s.head_groups};
  for (int i = 0; i < 7; ++i) v[i] = o[i];
}
"""


@pytest.fixture(scope="module")
def split(tmp_path_factory):
    d = tmp_path_factory.mktemp("split")
    src, so = d / "shim.cpp", d / "shim.so"
    src.write_text(SHIM)
    subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, "-o", str(so), str(src)], check=True)
    lib, v = C.CDLL(str(so)), (C.c_long * 7)()

    def call(rows, heads, d, rot, inter=0, cus=256):
        lib.split(rows, heads, d, rot, inter, cus, v)
        return list(v)
    return call


def _check(split, rows, heads, d, rot, inter, cus):
    items, h, r, per_item, per_row, row_groups, head_groups = split(rows, heads, d, rot, inter, cus)
    what = (rows, heads, d, rot, inter, cus)
    assert row_groups * 256 < 1 << 32 and head_groups < 65536, what              # the grid
    assert (row_groups - 1) * r < rows <= row_groups * r and (head_groups - 1) * h < heads <= head_groups * h, what
    assert 1 <= r <= 16 and items * h <= 4096 and r * rot * 4 <= 65536, what    # the workgroup and its LDS
    # quotients by the reciprocals are exact for every number that a workgroup forms
    last = r * items * h + 256 * 4
    for n in {0, 1, items - 1, items, items * h - 1, items * h, last - 1, last} | {random.Random(n).randrange(last) for n in range(20)}:
        for div, m in ((items, per_item), (items * h, per_row)):
            assert (n * m >> 32 if m else n) == n // div, what


def test_largest_grids(split):
    """2^25 rows of more than 512 items, one row of which fills a workgroup: two and three rows to a workgroup instead."""
    for rows in ((1 << 24) - 1, 1 << 24, (1 << 25) - 1, 1 << 25):
        for heads, d, rot in ((8192, 256, 0), (8192, 8, 0), (513, 8, 0), (600, 16, 16), (8192, 256, 256), (40, 256, 16)):
            for inter in (0, 1):
                _check(split, rows, heads, d, rot, inter, 256)
    assert split(1 << 25, 600, 16, 16)[2] == 3 and split((1 << 24) - 1, 600, 16, 16)[2] == 1


def test_every_size(split):
    r = random.Random(1)
    for _ in range(3000):
        d = 8 * r.randint(1, 32)
        _check(split, int(2 ** r.uniform(0, 25)), int(2 ** r.uniform(0, 13)), d, 16 * r.randint(0, d // 16), r.randint(0, 1), r.choice([1, 8, 170, 256]))
