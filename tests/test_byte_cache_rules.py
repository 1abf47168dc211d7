"""The decisions of the 8-bit cache's kernels that are host code too (csrc/launch_rules.h), compiled by the host compiler alone."""

import collections
import ctypes as C
import itertools
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_23431_amd", "csrc")
SOURCE = r"""
#include "launch_rules.h"
extern "C" int append_fits(int len, int count, int n_new, int n_block) { return byte_append_fits(len, count, n_new, n_block); }
extern "C" void one(int i, int heads, int groups, int splits, int *out) {
  const ByteGroup g = byte_attn_group(i, heads, groups, splits);
  out[0] = g.unit; out[1] = g.group; out[2] = g.split;
}
extern "C" void groups(int n, int heads, int groups, int splits, int (*out)[3]) {
  for (int i = 0; i < n; ++i) {
    const ByteGroup g = byte_attn_group(i, heads, groups, splits);
    out[i][0] = g.unit; out[i][1] = g.group; out[i][2] = g.split;
  }
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    (d / "r.cpp").write_text(SOURCE)
    # (signed overflow wraps, as it does on the device)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fwrapv", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC,
                           str(d / "r.cpp"), "-o", str(d / "r.so")])
    return C.CDLL(str(d / "r.so"))


LOW, HIGH = -(1 << 31), (1 << 31) - 1
NUMBERS = sorted({x for base in (LOW, -65536, 0, 64, 128, 256, 65536, 1 << 30, HIGH) for d in (-129, -65, -64, -63, -2, -1, 0, 1, 2, 63, 64, 65, 129)
                  for x in [base + d] if LOW <= x <= HIGH})


@pytest.mark.parametrize("n_block", [1, 4, 1 << 24])
@pytest.mark.parametrize("n_new", [1, 64, 130, 256, 1 << 30])
def test_what_append_takes(rules, n_new, n_block):
    """Against whole numbers of any size: every request that fits is taken, no other one, whatever its numbers are."""
    for length, count in itertools.product(NUMBERS, NUMBERS):
        fits = 1 <= count <= n_new and length - count >= 0 and length <= n_block * 64
        assert bool(rules.append_fits(length, count, n_new, n_block)) == fits, (length, count)


@pytest.mark.parametrize("heads", [1, 2, 4, 7, 8, 9, 12, 16, 33])
@pytest.mark.parametrize("groups", [1, 2, 3, 8, 65])
@pytest.mark.parametrize("splits", [1, 2, 5, 16])
def test_every_xcd_has_the_same_work(rules, heads, groups, splits):
    """Work-groups go to XCD (index mod 8): every part is dealt once, no XCD has more than one above another, and the work-groups
    of as many heads as are a multiple of eight share an XCD, whose cache holds their tokens."""
    n = heads * groups * splits
    out = (C.c_int * 3 * n)()
    rules.groups(n, heads, groups, splits, out)
    parts = [tuple(x) for x in out]
    assert sorted(parts) == sorted(itertools.product(range(heads), range(groups), range(splits)))
    count = collections.Counter(i % 8 for i in range(n))
    assert max(count.values()) - min(count[x] for x in range(8)) <= 1
    if groups > 1:
        xcds = collections.defaultdict(set)
        for i, (unit, _, _) in enumerate(parts):
            xcds[unit].add(i % 8)
        assert all(len(xcds[unit]) == 1 for unit in range(heads // 8 * 8))
        busy = collections.Counter(i % 8 for i, (unit, _, _) in enumerate(parts) if unit >= heads // 8 * 8)
        assert not busy or len(busy) == min(8, heads % 8 * groups * splits)


def test_large_launches_keep_their_parts(rules):
    last = (C.c_int * 3)()
    for heads, groups, splits in ((1 << 26, 31, 1), (9, (1 << 31) // 9, 1), (1, (1 << 31) - 1, 1), (1, 1, 256), (8, 1, 16)):
        rules.one(heads * groups * splits - 1, heads, groups, splits, last)
        assert tuple(last) == (heads - 1, groups - 1, splits - 1), (heads, groups, splits)
