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
extern "C" int pieces(int cols, int64_t heads) { return byte_attn_pieces(cols, heads); }
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


# columns, heads x requests, us with 32 columns to a wave and with work-groups of 128; type, head size, tokens, causal or not
PIECES = [(512, 16, 35.6, 79.02, "bf16", 128, 4096, True), (1024, 16, 58.68, 79.04, "bf16", 128, 4096, True),
          (1536, 16, 74.4, 79.85, "bf16", 128, 4096, True), (1792, 16, 81.43, 80.17, "bf16", 128, 4096, True),
          (2048, 16, 129.34, 116.46, "bf16", 128, 6144, True), (1024, 48, 81.36, 89.16, "bf16", 64, 3000, True),
          (256, 64, 22.25, 30.28, "bf16", 32, 2000, True), (1280, 48, 129.3, 122.84, "bf16", 128, 3000, True),
          (100, 224, 17.69, 10.25, "bf16", 128, 64, False), (100, 224, 10.89, 6.39, "bf16", 32, 64, False),
          (100, 224, 19.24, 13.39, "bf16", 96, 100, True), (200, 512, 502.26, 420.55, "bf16", 96, 6000, True),
          (512, 64, 153.46, 120.32, "bf16", 128, 6000, False), (1536, 16, 90.67, 102.13, "f16", 128, 4096, True),
          (2048, 16, 160.19, 148.21, "f16", 128, 6144, True), (1024, 48, 96.02, 106.12, "f16", 64, 3000, True),
          (100, 224, 18.88, 12.03, "f16", 128, 64, False), (100, 224, 21.56, 18.29, "f16", 128, 256, True),
          (100, 224, 27.98, 24.08, "f16", 32, 1000, True), (512, 64, 186.4, 151.82, "f16", 128, 6000, False)]


@pytest.mark.parametrize("cols,heads,small,large", [x[:4] for x in PIECES], ids=["-".join(map(str, x[4:] + x[:2])) for x in PIECES])
def test_pieces_of_every_length_and_head_size_go_where_they_are_faster(rules, cols, heads, small, large):
    assert bool(rules.pieces(cols, C.c_int64(heads))) == (large < small)
