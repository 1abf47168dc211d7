"""The decisions of the 8-bit cache's kernels that are host code too (csrc/launch_rules.h), compiled by the host compiler alone."""

import ctypes as C
import itertools
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_23431_amd", "csrc")
SOURCE = r"""
#include "launch_rules.h"
extern "C" int append_fits(int len, int count, int n_new, int n_block) { return byte_append_fits(len, count, n_new, n_block); }
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
