"""How attention over the 8-bit cache shapes its launches (byte_attn_shape in csrc/launch_rules.h), compiled by the host compiler
alone: against measured times of the shapes it chooses from, and within what the launch can hold."""

import ctypes as C
import itertools
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_23431_amd", "csrc")
SOURCE = r"""
#include "launch_rules.h"
extern "C" void shape(int cols, int64_t heads, int nblk, int head_dim, int *out) {
  const ByteAttnShape s = byte_attn_shape(cols, heads, nblk, head_dim);
  out[0] = s.tiles; out[1] = s.groups; out[2] = s.splits; out[3] = s.waves;
}
extern "C" int pieces(int cols, int64_t heads) { return byte_attn_pieces(cols, heads); }
"""
# head size, heads x requests, blocks of 64 tokens; us per launch (and its merge) by (waves, splits), bf16, one row
MEASURED = [
    (128, 1, 2, {(4, 1): 6.0, (8, 1): 6.1}),
    (64, 1, 5, {(4, 1): 5.35, (8, 1): 5.09}),
    (128, 1, 16, {(4, 1): 9.44, (8, 1): 8.41, (4, 4): 7.93, (4, 6): 8.44, (8, 3): 8.56}),
    (64, 1, 63, {(4, 1): 18.26, (8, 1): 14.69, (8, 8): 7.89, (4, 16): 7.97, (4, 8): 8.22}),
    (128, 1, 256, {(4, 1): 77.75, (8, 1): 72.63, (8, 32): 12.08, (4, 32): 12.47, (8, 16): 12.64}),
    (64, 4, 16, {(4, 1): 7.96, (8, 1): 7.08, (4, 4): 7.45, (4, 6): 7.74}),
    (128, 4, 32, {(4, 1): 15.87, (8, 1): 14.37, (4, 8): 9.52, (8, 4): 9.83, (8, 6): 10.21}),
    (128, 12, 63, {(4, 1): 25.16, (8, 1): 23.43, (8, 8): 11.31, (4, 16): 12.16}),
    (128, 12, 256, {(4, 1): 79.84, (8, 1): 76.35, (8, 16): 15.85, (4, 16): 16.05, (8, 12): 16.56}),
    (128, 16, 128, {(8, 1): 40.64, (8, 8): 13.18, (8, 15): 15.41, (8, 16): 13.95}),
    (128, 16, 133, {(8, 6): 15.47, (8, 8): 15.73, (8, 9): 13.75, (8, 12): 14.34, (8, 16): 15.98}),
    (128, 16, 71, {(8, 3): 14.65, (8, 4): 14.62, (8, 5): 12.57, (8, 6): 12.74, (8, 8): 13.18, (8, 9): 11.64}),
    (128, 4, 313, {(8, 14): 15.56, (8, 19): 15.70, (8, 20): 13.59, (8, 29): 14.82, (8, 39): 14.66, (8, 40): 14.02}),
    (128, 64, 71, {(8, 2): 21.73, (8, 3): 18.49, (8, 4): 20.42}),
    (128, 16, 16, {(4, 1): 11.02, (8, 1): 10.28, (4, 4): 9.72, (8, 2): 10.13}),
    (64, 32, 63, {(4, 1): 19.78, (8, 1): 15.64, (8, 8): 10.42, (8, 4): 10.43}),
    (128, 32, 128, {(4, 1): 43.77, (8, 1): 41.82, (8, 8): 17.72, (4, 16): 18.33}),
    (128, 64, 16, {(4, 1): 11.89, (8, 1): 10.62, (8, 2): 11.92, (8, 3): 11.97}),
    (128, 64, 256, {(4, 1): 87.77, (8, 1): 82.38, (8, 3): 44.86, (8, 4): 44.86}),
    (128, 128, 32, {(4, 1): 18.75, (8, 1): 17.58, (8, 2): 18.39, (4, 4): 18.68}),
    (64, 128, 256, {(4, 1): 67.32, (8, 1): 49.82, (4, 2): 44.93, (8, 2): 45.11}),
    (128, 256, 10, {(4, 1): 13.70, (8, 1): 12.68, (4, 2): 18.49}),
    (128, 256, 256, {(4, 1): 163.74, (8, 1): 157.79, (4, 2): 163.88}),
    (128, 1024, 2, {(4, 1): 21.92, (8, 1): 32.32}),
    (64, 1024, 16, {(4, 1): 26.14, (8, 1): 32.08, (4, 2): 33.52}),
    (128, 1024, 32, {(4, 1): 85.26, (8, 1): 89.20, (4, 2): 99.88}),
    (128, 1024, 63, {(4, 1): 161.46, (8, 1): 158.98, (4, 2): 177.17}),
]


@pytest.fixture(scope="module")
def shape(tmp_path_factory):
    d = tmp_path_factory.mktemp("shape")
    (d / "s.cpp").write_text(SOURCE)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, str(d / "s.cpp"),
                           "-o", str(d / "s.so")])
    lib = C.CDLL(str(d / "s.so"))

    lib.pieces.argtypes = [C.c_int, C.c_int64]

    def call(cols, heads, nblk, head_dim):
        out = (C.c_int * 4)()
        lib.shape(cols, C.c_int64(heads), nblk, head_dim, out)
        return tuple(out)
    call.pieces = lib.pieces
    return call


@pytest.mark.parametrize("hd,heads,nblk,us", MEASURED, ids=lambda x: str(x) if isinstance(x, int) else "")
def test_near_the_best_measured_shape(shape, hd, heads, nblk, us):
    tiles, groups, splits, waves = shape(1, heads, nblk, hd)
    assert (tiles, groups) == (1, 1)
    assert us[waves, splits] <= 1.1 * min(us.values())


def test_shapes_hold_what_there_is(shape):
    for cols, heads, nblk, hd in itertools.product((0, 1, 16, 17, 32, 33, 4096), (1, 3, 16, 255, 256, 257, 1 << 20),
                                                   (1, 4, 7, 8, 9, 100, 1 << 14, 1 << 24), (32, 64, 96, 128)):
        tiles, groups, splits, waves = shape(cols, heads, nblk, hd)
        assert groups * 16 * tiles >= cols > (groups - 1) * 16 * tiles or cols == groups == 0
        assert waves in (4, 8) and tiles == (1 if cols <= 16 else 2)
        assert splits == 1 or (splits * heads * groups <= 256 and (splits - 1) * 8 < nblk and waves == 8)


# columns, heads x requests, us of half queries with 32 columns to a wave and with work-groups of 128
PIECES = [(2048, 16, 212.07, 159.67), (1024, 16, 86.25, 101.91), (512, 16, 47.88, 100.09), (2048, 16, 121.11, 88.39),
          (512, 64, 51.32, 41.54), (2048, 24, 145.57, 148.43), (256, 16, 53.05, 192.41), (128, 16, 33.42, 191.33)]


@pytest.mark.parametrize("cols,heads,small,large", PIECES)
def test_pieces_go_where_they_are_faster(shape, cols, heads, small, large):
    assert bool(shape.pieces(cols, heads)) == (large < small)


def test_pieces_need_no_workspace(shape):
    for cols, heads in itertools.product((97, 128, 200, 1000, 5000, 1 << 20), (1, 7, 28, 56, 224, 1000, 1 << 16)):
        if shape.pieces(cols, heads):
            assert shape(cols, heads, 1 << 20, 128)[2] == 1
    assert not shape.pieces(96, 1 << 20) and not shape.pieces(0, 256) and shape.pieces(97, 224) and not shape.pieces(97, 223)
