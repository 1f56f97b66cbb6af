"""The rule that gives the grouped experts' products their tiles (csrc/grouped_shape.h), compiled for the host: every tile shape
is walked by a GPU test at widths and sums that do not divide into it."""
import ctypes
import os
import shutil
import subprocess

import pytest

from test_gpu_grouped_tiles import CASES, M

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DRIVER = r"""
#include "grouped_shape.h"
extern "C" int shape_of(int mx4, long long pairs, int experts, int cols)
{
    const teal::GroupedShape s = teal::grouped_shape(mx4, pairs, experts, cols);
    return s.bm * 1000 + s.bn;
}
"""
TILES = {"bf16": {(32, 128), (64, 128), (128, 128), (128, 256), (256, 256)}, "mx4": {(32, 128), (64, 128), (256, 128), (256, 256)}}


@pytest.fixture(scope="module")
def shape_of(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    d = tmp_path_factory.mktemp("grouped_shape")
    (d / "driver.cpp").write_text(DRIVER)
    subprocess.run([gxx, "-std=c++17", "-O2", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2408_14690_amd", "csrc"),
                    str(d / "driver.cpp"), "-o", str(d / "driver.so")], check=True)
    fn = ctypes.CDLL(str(d / "driver.so")).shape_of
    fn.argtypes = [ctypes.c_int, ctypes.c_longlong, ctypes.c_int, ctypes.c_int]
    return lambda fmt, pairs, experts, cols: divmod(fn(fmt == "mx4", pairs, experts, cols), 1000)


def test_the_cases_reach_every_tile_at_ragged_widths(shape_of):
    assert {fmt: {tile for g, tile, *_ in CASES if g == fmt} for fmt in TILES} == TILES
    for fmt, tile, sizes, f, n in CASES:
        pairs, experts = sum(sizes), len(sizes)
        assert shape_of(fmt, pairs, experts, 2 * f) == tile and shape_of(fmt, pairs, experts, n) == tile, (fmt, tile)
        assert f % (tile[1] // 2) and n % tile[1] and M % 64 and f % 64


@pytest.mark.parametrize("fmt", sorted(TILES))
def test_every_size_gets_a_tile_that_there_is(shape_of, fmt):
    for pairs in (1, 7, 8, 9, 64, 1000, 4096, 70001, 1 << 20, 1 << 24):
        for experts in (1, 2, 7, 64, 1024):
            for cols in (8, 128, 136, 4096, 14336, 1 << 20, 1 << 21):
                assert shape_of(fmt, pairs, experts, cols) in TILES[fmt]
