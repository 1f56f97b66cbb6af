"""The grouped experts' products in every tile shape they have, at widths that are no multiple of a tile's columns and sums that
are no multiple of a slab's channels, on the GPU.  Which shape a case gets is checked by test_grouped_shape.py."""
import numpy as np
import pytest

from test_gpu_grouped_experts import Case
from test_gpu_mx4 import T  # noqa: F401

pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

M = 136                                    # two whole slabs of 64 channels and one of 8
# rows of each expert: last tiles of a few rows, a quarter, half, three quarters and all of them, one more, and none
FEW = [1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 0, 0]
SOME = [20, 33, 1, 0, 65, 17, 9, 16]
MORE = [148, 32, 33, 64, 65, 96, 97, 1]
MANY = [276, 64, 65, 128, 129, 192, 193, 512, 7, 0]
# format, rows and columns of a tile (of gate and up half the columns are each one's), rows of the experts, f, n
CASES = [
    ("bf16", (32, 128), FEW, 1064, 1048), ("bf16", (64, 128), SOME, 1064, 1048), ("bf16", (128, 128), MORE, 1064, 1048),
    ("bf16", (128, 256), MANY, 1032, 2088), ("bf16", (256, 256), MANY, 1864, 4136),
    ("mx4", (32, 128), FEW, 1056, 1056), ("mx4", (64, 128), SOME, 1056, 1056), ("mx4", (256, 128), MANY, 544, 1056),
    ("mx4", (256, 256), MANY, 1504, 2976),
]


@pytest.mark.parametrize("fmt,tile,sizes,f,n", CASES)
def test_every_tile_at_ragged_widths(T, fmt, tile, sizes, f, n):   # noqa: F811
    choose = np.random.default_rng(f + n).permutation(np.repeat(np.arange(len(sizes), dtype=np.int32), sizes))[:, None]
    Case(T, fmt, choose.shape[0], 1, len(sizes), M, f, n, choose=choose).check()
