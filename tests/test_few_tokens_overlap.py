"""moe_forward_few refuses a y that shares memory with an input, wherever in it: rows of x and weights are read until the last of y are written."""
import ctypes

import pytest
import torch

from paper_1701_06538_b200 import binding as B
from paper_1701_06538_b200 import build as moe_build

INVALID = 1
T, D, H, N, K = 16, 64, 96, 8, 2


@pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses")
@pytest.mark.parametrize("act,size", [("f32", 4), ("bf16", 2)])
def test_places_of_y(act, size):
    moe_build.build()
    cfg = B.make_config(T, D, H, N, K, act)
    sizes = [T * D * size, D * N * 4, N * D * H * size, N * H * size, N * H * D * size, N * D * size]  # x, Wg, W1, b1, W2, b2
    at = [(i + 1) << 30 for i in range(len(sizes))]
    of_y = T * D * size

    def call(y):
        p = [ctypes.c_void_p(a) for a in at + [y]]
        return B.lib().moe_forward_few(ctypes.byref(cfg), *p, ctypes.c_void_p(0), ctypes.c_void_p(0), ctypes.c_void_p(1 << 40), ctypes.c_void_p(0))

    for a, n in zip(at, sizes):
        for y in (a, a + 32, a + n - 32, a - 32, a - of_y + 32):
            assert call(y) == INVALID, (hex(a), y - a)
        for y in (a + n, a - of_y):  # beside it: whatever comes next on a machine without a GPU, the arguments are good
            assert call(y) != INVALID, (hex(a), y - a)
