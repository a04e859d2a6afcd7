"""CPU checks of the block product's exact route into 16-bit outputs: its type flag and its plans."""
import ctypes

import pytest
import torch

from paper_2609_33496_amd import cham


@pytest.mark.parametrize("y_type", [-1, 3, 256 + 3, 257 - 512, 512, 512 + 1])
def test_types_that_do_not_exist_are_refused(y_type):
    L, out = cham.lib(), (ctypes.c_int32 * 3)()
    x, w = cham._BQ(4, 64, 0, 64, 64), cham._BW(4, 64, 0, 64, 64)
    assert L.cham_block_linear(ctypes.byref(x), ctypes.byref(w), ctypes.c_void_p(64), y_type, 4, None) == cham.EFORMAT
    assert L.cham_block_linear_plan(64, 64, 64, y_type, out, 3) == cham.EFORMAT


def test_the_exact_route_has_the_binary32_plans():
    sizes = [(M, N, K) for M in (1, 17, 240, 2048, 8192) for N in (64, 1152, 10240) for K in (32, 1280, 8192)]
    for s in sizes:
        for dt in (torch.float16, torch.bfloat16, torch.float32):
            assert cham.block_linear_plan(*s, dt, exact=True) == cham.block_linear_plan(*s, torch.float32)
    x, w = cham._BQ(0, 64, 0, None, None), cham._BW(4, 64, 0, 64, 64)
    assert cham.lib().cham_block_linear(ctypes.byref(x), ctypes.byref(w), None, cham._EXACT + 2, 4, None) == cham.OK
