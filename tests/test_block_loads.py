"""The block product prefetches two steps past the last block: those loads, and the rows past the
last one, must fall outside their buffer for any size of the last tile.  Its offsets are checked on
the host against the documented range check of buffer loads."""
import ctypes
import os
import subprocess

import pytest

from paper_2609_33496_amd import build

SRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "native", "block_load.hip")


@pytest.fixture(scope="module")
def faults(tmp_path_factory):
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    lib = tmp_path_factory.mktemp("load") / "block_load.so"
    subprocess.run([build.HIPCC, *build.FLAGS, "-shared", SRC, "-o", str(lib)], check=True, stderr=subprocess.DEVNULL)
    f = ctypes.CDLL(str(lib)).block_load_faults
    f.restype = ctypes.c_long
    return f


@pytest.mark.parametrize("bm,groups", [(32, 1), (32, 2), (64, 1), (64, 2), (128, 1), (192, 1), (256, 1)])
def test_every_load_reads_its_chunk_or_zeros(faults, bm, groups):
    for rows in {1, 2, 3, 7, 8, 31, 32, 33, bm // 2, bm - 1, bm}:
        for K in (32, 64, 96, 128, 160, 256, 288, 1152, 1280, 4128):
            assert rows > bm or faults(bm, rows, K, 2 * groups + groups) == 0, (bm, rows, K)
    assert faults(bm, bm, 1 << 20, 3 * groups) == 0  # the longest rows
