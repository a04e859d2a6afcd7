"""The linear layer leaves it to the range check of buffer stores to drop the rows past the last of a
ragged tile.  Its offsets are checked on the host against that check as it is documented."""
import ctypes
import os
import subprocess

import pytest

from paper_2609_33496_amd import build

SRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "native", "store_rows.hip")


@pytest.fixture(scope="module")
def faults(tmp_path_factory):
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    lib = tmp_path_factory.mktemp("store") / "store_rows.so"
    subprocess.run([build.HIPCC, *build.FLAGS, "-shared", SRC, "-o", str(lib)], check=True, stderr=subprocess.DEVNULL)
    f = ctypes.CDLL(str(lib)).store_faults
    f.restype = ctypes.c_long
    return f


@pytest.mark.parametrize("tm", [2, 4])
def test_rows_past_the_last_are_dropped_and_no_others(faults, tm):
    for rows in range(1, 32 * tm + 1):
        for N in (1, 31, 32, 640, 9119, (1 << 21) - 1):
            assert faults(tm, rows, N) == 0, (rows, N)
