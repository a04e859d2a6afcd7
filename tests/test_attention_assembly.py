"""The tiled attention kernel's 16-bit rows go from memory into LDS directly, two buffers in turn.
That is right only if every load has landed before the barrier behind which it is read and before the
workgroup gives its LDS back, and fast only if nothing waits for loads in between and nothing spills.
This compiles the source to assembly and checks it, kernel by kernel."""
import os
import re
import subprocess

import pytest

from paper_2609_33496_amd import build

SRC = os.path.join(build.CSRC, "cham_attention.hip")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    out = tmp_path_factory.mktemp("asm") / "attention.s"
    subprocess.run([build.HIPCC, *build.FLAGS, "-S", "--cuda-device-only", SRC, "-o", str(out)], check=True,
                   stderr=subprocess.DEVNULL)
    found = re.findall(r"^(_ZN4cham\S*?kernelI\S*?):(.*?)^\.Lfunc_end", out.read_text(), re.S | re.M)
    assert len([n for n, _ in found if "tile_kernel" in n]) == 24
    return found


def _direct(kernels):
    """The tiled kernels whose rows go to LDS directly (packed rows and 16-bit pages)."""
    return [(n, b) for n, b in kernels if re.search(r"tile_kernelILi\dELi\dELi\dELi[01]E", n)]


def _lines(body):
    return [x for x in (re.sub(r"\s*;.*", "", line).strip() for line in body.splitlines()) if x]


def test_loads_land_before_the_barriers_that_open_a_step(kernels):
    """The loop holds two steps, one a buffer, and each opens with a barrier behind which the other waves' loads
    are read: each of the two waits for all loads first.  A wait also follows the last load of the text."""
    for name, body in _direct(kernels):
        text = "\n".join(_lines(body))
        loads = [m.start() for m in re.finditer(r"buffer_load_dwordx4 [^\n]* lds\n", text)]
        assert loads, name
        assert len(re.findall(r"s_waitcnt vmcnt\(0\)[^\n]*\ns_barrier", text)) == 2, name
        assert text.find("s_waitcnt vmcnt(0)", loads[-1]) > 0, name


def test_products_do_not_wait_for_loads(kernels):
    """In a run of products no instruction waits for loads from memory: those under way are the next step's."""
    for name, body in _direct(kernels):
        for block in re.split(r"^\.LBB\S+:.*$", body, flags=re.M):
            if len(re.findall(r"v_mfma", block)) >= 8:
                first, last = block.index("v_mfma"), block.rindex("v_mfma")
                assert "vmcnt" not in block[first:last], name


def test_nothing_spills(kernels):
    for name, body in kernels:
        assert not re.search(r"\bscratch_", body), name
