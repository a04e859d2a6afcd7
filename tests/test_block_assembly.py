"""The tile kernels of the block product wait by counting: a step's barrier lets exactly the loads
of the step behind it stay in flight.  That holds only if the compiler leaves every load between
the barriers where the source puts it, reads LDS as LDS, and spills nothing (a spill is a memory
operation of its own).  This compiles the source to assembly and checks it, kernel by kernel."""
import os
import re
import subprocess

import pytest

from paper_2609_33496_amd import build

SRC = os.path.join(build.CSRC, "cham_block.hip")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    out = tmp_path_factory.mktemp("asm") / "block.s"
    subprocess.run([build.HIPCC, *build.FLAGS, "-S", "--cuda-device-only", SRC, "-o", str(out)], check=True,
                   stderr=subprocess.DEVNULL)
    text = out.read_text()
    found = re.findall(r"^(_ZN4cham\S*tile_kernel\S*?):(.*?)s_endpgm", text, re.S | re.M)
    assert len(found) >= 30
    return found


def _events(body):
    """The memory operations of a kernel in order: s a scale's load, d a load into LDS, B a barrier."""
    for line in map(str.strip, body.splitlines()):
        if re.match(r"buffer_load_(dword|ubyte)\s", line):
            yield "s"
        elif re.match(r"buffer_load_dwordx4\s.*\blds$", line):
            yield "d"
        elif line.startswith("s_barrier"):
            yield "B"


def test_every_step_holds_exactly_its_loads(kernels):
    for name, body in kernels:
        wm, wn, tm, tn, _ = map(int, re.search(r"TileILi(\d)ELi(\d)ELi(\d)ELi(\d)ELi(\d)E", name).groups())
        loads = (16 * tm * wm + 16 * tn * wn) // 8 // (wm * wn)
        scales = tm + (1 if 128 % (16 * tn) == 0 else tn // 2)  # of rows, and of blocks of weights
        step = sorted("s" * scales + "d" * loads)
        parts = "".join(_events(body)).split("B")
        # in front of the first barrier: the first step's loads, then the second's
        n = len(step)
        assert len(parts[0]) == 2 * n and sorted(parts[0][:n]) == step and sorted(parts[0][n:]) == step, (name, parts[0])
        # the six steps of the loop: from one landing barrier to the next, over the one between
        for i in range(1, 13, 2):
            assert sorted(parts[i] + parts[i + 1]) == step, (name, i, parts[i], parts[i + 1])
        # the waits: the loop's barriers let one step's loads stay in flight
        assert len(re.findall(r"s_waitcnt vmcnt\(%d\)\n\s*s_barrier" % n, body)) >= 6, name


def test_lds_is_read_as_lds_and_nothing_spills(kernels):
    for name, body in kernels:
        assert not re.search(r"\b(flat|global)_load|\bscratch_", body), name
