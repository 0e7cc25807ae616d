"""Rows moved inside a cache in pages are read by all of a workgroup's waves before one
writes: in the built kernels a wave waits for its loads in front of the barrier, which by
itself waits for none.  These loads are three round trips: a thread's sources, their pages
and the rows, all of a kind at once."""
import glob
import os
import re
import shutil
import subprocess

import pytest

import paper_2606_00724_amd as wf
from test_build_m0 import OBJDUMP

KERNEL = "move_kernel"


def loads_in_flight(lines):
    """The loads that may be in flight at a barrier, going back from it to the last wait
    for all of them (or to the kernel's beginning): whichever way leads there, the wait
    is on it if there is none."""
    text = [re.sub(r"\s*//.*", "", s).strip() for s in lines]
    out = []
    for i, x in enumerate(text):
        if x.startswith("s_barrier"):
            for y in reversed(text[:i]):
                if y.startswith("s_waitcnt") and "vmcnt(0)" in y:
                    break
                # (a jump that comes between them may pass the wait by)
                if y.startswith(("global_load", "buffer_load", "flat_load", "s_cbranch",
                                 "s_branch")):
                    out.append(y)
    return out


def test_the_check_finds_a_load_in_flight():
    load, wait = "\tglobal_load_ushort v20, v[18:19], off // 00", "s_waitcnt vmcnt(0) lgkmcnt(0)"
    assert loads_in_flight([load, wait, "v_mov_b32_e32 v0, v1", "s_barrier"]) == []
    for bad in ([load, "s_barrier"], [wait, load, "s_barrier"],
                [load, "s_waitcnt vmcnt(1)", "s_waitcnt lgkmcnt(0)", "s_barrier"],
                [load, "s_cbranch_execz 3", wait, "s_cbranch_vccz 4", "s_barrier"]):
        assert loads_in_flight(bad)


def round_trips(lines):
    """The longest chain of loads in front of the barrier, each behind a wait for the one
    before it (loads return in order: a wait for all but n is for all older ones)."""
    flight, done, deepest = [], 0, 0
    for x in (re.sub(r"\s*//.*", "", s).strip() for s in lines):
        wait = re.match(r"s_waitcnt.*vmcnt\((\d+)\)", x)
        if x.startswith("global_load"):
            flight.append(done + 1)
            deepest = max(deepest, done + 1)
        elif wait:
            while len(flight) > int(wait[1]):
                done = max(done, flight.pop(0))
        elif x.startswith("s_barrier"):
            return deepest
    raise AssertionError("no barrier")


def test_the_count_of_round_trips():
    load, wait = "global_load_dword v1, v[2:3], off", "s_waitcnt vmcnt(0)"
    assert round_trips([load, load, wait, load, load, wait, "s_barrier"]) == 2
    assert round_trips([load, load, "s_waitcnt vmcnt(1)", load, "s_waitcnt vmcnt(1)", load,
                        "s_barrier"]) == 2
    assert round_trips([load, wait, load, wait, load, "s_barrier", load]) == 3


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no llvm-objdump")
def test_rows_are_read_before_any_is_written(tmp_path):
    shutil.copy(wf.LIB_PATH, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True,
                   capture_output=True)
    seen = 0
    for obj in sorted(glob.glob(str(tmp_path / "lib.so.*gfx950"))):
        names = subprocess.run([OBJDUMP, "-t", obj], check=True, capture_output=True,
                               text=True).stdout
        for name in re.findall(r"\bF \.text\b.*\s(\S*" + KERNEL + r"\S*)$", names, re.M):
            asm = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn",
                                  f"--disassemble-symbols={name}", obj], check=True,
                                 capture_output=True, text=True).stdout.splitlines()
            assert sum("global_load" in s for s in asm) >= 4
            assert sum("s_barrier" in s for s in asm) == 1
            assert loads_in_flight(asm) == [], name
            assert round_trips(asm) == 3, name
            seen += 1
    assert seen == 12
