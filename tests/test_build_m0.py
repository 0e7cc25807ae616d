"""The prefix attention's tile loads set m0 and do not restore it, which holds
as long as the compiler has no use of its own for it: in the built kernels every
mention of m0 is the write in front of such a load."""
import glob
import os
import re
import shutil
import subprocess

import pytest

import paper_2606_00724_amd as wf

OBJDUMP = shutil.which("llvm-objdump") or "/opt/rocm/llvm/bin/llvm-objdump"
WRITE = re.compile(r"s_(mov_b32 m0, s\d+|add_u32 m0, s\d+, (0x[0-9a-f]+|\d+))$")


def foreign_uses(lines):
    """Instructions that name m0 and are not the write of a tile load."""
    text = [re.sub(r"\s*//.*", "", s).strip() for s in lines]
    return [x for i, x in enumerate(text) if re.search(r"\bm0\b", x)
            and not (WRITE.match(x) and text[i + 1] == "s_nop 0"
                     and text[i + 2].startswith("global_load_lds_dwordx4 "))]


def test_the_check_finds_other_uses():
    load = ["s_mov_b32 m0, s3 // 00", "s_nop 0", "global_load_lds_dwordx4 v[0:1], off offset:64"]
    assert foreign_uses(load) == []
    for other in (["s_mov_b32 s4, m0"], ["s_mov_b32 m0, -1", "s_nop 0", load[2]],
                  ["s_mov_b32 m0, s3", "v_movrels_b32_e32 v0, v1", load[2]],
                  ["s_add_u32 m0, m0, 64", "s_nop 0", load[2]]):
        assert len(foreign_uses(load + other + load)) == 1


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no llvm-objdump")
def test_prefix_kernels_have_no_other_use_of_m0(tmp_path):
    shutil.copy(wf.LIB_PATH, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True,
                   capture_output=True)
    seen = 0
    for obj in sorted(glob.glob(str(tmp_path / "lib.so.*gfx950"))):
        names = subprocess.run([OBJDUMP, "-t", obj], check=True, capture_output=True,
                               text=True).stdout
        if "prefix_attn_kernel" not in names:
            continue
        asm = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", obj], check=True,
                             capture_output=True, text=True).stdout.splitlines()
        assert sum("global_load_lds_dwordx4" in s for s in asm) > 100
        assert foreign_uses(asm) == []
        seen += 1
    assert seen == 1
