"""As test_build_m0, for the attention over a cache in pages: its kernel of few query
rows also loads single words (the exponents of a block) to LDS."""
import glob
import os
import shutil
import subprocess

import pytest

import paper_2606_00724_amd as wf
from test_build_m0 import OBJDUMP, foreign_uses

WORD = "global_load_lds_dword "


def foreign_uses_of_tree(lines):
    return foreign_uses([s.replace(WORD, "global_load_lds_dwordx4 ") for s in lines])


def test_the_check_finds_other_uses():
    load = ["s_mov_b32 m0, s3 // 00", "s_nop 0", "\t" + WORD + "v[0:1], off"]
    assert foreign_uses_of_tree(load) == []
    for other in (["s_mov_b32 s4, m0"], ["s_mov_b32 m0, s3", "s_nop 0", "ds_read_b32 v0, v1"]):
        assert len(foreign_uses_of_tree(load + other + load)) == 1


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no llvm-objdump")
@pytest.mark.parametrize("kernel,tiles,words", [("tree_attn_kernel", 50, 0),
                                                ("tree_few_kernel", 50, 10)])
def test_tree_kernels_have_no_other_use_of_m0(tmp_path, kernel, tiles, words):
    shutil.copy(wf.LIB_PATH, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True,
                   capture_output=True)
    seen = 0
    for obj in sorted(glob.glob(str(tmp_path / "lib.so.*gfx950"))):
        names = subprocess.run([OBJDUMP, "-t", obj], check=True, capture_output=True,
                               text=True).stdout
        if kernel not in names:
            continue
        asm = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", obj], check=True,
                             capture_output=True, text=True).stdout.splitlines()
        assert sum("global_load_lds_dwordx4" in s for s in asm) > tiles
        assert sum(WORD in s for s in asm) >= words
        assert foreign_uses_of_tree(asm) == []
        seen += 1
    assert seen == 1
