"""As test_build_m0, for the attention over a cache in pages."""
import glob
import os
import shutil
import subprocess

import pytest

import paper_2606_00724_amd as wf
from test_build_m0 import OBJDUMP, foreign_uses


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no llvm-objdump")
def test_tree_kernels_have_no_other_use_of_m0(tmp_path):
    shutil.copy(wf.LIB_PATH, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True,
                   capture_output=True)
    seen = 0
    for obj in sorted(glob.glob(str(tmp_path / "lib.so.*gfx950"))):
        names = subprocess.run([OBJDUMP, "-t", obj], check=True, capture_output=True,
                               text=True).stdout
        if "tree_attn_kernel" not in names:
            continue
        asm = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", obj], check=True,
                             capture_output=True, text=True).stdout.splitlines()
        assert sum("global_load_lds_dwordx4" in s for s in asm) > 50
        assert foreign_uses(asm) == []
        seen += 1
    assert seen == 1
