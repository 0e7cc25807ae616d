"""Without the library, or with one of an older build, importing the binding
fails with the command that builds it, which does not import the binding."""
import os
import re
import shutil
import subprocess
import sys

import pytest

PKG = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                   "paper_2606_00724_amd")


@pytest.mark.parametrize("older", [False, True], ids=["missing", "older"])
def test_import_names_the_build(tmp_path, older):
    pkg = tmp_path / "paper_2606_00724_amd"
    pkg.mkdir()
    for f in ("__init__.py", "build.py"):
        shutil.copy(os.path.join(PKG, f), pkg / f)
    if older:  # a library without any of the functions
        (tmp_path / "empty.c").write_text("int nothing;\n")
        subprocess.run(["gcc", "-shared", "-fPIC", "-o", pkg / "libwavefilter.so",
                        tmp_path / "empty.c"], check=True)
    r = subprocess.run([sys.executable, "-c", "import paper_2606_00724_amd"], cwd=tmp_path,
                       capture_output=True, text=True)
    assert r.returncode != 0 and "ImportError" in r.stderr
    command = re.search(r"`python (\S+)`", r.stderr).group(1)
    assert os.path.samefile(command, pkg / "build.py")
    assert not re.search(r"^\s*(import|from) (paper_|torch)", open(command).read(), re.M)
