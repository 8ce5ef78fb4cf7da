"""The optimizer's step, the norm and the loss from C: the program compiles as strict C
(CPU), calls each of them on the GPU and compares with plain loops."""
import os
import subprocess
import sys

import pytest

from paper_2501_04266_amd import _lib

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, os.path.join(HERE, "c"))
import build as cbuild  # noqa: E402

CHECK = os.path.join(HERE, "c", "step_check.c")


def test_consumer_is_strict_c():
    subprocess.run(["gcc", *cbuild.flags(), "-fsyntax-only", CHECK], check=True)


@pytest.mark.gpu
def test_c_program_matches_loops(tmp_path):
    if not os.path.exists(_lib.LIB_PATH):
        pytest.fail("libzq.so is not built")
    exe, lib = str(tmp_path / "step_check"), os.path.join(cbuild.ROCM, "lib")
    subprocess.run(["gcc", *cbuild.flags(), "-o", exe, CHECK, "-L", cbuild.PKG, "-lzq", "-L", lib, "-lamdhip64",
                    "-Wl,-rpath," + cbuild.PKG, "-Wl,-rpath," + lib, "-lm"], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "step_check ok" in r.stdout
