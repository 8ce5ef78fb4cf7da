"""The calls around the path from C: the structures' layouts as the binding mirrors them
(CPU), and a C program (tests/c/operators_check.c) that calls each of them on the GPU
and compares with plain loops."""
import ctypes
import os
import subprocess
import sys

import pytest

from paper_2501_04266_amd import _lib

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, os.path.join(HERE, "c"))
import build as cbuild  # noqa: E402

CHECK = os.path.join(HERE, "c", "operators_check.c")


def test_layouts_of_the_binding(tmp_path):
    exe = str(tmp_path / "layouts")
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I",
                    os.path.join(cbuild.ROOT, "include"), os.path.join(HERE, "c", "layouts.c"), "-o", exe], check=True)
    said = subprocess.run([exe], capture_output=True, text=True, check=True).stdout.splitlines()
    header = {f[0]: tuple(int(v) for v in f[1:]) for f in (line.split() for line in said)}
    mirror = {name: (getattr(_lib, name),) for name in ("ZQ_F32", "ZQ_F16", "ZQ_BF16", "ZQ_I32", "ZQ_I64", "ZQ_INT4")}
    for name, cls in (("zq_grad", _lib._Grad), ("zq_grad_plan", _lib._GradPlan)):
        mirror[name] = (ctypes.sizeof(cls),)
        for field, _ in cls._fields_:
            d = getattr(cls, field)
            mirror[f"{name}.{field}"] = (d.offset, d.size)
    assert mirror == header


def test_consumer_is_strict_c():
    subprocess.run(["gcc", *cbuild.flags(), "-fsyntax-only", CHECK], check=True)


@pytest.mark.gpu
def test_c_program_matches_loops(tmp_path):
    if not os.path.exists(_lib.LIB_PATH):
        pytest.fail("libzq.so is not built")
    exe, lib = str(tmp_path / "operators_check"), os.path.join(cbuild.ROCM, "lib")
    subprocess.run(["gcc", *cbuild.flags(), "-o", exe, CHECK, "-L", cbuild.PKG, "-lzq", "-L", lib, "-lamdhip64",
                    "-Wl,-rpath," + cbuild.PKG, "-Wl,-rpath," + lib, "-lm"], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "operators_check ok" in r.stdout
