"""How the calls that fill gradient tensors check their arguments: what that costs, and which memory may lie where.  No GPU call is
made."""
import os
import shutil
import subprocess

import pytest

from paper_2004_14020_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_calls_allocate_nothing(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("gcc not available")
    exe, libdir = str(tmp_path / "alloc_check"), os.path.dirname(binding.LIB_PATH)
    subprocess.run(["gcc", "-std=gnu99", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"),
                    os.path.join(ROOT, "tests", "host", "alloc_check.c"), "-L", libdir, "-l:libcaramel.so",
                    "-Wl,-rpath," + libdir, "-o", exe], check=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0 and "alloc_check ok" in res.stdout, res.stdout + res.stderr
