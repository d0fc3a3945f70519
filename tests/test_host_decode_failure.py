"""Decode steps and calls of the decoder stack that fail leave the plan as it was (CPU only).

tests/host/decode_step_check.cpp and model_step_check.cpp are linked to the built library and bring a device runtime of
their own, on host memory, whose calls fail one after another; so do the host's allocations."""
import os
import shutil
import subprocess

import pytest

from paper_2511_02749_amd import _lib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("name", ["decode_step_check", "model_step_check"])
def test_a_step_that_fails_appends_nothing(tmp_path, name):
    lib, source = _lib.library_path(), os.path.join(ROOT, "tests", "host", name + ".cpp")
    if shutil.which("g++") is None or not os.path.exists(lib) or not os.path.exists(source):
        pytest.skip("needs g++, the built library and the host checks")
    exe = os.path.join(str(tmp_path), name)
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-Wall", "-Wextra", "-rdynamic", "-I", os.path.join(ROOT, "include"),
                        source, lib, f"-Wl,-rpath,{os.path.dirname(lib)}", "-Wl,--allow-shlib-undefined", "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    print(r.stdout, end="")
    assert r.returncode == 0 and "all checks passed" in r.stdout, r.stdout + r.stderr[-4000:]
