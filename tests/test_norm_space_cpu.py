"""The group norm's workspace (csrc/rf_norm_plan.h) holds what its launches put there; a small C++ program without a GPU."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_workspace_holds_sums_and_rests(tmp_path):
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("no g++")
    exe = str(tmp_path / "norm_space")
    subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-D__HIP_PLATFORM_AMD__", "-I",
                    os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2606_06309_amd", "csrc"), "-I",
                    "/opt/rocm/include", os.path.join(ROOT, "tests", "c", "norm_space.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]
    assert r.stdout.startswith("ok ")
