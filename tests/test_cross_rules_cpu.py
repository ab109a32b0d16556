"""Host rules of a cross attention's launch (csrc/rf_cross_plan.h), run by a small C++ program without a GPU."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_cross_rules(tmp_path):
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("no g++")
    exe = str(tmp_path / "cross_rules")
    subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-D__HIP_PLATFORM_AMD__", "-I",
                    os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2606_06309_amd", "csrc"), "-I",
                    "/opt/rocm/include", os.path.join(ROOT, "tests", "c", "cross_rules.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]
    assert r.stdout.startswith("ok ")


def test_sizes_past_the_largest_launch_are_refused():
    """2^24 tiles of 128 fp32 queries; fabricated addresses, as nothing is launched."""
    import ctypes
    rf = pytest.importorskip("paper_2606_06309_amd.binding")
    n = ctypes.c_int64(0)
    for B, Lq, heads in ((1 << 20, 32, 16), ((1 << 24) - 63, 1, 1), (1 << 16, 1, 256)):
        args = [0x100000000000 + i * 0x10000000000 for i in range(4)]
        assert rf.lib.rf_cross_attention(*args, None, None, B, Lq, 7, heads, heads, 64, None, rf.RF_F32, None, 0,
                                         None) == rf.RF_ERR_RANGE, rf.lib.rf_last_error()
        assert rf.lib.rf_cross_attention_workspace(B, Lq, 7, heads, heads, 64, rf.RF_F32, 256,
                                                   ctypes.byref(n)) == rf.RF_ERR_RANGE
        assert rf.lib.rf_cross_attention_workspace(B, Lq, 7, heads, heads, 64, rf.RF_BF16, 256,
                                                   ctypes.byref(n)) == rf.RF_OK
    assert rf.lib.rf_cross_attention_workspace((1 << 24) - 64, 1, 7, 1, 1, 64, rf.RF_F32, 256, ctypes.byref(n)) == rf.RF_OK
