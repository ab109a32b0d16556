"""Host rules of the frame matrix product's launch (csrc/rf_linear_plan.h), run by a small C++ program without a GPU."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_linear_rules(tmp_path):
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("no g++")
    exe = str(tmp_path / "linear_rules")
    subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-D__HIP_PLATFORM_AMD__", "-I",
                    os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2606_06309_amd", "csrc"), "-I",
                    "/opt/rocm/include", os.path.join(ROOT, "tests", "c", "linear_rules.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]
    assert r.stdout.startswith("ok ")


def test_sizes_past_the_largest_launch_are_refused():
    """2^24 - 63 tiles and more; fabricated addresses, as nothing is launched."""
    import ctypes
    rf = pytest.importorskip("paper_2606_06309_amd.binding")
    ids = (ctypes.c_int32 * 256)(*range(256))
    x, w, y = (0x10000000000000 * i for i in (1, 2, 3))
    for M, N, n in ((1, 2 ** 31 - 1, 8), (255, 2 ** 23, 264), (1, ((1 << 24) - 64) * 128 + 1, 128), (1, 129, 2 ** 31 - 8)):
        assert rf.lib.rf_frame_linear(x, w, None, None, None, y, ctypes.cast(ids, ctypes.c_void_p), M, M, N, 8, n, 0, 0,
                                      rf.RF_F32, None, 0, None) == rf.RF_ERR_RANGE, rf.lib.rf_last_error()
        assert b"tiles" in rf.lib.rf_last_error()
