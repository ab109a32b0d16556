"""The host side of group norm, rows in 8 bits and their products (csrc/rf_abi.cpp) built with AddressSanitizer and
UndefinedBehaviorSanitizer by g++ (host code only; the kernel launchers come from the built library and are never
reached) and driven by tests/c/rows_errors.c in a process of its own. Skipped when g++ or the built library is missing."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2606_06309_amd")
SAN = ["-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-fno-omit-frame-pointer", "-g", "-O1"]


def test_refusals_are_clean(tmp_path):
    gxx, gcc = shutil.which("g++"), shutil.which("gcc")
    if not gxx or not gcc or not os.path.exists(os.path.join(PKG, "librhymeflow.so")):
        pytest.skip("no compiler or library")
    inc = ["-I", os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "csrc"), "-I", "/opt/rocm/include",
           "-D__HIP_PLATFORM_AMD__"]
    abi, main, exe = (str(tmp_path / n) for n in ("abi.o", "main.o", "rows_errors"))
    subprocess.run([gxx, "-std=c++17", *SAN, *inc, "-c", os.path.join(PKG, "csrc", "rf_abi.cpp"), "-o", abi], check=True)
    subprocess.run([gcc, "-std=c99", "-Wall", "-Wextra", "-Werror", *SAN, "-I", os.path.join(ROOT, "include"), "-c",
                    os.path.join(ROOT, "tests", "c", "rows_errors.c"), "-o", main], check=True)
    subprocess.run([gxx, *SAN, main, abi, "-L", PKG, "-lrhymeflow", f"-Wl,-rpath,{PKG}", "-L", "/opt/rocm/lib",
                    "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib", "-lm", "-o", exe], check=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=0",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120, env=env)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr, r.stderr[-4000:]
    assert r.stdout.strip().splitlines()[-1].startswith("ok "), r.stdout[-2000:]
