"""What lists of tensors ask of the HIP runtime, on a stand-in for it (tests/pins/list_calls.cpp).  No GPU: the kernels don't run."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PINS = os.path.join(ROOT, "tests", "pins")
PKG = os.path.join(ROOT, "paper_2406_08334_amd")


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    from paper_2406_08334_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2406_08334_amd import build
        build.build()
    out = str(tmp_path_factory.mktemp("list_calls") / "list_calls")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-rdynamic", "-Wno-unused-result", "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I",
           os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "csrc"), os.path.join(PINS, "list_calls.cpp"), "-o", out, "-L", PKG, "-lptchunk",
           "-Wl,-rpath," + PKG, "-Wl,--allow-shlib-undefined"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-4000:]
    return out


@pytest.mark.parametrize("check", ["destroyed_from_another_device", "betas_behind_an_update_that_failed"])
def test_calls(exe, check):
    res = subprocess.run([exe, check], capture_output=True, text=True, timeout=60)
    assert res.returncode == 0 and "held" in res.stdout, (res.stdout + res.stderr)[-4000:]
