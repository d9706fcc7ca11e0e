"""That the sizes of tests/layers_sizes.py take the kernels they are there for, seen on a stand-in for the HIP runtime (tests/pins/layer_launches.cpp).  No GPU:
the kernels don't run."""
import os
import subprocess

import pytest

import layers_sizes as sizes

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PINS = os.path.join(ROOT, "tests", "pins")
PKG = os.path.join(ROOT, "paper_2406_08334_amd")


@pytest.fixture(scope="module")
def launched(tmp_path_factory):
    from paper_2406_08334_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2406_08334_amd import build
        build.build()
    out = str(tmp_path_factory.mktemp("layer_launches") / "layer_launches")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-rdynamic", "-Wno-unused-result", "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I",
           os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "csrc"), os.path.join(PINS, "layer_launches.cpp"), "-o", out, "-L", PKG, "-lptchunk",
           "-Wl,-rpath," + PKG, "-Wl,--allow-shlib-undefined"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-4000:]

    def ask(line):
        res = subprocess.run([out], input=line + "\n", capture_output=True, text=True, timeout=60)
        assert res.returncode == 0 and "refused" not in res.stdout, res.stdout + res.stderr
        return res.stdout.strip().split(" | ")
    return ask


def product(rows, width, outs, dtype=0, act=2, bits=16, pad=0, shift=0, has="bprga"):
    return f"linear out {rows} {width} {outs} {dtype} {act} {bits} {pad} {shift} {has}"


@pytest.mark.parametrize("act", range(5))
@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("which", ["LARGEST", "LARGEST_8"])
def test_products_in_the_largest_tiles(launched, which, dtype, act):
    for name, (rows, width, outs, more) in getattr(sizes, which).items():
        for shift in (0, 1):
            calls = launched(product(rows, width, outs, dtype, act, more.get("bits", 16), more.get("pad", 0), shift))
            mul = 16 if more.get("bits") == 8 else dtype
            at = [c for c in calls if c.startswith(f"k_linear_product<{mul}, {dtype}, {act}, {sizes.BIG}")]
            assert len(at) == 1 and "Layer" in at[0], calls
            assert any(sizes.JOIN in c for c in calls) == (name == "shared")
            left = outs % 256
            assert {"64 at the end": 0 < left <= 64, "128 at the end": 64 < left <= 128, "whole": left == 0, "shared": True}[name]


@pytest.mark.parametrize("variant", sizes.THIN)
@pytest.mark.parametrize("dtype,bits", [(0, 16), (1, 16), (0, 8), (1, 8)])
def test_products_of_few_rows(launched, variant, dtype, bits):
    for size in sizes.THIN[variant]:
        calls = launched(product(*size, dtype=dtype, bits=bits))
        assert len(calls) == 1 and calls[0].startswith(f"k_linear_thin<{16 if bits == 8 else dtype}, {dtype}, {variant}>"), calls


def test_products_of_33_to_64_rows_share_k(launched):
    parts = []
    for rows, width, outs in sizes.FEW_SHARED:
        calls = launched(product(rows, width, outs))
        assert sizes.FEW in calls[-2] and calls[-1].startswith(sizes.JOIN), calls
        parts.append(int(calls[-2].split()[-1]) // -(-outs // 128))
    assert parts == [6, 16, 8]


def test_gradients_in_unshared_largest_tiles(launched):
    for name, (rows, width, outs) in sizes.GRADS.items():
        calls = launched(f"linear grads {rows} {width} {outs} 0 4 16 0 0 bpgxwde")
        x, w = ([i for i, c in enumerate(calls) if c.startswith("k_linear_product") and f"false, {k}, Plain" in c] for k in ("true", "false"))
        for what, at in (("d_x", x), ("d_weight", w)):
            if name in (what, "both"):
                assert sizes.BIG in calls[at[0]] and calls[at[0]].endswith("grid 256"), calls
                assert at[0] + 1 == len(calls) or not calls[at[0] + 1].startswith(sizes.JOIN)


def test_norms_of_rows_one_after_the_other(launched):
    for rows, width in sizes.RMS_AHEAD:
        for dtype in (0, 1):
            calls = launched(f"rms norm {rows} {width} {dtype} 8 r")
            assert len(calls) == 1 and calls[0].endswith(", true> grid 512"), calls
    for rows, width in sizes.RMS_GRADS_RELOAD:
        calls = launched(f"rms grads {rows} {width} 0 16 rgx")
        waves, pieces = (int(x) for x in calls[0][len("k_rms_grads<"):].split(">")[0].split(", ")[1:])
        assert waves * pieces > 16 and int(calls[0].split()[-1]) < rows, calls
