"""Every kernel of the product with its epilogue, at the sizes of layers_sizes.py (test_layer_launches.py: that they take it), against the formulas in 64 bits
(bounds: layers_reference.py; sums of products in 8 bits: layers_codes.py)."""
import functools

import pytest

import layers_codes as codes
import layers_reference as ref
import layers_sizes as sizes
from test_gpu_linear import call, case

pytestmark = pytest.mark.gpu

# whole tiles on their sums where they are: with nothing, with all that they take; through LDS: with a gate, and with all at odd addresses
EPILOGUES = {"bare": dict(), "bias": dict(bias=True), "sums": dict(bias=True, residual=True, drop=0.1), "gate": dict(gate=True),
             "odd": dict(bias=True, gate=True, residual=True, drop=0.25, shift=1)}


@pytest.fixture(autouse=True)
def masks_once(monkeypatch, kept=functools.lru_cache(maxsize=4)(ref.kept)):
    """The masks of large arrays are worked out on the host: once for all activations."""
    monkeypatch.setattr(ref, "kept", kept)


def check(c, grads=False):
    want = ref.linear_grads(c) if grads else codes.linear(c) if c.get("x_scale") is not None else ref.linear(c)
    for name, (v, b) in want.items():
        if c.get(name) is not None:
            ref.within(name, c[name], v, b)


# where sums of several workgroups are joined, two activations an epilogue
@pytest.mark.parametrize("size,epilogue,act", [(s, e, a) for i, a in enumerate(ref.ACTS) for j, e in enumerate(EPILOGUES) for s in sizes.LARGEST
                                               if s != "shared" or (i - j) % 5 < 2])
def test_largest_tiles(size, epilogue, act):
    rows, width, outs, more = sizes.LARGEST[size]
    c = case(rows, width, outs, "fp16" if ref.ACTS.index(act) % 2 else "bf16", act=act, **more, **EPILOGUES[epilogue])
    call(c)
    check(c)


@pytest.mark.parametrize("act", ref.ACTS)
@pytest.mark.parametrize("epilogue", ["bias", "sums", "gate", "odd"])
@pytest.mark.parametrize("size", sizes.LARGEST_8)
def test_8_bits_in_the_largest_tiles(size, epilogue, act):
    rows, width, outs, more = sizes.LARGEST_8[size]
    c = case(rows, width, outs, "bf16" if ref.ACTS.index(act) % 2 else "fp16", act=act, **more, **EPILOGUES[epilogue])
    call(c)
    check(c)


@pytest.mark.parametrize("more", [dict(), dict(drop=0.3), dict(gate=True), dict(shift=1, drop=0.3)])
@pytest.mark.parametrize("size", ["64 at the end", "whole"])
def test_out_is_the_residual_in_the_largest_tiles(size, more):
    rows, width, outs, at = sizes.LARGEST[size]
    c = case(rows, width, outs, act="gelu", residual=True, **at, **more)
    want = ref.linear(c)["out"]
    c["out"] = c["residual"]
    call(c)
    ref.within("out", c["out"], *want)


@pytest.mark.parametrize("variant", sizes.THIN)
@pytest.mark.parametrize("dtype,bits", [("bf16", 16), ("fp16", 16), ("bf16", 8), ("fp16", 8)])
def test_up_to_32_rows(variant, dtype, bits):
    for i, (rows, width, outs) in enumerate(sizes.THIN[variant]):
        for pad, shift in ((0, 0), (3, 1)):
            c = case(rows, width, outs, dtype, act=ref.ACTS[(i * 2 + shift + 1) % 5], bias=True, gate=True, residual=True, drop=0.2, bits=bits, pad=pad, shift=shift)
            call(c)
            check(c)


@pytest.mark.parametrize("act", ref.ACTS)
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("rows,width,outs", sizes.FEW_SHARED)
def test_33_to_64_rows_whose_k_is_shared(rows, width, outs, bits, act):
    c = case(rows, width, outs, "fp16" if rows % 2 else "bf16", act=act, bias=True, gate=True, residual=True, drop=0.2, bits=bits)
    call(c)
    check(c)
    c = case(rows, width, outs, act=act, residual=act != "relu", pad=1, shift=1)
    call(c)
    check(c)


@pytest.mark.parametrize("what", sizes.GRADS)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_gradients_in_unshared_largest_tiles(what, dtype):
    rows, width, outs = sizes.GRADS[what]
    c = case(rows, width, outs, dtype, act="silu", gate=True, drop=0.1, grads=True)
    call(c, True)
    check(c, True)
