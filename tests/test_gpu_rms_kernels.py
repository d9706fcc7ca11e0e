"""The norm's kernels that take a workgroup's rows one after the other, at the sizes of layers_sizes.py (test_layer_launches.py: that they take them)."""
import pytest
import torch

import layers_reference as ref
import layers_sizes as sizes
from paper_2406_08334_amd import binding as B
from test_gpu_rms import arrays, grads, norm

pytestmark = pytest.mark.gpu
E = ref.E


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,width", sizes.RMS_AHEAD)
def test_8_bits_of_many_rows(rows, width, dtype):
    norm(rows, width, dtype, bits=8)
    norm(rows, width, dtype, bits=8, residual=False, gain=False, pad=3, shift=1)


@pytest.mark.parametrize("over", ["x", "residual"])
@pytest.mark.parametrize("rows,width", sizes.RMS_AHEAD)
def test_8_bits_of_many_rows_in_place(rows, width, over):
    (x, r, _, _), g = arrays(rows, width, "bf16")
    want_s, want_r, want_y, err = ref.rms(x[1], r[1], g, 1e-5)
    y, y_scale, rstd = torch.empty(rows, width, dtype=torch.uint8, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    s = (x if over == "x" else r)[1]
    B.pt_rms_norm(B.rms(x[1], y, gain=g, residual=r[1], sum=s, rstd=rstd, y_scale=y_scale))
    torch.cuda.synchronize()
    ref.within("rstd", rstd, want_r, err * want_r)
    ref.within("sum", s, want_s, ref.rounding(want_s, s.dtype) * 1.001 + E * want_s.abs())
    ref.codes_within("y", y, y_scale, want_y, err * want_y.abs())


@pytest.mark.parametrize("rows,width", sizes.RMS_AHEAD)
def test_rows_of_zero_inf_and_nan_among_many(rows, width):
    """What a row holds reaches no other one: not the next of its workgroup (512 on), nor the one after that, which has the same shared sums."""
    (x, _, _, _), g = arrays(rows, width, "bf16")
    x = x[1].contiguous()
    bad = [0, 511, 513, 1025, 2000, rows - 1]
    x[0], x[513] = 0, 0
    x[511, 3], x[1025, width - 1] = float("inf"), float("-inf")
    x[2000, 9], x[rows - 1, 0] = float("nan"), float("nan")
    y, y_scale, rstd = torch.empty(rows, width, dtype=torch.uint8, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    B.pt_rms_norm(B.rms(x, y, gain=g, rstd=rstd, y_scale=y_scale))
    torch.cuda.synchronize()
    good = torch.ones(rows, dtype=torch.bool, device="cuda")
    good[bad] = False
    _, want_r, want_y, err = ref.rms(x[good], None, g, 1e-5)
    ref.within("rstd", rstd[good], want_r, err * want_r)
    ref.codes_within("y", y[good], y_scale[good], want_y, err * want_y.abs())
    assert bool((y[[0, 513]] & 0x7F == 0).all()) and bool((y_scale[[0, 513]] == 0).all())
    assert bool(y_scale[[511, 1025, 2000, rows - 1]].isnan().all()) and bool(rstd[[2000, rows - 1]].isnan().all())


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,width", sizes.RMS_GRADS_RELOAD)
def test_gradients_of_wide_rows(rows, width, dtype):
    grads(rows, width, dtype)
    grads(rows, width, dtype, d_sum=False, pad=1, shift=1)
    grads(rows, width, dtype, only="d_gain")
    grads(rows, width, dtype, only="d_x")


@pytest.mark.parametrize("rows,width", sizes.RMS_GRADS_RELOAD)
def test_gradients_of_wide_rows_in_place(rows, width):
    (s, dy, ds, _), g = arrays(rows, width, "bf16", seed=4)
    rstd = (s[1].float().square().mean(1) + 1e-5) ** -0.5
    want = ref.rms_grads(s[1], rstd, g, dy[1], ds[1])
    d_gain = torch.empty_like(g)
    d = B.rms(s[1], gain=g, rstd=rstd, d_y=dy[1], d_sum=ds[1], d_x=ds[1], d_gain=d_gain)
    B.pt_rms_grads(d, torch.empty(B.pt_rms_workspace(d), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    ref.within("d_x", ds[1], *want["d_x"])
    ref.within("d_gain", d_gain, *want["d_gain"])
