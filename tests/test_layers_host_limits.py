"""What the layers before the head refuse, and ask for, at the limits of their arguments, without a GPU."""
import ctypes as C

import pytest

from paper_2406_08334_amd import binding as B
from test_layers_host import ARG, LINEAR, NOMEM, RMS, made, refused


@pytest.mark.parametrize("eps", [float("inf"), 1e39, 3.4029e38])
def test_an_eps_beyond_fp32_is_refused(eps):
    d = made(B.pt_rms, RMS, dict(eps=eps))
    refused(ARG, lambda: B.pt_rms_workspace(d), lambda: B.pt_rms_norm(d, 0), lambda: B.pt_rms_grads(d, None, 0))


def test_an_eps_in_fp32s_range():
    for eps in (0.0, 1e-300, 1.0, 3.4028e38):
        assert B.pt_rms_workspace(made(B.pt_rms, RMS, dict(eps=eps))) > 0


def test_a_gradient_without_products_needs_no_room_for_dz():
    """With frozen weights and inputs: of the gate's nothing, of the bias's sums for groups of 16 rows or more, and both of no more than that."""
    rows, outs = 8192, 11008
    layer = dict(LINEAR, rows=rows, outs=outs, **{k: 1 << 14 for k in LINEAR if k.endswith("_stride")}, d_x=0, d_weight=0)
    gate, bias, both = (B.pt_linear_workspace(made(B.pt_linear, layer, change))[1] for change in (dict(d_bias=0), dict(d_gate=0), dict()))
    assert gate == 0 and 4 * outs <= bias <= 4 * outs * rows // 16 and both == bias
    for what in ("d_x", "d_weight"):
        assert B.pt_linear_workspace(made(B.pt_linear, layer, {what: 0x7000}))[1] >= bias + 2 * rows * outs
    L, d = B.lib(), made(B.pt_linear, layer, dict())
    assert L.pt_linear_grads(C.byref(d), 0x1000, bias - 1, None) == NOMEM
