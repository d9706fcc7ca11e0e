"""What the layers before the head refuse, and ask for, at the limits of their arguments, without a GPU."""
import pytest

from paper_2406_08334_amd import binding as B
from test_layers_host import ARG, RMS, made, refused


@pytest.mark.parametrize("eps", [float("inf"), 1e39, 3.4029e38])
def test_an_eps_beyond_fp32_is_refused(eps):
    d = made(B.pt_rms, RMS, dict(eps=eps))
    refused(ARG, lambda: B.pt_rms_workspace(d), lambda: B.pt_rms_norm(d, 0), lambda: B.pt_rms_grads(d, None, 0))


def test_an_eps_in_fp32s_range():
    for eps in (0.0, 1e-300, 1.0, 3.4028e38):
        assert B.pt_rms_workspace(made(B.pt_rms, RMS, dict(eps=eps))) > 0
