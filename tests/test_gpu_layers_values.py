"""What infinite, saturated and extreme values make of the layers' results."""
import pytest
import torch

import layers_reference as ref
from test_gpu_linear import call, case

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
NAMES = ("d_x", "d_weight", "d_bias", "d_gate")


def gradients(c, **change):
    """What is left of c with some arrays changed."""
    c = dict(c, **change)
    for n in NAMES:
        if c.get(n) is not None:
            c[n] = torch.full_like(c[n], 7.0)
    c["buffers"] = {}
    call(c, True)
    return {n: c[n] for n in NAMES if c.get(n) is not None}


@pytest.mark.parametrize("exact", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,outs", [(1, 64), (3, 96), (20, 130), (32, 1000), (33, 96), (300, 130)])
def test_infinite_operands_of_gradients(rows, outs, dtype, exact):
    """An infinity in x makes d_weight's column +-inf, by the sign of dz, one in the weight d_x's; nothing else sees them.  exact: dz needs no rounding."""
    c = case(rows, 72, outs, dtype, act="none" if exact else "silu", gate=True, grads=True)
    if exact:
        c["gate"] = torch.where(c["gate"] < 0, -0.5, 2.0).to(c["gate"].dtype)
    want = gradients(c)
    e, g = c["d_out"].double(), c["gate"].double()
    dz = e * g * ref.act(c["act"], c["pre"].double())[1]
    there = dz.abs() > 2.0 ** -12                          # in fp16 some of the others may round to nothing
    row, k, out = rows // 2, 5, 9
    for bad in (INF, -INF):
        x, w = c["x"].clone(), c["weight"].clone()
        x[row, k] = bad
        got = gradients(c, x=x)
        col = got["d_weight"][:, k].double()
        assert bool((col == dz[row].sign() * bad)[there[row]].all())
        rest = [i for i in range(72) if i != k]
        assert torch.equal(got["d_weight"][:, rest], want["d_weight"][:, rest])
        assert all(torch.equal(got[n], want[n]) for n in ("d_x", "d_bias", "d_gate"))
        w[out, k] = bad
        got = gradients(c, weight=w)
        col = got["d_x"][:, k].double()
        assert bool((col == dz[:, out].sign() * bad)[there[:, out]].all())
        assert torch.equal(got["d_x"][:, rest], want["d_x"][:, rest])
        assert all(torch.equal(got[n], want[n]) for n in ("d_weight", "d_bias", "d_gate"))
    x[row, k], w[out, k] = NAN, NAN
    got = gradients(c, x=x, weight=w)
    assert bool(got["d_weight"][:, k].isnan().all()) and bool(got["d_x"][:, k].isnan().all())
    assert torch.equal(got["d_weight"][:, rest], want["d_weight"][:, rest]) and torch.equal(got["d_x"][:, rest], want["d_x"][:, rest])
