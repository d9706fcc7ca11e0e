"""What infinite, saturated and extreme values make of the layers' results."""
import pytest
import torch

import layers_reference as ref
from paper_2406_08334_amd import binding as B
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


@pytest.mark.parametrize("act", ref.ACTS)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows", [3, 100])
def test_gradients_of_a_saturated_z(rows, dtype, act):
    """z beyond the type's range is kept as +-inf: there an activation is its limit, 0 or z, and its derivative 0 or 1."""
    c = case(rows, 64, 96, dtype, act=act, gate=True, grads=True)
    e, g = c["d_out"].double(), c["gate"].double()
    want = gradients(c)
    pre = c["pre"].clone()
    pre[1, 5], pre[2, 7] = -INF, INF
    got = gradients(c, pre=pre)
    assert bool(got["d_x"].isfinite().all()) and bool(got["d_weight"].isfinite().all())
    assert float(got["d_gate"][1, 5]) == (-INF * float(e[1, 5].sign()) if act == "none" else 0.0)
    assert float(got["d_gate"][2, 7]) == INF * float(e[2, 7].sign())
    for where, slope in (((1, 5), 1.0 if act == "none" else 0.0), ((2, 7), 1.0)):
        rest = [r for r in range(rows) if r != where[0]]
        bias = (e[rest, where[1]] * g[rest, where[1]] * ref.act(act, c["pre"][rest, where[1]].double())[1])
        v = bias.sum() + slope * e[where] * g[where]
        # as in ref.linear_grads: the activation's derivative, the sum, one rounding
        bound = (ref.ACT_ERR + (rows + 64) * ref.E) * (e[:, where[1]] * g[:, where[1]]).abs().sum() * 1.2 + 1.001 * ref.rounding(v, c["pre"].dtype)
        assert abs(float(got["d_bias"][where[1]]) - float(v)) <= float(bound)
    same = torch.ones(rows, 96, dtype=torch.bool, device="cuda")
    same[1, 5], same[2, 7] = False, False
    assert torch.equal(got["d_gate"][same], want["d_gate"][same])


@pytest.mark.parametrize("act", ref.ACTS)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,width,outs", [(16, 64, 32), (48, 64, 40), (200, 64, 136), (2048, 1024, 4104)])
def test_activations_of_infinite_z(rows, width, outs, dtype, act):
    """Through every kind of product and epilogue: +inf stays, -inf becomes what its product with 0 is, NaN stays NaN, other rows keep their bits."""
    dt = ref.TYPES[dtype][0]
    for gate in (None, torch.full((rows, outs), 2.0, dtype=dt, device="cuda")):
        x, w = torch.zeros(rows, width, dtype=dt, device="cuda"), torch.zeros(outs, width, dtype=dt, device="cuda")
        x[:, 0] = torch.linspace(-4.0, 4.0, rows, device="cuda")
        w[:, 0] = 1.0
        outs_ = []
        for bad in (None, INF, -INF, NAN):
            if bad is not None:
                x[rows // 3, 0] = bad
            c = dict(x=x, weight=w, act=act, gate=gate, out=torch.full((rows, outs), 7.0, dtype=dt, device="cuda"), buffers={})
            call(c)
            outs_.append(c["out"])
        for bad, out in zip((INF, -INF, NAN), outs_[1:]):
            f = out[rows // 3].float()
            if bad != bad or bad < 0 and act not in ("none", "relu"):
                assert bool(f.isnan().all()), bad
            else:
                assert bool((f == (0.0 if bad < 0 and act == "relu" else bad)).all()), bad
            out[rows // 3] = outs_[0][rows // 3]
            assert torch.equal(out, outs_[0])


def test_silu_derivative_far_below_zero():
    """(1 + z) sigmoid(z) to fp32's accuracy as far as it is a normal number: the exponential's argument counts up to 123, each unit E twice over, and the factors
    a few E; one rounding to bf16."""
    z = torch.tensor([-20.0, -31.0, -32.0, -33.0, -40.0, -48.5, -57.0, -64.0, -71.0, -80.0, -84.0], dtype=torch.bfloat16, device="cuda")
    n = z.numel()
    for rows in (1, 40):
        dt, dev = torch.bfloat16, "cuda"
        pre, d_out = z.expand(rows, n).contiguous(), torch.zeros(rows, n, dtype=dt, device=dev)
        d_out[rows - 1] = 1.0
        d_bias = torch.empty(n, dtype=dt, device=dev)
        c = dict(x=torch.zeros(rows, 8, dtype=dt, device=dev), weight=torch.zeros(n, 8, dtype=dt, device=dev), act="silu", pre=pre, d_out=d_out, d_bias=d_bias, buffers={})
        call(c, True)
        want = (1 + z.double()) * torch.sigmoid(z.double())
        ref.within("d_bias", d_bias, want, 300 * ref.E * want.abs() + 1.001 * ref.rounding(want, dt))


@pytest.mark.parametrize("bits", [16, 8])
def test_an_eps_that_fp32_has_not(bits):
    """Above 0, and so a row of zeros stays zero; its rstd is a number."""
    x = torch.randn(4, 100).bfloat16().cuda()
    x[2] = 0
    y = torch.empty(4, 100, dtype=torch.uint8 if bits == 8 else torch.bfloat16, device="cuda")
    y_scale, rstd = torch.empty(4, device="cuda") if bits == 8 else None, torch.empty(4, device="cuda")
    B.pt_rms_norm(B.rms(x, y, rstd=rstd, y_scale=y_scale, eps=1e-60))
    torch.cuda.synchronize()
    v = y.float() if bits == 16 else y.view(torch.float8_e4m3fn).float() * y_scale[:, None]
    assert bool(rstd.isfinite().all()) and bool((v[2] == 0).all()) and bool(v.isfinite().all())
    _, want_r, want, err = ref.rms(x[[0, 1, 3]], None, None, 0.0)
    ref.within("rstd", rstd[[0, 1, 3]], want_r, err * want_r)
