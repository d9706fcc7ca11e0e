"""What products of e4m3 codes keep: as layers_codes.py says, with codes made for it, and over random ones of every size of power."""
import pytest
import torch

import layers_codes as codes
import layers_reference as ref
from paper_2406_08334_amd import binding as B

pytestmark = pytest.mark.gpu


def product(x, w, scale=1.0):
    """Sums of codes times a power of two, rounded to bf16."""
    rows, outs = x.shape[0], w.shape[0]
    x8, w8 = x.to(torch.float8_e4m3fn), w.to(torch.float8_e4m3fn)
    assert torch.equal(x8.to(x.dtype), x) and torch.equal(w8.to(w.dtype), w)
    out = torch.empty(rows, outs, dtype=torch.bfloat16, device="cuda")
    xs, ws = torch.ones(rows, device="cuda"), torch.full((outs,), scale, device="cuda")
    layer = B.linear(x8, w8, out, x_scale=xs, weight_scale=ws)
    work = torch.empty(max(1, B.pt_linear_workspace(layer)[0]), dtype=torch.uint8, device="cuda")
    B.pt_linear_out(layer, work)
    torch.cuda.synchronize()
    return out.double() / scale


SMALL = [2.0 ** e for e in range(8, -10, -1)]


@pytest.mark.parametrize("rows,outs", [(16, 64), (48, 64), (300, 256)])
@pytest.mark.parametrize("pair,small,scale,cut", [((256.0, 256.0), 1.0, 1.0, 3), ((448.0, 448.0), 1.0, 1.0, 3), ((2.0 ** -9, 256.0), 2.0 ** -6, 2.0 ** 20, -11),
                                                  ((0.0, 448.0), 2.0 ** -9, 2.0 ** 20, None)])
def test_a_small_product_beside_two_that_cancel(pair, small, scale, cut, rows, outs):
    """Among the same eight it is there down to 2^cut, and elsewhere down to what fp32 keeps, 2^-24 of the largest."""
    for at in (2, 7, 8, 20):
        x, w = torch.zeros(rows, 128, device="cuda"), torch.zeros(outs, 128, device="cuda")
        x[:, 0], x[:, 1], x[:, at] = pair[0], pair[0], small
        w[:, 0], w[:, 1], w[:len(SMALL), at] = pair[1], -pair[1], torch.tensor(SMALL, device="cuda")
        got = product(x, w, scale)[:, :len(SMALL)]
        for i, v in enumerate(SMALL):
            exact = v * small
            least = 2.0 ** cut if at < 8 and cut is not None else pair[0] * pair[1] * 2.0 ** -23
            if exact >= least:
                assert bool((got[:, i] == exact).all()), (at, v)
            elif at < 8:
                assert bool((got[:, i] == 0).all()), (at, v)


def test_cut_towards_zero():
    v = [9.0, 13.0, 15.0, 30.0, 60.0, 7.0, 0.5]
    x, w = torch.zeros(16, 64, device="cuda"), torch.zeros(16, 64, device="cuda")
    x[:, 40], x[:, 41], x[:, 47], w[:, 40], w[:, 41] = 256.0, 256.0, 1.0, 256.0, -256.0
    w[:14, 47] = torch.tensor(v + [-a for a in v], device="cuda")
    want = [8.0, 8.0, 8.0, 24.0, 56.0, 0.0, 0.0]
    assert product(x, w)[0, :14].tolist() == want + [-a for a in want]


@pytest.mark.parametrize("rows,width,outs", [(1, 8, 40), (16, 77, 300), (40, 200, 130), (300, 1000, 200), (2040, 264, 4456)])
def test_codes_of_every_power(rows, width, outs):
    """All codes but NaN's, so that among every eight there are ones that are cut, below the normal range, and zero."""
    gen = torch.Generator().manual_seed(rows)
    x, w = (torch.randint(0, 256, (n, width), generator=gen, dtype=torch.uint8) for n in (rows, outs))
    x, w = (torch.where(a & 0x7F == 0x7F, 0, a).cuda().view(torch.float8_e4m3fn).float() for a in (x, w))
    got = product(x, w)
    want = codes.sums_of_codes(x.to(torch.float8_e4m3fn), w.to(torch.float8_e4m3fn))
    big = x.double().abs() @ w.double().abs().t()
    ref.within("out", got, want, (width + 64) * ref.E * big + ref.rounding(want, torch.bfloat16) * 1.001)
