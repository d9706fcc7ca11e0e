"""Rows that lie more than 2^32 elements behind the first: the bits of the same call on rows next to each other."""
import pytest
import torch

from paper_2406_08334_amd import binding as B

pytestmark = pytest.mark.gpu
ROWS, STRIDE = 66000, 1 << 16                               # 2^32 elements end at row 65536


def far(x):
    view = torch.zeros(ROWS, STRIDE, dtype=x.dtype, device="cuda")[:, :x.shape[1]]
    view.copy_(x)
    return view


def work(size):
    return torch.empty(max(1, size), dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("width,outs", [(128, 64), (77, 300)])
def test_products(width, outs):
    gen = torch.Generator(device="cuda").manual_seed(outs)
    r = lambda *shape: torch.randn(shape, generator=gen, device="cuda").bfloat16()  # noqa: E731
    x, w, res, pre, d_out = r(ROWS, width), r(outs, width), r(ROWS, outs), r(ROWS, outs), r(ROWS, outs)
    results = []
    for place in (lambda t: t.clone(), far):
        out, z = place(res), place(torch.zeros_like(pre))
        a, b, c = place(x), place(pre), place(d_out)
        layer = B.linear(a, w, out, residual=out, pre=z, act="gelu", drop=0.1, seed=3)
        B.pt_linear_out(layer, work(B.pt_linear_workspace(layer)[0]))
        d_x, d_weight, d_bias = place(torch.zeros_like(x)), torch.empty_like(w), torch.empty_like(w[:, 0])
        grads = B.linear(a, w, pre=b, act="gelu", drop=0.1, seed=3, d_out=c, d_x=d_x, d_weight=d_weight, d_bias=d_bias)
        B.pt_linear_grads(grads, work(B.pt_linear_workspace(grads)[1]))
        torch.cuda.synchronize()
        results.append([t.clone() for t in (out, z, d_x, d_weight, d_bias)])
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert bool(results[0][0][-1].any()) and bool(results[0][2][-1].any())


@pytest.mark.parametrize("width", [128, 2056])
def test_norms_and_rows(width):
    gen = torch.Generator(device="cuda").manual_seed(width)
    x, d_y = (torch.randn(ROWS, width, generator=gen, device="cuda").bfloat16() for _ in range(2))
    results = []
    for place in (lambda t: t.clone(), far):
        a, d = place(x), place(d_y)
        y, rstd = place(torch.zeros_like(x)), torch.empty(ROWS, device="cuda")
        B.pt_rms_norm(B.rms(a, y, rstd=rstd))
        y8, s8, codes, scale = (place(torch.zeros(ROWS, width, dtype=torch.uint8, device="cuda")), torch.empty(ROWS, device="cuda"),
                                place(torch.zeros(ROWS, width, dtype=torch.uint8, device="cuda")), torch.empty(ROWS, device="cuda"))
        B.pt_rms_norm(B.rms(a, y8, y_scale=s8))
        B.pt_rows8(B.rows8(a, codes, scale))
        d_gain = torch.empty_like(x[0])
        d_x = place(torch.zeros_like(x))
        grads = B.rms(a, rstd=rstd, d_y=d, d_sum=d, d_x=d_x, d_gain=d_gain)
        B.pt_rms_grads(grads, work(B.pt_rms_workspace(grads)))
        torch.cuda.synchronize()
        results.append([t.clone() for t in (y, rstd, y8, s8, codes, scale, d_x, d_gain)])
        del a, d, y, y8, codes, d_x
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert bool(results[0][0][-1].any()) and bool(results[0][4][-1].any()) and bool(results[0][6][-1].any())
