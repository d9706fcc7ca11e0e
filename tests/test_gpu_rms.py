"""RMS norm with the residual's addition, its gradients, and rows in 8 bits, against the formulas in 64 bits (bounds: layers_reference.py)."""
import pytest
import torch

import layers_reference as ref
from paper_2406_08334_amd import binding as B

pytestmark = pytest.mark.gpu
E = ref.E
# widths on both sides of every change of a row's waves and pieces, rows that end inside a piece, fewer elements than a piece
WIDTHS = [1, 3, 7, 8, 9, 64, 511, 512, 513, 771, 1024, 1030, 2048, 2049, 4096, 4100, 5120, 8192, 8200, 16384, 16390, 32768]


def arrays(rows, width, dtype, pad=0, shift=0, seed=0, n=4):
    gen = torch.Generator().manual_seed(seed * 7919 + rows * 31 + width)
    dt = ref.TYPES[dtype][0]
    size = torch.exp(torch.randn(rows, 1, generator=gen))
    return [ref.place((torch.randn(rows, width, generator=gen) * size).to(dt).cuda(), pad, shift) for _ in range(n)], \
        (1 + 0.2 * torch.randn(width, generator=gen)).to(dt).cuda()


def norm(rows, width, dtype="bf16", residual=True, bits=16, gain=True, eps=1e-5, pad=0, shift=0, x=None):
    (a, b, s, y), g = arrays(rows, width, dtype, pad, shift)
    if x is not None:
        a[1].copy_(x)
    y_scale = None
    if bits == 8:
        y, y_scale = ref.place(torch.zeros(rows, width, dtype=torch.uint8, device="cuda"), pad, shift), torch.empty(rows, device="cuda")
    rstd = torch.empty(rows, device="cuda")
    d = B.rms(a[1], y[1], gain=g if gain else None, residual=b[1] if residual else None, sum=s[1] if residual else None, rstd=rstd, y_scale=y_scale, eps=eps)
    B.pt_rms_norm(d)
    torch.cuda.synchronize()
    for buf, view in (a, b, s, y):
        assert ref.untouched(buf, view)
    want_s, want_r, want_y, err = ref.rms(a[1], b[1] if residual else None, g if gain else None, eps)
    ref.within("rstd", rstd, want_r, err * want_r)
    if residual:
        ref.within("sum", s[1], want_s, ref.rounding(want_s, a[1].dtype) * 1.001 + E * want_s.abs())
    if bits == 8:
        ref.codes_within("y", y[1], y_scale, want_y, err * want_y.abs())
    else:
        ref.within("y", y[1], want_y, err * want_y.abs() + ref.rounding(want_y, a[1].dtype) * 1.001)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("width", WIDTHS)
def test_norm_against_64_bits(width, bits):
    norm(5, width, "bf16" if width % 2 else "fp16", residual=width % 3 != 0, bits=bits, gain=width % 5 != 0)
    norm(1, width, "fp16" if width % 2 else "bf16", bits=bits)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("width,pad,shift", [(64, 1, 0), (77, 0, 1), (520, 3, 7), (1600, 8, 0), (4096, 0, 1), (771, 5, 3)])
def test_norm_at_any_address_and_stride(width, pad, shift, bits):
    norm(37, width, bits=bits, pad=pad, shift=shift)


def grads(rows, width, dtype="bf16", d_sum=True, gain=True, pad=0, shift=0, only=None):
    (s, dy, ds, dx), g = arrays(rows, width, dtype, pad, shift, seed=1)
    rstd = (s[1].float().square().mean(1) + 1e-5) ** -0.5
    d_gain = torch.empty_like(g)
    d = B.rms(s[1], gain=g if gain else None, rstd=rstd, d_y=dy[1], d_sum=ds[1] if d_sum else None, d_x=dx[1] if only != "d_gain" else None,
              d_gain=d_gain if only != "d_x" else None)
    size = B.pt_rms_workspace(d)
    work = torch.full((size + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    work[:size] = 0xFF
    B.pt_rms_grads(d, work[:size])
    torch.cuda.synchronize()
    assert bool((work[size:] == 0x5A).all())
    for buf, view in (s, dy, ds, dx):
        assert ref.untouched(buf, view)
    want = ref.rms_grads(s[1], rstd, g if gain else None, dy[1], ds[1] if d_sum else None)
    if only != "d_gain":
        ref.within("d_x", dx[1], *want["d_x"])
    if only != "d_x":
        ref.within("d_gain", d_gain, *want["d_gain"])


@pytest.mark.parametrize("width", WIDTHS)
def test_grads_against_64_bits(width):
    grads(5, width, "bf16" if width % 2 else "fp16", d_sum=width % 3 != 0, gain=width % 5 != 0)
    grads(1, width)


@pytest.mark.parametrize("rows,width,pad,shift", [(2500, 64, 0, 0), (2049, 771, 0, 1), (3000, 600, 2, 0), (1100, 1600, 0, 0), (513, 4096, 8, 8), (700, 5121, 0, 0)])
def test_grads_of_more_rows_than_are_taken_at_a_time(rows, width, pad, shift):
    grads(rows, width, pad=pad, shift=shift)


@pytest.mark.parametrize("only", ["d_x", "d_gain"])
def test_one_gradient_alone(only):
    grads(300, 520, only=only)


def test_gradients_against_differences():
    R, K, h = 3, 12, 1e-6
    gen = torch.Generator().manual_seed(5)
    x = torch.randn(R, K, generator=gen).half().cuda()
    g = (1 + 0.2 * torch.randn(K, generator=gen)).half().cuda()
    dy = torch.randn(R, K, generator=gen).half().cuda()
    rstd = (x.double().square().mean(1) + 1e-5).pow(-0.5).float()
    dx, dg = torch.empty_like(x), torch.empty_like(g)
    d = B.rms(x, gain=g, rstd=rstd, d_y=dy, d_x=dx, d_gain=dg)
    B.pt_rms_grads(d, torch.empty(B.pt_rms_workspace(d), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()

    def total(a, b):
        return float((ref.rms(a, None, b, 1e-5)[2] * dy.double()).sum())
    for i, got in ((0, dx), (1, dg)):
        args = [x.double(), g.double()]
        for at in range(args[i].numel()):
            two = []
            for s in (h, -h):
                a = [t.clone() for t in args]
                a[i].view(-1)[at] += s
                two.append(total(*a))
            want = (two[0] - two[1]) / (2 * h)
            assert abs(float(got.flatten()[at]) - want) < 2.0 ** -11 * abs(want) + 1e-4        # differences: 1e-15 / h and h^2; fp32 sums


def test_in_place():
    """The sum over the residual, its gradient over the one that reaches it."""
    (x, r, _, y), g = arrays(40, 600, "bf16")
    want_s, _, want_y, err = ref.rms(x[1], r[1], g, 1e-5)
    rstd = torch.empty(40, device="cuda")
    B.pt_rms_norm(B.rms(x[1], y[1], gain=g, residual=r[1], sum=r[1], rstd=rstd))
    torch.cuda.synchronize()
    ref.within("sum", r[1], want_s, ref.rounding(want_s, torch.bfloat16) * 1.001)
    ref.within("y", y[1], want_y, err * want_y.abs() + ref.rounding(want_y, torch.bfloat16) * 1.001)
    (dy, ds, _, _), _ = arrays(40, 600, "bf16", seed=2)
    want = ref.rms_grads(r[1], rstd, g, dy[1], ds[1])["d_x"]
    B.pt_rms_grads(B.rms(r[1], gain=g, rstd=rstd, d_y=dy[1], d_sum=ds[1], d_x=ds[1]))
    torch.cuda.synchronize()
    ref.within("d_x", ds[1], *want)


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("width", WIDTHS)
def test_rows8(width, kind):
    gen = torch.Generator().manual_seed(width)
    for rows, pad, shift in ((6, 0, 0), (3, 3, 1)):
        x = torch.randn(rows, width, generator=gen) * torch.logspace(-3, 3, rows)[:, None]
        x = ref.place(x.to(kind).cuda(), pad, shift)
        codes, scale = ref.place(torch.zeros(rows, width, dtype=torch.uint8, device="cuda"), pad, shift), torch.empty(rows, device="cuda")
        B.pt_rows8(B.rows8(x[1], codes[1], scale))
        torch.cuda.synchronize()
        assert ref.untouched(*codes) and ref.untouched(*x)
        ref.codes_within("codes", codes[1], scale, x[1].double(), torch.zeros_like(x[1].double()))


def test_rows8_of_nothing_and_of_what_is_no_number():
    x = torch.randn(7, 100).cuda()
    x[1] = 0
    x[2, 5], x[3, 99], x[4, 0] = float("inf"), float("nan"), float("-inf")
    x[5] *= 2.0 ** -110
    x[6] *= 2.0 ** 120
    codes, scale = torch.empty(7, 100, dtype=torch.uint8, device="cuda"), torch.empty(7, device="cuda")
    B.pt_rows8(B.rows8(x, codes, scale))
    torch.cuda.synchronize()
    v = codes.view(torch.float8_e4m3fn).float()
    assert bool((codes[[1, 5]] & 0x7F == 0).all()) and scale[1] == 0 and scale[5] == 0
    assert bool(scale[2:5].isnan().all()) and bool(v[2:5].isnan().all())
    ref.codes_within("codes", codes[[0, 6]], scale[[0, 6]], x[[0, 6]].double(), torch.zeros(2, 100, dtype=torch.float64, device="cuda"))


@pytest.mark.parametrize("bits", [16, 8])
def test_rows_of_zero_inf_and_nan(bits):
    """What a row holds reaches no other one; a row of zeros stays zero."""
    x = torch.randn(6, 300).bfloat16().cuda()
    x[1] = 0
    x[2, 7], x[4, 299] = float("inf"), float("nan")
    y = torch.empty(6, 300, dtype=torch.uint8 if bits == 8 else torch.bfloat16, device="cuda")
    y_scale = torch.empty(6, device="cuda") if bits == 8 else None
    B.pt_rms_norm(B.rms(x, y, y_scale=y_scale))
    torch.cuda.synchronize()
    v = y.float() if bits == 16 else y.view(torch.float8_e4m3fn).float() * y_scale[:, None]
    _, _, want, err = ref.rms(x, None, None, 1e-5)
    good = [0, 3, 5]
    if bits == 16:
        ref.within("y", y[good], want[good], err * want[good].abs() + ref.rounding(want[good], torch.bfloat16) * 1.001)
    else:
        ref.codes_within("y", y[good], y_scale[good], want[good], err * want[good].abs())
    assert bool((v[1] == 0).all()) and bool(v[4].isnan().all()) and bool(v[2, 7].isnan())


def test_captured():
    (x, r, s, y), g = arrays(300, 1024, "fp16")
    (dy, ds, dx, _), _ = arrays(300, 1024, "fp16", seed=3)
    rstd, dg = torch.empty(300, device="cuda"), torch.empty_like(g)
    fwd = B.rms(x[1], y[1], gain=g, residual=r[1], sum=s[1], rstd=rstd)
    bwd = B.rms(s[1], gain=g, rstd=rstd, d_y=dy[1], d_sum=ds[1], d_x=dx[1], d_gain=dg)
    work = torch.empty(B.pt_rms_workspace(bwd), dtype=torch.uint8, device="cuda")
    B.pt_rms_norm(fwd), B.pt_rms_grads(bwd, work)
    torch.cuda.synchronize()
    first = [t.clone() for t in (y[1], s[1], rstd, dx[1], dg)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.pt_rms_norm(fwd), B.pt_rms_grads(bwd, work)
    for _ in range(3):
        for t in (y[1], s[1], rstd, dx[1], dg):
            t.zero_()
        work.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, (y[1], s[1], rstd, dx[1], dg)))


def test_no_rows():
    x, g = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"), torch.ones(64, dtype=torch.bfloat16, device="cuda")
    dg = torch.full_like(g, 5.0)
    B.pt_rms_norm(B.rms(x, x.clone(), gain=g))
    d = B.rms(x, gain=g, rstd=torch.empty(0, device="cuda"), d_y=x.clone(), d_x=x.clone(), d_gain=dg)
    B.pt_rms_grads(d, torch.empty(max(1, B.pt_rms_workspace(d)), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    assert not bool(dg.any())


def test_more_rows_than_a_launch_takes():
    """The rows behind the first 2^21, in their places."""
    rows, width = (1 << 21) + 77, 9
    x = torch.randn(rows, width, device="cuda").bfloat16()
    y, rstd = torch.empty_like(x), torch.empty(rows, device="cuda")
    y8, codes = (torch.empty(rows, width, dtype=torch.uint8, device="cuda") for _ in range(2))
    ys, scale = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    s = torch.empty_like(x)
    B.pt_rms_norm(B.rms(x, y, residual=x, sum=s, rstd=rstd))
    B.pt_rms_norm(B.rms(x, y8, residual=x, y_scale=ys))
    B.pt_rows8(B.rows8(x, codes, scale))
    torch.cuda.synchronize()
    want_s, want_r, want, err = ref.rms(x, x, None, 1e-5)
    ref.within("rstd", rstd, want_r, err * want_r)
    ref.within("sum", s, want_s, ref.rounding(want_s, x.dtype) * 1.001)
    ref.within("y", y, want, err * want.abs() + ref.rounding(want, x.dtype) * 1.001)
    ref.codes_within("y8", y8, ys, want, err * want.abs())
    ref.codes_within("codes", codes, scale, x.double(), torch.zeros_like(want))
