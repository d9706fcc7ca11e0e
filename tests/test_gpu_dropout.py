"""Dropout: the mask bit for bit as it is defined, the values to one rounding."""
import pytest
import torch

import layers_reference as ref
from paper_2406_08334_amd import binding as B

pytestmark = pytest.mark.gpu


def run(rows, width, dtype="bf16", p=0.1, residual=True, pad=0, shift=0, seed=11, step=None, in_place=None):
    gen = torch.Generator().manual_seed(rows * 31 + width)
    dt = ref.TYPES[dtype][0]
    x, r, out = (ref.place((torch.randn(rows, width, generator=gen) + 3).to(dt).cuda(), pad, shift) for _ in range(3))
    to = {None: out, "x": x, "residual": r}[in_place]
    a, b = x[1].double(), r[1].double()
    s = None if step is None else torch.full((1,), step, dtype=torch.int64, device="cuda")
    B.pt_dropout(B.dropout(x[1], to[1], p, seed, step=s, residual=r[1] if residual else None))
    torch.cuda.synchronize()
    for buf, view in (x, r, out):
        assert ref.untouched(buf, view)
    k = ref.kept(rows, width, p, seed, step or 0)
    want = a * k + (b if residual else 0)
    if not residual:
        assert torch.equal(to[1] == 0, k == 0)              # no x is zero
    ref.within("out", to[1], want, 3 * ref.E * (a * k).abs() + ref.E * want.abs() + ref.rounding(want, dt) * 1.001)
    return to[1]


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("rows,width", [(1, 1), (1, 5), (3, 7), (2, 8), (5, 9), (48, 771), (7, 4), (33, 12), (1, 100000), (300, 64), (2, 16385), (4097, 3)])
def test_against_64_bits(rows, width, residual):
    run(rows, width, "fp16" if rows % 2 else "bf16", residual=residual)


@pytest.mark.parametrize("p", [0.0, 1e-6, 1.0 / 65536, 0.25, 0.9, 0.99999, 1 - 2.0 ** -40])
def test_probabilities(p):
    run(64, 160, p=p, residual=False)
    run(64, 163, p=p)


@pytest.mark.parametrize("pad,shift", [(1, 0), (0, 1), (4, 3), (8, 8)])
@pytest.mark.parametrize("width", [16, 61])
def test_any_address_and_stride(width, pad, shift):
    run(21, width, pad=pad, shift=shift)


@pytest.mark.parametrize("in_place", ["x", "residual"])
@pytest.mark.parametrize("width", [77, 128])
def test_in_place(width, in_place):
    run(50, width, in_place=in_place)


def test_steps_and_seeds_give_other_masks_and_the_same_ones_again():
    a = [run(20, 100, seed=s, step=t, p=0.5, residual=False).clone() for s, t in ((1, None), (1, 0), (1, 1), (2, 0), (2 ** 64 - 1, 2 ** 62), (1, 1))]
    assert torch.equal(a[0], a[1]) and torch.equal(a[2], a[5])
    assert not torch.equal(a[1], a[2]) and not torch.equal(a[1], a[3]) and not torch.equal(a[3], a[4])


def test_how_many_are_dropped_and_nothing_that_they_hold_is_seen():
    """Binomial: 2^20 elements, six standard deviations."""
    n, p = 1 << 20, 0.3
    x = torch.full((1024, 1024), float("nan"), dtype=torch.bfloat16, device="cuda")
    k = ref.kept(1024, 1024, p, 5, 0)
    x[k != 0] = 1.0
    out = torch.empty_like(x)
    B.pt_dropout(B.dropout(x, out, p, 5))
    torch.cuda.synchronize()
    zero = int((out == 0).sum())
    assert abs(zero - n * p) < 6 * (n * p * (1 - p)) ** 0.5 + n / 65536
    assert not bool(out.isnan().any())


def test_places_beyond_32_bits():
    """An array of 2^32 and a few elements: the last ones have words of their own."""
    rows, width = (1 << 20) + 1, 4100
    x = torch.ones(rows, width, dtype=torch.bfloat16, device="cuda")
    for wide in (width, width - 1):                         # back to back, and row by row
        v = x[:, :wide]
        out = torch.zeros(rows, width, dtype=torch.bfloat16, device="cuda")[:, :wide]
        B.pt_dropout(B.dropout(v, out, 0.5, 9))
        torch.cuda.synchronize()
        for r0 in (0, rows // 2, rows - 3):
            import numpy as np
            words = (wide + 3) // 4
            r, c = np.arange(r0, r0 + 3, dtype=np.uint64)[:, None], np.arange(wide, dtype=np.uint64)[None]
            with np.errstate(over="ignore"):
                phi = np.uint64(0x9E3779B97F4A7C15)
                z = ref.mix(ref.mix(np.uint64(9)) + (r * np.uint64(words) + c // np.uint64(4) + np.uint64(1)) * phi)
            bits = (z >> (np.uint64(16) * (c % np.uint64(4)))) & np.uint64(0xFFFF)
            assert (out[r0:r0 + 3].float().cpu().numpy() == np.where(bits < 32768, 0.0, 2.0)).all()
        del out


def test_captured_with_another_step_at_each_replay():
    x = torch.randn(100, 256, device="cuda").bfloat16()
    out, step = torch.empty_like(x), torch.zeros(1, dtype=torch.int64, device="cuda")
    d = B.dropout(x, out, 0.5, 77, step=step)
    B.pt_dropout(d)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.pt_dropout(d)
        step.add_(1)
    for t in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert int(step) == t + 1 and torch.equal(out != 0, ref.kept(100, 256, 0.5, 77, t) != 0)
