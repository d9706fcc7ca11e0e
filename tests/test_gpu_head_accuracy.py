"""What the head's loss and gradients keep of small losses beside large logits.  Bounds, with e = 2^-24 and u as in test_gpu_head:

  S = sum exp(z - largest)   1 and more; at most 64 additions on an element's way into it, each e of S, and 2e-6 of what is added for exp of it:
                             |dS| <= 64 e S + 2e-6 (S - 1) =: T S.  Logits here are exact, so nothing else is off
  loss                       (largest - z_y) + log S: T, and 4 e of the loss.  The logits' size does not enter
  G                          at the target s expm1(-loss): s (T p + 8 e |expm1|); elsewhere s p (T + 2e-6); rounded by u of it, of bf16 by 2^-11 before;
                             16-bit numbers below the type's normal range are 2^-38 of the largest s apart at most"""
import pytest
import torch

from paper_2406_08334_amd import binding as B
from test_gpu_head import DTYPES, E, call, case

pytestmark = pytest.mark.gpu
C = 8.0                                                    # the first element of every row of the weight


def large_logits(rows, dtype, offset, seed=0):
    """Logits offset + b_r w_v, exact in fp32 in any order: b and w are multiples of 1/4.  Most targets are the word with w = 1, ahead of the others by b: losses of 1e-6 to 1;
    some are hopeless."""
    gen = torch.Generator().manual_seed(seed)
    vocab, width = 300, 64
    dt = DTYPES[dtype][0]
    w = torch.zeros(vocab, width)
    w[:, 0] = C
    w[:, 1] = torch.randint(-4, 1, (vocab,), generator=gen) / 4
    y = torch.zeros(rows, dtype=torch.int64)
    w[0, 1] = 1.0
    h = torch.zeros(rows, width)
    h[:, 0] = offset / C
    h[:, 1] = torch.randint(20, 80, (rows,), generator=gen) / 4
    y[::7] = torch.randint(1, vocab, (len(y[::7]),), generator=gen)
    assert bool((h.to(dt).float() == h).all()) and bool((w.to(dt).float() == w).all())
    return dict(hidden=h.to(dt).cuda(), weight=w.to(dt).cuda(), target=y.cuda(), scale=torch.full((rows,), 1.0 / rows).cuda())


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("offset", [0.0, 1000.0, -1000.0, 4000.0])
@pytest.mark.parametrize("rows", [5, 64, 100, 300])
def test_small_losses_beside_large_logits(rows, offset, dtype):
    c = large_logits(rows, dtype, offset)
    _, u, tiny = DTYPES[dtype]
    h, w, y = c["hidden"].double().cpu(), c["weight"].double().cpu(), c["target"].cpu()
    s = c["scale"].double().cpu()[:, None]
    z = h @ w.t()
    logp = torch.log_softmax(z, 1)
    i = torch.arange(rows)
    want = -logp[i, y]
    S = torch.exp(z - z.amax(1, keepdim=True)).sum(1)
    T = 64 * E + 2e-6 * (S - 1) / S
    assert float(want.min()) < 1e-4
    p = logp.exp()
    g = p.clone()
    g[i, y] = torch.expm1(logp[i, y])
    dg = p * (T[:, None] + 2e-6)
    dg[i, y] = T * p[i, y] + 8 * E * g[i, y].abs()
    dg = s * (dg + g.abs() * (u + (2.0 ** -11 if dtype == "bf16" else 0.0))) + float(s.max()) * 2.0 ** -38
    g = g * s
    for grads in ("none", "both"):
        loss, dh, dw = call(c, grads=grads)
        off = (loss.double().cpu() - want).abs()
        assert bool((off <= T + 4 * E * want).all()), f"{grads}: {float((off / (T + 4 * E * want)).max()):.3g} of the bound"
    for name, got, want, bound in (("d_hidden", dh, g @ w, dg @ w.abs() + 400 * E * (g.abs() @ w.abs())),
                                   ("d_weight", dw, g.t() @ h, dg.t() @ h.abs() + (rows + 64) * E * (g.abs().t() @ h.abs()))):
        bound = bound * (1 + u) + u * want.abs().clamp(min=tiny)
        off = (got.double().cpu() - want).abs()
        assert bool((off <= bound).all()), f"{name}: {float((off / bound).max()):.3g} of the bound"


# ---- what rounding G leaves at the target ----------------------------------------------------------------

def expected(c, where="cuda"):
    """Gradients in 64 bits and their bounds.  D: what z can be off by (sums of `width` exact products in fp32, any order); G is rounded by u away from the target, where bf16's
    exponentials are rounded to 11 bits before; at the target what the rounding leaves is multiplied too, rounded by u itself: u^2."""
    dt = c["hidden"].dtype
    u, tiny = next((u, t) for d, u, t in DTYPES.values() if d == dt)
    w, y = c["weight"].double().to(where), c["target"].to(where)
    rows, width = c["hidden"].shape
    on = ((y >= 0) & (y < w.shape[0])).nonzero()[:, 0]
    h, s, yy = c["hidden"].double().to(where)[on], c["scale"].double().to(where)[on], y[on]
    D = 2 * (width + 64) * E * (h.abs() @ w.abs().t()).amax(1) + 2e-5
    logp = torch.log_softmax(h @ w.t(), 1)
    i = torch.arange(len(on), device=where)
    p = logp.exp()
    g = p.clone()
    g[i, yy] = torch.expm1(logp[i, yy])
    dg = g.abs() * (u + (2.0 ** -11 if dt == torch.bfloat16 else 0.0))
    dg[i, yy] = g[i, yy].abs() * (u * u + 8 * E)
    dg = s.abs()[:, None] * (dg + D[:, None] * p) + float(s.abs().max()) * 2.0 ** -38
    g = g * s[:, None]
    dh, dh_b = (torch.zeros(rows, width, dtype=torch.float64, device=where) for _ in range(2))
    dh[on], dh_b[on] = g @ w, dg @ w.abs() + (w.shape[0] + 64) * E * (g.abs() @ w.abs())
    dw, dw_b = g.t() @ h, dg.t() @ h.abs() + (2 * len(on) + 64) * E * (g.abs().t() @ h.abs())
    return [(x, b * (1 + u) + u * x.abs().clamp(min=tiny)) for x, b in ((dh, dh_b), (dw, dw_b))]


def check(got, want):
    for name, x, (w, b) in zip(("d_hidden", "d_weight"), got[1:], want):
        if x is None:
            continue
        off = (x.double().to(w.device) - w).abs()
        assert bool((off <= b).all()), f"{name}: {float((off / b.clamp(min=1e-300)).max()):.3g} of the bound"


# few rows and many, listed by one workgroup and by all; tiles of both kinds, shared and not; widths that end inside one; a vocabulary inside one
# tile, and one word
ROWS = [(64, 128, 900, None), (128, 200, 900, None), (129, 200, 900, None), (300, 771, 1500, None), (1024, 320, 12800, None), (1025, 96, 700, "least"),
        (2100, 640, 9000, None), (2600, 64, 3000, "least"), (3000, 203, 700, None), (9000, 64, 40, None), (5000, 130, 300, "least"), (700, 72, 2, None)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,width,vocab,workspace", ROWS)
def test_the_target_takes_part_unrounded(rows, width, vocab, workspace, dtype):
    c = case(rows, width, vocab, dtype, ignored=0.2)
    want = expected(c)
    check(call(c, workspace=workspace), want)
    check(call(c, grads="weight", workspace=workspace), want)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,workspace", [(400, None), (5000, "least"), (9000, None)])
def test_targets_that_repeat(rows, workspace, dtype):
    """Half of the rows have one word, a quarter the last one, some words none."""
    c = case(rows, 96, 2000, dtype, ignored=0.1)
    at = torch.arange(rows, device="cuda")
    c["target"][(at % 2 == 0) & (c["target"] >= 0)] = 1234
    c["target"][(at % 4 == 1) & (c["target"] >= 0)] = 1999
    check(call(c, workspace=workspace), expected(c))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows", [40, 200])
@pytest.mark.parametrize("big", [2.0 ** 120, 2.0 ** 127, 2.0 ** -120])
def test_scales_at_the_ends_of_their_range(rows, big, dtype):
    """Any finite scale: right where the results are in the type's range; where they are not, inf and no NaN, and zero where the weight or h is."""
    c = case(rows, 64, 300, dtype)
    c["scale"] = torch.full((rows,), big, device="cuda")
    c["weight"][:, 5:9] = 0.0
    c["hidden"][:, 5:9] = 0.0
    loss, dh, dw = call(c)
    assert not bool(dh.isnan().any()) and not bool(dw.isnan().any())
    assert bool((dh[:, 5:9] == 0).all()) and bool((dw[:, 5:9] == 0).all())
    if dtype == "bf16" and big < 2.0 ** 127:
        check((loss, dh, dw), expected(c))
