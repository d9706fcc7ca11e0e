"""What the head's loss and gradients keep of small losses beside large logits.  Bounds, with e = 2^-24 and u as in test_gpu_head:

  S = sum exp(z - largest)   1 and more; at most 64 additions on an element's way into it, each e of S, and 2e-6 of what is added for exp of it:
                             |dS| <= 64 e S + 2e-6 (S - 1) =: T S.  Logits here are exact, so nothing else is off
  loss                       (largest - z_y) + log S: T, and 4 e of the loss.  The logits' size does not enter
  G                          at the target s expm1(-loss): s (T p + 8 e |expm1|); elsewhere s p (T + 2e-6); rounded by u of it, of bf16 by 2^-11 before;
                             16-bit numbers below the type's normal range are 2^-38 of the largest s apart at most"""
import pytest
import torch

from paper_2406_08334_amd import binding as B
from test_gpu_head import DTYPES, E, call

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
