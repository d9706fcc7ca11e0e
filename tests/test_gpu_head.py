"""Loss of a language model's head and its gradients against the formulas in 64 bits.

Bounds, with u the unit roundoff of the 16-bit type (8 and 11 significant bits: 2^-8 bf16, 2^-11 fp16) and e = 2^-24:
  z        sums of `width` exact products in fp32: |dz| <= (width + 64) e max_v sum_k |h_k W_vk| =: D, for any order
  loss     lse and the target's z: 2 D, and 2e-5 for exp, the sum over the vocabulary and log in fp32
  G        D' = 2 D + 2e-5 is the error of z - lse, so |dG| <= u |G| + s D' p; 16-bit numbers below the type's normal range are
           2^-38 of the largest s apart at most (G is scaled to it)
  results  the sums of |dG| times the other operand, fp32 sums, and u of the result (of the smallest normal number at least)
"""
import numpy as np
import pytest
import torch

from paper_2406_08334_amd import binding as B

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": (torch.bfloat16, 2.0 ** -8, 2.0 ** -126), "fp16": (torch.float16, 2.0 ** -11, 2.0 ** -14)}
E = 2.0 ** -24


def place(x, pad, shift):
    """x with `pad` elements behind every row, the first `shift` elements behind a 256-byte boundary."""
    rows, width = x.shape
    buf = torch.full((shift + rows * (width + pad) + 8,), 7.0, dtype=x.dtype, device="cuda")
    view = buf[shift:shift + rows * (width + pad)].view(rows, width + pad)[:, :width]
    view.copy_(x)
    return buf, view


def case(rows, width, vocab, dtype, seed=0, ignored=0.0, scale="mean", pad=0, shift=0, spread=1.0):
    """Inputs on the device."""
    gen = torch.Generator().manual_seed(seed * 1000003 + rows * 31 + width * 7 + vocab)
    dt = DTYPES[dtype][0]
    w = (torch.randn(vocab, width, generator=gen) * 0.02 * spread).to(dt)
    y = torch.randint(0, vocab, (rows,), generator=gen)
    lean = torch.rand(rows, 1, generator=gen) * 8.0 / (4e-4 * width)
    h = (torch.randn(rows, width, generator=gen) + lean / spread * w[y].float()).to(dt)
    y[torch.rand(rows, generator=gen) < ignored] = -100
    n = max(1, int((y >= 0).sum()))
    s = {"mean": torch.full((rows,), 1.0 / n), "none": None, "mixed": torch.randn(rows, generator=gen) * torch.logspace(-3, 3, rows)}[scale]
    hb, h = place(h.cuda(), pad, shift)
    wb, w = place(w.cuda(), pad, shift)
    return dict(hidden=h, weight=w, target=y.cuda(), scale=None if s is None else s.cuda(), keep=(hb, wb))


def call(c, grads="both", workspace=None, pad=0, shift=0, stream=None):
    """-> loss, d_hidden, d_weight, and the buffers that the gradients lie in."""
    rows, width = c["hidden"].shape
    vocab = c["weight"].shape[0]
    loss = torch.full((rows,), float("nan"), device="cuda")
    dhb, dh = place(torch.full((rows, width), 9.0, dtype=c["hidden"].dtype, device="cuda"), pad, shift) if grads in ("both", "hidden") else (None, None)
    dwb, dw = place(torch.full((vocab, width), 9.0, dtype=c["hidden"].dtype, device="cuda"), pad, shift) if grads in ("both", "weight") else (None, None)
    head = B.head(c["hidden"], c["weight"], c["target"], loss, row_scale=c["scale"], d_hidden=dh, d_weight=dw)
    least, best = B.pt_head_workspace(head)
    size = {None: best, "least": least}.get(workspace, workspace)
    guard = 4096
    work = torch.full((size + guard,), 0x5A, dtype=torch.uint8, device="cuda")
    work[:size] = 0xFF                                     # NaN, if anything read it
    torch.cuda.synchronize()
    B.pt_head_loss(head, work[:size], stream)
    torch.cuda.synchronize()
    assert bool((work[size:] == 0x5A).all()), "wrote behind the workspace"
    for buf, x in ((dhb, dh), (dwb, dw)):
        if buf is not None:                                # nothing between the rows
            mask = torch.ones_like(buf, dtype=torch.bool)
            mask.as_strided(x.shape, x.stride(), x.storage_offset()).fill_(False)
            assert bool((buf[mask] == 7.0).all()), "wrote between the rows"
    return loss, dh, dw


def expected(c, where="cpu"):
    """Loss and gradients in 64 bits and their bounds, on the host or the device."""
    dt = c["hidden"].dtype
    u, tiny = next((u, t) for d, u, t in DTYPES.values() if d == dt)
    w = c["weight"].double().to(where)
    y = c["target"].to(where)
    on = ((y >= 0) & (y < w.shape[0])).nonzero()[:, 0]
    rows, width = c["hidden"].shape
    h = c["hidden"].double().to(where)[on]
    s = torch.ones(rows, dtype=torch.float64, device=where) if c["scale"] is None else c["scale"].double().to(where)
    s, yy = s[on], y[on]
    z = h @ w.t()
    D = (width + 64) * E * (h.abs() @ w.abs().t()).amax(1) if len(on) else torch.zeros(0, dtype=torch.float64, device=where)
    logp = torch.log_softmax(z, 1)
    del z
    i = torch.arange(len(on), device=where)
    loss, loss_b = (torch.zeros(rows, dtype=torch.float64, device=where) for _ in range(2))
    loss[on], loss_b[on] = -logp[i, yy], 2 * D + 2e-5 + 4 * E * logp[i, yy].abs()
    p = logp.exp()
    g = p.clone()
    g[i, yy] = torch.expm1(logp[i, yy])
    big = float(s.abs().max()) if len(on) else 0.0
    dg = s.abs()[:, None] * (u * g.abs() + (2 * D + 2e-5)[:, None] * p) + big * 2.0 ** -38
    g = g * s[:, None]
    dh, dh_b = (torch.zeros(rows, width, dtype=torch.float64, device=where) for _ in range(2))
    dh[on] = g @ w
    dh_b[on] = dg @ w.abs() + (w.shape[0] + 64) * E * (g.abs() @ w.abs())
    dw, dw_b = g.t() @ h, dg.t() @ h.abs() + (len(on) + 64) * E * (g.abs().t() @ h.abs())
    out = []
    for x, b in ((dh, dh_b), (dw, dw_b)):
        out += [x, b * (1 + u) + u * torch.clamp(x.abs(), min=tiny)]
    return loss, loss_b, *out


def check(got, want, grads="both"):
    loss, loss_b, dh, dh_b, dw, dw_b = want
    for name, x, w, b in (("loss", got[0], loss, loss_b), ("d_hidden", got[1], dh, dh_b), ("d_weight", got[2], dw, dw_b)):
        if x is None:
            continue
        off = (x.double().to(w.device) - w).abs()
        assert bool((off <= b).all()), f"{name}: worst {float((off / b.clamp(min=1e-300)).max()):.3g} of the bound"


SHAPES = [(1, 8, 2), (1, 64, 300), (3, 1, 5), (7, 65, 257), (64, 128, 512), (100, 72, 1000), (257, 200, 511), (300, 256, 256), (513, 771, 999),
          (2, 40, 20011), (1030, 24, 130), (33, 513, 3001)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,width,vocab", SHAPES)
def test_against_64_bits(rows, width, vocab, dtype):
    c = case(rows, width, vocab, dtype, ignored=0.2 if rows > 6 else 0.0)
    want = expected(c)
    check(call(c), want)
    check(call(c, grads="none"), want)


# sizes that take tiles of 256 x 256: with the last 64, 128 and 3 of the width in narrower ones, workgroups that share a tile's k, several pieces
LARGE = [(1024, 320, 12800, None), (1024, 384, 12800, None), (700, 515, 20000, None), (300, 320, 40000, None), (1300, 256, 25000, "least"),
         (2100, 640, 9000, None)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,width,vocab,workspace", LARGE)
def test_large_tiles(rows, width, vocab, workspace, dtype):
    c = case(rows, width, vocab, dtype, ignored=0.1)
    check(call(c, workspace=workspace), expected(c, "cuda"))


# a small vocabulary: workgroups that share the rows of a tile of the weight's gradient, in either kind of tile, one piece of more rows than usual, widths
# whose sums end inside four numbers
SHARED = [(8192, 512, 1000), (3000, 203, 700), (9000, 64, 40), (20000, 130, 300), (1500, 1100, 2100), (33000, 16, 17)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,width,vocab", SHARED)
def test_small_vocabularies(rows, width, vocab, dtype):
    c = case(rows, width, vocab, dtype, ignored=0.3)
    want = expected(c, "cuda")
    check(call(c), want)
    check(call(c, grads="weight"), want)


def test_a_small_vocabulary_without_a_row():
    c = case(3000, 128, 200, "bf16")
    c["target"][:] = -1
    loss, dh, dw = call(c)
    assert not bool(loss.any()) and not bool(dh.any()) and not bool(dw.any())


@pytest.mark.parametrize("rows", [1, 9, 40, 64])
def test_rows_without_a_target_that_are_multiplied_all_the_same(rows):
    """Few rows whose hidden states are taken where they lie: those without a target hold what must not reach a result."""
    c = case(rows, 128, 500, "bf16", ignored=0.4)
    off = c["target"] < 0
    c["hidden"][off] = float("nan")
    c["hidden"][off, ::2] = float("inf")
    want = expected(c)
    for grads in ("both", "hidden", "weight"):
        got = call(c, grads=grads)
        check(got, want)
        assert not bool(got[0][off].any()) and (got[1] is None or not bool(got[1][off].any()))


def test_logits_beyond_32_bits():
    """What is kept of a piece's logits is 4.3 GB: rows whose place passes 2^32 bytes."""
    c = case(8192, 64, 131072, "fp16")
    c["scale"] *= 1024.0
    check(call(c), expected(c, "cuda"))


@pytest.mark.parametrize("rows", [1, 20, 64, 65])
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 8), (4, 0), (0, 1)])
def test_losses_alone_of_few_rows(rows, pad, shift):
    """Rows that are multiplied where they lie, and those that cannot be; ones without a target hold infinities."""
    c = case(rows, 192, 1000, "bf16", ignored=0.3, pad=pad, shift=shift)
    c["hidden"][c["target"] < 0] = float("inf")
    check(call(c, grads="none"), expected(c))


@pytest.mark.parametrize("rows", [128, 129])
def test_either_side_of_the_rows_whose_rounding_is_made_good(rows):
    c = case(rows, 200, 900, "bf16", ignored=0.1)
    check(call(c), expected(c))


@pytest.mark.parametrize("grads", ["hidden", "weight"])
def test_one_gradient(grads):
    c = case(130, 96, 700, "bf16")
    check(call(c, grads=grads), expected(c))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("grads", ["hidden", "weight"])
def test_one_gradient_in_pieces_the_last_of_few_rows(grads, dtype):
    c = case(1300, 96, 700, dtype, ignored=0.2)
    check(call(c, grads=grads, workspace="least"), expected(c))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows", [1, 40, 300])
def test_a_vocabulary_of_one_word(rows, dtype):
    """The word is certain: no loss, no gradient."""
    c = case(rows, 72, 1, dtype, scale="none")
    loss, dh, dw = call(c)
    assert not bool(loss.any()) and not bool(dh.any()) and not bool(dw.any())


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows", [50, 600])
def test_no_loss_is_below_zero(rows, dtype):
    """The target's z is the largest by far, and far from 0: nothing but roundings is left of the loss."""
    c = case(rows, 64, 500, dtype)
    w = c["weight"].float()
    c["hidden"].copy_(100.0 * w[c["target"]] / w[c["target"]].square().sum(1, keepdim=True))
    for grads in ("none", "both"):
        loss = call(c, grads=grads)[0]
        assert bool((loss >= 0).all()) and float(loss.max()) < 1e-3
    check(call(c), expected(c))


@pytest.mark.parametrize("rows", [30, 200])
def test_scales_of_zero(rows):
    """Rows whose gradient is wanted zero times, and none but such."""
    c = case(rows, 64, 300, "bf16")
    c["scale"][::3] = 0.0
    check(call(c), expected(c))
    c["scale"][:] = 0.0
    loss, dh, dw = call(c)
    check((loss, None, None), expected(c))
    assert not bool(dh.any()) and not bool(dw.any())


@pytest.mark.parametrize("scale", ["none", "mixed"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_scales_of_rows(dtype, scale):
    """None: 1 for every row; scales of both signs over six powers of ten."""
    c = case(150, 64, 400, dtype, scale=scale, ignored=0.3)
    if dtype == "fp16" and scale == "mixed":
        c["scale"] *= 0.01                                # results stay in the type's range
    check(call(c), expected(c))


def test_fp16_without_a_loss_scale():
    """Scales so small that s p is far below fp16's range; the results are small too, but in it."""
    c = case(40, 64, 3000, "fp16")
    c["scale"] = torch.full((40,), 2e-4, device="cuda")
    check(call(c), expected(c))


@pytest.mark.parametrize("pad,shift", [(8, 0), (8, 8), (3, 0), (0, 1), (5, 3), (4, 4)])
def test_strides_and_alignments(pad, shift):
    c = case(70, 136, 300, "bf16", pad=pad, shift=shift)
    check(call(c, pad=pad, shift=shift), expected(c))


def test_rows_in_pieces_give_the_same_within_the_bounds_and_the_least_workspace_does():
    c = case(1300, 80, 600, "bf16", ignored=0.3)
    want = expected(c)
    check(call(c, workspace="least"), want)
    loss = torch.empty(1300, device="cuda")
    dh, dw = torch.empty_like(c["hidden"]), torch.empty_like(c["weight"])
    least, best = B.pt_head_workspace(B.head(c["hidden"], c["weight"], c["target"], loss, d_hidden=dh, d_weight=dw))
    assert least < best
    check(call(c, workspace=(least + best) // 2 // 256 * 256), want)


def test_pieces_without_a_row():
    """All rows with a target in the first piece, all in the last, and none at all."""
    for lo, hi in ((0, 100), (900, 1000), (0, 0)):
        c = case(1000, 64, 300, "bf16")
        off = torch.ones(1000, dtype=torch.bool)
        off[lo:hi] = False
        c["target"][off.cuda()] = -1
        c["hidden"][off.cuda()] = float("nan")
        want = expected(c)
        for workspace in (None, "least"):
            got = call(c, workspace=workspace)
            check(got, want)
            assert bool((got[0][off.cuda()] == 0).all()) and bool((got[1][off.cuda()] == 0).all())


@pytest.mark.parametrize("bad", [-1, -100, 300, 1 << 40, -(1 << 63)])
def test_any_target_outside_the_vocabulary_is_ignored(bad):
    c = case(90, 64, 300, "bf16")
    c["target"][::3] = bad
    c["hidden"][::3] = float("inf")
    check(call(c), expected(c))


def test_not_a_number_in_a_row_that_counts_reaches_its_results():
    c = case(20, 64, 300, "bf16")
    c["hidden"][3, 5] = float("nan")
    loss, dh, dw = call(c)
    assert bool(loss[3].isnan()) and bool(dh[3].isnan().all()) and bool(dw.isnan().all())
    fine = [r for r in range(20) if r != 3]
    want = expected({**c, "hidden": torch.nan_to_num(c["hidden"])})
    check((loss[fine], dh[fine], None), [x[fine] for x in want[:4]] + [None, None])


def test_certain_and_hopeless_targets():
    """Probabilities of the target from 1 - 1e-12 to 1e-40: no cancellation at the one, no log of 0 at the other."""
    c = case(64, 64, 500, "bf16")
    w = c["weight"].float()
    sign = torch.linspace(-40, 40, 64, device="cuda")[:, None]
    y = c["target"]
    c["hidden"].copy_(sign * w[y] / w[y].square().sum(1, keepdim=True))
    want = expected(c)
    assert float(want[0].max()) > 35 and float(want[0].min()) < 1e-6
    check(call(c), want)


def test_gradient_against_differences_of_the_loss():
    """d(total) along random directions of h and W from losses alone, against the gradients: the difference quotient's error is that of the
    losses (2e-5 each, n of them with a scale of 1 / n) over the step, and the third derivative's share."""
    c = case(60, 128, 400, "fp16", scale="mean")
    loss, dh, dw = call(c)
    gen = torch.Generator(device="cuda").manual_seed(5)
    eps = 2.0 ** -5
    for name, grad in (("hidden", dh), ("weight", dw)):
        x = c[name]
        step = torch.randint(0, 2, x.shape, generator=gen, device="cuda") * 2.0 - 1.0
        step = step * (eps if name == "hidden" else eps * 2.0 ** -5)
        plus, minus = (x.float() + step).to(x.dtype), (x.float() - step).to(x.dtype)
        total = [float((call({**c, name: v.clone()}, grads="none")[0].double() * c["scale"].double()).sum()) for v in (plus, minus)]
        want = float((grad.double() * (plus.double() - minus.double())).sum())
        size = float((grad.double() * (plus.double() - minus.double())).square().sum().sqrt())
        assert abs(total[0] - total[1] - want) <= 4e-5 + 0.05 * size, (name, total, want)


def test_the_same_bits_again_also_on_another_stream_and_in_a_graph():
    c = case(300, 96, 800, "bf16", ignored=0.1)
    first = [x.clone() for x in call(c)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = call(c, stream=side)
    for a, b in zip(first, again):
        assert torch.equal(a, b)
    loss = torch.empty(300, device="cuda")
    dh, dw = torch.empty_like(c["hidden"]), torch.empty_like(c["weight"])
    head = B.head(c["hidden"], c["weight"], c["target"], loss, row_scale=c["scale"], d_hidden=dh, d_weight=dw)
    work = torch.empty(B.pt_head_workspace(head)[1], dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.pt_head_loss(head, work)
    for k in range(3):
        for x in (loss, dh, dw):
            x.fill_(3.0)
        c["target"].copy_(torch.roll(c["target"], k))     # other rows are ignored: their number is the device's
        graph.replay()
        torch.cuda.synchronize()
        want = call(c)
        for a, b in zip((loss, dh, dw), want):
            assert torch.equal(a, b), k


def test_no_rows_clear_the_weight_gradient():
    w = torch.randn(50, 24, device="cuda").bfloat16()
    dw = torch.full_like(w, 5.0)
    empty = torch.empty(0, 24, dtype=torch.bfloat16, device="cuda")
    head = B.head(empty, w, torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda"), d_hidden=empty.clone(), d_weight=dw)
    assert B.pt_head_workspace(head) == (0, 0)
    B.pt_head_loss(head, None)
    assert bool((dw == 0).all())


def test_refusals():
    c = case(20, 64, 300, "bf16")
    loss = torch.empty(20, device="cuda")
    head = B.head(c["hidden"], c["weight"], c["target"], loss)
    least, _ = B.pt_head_workspace(head)
    work = torch.empty(least + 256, dtype=torch.uint8, device="cuda")
    for args, status in (((None,), B.PT_ERR_INVALID_ARG), ((work[:least - 1],), B.PT_ERR_NOMEM), ((work[16:],), B.PT_ERR_ALIGNMENT)):
        with pytest.raises(B.PtError) as e:
            B.pt_head_loss(head, *args)
        assert e.value.status == status
