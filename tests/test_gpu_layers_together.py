"""The layers before the head one behind the other, as a model uses them: gradients of a whole block against torch's own in 64 bits, in 8 bits, captured, and the
example that trains with them."""
import math

import pytest
import torch

import layers_reference as ref
from paper_2406_08334_amd import binding as B
from paper_2406_08334_amd import train_head

pytestmark = pytest.mark.gpu


def block64(h, params, drop_mask):
    g1, w1, b1, w2, b2, g2 = params

    def norm(x, g):
        return x * (x.square().mean(1, keepdim=True) + 1e-5) ** -0.5 * g
    a = torch.nn.functional.gelu(norm(h, g1) @ w1.t() + b1)
    s = h + (a @ w2.t() + b2) * drop_mask
    return norm(s, g2)


@pytest.mark.parametrize("rows,width,mlp,dtype", [(200, 96, 200, "fp16"), (33, 77, 131, "fp16"), (300, 128, 512, "bf16"), (1, 64, 96, "fp16")])
def test_a_block_and_its_gradients(rows, width, mlp, dtype):
    """Values between the kernels are rounded to 16 bits, ten roundings or fewer on each way: 2-norms within 10 u, where u is one rounding's."""
    dt, u, _ = ref.TYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(rows)
    h = torch.randn(rows, width, generator=gen, device="cuda").to(dt)
    block = train_head.Block(h, mlp, 0.25, 9, gen)
    d = torch.randn(rows, width, generator=gen, device="cuda").to(dt)
    block.forward()
    block.d_out.copy_(d)
    block.backward()
    torch.cuda.synchronize()
    leaves = [h.double().requires_grad_(True)] + [p.double().requires_grad_(True) for p in block.params]
    out = block64(leaves[0], leaves[1:], ref.kept(rows, width, 0.25, 9, 0))
    want = [out.detach()] + list(torch.autograd.grad((out * d.double()).sum(), leaves))
    for name, x, w in zip(["out", "d_hidden", "g1", "w1", "b1", "w2", "b2", "g2"], [block.out, block.d_hidden] + block.grads, want):
        off = float((x.double() - w).norm() / w.norm())
        assert off < 10 * u, (name, off)
    assert int(block.step) == 1


def test_a_block_captured_beside_an_eager_one():
    """Forward and backward in two graphs that share a workspace, replayed several times with eager work of the same arrays in between."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    h = torch.randn(256, 128, generator=gen, device="cuda").bfloat16()
    block = train_head.Block(h, 320, 0.25, 9, gen)
    block.d_out.copy_(torch.randn(256, 128, generator=gen, device="cuda"))
    results = lambda: [x.clone() for x in [block.out, block.d_hidden] + block.grads]  # noqa: E731
    want = []
    for step in range(3):
        block.step.fill_(step)
        block.forward(), block.backward()
        want.append(results())
    torch.cuda.synchronize()
    fwd, bwd = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(fwd):
        block.forward()
    with torch.cuda.graph(bwd):
        block.backward()
    block.step.zero_()
    for step in range(3):
        assert int(block.step) == step
        for x in [block.out, block.d_hidden] + block.grads:
            x.fill_(7.0)
        block.work.fill_(0xFF)
        fwd.replay()
        bwd.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results(), want[step]))
        block.forward()                                     # eager, with the next step's mask
        torch.cuda.synchronize()
    assert not torch.equal(want[0][0], want[1][0])


@pytest.mark.parametrize("rows", [1, 40, 300])
def test_a_norm_in_8_bits_before_a_product_in_8_bits(rows):
    """Norm with codes, weights laid out by rows8, their product: each against what the one before has left."""
    gen = torch.Generator().manual_seed(rows)
    width, outs = 520, 300
    x, r = (torch.randn(rows, width, generator=gen).bfloat16().cuda() for _ in range(2))
    w = (torch.randn(outs, width, generator=gen) * 0.05).cuda()
    gate = torch.randn(rows, outs, generator=gen).bfloat16().cuda()
    y, w8 = torch.empty(rows, width, dtype=torch.uint8, device="cuda"), torch.empty(outs, width, dtype=torch.float8_e4m3fn, device="cuda")
    ys, ws = torch.empty(rows, device="cuda"), torch.empty(outs, device="cuda")
    out = torch.empty(rows, outs, dtype=torch.bfloat16, device="cuda")
    B.pt_rows8(B.rows8(w, w8, ws))
    B.pt_rms_norm(B.rms(x, y, residual=r, sum=r, y_scale=ys))
    layer = B.linear(y, w8, out, gate=gate, act="silu", x_scale=ys, weight_scale=ws)
    B.pt_linear_out(layer, torch.empty(max(1, B.pt_linear_workspace(layer)[0]), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    c = dict(x=y.view(torch.float8_e4m3fn), weight=w8, x_scale=ys, weight_scale=ws, gate=gate, act="silu", out=out)
    ref.within("out", out, *ref.linear(c)["out"])


def test_two_streams_at_once():
    """The same block on two streams with a workspace each, call behind call without waiting: the results of one after the other."""
    blocks, want = [], []
    for seed in (1, 2):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        h = torch.randn(700, 192, generator=gen, device="cuda").bfloat16()
        b = train_head.Block(h, 640, 0.25, seed, gen)
        b.d_out.copy_(torch.randn(700, 192, generator=gen, device="cuda"))
        b.forward(), b.backward()
        blocks.append(b)
        want.append([x.clone() for x in [b.out, b.d_hidden] + b.grads])
        b.step.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in blocks]
    for _ in range(5):
        for b, s in zip(blocks, streams):
            with torch.cuda.stream(s):
                b.forward()
        for b, s in zip(blocks, streams):
            with torch.cuda.stream(s):
                b.backward()
                b.step.zero_()
    torch.cuda.synchronize()
    for b, w in zip(blocks, want):
        assert all(torch.equal(x, y) for x, y in zip([b.out, b.d_hidden] + b.grads, w))


@pytest.mark.parametrize("bits,dtype", [(8, "bf16"), (32, "fp16")])
def test_the_example_runs_with_a_block(bits, dtype):
    losses = train_head.train(steps=30, vocab=256, width=64, rows=512, bits=bits, dtype=dtype, mlp=128, drop=0.1)
    assert len(losses) == 30 and all(math.isfinite(x) for x in losses)
    assert abs(losses[0] - math.log(256)) < 1.0
