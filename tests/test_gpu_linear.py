"""Matrix product with its epilogue, and its gradients, against the formulas in 64 bits (bounds: layers_reference.py)."""
import pytest
import torch

import layers_reference as ref
from paper_2406_08334_amd import binding as B

pytestmark = pytest.mark.gpu
SEED, STEP = 0xC0FFEE1234567, 3


def case(rows, width, outs, dtype="bf16", act="none", bias=False, gate=False, residual=False, drop=0.0, bits=16, pad=0, shift=0, seed=0, grads=False):
    """Arrays on the device, as binding.linear takes them; `buffers`: those that lie in larger ones."""
    gen = torch.Generator().manual_seed(seed * 1000003 + rows * 31 + width * 7 + outs)
    dt = ref.TYPES[dtype][0]
    r = lambda std, *shape: torch.randn(*shape, generator=gen) * std  # noqa: E731
    c, buffers = dict(act=act, drop=drop, seed=SEED, step=torch.full((1,), STEP, dtype=torch.int64, device="cuda"), step_value=STEP), {}

    def put(name, x):
        buffers[name] = ref.place(x.cuda(), pad, shift)
        c[name] = buffers[name][1]
    x, w = r(1.0, rows, width), r(1.0 / max(1, width) ** 0.5, outs, width)
    if bits == 8:
        for name, a in (("x", x), ("weight", w)):
            scale = a.abs().amax(1) / 448
            put(name, (a / scale.clamp(min=1e-30)[:, None]).to(torch.float8_e4m3fn))
            c[("x" if name == "x" else "weight") + "_scale"] = scale.cuda()
    else:
        put("x", x.to(dt))
        put("weight", w.to(dt))
    if bias:
        c["bias"] = r(0.5, outs).to(dt).cuda()
    for name, on in (("gate", gate), ("residual", residual)):
        if on:
            put(name, r(1.0, rows, outs).to(dt))
    blank = torch.zeros(rows, outs, dtype=dt)
    if grads:
        if act != "none" or gate:
            put("pre", (r(2.0, rows, outs)).to(dt))
        put("d_out", r(0.3, rows, outs).to(dt))
        put("d_x", torch.zeros(rows, width, dtype=dt))
        put("d_weight", torch.zeros(outs, width, dtype=dt))
        c["d_bias"] = torch.empty(outs, dtype=dt, device="cuda")
        if gate:
            put("d_gate", blank)
    else:
        put("pre", blank)
        put("out", blank)
    c["buffers"] = buffers
    return c


def call(c, grads=False, stream=None, work=None):
    """Runs it in a workspace of exactly its size, filled with what no result may come from."""
    layer = B.linear(**{k: v for k, v in c.items() if k not in ("step_value", "buffers")})
    size = B.pt_linear_workspace(layer)[grads]
    guard = torch.full((size + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    guard[:size] = 0xFF
    torch.cuda.synchronize()
    (B.pt_linear_grads if grads else B.pt_linear_out)(layer, guard[:size], stream)
    torch.cuda.synchronize()
    assert bool((guard[size:] == 0x5A).all()), "wrote behind the workspace"
    for name, (buf, view) in c["buffers"].items():
        assert ref.untouched(buf, view), f"wrote beside {name}"


def check(c, grads=False):
    want = (ref.linear_grads if grads else ref.linear)(c)
    for name, (v, b) in want.items():
        if c.get(name) is not None:
            ref.within(name, c[name], v, b)


SIZES = [(1, 1, 1), (1, 64, 300), (3, 7, 5), (2, 8, 129), (16, 200, 64), (17, 65, 257), (48, 512, 96), (64, 128, 512), (65, 130, 130), (100, 72, 1000), (129, 256, 128),
         (257, 200, 511), (300, 771, 999), (1030, 64, 130), (513, 1000, 260)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,width,outs", SIZES)
def test_out_against_64_bits(rows, width, outs, dtype):
    i = SIZES.index((rows, width, outs))
    c = case(rows, width, outs, dtype, act=ref.ACTS[i % 5], bias=i % 2 == 0, gate=i % 3 == 0, residual=i % 4 < 2, drop=(0.0, 0.1, 0.5)[i % 3])
    call(c)
    check(c)


@pytest.mark.parametrize("act", ref.ACTS)
@pytest.mark.parametrize("rows", [5, 40, 200])
def test_every_epilogue(rows, act):
    c = case(rows, 192, 264, act=act, bias=True, gate=True, residual=True, drop=0.25)
    call(c)
    check(c)


@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (3, 5), (8, 8), (64, 0)])
@pytest.mark.parametrize("rows,width,outs", [(4, 64, 40), (33, 128, 136), (150, 192, 200), (70, 77, 131)])
def test_rows_at_any_address_and_stride(rows, width, outs, pad, shift):
    c = case(rows, width, outs, act="silu", bias=True, gate=True, residual=True, pad=pad, shift=shift)
    call(c)
    check(c)
    g = case(rows, width, outs, act="gelu", gate=True, pad=pad, shift=shift, grads=True)
    call(g, True)
    check(g, True)


# sizes that take 256 x 256 tiles, whole, narrower at the end, and shared by several workgroups
LARGE = [(2048, 256, 2048), (1024, 1600, 3264), (4096, 320, 1100), (300, 4096, 1088), (700, 8192, 515)]


@pytest.mark.parametrize("rows,width,outs", LARGE)
def test_large_tiles(rows, width, outs):
    c = case(rows, width, outs, "fp16" if rows == 700 else "bf16", act="gelu_tanh", bias=True, residual=True, drop=0.1)
    call(c)
    check(c)


# one round of 256 x 256 tiles and a few of 64 x 256 at the end of the outs; rows at multiples of 16 bytes (stored from the sums) or not (through LDS)
@pytest.mark.parametrize("act", ref.ACTS)
@pytest.mark.parametrize("dtype,pad,shift,more", [("bf16", 4, 0, dict(residual=True, drop=0.1)), ("fp16", 4, 8, dict()), ("bf16", 4, 0, dict(gate=True)),
                                                  ("fp16", 0, 1, dict(residual=True, drop=0.5, gate=True))])
def test_every_epilogue_of_the_largest_tiles(dtype, pad, shift, more, act):
    c = case(4096, 1024, 4100, dtype, act=act, bias=True, pad=pad, shift=shift, **more)
    call(c)
    check(c)


@pytest.mark.parametrize("act,dtype,more", [("none", "bf16", dict(pad=4)), ("gelu", "fp16", dict(pad=4, residual=True, drop=0.1)), ("silu", "bf16", dict(gate=True))])
def test_8_bits_in_the_largest_tiles(act, dtype, more):
    c = case(4096, 2048, 4100, dtype, act=act, bias=True, bits=8, **more)
    call(c)
    check(c)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,width,outs", SIZES)
def test_grads_against_64_bits(rows, width, outs, dtype):
    i = SIZES.index((rows, width, outs))
    c = case(rows, width, outs, dtype, act=ref.ACTS[i % 5], gate=i % 3 == 0, drop=(0.0, 0.1, 0.5)[i % 3], grads=True)
    call(c, True)
    check(c, True)


@pytest.mark.parametrize("rows,width,outs", LARGE + [(8192, 128, 192), (20, 2048, 4096)])
def test_grads_of_large_tiles(rows, width, outs):
    c = case(rows, width, outs, act="silu", gate=True, grads=True)
    call(c, True)
    check(c, True)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,width,outs", [(1, 64, 64), (2, 96, 64), (31, 200, 130), (32, 64, 1000), (7, 4096, 65), (16, 77, 2048), (33, 64, 64)])
def test_grads_of_few_rows_have_one_rounding(rows, width, outs, dtype):
    """Up to 32 rows the bound has no term for rounding dz but its square."""
    for k in range(3):
        c = case(rows, width, outs, dtype, act=("gelu", "silu", "none")[k], gate=k != 0, drop=0.2 * k, grads=True, seed=k)
        call(c, True)
        check(c, True)


def test_grads_beyond_the_type_stay_infinite():
    for rows in (3, 40):
        c = case(rows, 64, 96, "fp16", gate=True, grads=True)
        c["d_out"][1, 5], c["gate"][1, 5] = 60000.0, 8.0
        call(c, True)
        assert bool(c["d_bias"][5].isinf()) and bool(c["d_x"][1].float().abs().isinf().all())
        assert bool(c["d_x"][[0, 2]].isfinite().all()) and bool(c["d_weight"][[4, 6]].isfinite().all())


@pytest.mark.parametrize("what", ["d_x", "d_weight", "d_bias", "d_gate"])
def test_one_gradient_alone(what):
    c = case(130, 96, 140, act="gelu", gate=True, drop=0.2, grads=True)
    want = ref.linear_grads(c)
    for name in ("d_x", "d_weight", "d_bias", "d_gate"):
        if name != what:
            c[name] = None
    call(c, True)
    ref.within(what, c[what], *want[what])


@pytest.mark.parametrize("rows,width,outs,pad,shift", [(1, 16, 8, 0, 0), (1, 128, 300, 0, 0), (5, 100, 33, 3, 1), (17, 256, 130, 0, 16), (64, 200, 77, 1, 0),
                                                       (200, 128, 256, 0, 0), (300, 1000, 600, 24, 0), (1500, 512, 1030, 0, 0), (2048, 1536, 2304, 0, 0)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_8_bits(rows, width, outs, pad, shift, dtype):
    c = case(rows, width, outs, dtype, act="silu", bias=True, gate=rows % 2 == 1, bits=8, pad=pad, shift=shift)
    call(c)
    check(c)


def test_out_is_the_residual():
    for rows in (3, 90, 600):
        c = case(rows, 128, 200, residual=True, drop=0.3)
        want = ref.linear(c)["out"]
        c["out"] = c["residual"]
        call(c)
        ref.within("out", c["out"], *want)


@pytest.mark.parametrize("act", ref.ACTS)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_activations_at_the_ends_of_their_range(act, dtype):
    """z as large as the type has it, infinite and NaN: an identity weight hands x through."""
    dt = ref.TYPES[dtype][0]
    big = torch.finfo(dt).max
    v = torch.tensor([0.0, -0.0, 1e-3, -1e-3, 3.0, -3.0, 5.5, -5.5, 9.0, -9.0, 13.0, -13.0, 40.0, -40.0, big, -big], device="cuda")
    x = torch.zeros(16, 64, device="cuda")
    x[:, 0] = v
    w = torch.zeros(32, 64, device="cuda")
    w[:, 0] = 1.0
    c = dict(x=x.to(dt), weight=w.to(dt), act=act, out=torch.empty(16, 32, dtype=dt, device="cuda"), buffers={})
    call(c)
    want, _ = ref.act(act, c["x"].double()[:, :1].expand(16, 32))
    ref.within("out", c["out"], want, ref.rounding(want, dt) * 1.01 + 1e-17)
    g = dict(c, pre=c["x"][:, :1].expand(16, 32).contiguous(), d_out=torch.ones(16, 32, dtype=dt, device="cuda"), out=None,
             d_bias=torch.empty(32, dtype=dt, device="cuda"), d_x=torch.empty(16, 64, dtype=dt, device="cuda"))
    call(g, True)
    slope = ref.act(act, c["x"].double()[:, 0].clamp(-64, 64))[1]
    ref.within("d_x", g["d_x"][:, 0] / 32, slope, 2 * ref.rounding(slope, dt) + 2 * ref.ACT_ERR)
    for bad in (float("inf"), float("-inf"), float("nan")):
        x = c["x"].clone()
        x[3, 0] = bad
        d = dict(c, x=x, out=torch.empty(16, 32, dtype=dt, device="cuda"))
        call(d)
        torch.testing.assert_close(d["out"][[0, 1, 2, 4, 5]], c["out"][[0, 1, 2, 4, 5]], rtol=0, atol=0)
        f = d["out"][3].float()
        if bad == float("inf"):
            assert bool((f == bad).all() if act in ("none", "relu") else (f == bad).all() | f.isnan().all())
        elif bad != bad:
            assert bool(f.isnan().all())


def test_what_a_dropped_element_holds_reaches_nothing():
    for rows in (4, 100):
        c = case(rows, 64, 96, gate=True, residual=True, drop=0.5)
        off = ref.kept(rows, 96, 0.5, SEED, STEP) == 0
        want = ref.linear(c)["out"]
        c["gate"][off] = float("nan")
        call(c)
        ref.within("out", c["out"], *want)
        g = case(rows, 64, 96, act="silu", gate=True, drop=0.5, grads=True)
        want = ref.linear_grads(g)
        g["d_out"][off] = float("inf")
        g["pre"][off] = float("nan")
        g["gate"][off] = float("-inf")
        call(g, True)
        for name, (v, b) in want.items():
            ref.within(name, g[name], v, b)


def test_gradients_against_differences():
    """Of sum(out * weights) by each input, central differences of the plain evaluation in 64 bits around the same point."""
    R, K, N, h = 6, 10, 9, 1e-5
    c = case(R, K, N, "fp16", act="gelu_tanh", gate=True, drop=0.25, grads=True)
    bias = torch.randn(N, dtype=torch.float64).cuda()
    z = c["x"].double() @ c["weight"].double().t() + bias
    c["pre"].copy_(z)
    call(c, True)
    k = ref.kept(R, N, 0.25, SEED, STEP)

    def total(x, w, b, g):
        return float((ref.act("gelu_tanh", x @ w.t() + b)[0] * g * k * c["d_out"].double()).sum())
    args = [c["x"].double(), c["weight"].double(), bias, c["gate"].double()]
    for i, name in enumerate(("d_x", "d_weight", "d_bias", "d_gate")):
        flat = args[i].flatten()
        for at in range(0, flat.numel(), 7):
            two = []
            for s in (h, -h):
                a = [t.clone() for t in args]
                a[i].view(-1)[at] += s
                two.append(total(*a))
            got = float(c[name].flatten()[at])
            # pre is rounded to 2^-11 of itself, the slope's own slope is at most 1.2; sums of up to ten terms of size one
            assert abs(got - (two[0] - two[1]) / (2 * h)) < 2e-2, (name, at)


def test_captured_with_another_step_at_each_replay():
    """The step is read when the graph runs; eager work lies between the replays."""
    c = case(70, 128, 192, drop=0.4, residual=True)
    layer = B.linear(**{k: v for k, v in c.items() if k not in ("step_value", "buffers")})
    work = torch.empty(max(1, B.pt_linear_workspace(layer)[0]), dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        B.pt_linear_out(layer, work)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.pt_linear_out(layer, work)
    seen = []
    for step in (0, 1, 2 ** 40, 1):
        c["step"].fill_(step)
        graph.replay()
        torch.cuda.synchronize()
        ref.within("out", c["out"], *ref.linear(dict(c, step_value=step))["out"])
        seen.append(c["out"].clone())
        B.pt_linear_out(layer, work)
        torch.cuda.synchronize()
        assert torch.equal(seen[-1], c["out"])
    assert torch.equal(seen[1], seen[3]) and not torch.equal(seen[0], seen[1])


def test_grads_captured_and_on_another_stream():
    c = case(300, 256, 384, act="silu", gate=True, drop=0.1, grads=True)
    want = ref.linear_grads(c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(c, True, stream=side)
    for name, (v, b) in want.items():
        ref.within(name, c[name], v, b)
    first = {n: c[n].clone() for n in want}
    layer = B.linear(**{k: v for k, v in c.items() if k not in ("step_value", "buffers")})
    work = torch.empty(B.pt_linear_workspace(layer)[1], dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.pt_linear_grads(layer, work)
    for _ in range(3):
        for n in want:
            c[n].zero_()
        work.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(c[n], first[n]) for n in want)


def test_no_rows():
    c = case(1, 96, 40, grads=True)
    for n in ("x", "d_out", "d_x"):
        c[n] = c[n][:0]
    c["d_weight"].fill_(3.0)
    c["d_bias"].fill_(3.0)
    layer = B.linear(**{k: v for k, v in c.items() if k not in ("step_value", "buffers")})
    assert B.pt_linear_workspace(layer) == (0, 0)
    B.pt_linear_grads(layer)
    torch.cuda.synchronize()
    assert not bool(c["d_weight"].any()) and not bool(c["d_bias"].any())
    assert ref.untouched(*c["buffers"]["d_weight"])
