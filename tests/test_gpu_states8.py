"""Lists of tensors with states in 8 bits over several steps, against a plain evaluation in fp32 that goes its own way.

The plain evaluation takes the multiplier of the gradients (clip over loss scale) from the list and nothing else: states, codes and weights are its own from
the first step on.  Products, sums and codes are then the same fp32 operations on the same numbers, so the codes have to be equal, all of them; the
weight's quotient may be two units in the last place off, so each step may add 16 e of the magnitudes that enter it (e = 2^-24)."""
import pytest
import torch

from paper_2406_08334_amd import binding as B
from test_gpu_tensors import E, HP, SIZES, List, randoms

gpu = pytest.mark.gpu


class Plain:
    """The update of a list in elementary fp32 operations, from a copy of its arrays."""

    def __init__(self, l):
        self.l, self.w = l, [w.clone() for w in l.w]
        value = lambda c, s: c.clone().view(torch.float8_e4m3fn).float() * s.repeat_interleave(256)[:len(c)]  # noqa: E731
        self.codes = [(m.clone(), v.clone()) for m, v in zip(l.m, l.v)]
        self.m = [value(c, s) for c, s in zip(l.m, l.ms)]
        self.v = [value(c, s).square() for c, s in zip(l.v, l.vs)]
        self.off = [torch.zeros(n, dtype=torch.float64, device="cuda") for n in l.sizes]         # how far the weights may be off by now

    def step(self, t, mult, **hp):
        hp = {**HP, **hp}
        for i, (n, u) in enumerate(zip(self.l.sizes, randoms(self.l.sizes, self.l.seed, t))):
            if not n:
                continue
            g = self.l.g[i].float() * mult
            m = self.m[i] * hp["beta1"] + g * (1.0 - hp["beta1"])
            v = self.v[i] * hp["beta2"] + g * (1.0 - hp["beta2"]) * g
            d = v.sqrt() / (1.0 - hp["beta2"] ** t) ** 0.5 + hp["eps"]
            rate = hp["lr"] / (1.0 - hp["beta1"] ** t)
            keep = 1.0 if i in self.l.no_decay else 1.0 - hp["lr"] * hp["weight_decay"]
            size = self.w[i].abs().double() * keep + rate * (self.m[i].abs() * hp["beta1"] + g.abs() * (1.0 - hp["beta1"])).double() / d.double()
            self.off[i] += 16 * E * size
            self.w[i] = self.w[i] * keep - rate * (m / d)
            (cm, self.m[i]), (cv, r) = (to8(x, torch.from_numpy(k).float().cuda(), lift) for x, k, lift in ((m, u[0], False), (v.sqrt(), u[1], True)))
            self.v[i] = r.square()
            self.codes[i] = cm, cv


def to8(x, u, lift):
    """Codes of x, 256 that share a scale, and the values they stand for."""
    n = len(x)
    x = torch.nn.functional.pad(x, (0, -n % 256)).view(-1, 256)
    u = torch.nn.functional.pad(u, (0, -n % 256)).view(-1, 256)
    big = x.abs().amax(1, keepdim=True)
    there = big >= 2.0 ** -100
    y = x.abs() * torch.where(there, big.reciprocal() * 448.0, 0.0)
    _, e = torch.frexp(y.clamp(min=2.0 ** -6))
    step = torch.exp2((e - 4).float())
    q = (torch.floor(y / step + u) * step).clamp(max=448.0)
    if lift:
        q = torch.where(y > 0, q.clamp(min=2.0 ** -9), q)
    q = torch.where(x < 0, -q, q).to(torch.float8_e4m3fn)
    scale = torch.where(there, big * (1.0 / 448.0), 0.0)
    return q.view(-1)[:n].view(torch.uint8), (q.float() * scale).view(-1)[:n]


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("zero", [True, False])
def test_steps_that_go_on_from_each_other(zero, dtype):
    """From states of zero, which only reach what a run can, and from momentum and variance that know nothing of each other: momenta up to hundreds of
    times the root of the variance beside them, where a code of it decides over the weight's next step."""
    l = List(SIZES + [200_000], 8, dtype, zero=zero, no_decay=(1, 5))
    plain = Plain(l)
    gen = torch.Generator(device="cuda").manual_seed(11)
    for t in range(1, 9):
        for g in l.g:
            g.copy_(torch.randn(g.shape, generator=gen, device="cuda") * 1e-2)
        l.step()
        plain.step(t, B.pt_tensors_report_read(l.list).grad_mult)
        for i, n in enumerate(l.sizes):
            for name, code, want in (("m", l.m[i], plain.codes[i][0]), ("v", l.v[i], plain.codes[i][1])):
                same = (code == want) | ((code | want) & 0x7F == 0)                   # zero has two signs
                assert bool(same.all()), (t, i, name, int((~same).sum()))
            assert bool(((l.w[i].double() - plain.w[i].double()).abs() <= plain.off[i]).all()), (t, i)
    l.close()


# ---- rounding that keeps the mean ----------------------------------------------------------------------

N, SCALE, CODE, UP = 1 << 18, 1e-4, 288.0, 320.0          # elements; a block's scale; their code, and the next one
PULL, SMALL, STEPS = 12.6, 0.4, 20                        # one pull by 0.39 of the distance; many by 0.0125 of it


def mean_is_kept(values, want, steps):
    """values: in codes.  Each step leaves an element one of two codes 32 apart, their spread at most half of that; so the mean of N is off by 16 / sqrt(N) times the root of
    the steps, of which six times are allowed, and 1e-6 for the fp32 operations."""
    return abs(float(values.mean()) - want) <= 6 * 16 * (steps / N) ** 0.5 + 1e-6 * want * steps


@pytest.mark.parametrize("rounding", ["random", "nearest"])
def test_what_the_mean_tells(rounding):
    """On the host: the two tests below hold for rounding at random and fail by ten times their bound for rounding to nearest."""
    gen = torch.Generator().manual_seed(1)

    def one(y):
        return (torch.floor(y / 32 + (torch.rand(N, generator=gen) if rounding == "random" else 0.5))) * 32
    once, many = one(torch.full((N,), CODE + PULL)), torch.full((N,), CODE)
    for _ in range(STEPS):
        many = one(many + SMALL)
    for values, want, steps in ((once, CODE + PULL, 1), (many, CODE + STEPS * SMALL, STEPS)):
        assert mean_is_kept(values, want, steps) == (rounding == "random")
        if rounding == "nearest":
            assert abs(float(values.mean()) - want) > 6 * 1.5 * 16 * (steps / N) ** 0.5


@gpu
@pytest.mark.parametrize("pull,steps", [(PULL, 1), (SMALL, STEPS)])
def test_the_mean_of_what_moves_by_part_of_a_code(pull, steps):
    """Momenta of code 288 beside a block's largest of 448 that stays what it is: beta1 next to 1 and a gradient that pulls each by `pull` codes a step."""
    l = List([N], 8, zero=True, dtype=torch.bfloat16, grad32=True)
    code = lambda x: torch.tensor(x).to(torch.float8_e4m3fn).view(torch.uint8)  # noqa: E731
    l.m[0].copy_(code(CODE).expand(N))
    l.m[0][::256] = code(448.0)
    l.ms[0].fill_(SCALE)
    beta1 = 1.0 - 2.0 ** -9
    # the largest's gradient is its own value: it stays; the others' is theirs and the pull over 1 - beta1
    rest = torch.arange(N, device="cuda") % 256 != 0
    B.pt_tensors_set_state(l.list, 10, 1.0, 0)
    for t in range(steps):
        torch.cuda.synchronize()
        m = l.m[0].view(torch.float8_e4m3fn).float() * l.ms[0].repeat_interleave(256)
        l.g[0].copy_(torch.where(rest, m + pull * SCALE * 2.0 ** 9, m))
        l.step(beta1=beta1, max_norm=0.0)
    torch.cuda.synchronize()
    q = l.m[0].view(torch.float8_e4m3fn).float()[rest].double()
    assert bool((l.ms[0] - SCALE).abs().max() <= 1e-6 * SCALE * steps)
    if steps == 1:
        assert sorted(q.unique().tolist()) == [CODE, UP]
    assert mean_is_kept(q, CODE + steps * pull, steps)
    l.close()


# ---- a gradient whose square is no fp32 number -----------------------------------------------------------

@gpu
@pytest.mark.parametrize("grad32", [False, True])
def test_a_variance_beyond_fp32(grad32):
    """Finite gradients of 1e20 without a clip: the norm is finite, so the step is taken, and the variance is inf in 32 bits.  The weight gets its decay and
    nothing else, as with states in 32 bits; in 8 bits the state stays finite, so that its block comes back."""
    sizes = [700, 300]
    lists = [List(sizes, bits, zero=True, grad32=grad32) for bits in (8, 32)]
    for l in lists:
        l.g[0][5], l.g[0][600], l.g[1][299] = 1e20, -1e20, 3e38
    start = [w.double() for w in lists[0].w]
    for l in lists:
        l.step(max_norm=0.0)
        torch.cuda.synchronize()
        assert B.pt_tensors_report_read(l.list).step == 1
    small, large = lists
    keep = 1.0 - HP["lr"] * HP["weight_decay"]
    for i in range(2):
        assert bool(small.w[i].isfinite().all()) and bool(small.p[i].float().isfinite().all())
        size = start[i].abs() * keep + HP["lr"] * 1.1            # of a first step, which moves a weight by lr at most
        assert bool(((small.w[i].double() - large.w[i].double()).abs() <= 16 * E * size).all())
    for i, k in ((0, 5), (0, 600), (1, 299)):
        assert abs(float(small.w[i][k]) - float(start[i][k]) * keep) <= 2 * E * abs(float(start[i][k]))
    assert bool(large.v[0][5].isinf())
    for _ in range(3):                                           # gradients as usual again
        for l in lists:
            for g in l.g:
                g.fill_(1e-2)
        small.step()
        for i in range(2):
            r = small.v[i].view(torch.float8_e4m3fn).float() * small.vs[i].repeat_interleave(256)[:sizes[i]]
            assert bool(r.square().isfinite().all()) and bool(small.ms[i].isfinite().all())
            assert bool(small.w[i].isfinite().all())
    for l in lists:
        l.check_guards()
        l.close()
