"""Plain evaluations of the layers before the head, in 64 bits, with the bounds that the GPU's results are held to.

u is the largest relative error of one rounding to the 16-bit type (2^-8 bf16, 2^-11 fp16; of numbers below its normal range, that of the smallest
normal one), E = 2^-24 that of fp32.
"""
import math

import numpy as np
import torch

TYPES = {"bf16": (torch.bfloat16, 2.0 ** -8, 2.0 ** -126), "fp16": (torch.float16, 2.0 ** -11, 2.0 ** -14)}
E = 2.0 ** -24
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]
ACT_ERR = 2.0 ** -15       # of an activation relative to its value, and of its derivative: see `act`


def unit(dt):
    return next((u, t) for d, u, t in TYPES.values() if d == dt)


def rounding(x, dt):
    u, tiny = unit(dt)
    return u * x.abs().clamp(min=tiny)


def place(x, pad=0, shift=0, fill=7.0):
    """-> (buffer, x in it): `pad` elements behind every row, the first `shift` elements behind a 256-byte boundary."""
    rows, width = x.shape
    buf = torch.empty(shift + rows * (width + pad) + 8, dtype=x.dtype, device="cuda")
    buf.view(torch.uint8).fill_(0x47)
    view = buf[shift:shift + rows * (width + pad)].view(rows, width + pad)[:, :width]
    view.copy_(x)
    return buf, view


def untouched(buf, view):
    """Whether nothing between the rows, before or behind them was written."""
    mask = torch.ones(buf.shape, dtype=torch.bool, device=buf.device)
    mask.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(False)
    rest = buf.view(torch.uint8).view(-1, buf.element_size())[mask]
    return bool((rest == 0x47).all())


def mix(x):
    """splitmix64's output function on numpy's 64-bit words."""
    with np.errstate(over="ignore"):
        x = (x ^ (x >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        x = (x ^ (x >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        return x ^ (x >> np.uint64(31))


def kept(rows, width, p, seed, step):
    """What dropout multiplies each element by, in 64 bits on the device."""
    off = min(65535, round(p * 65536))
    if not off:
        return torch.ones(rows, width, dtype=torch.float64, device="cuda")
    phi = np.uint64(0x9E3779B97F4A7C15)
    with np.errstate(over="ignore"):
        key = mix(np.uint64(seed) + np.uint64(step) * phi)
        r, c = np.arange(rows, dtype=np.uint64)[:, None], np.arange(width, dtype=np.uint64)[None, :]
        words = np.uint64((width + 3) // 4)
        z = mix(key + (r * words + c // np.uint64(4) + np.uint64(1)) * phi)
        bits = (z >> (np.uint64(16) * (c % np.uint64(4)))) & np.uint64(0xFFFF)
    return torch.from_numpy(np.where(bits < off, 0.0, 65536.0 / (65536 - off))).cuda()


def act(name, z):
    """act(z) and its derivative in 64 bits.

    In fp32 an activation's relative error is a few E times 1 plus the exponential's argument, which counts up to 100 (beyond it the result is below 1e-38):
    under 450 E < ACT_ERR; the fit of the normal distribution's function adds 2^-18.  A derivative's terms are at most 1.2 with factors as exact,
    but for 1 - sigmoid, which is E off where the other factors are under 40 (beyond that it is 0): 40 E and a few more E, under ACT_ERR."""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "relu":
        return z.clamp(min=0), (z > 0).double()
    if name == "silu":
        f = torch.sigmoid(z)
        return z * f, f * (1 + z * (1 - f))
    if name == "gelu":
        f = 0.5 * torch.special.erfc(-z / math.sqrt(2))
        return z * f, f + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    k, b = math.sqrt(8 / math.pi), 0.044715
    f = torch.sigmoid(k * (z + b * z ** 3))
    return z * f, f + z * f * (1 - f) * k * (1 + 3 * b * z * z)


def within(name, got, want, bound):
    off = (got.double() - want).abs()
    bad = ~(off <= bound)
    assert not bool(bad.any()), (f"{name}: {int(bad.sum())} of {bad.numel()} outside, worst {float((off / bound.clamp(min=1e-300))[bad].max()):.3g} of the bound, "
                                 f"first at {bad.nonzero()[0].tolist()}")


def linear(c):
    """c: dict of arrays and options as binding.linear's.  -> {"out", "pre"}: (value, bound)."""
    x, w = c["x"].double(), c["weight"].double()
    K = x.shape[1]
    dt = c["out"].dtype
    z, big = x @ w.t(), x.abs() @ w.abs().t()
    if c.get("x_scale") is not None:
        s = c["x_scale"].double()[:, None] * c["weight_scale"].double()
        z, big = z * s, big * s
    dz = (K + 64) * E * big + 3 * E * z.abs()
    if c.get("bias") is not None:
        z = z + c["bias"].double()
        dz = dz + E * z.abs()
    y, _ = act(c.get("act", "none"), z)
    dy = 1.2 * dz + ACT_ERR * y.abs() + 1e-17
    k = kept(*y.shape, c.get("drop", 0.0), c.get("seed", 0), c.get("step_value", 0))
    g = c["gate"].double() if c.get("gate") is not None else torch.ones_like(y)
    y, dy = y * g * k, dy * g.abs() * k + 3 * E * (y * g * k).abs()
    if c.get("residual") is not None:
        y = y + c["residual"].double()
        dy = dy + E * y.abs()
    return {"out": (y, dy + rounding(y, dt) * 1.001), "pre": (z, dz + rounding(z, dt) * 1.001)}


def linear_grads(c):
    x, w, e = c["x"].double(), c["weight"].double(), c["d_out"].double()
    dt = c["x"].dtype
    R, N = e.shape
    e = e * kept(R, N, c.get("drop", 0.0), c.get("seed", 0), c.get("step_value", 0))
    g = c["gate"].double() if c.get("gate") is not None else torch.ones_like(e)
    out = {}
    dz = e * g
    ddz = 4 * E * dz.abs()
    if c.get("pre") is not None:
        y, slope = act(c.get("act", "none"), c["pre"].double())
        out["d_gate"] = (e * y, (ACT_ERR + 4 * E) * (e * y).abs() + 1e-17 * e.abs() + rounding(e * y, dt) * 1.001)
        ddz = ACT_ERR * dz.abs() + 4 * E * (dz * slope).abs()
        dz = dz * slope
    out["d_bias"] = (dz.sum(0), None)
    bound = ddz.sum(0) + (R + 64) * E * dz.abs().sum(0)
    out["d_bias"] = (dz.sum(0), bound + rounding(dz.sum(0), dt) * 1.001)
    # up to 32 rows what rounding dz leaves is multiplied as well, and rounded itself
    ddz = ddz + rounding(dz, dt) * (unit(dt)[0] if R <= 32 else 1.0) + unit(dt)[1] * unit(dt)[0]
    for name, a, b, da, n in (("d_x", dz, w, ddz, N), ("d_weight", dz.t(), x, ddz.t(), R)):
        v = a @ b
        bound = da @ b.abs() + (n + 64) * E * (a.abs() @ b.abs())
        out[name] = (v, bound * 1.01 + rounding(v, dt) * 1.001)
    return out


def codes_within(name, codes, scale, y, dy):
    """Codes times scale against y, whose error is dy: half a step of the format, 2^-4 of a number or 2^-10 of the scale below its normal range."""
    top = y.abs().amax(1)
    want = torch.where(top < 2.0 ** -100, 0.0, top / 448)
    within(name + " scale", scale, want, (dy.abs() / y.abs().clamp(min=1e-300)).nan_to_num(0).amax(1).clamp(max=1) * want + 4 * E * want)
    v = codes.view(torch.float8_e4m3fn).double() * scale.double()[:, None]
    y = torch.where(top[:, None] < 2.0 ** -100, 0.0, y)
    within(name, v, y, torch.maximum(2.0 ** -4 * y.abs(), 2.0 ** -10 * want[:, None]) * 1.0001 + dy + 8 * E * y.abs())


def rms(x, residual, gain, eps):
    """-> s, rstd, y and the relative error of the last two."""
    s = x.double() if residual is None else x.double() + residual.double()
    K = s.shape[1]
    rstd = (s.square().mean(1) + eps) ** -0.5
    y = s * rstd[:, None]
    if gain is not None:
        y = y * gain.double()
    return s, rstd, y, (K + 64) * E


def rms_grads(s, rstd, gain, d_y, d_sum):
    """-> {"d_x", "d_gain"}: (value, bound)."""
    dt = s.dtype
    s, k, g = s.double(), rstd.double()[:, None], d_y.double()
    R, K = s.shape
    t = g if gain is None else g * gain.double()
    h = s * k
    c, cb = (t * h).mean(1, keepdim=True), (t * h).abs().mean(1, keepdim=True)
    d = k * (t - h * c)
    bound = k * (8 * E * t.abs() + h.abs() * ((K + 72) * E * cb)) + 4 * E * k * (t.abs() + (h * c).abs())
    if d_sum is not None:
        d = d + d_sum.double()
        bound = bound + E * d.abs()
    v = (g * h).sum(0)
    vb = (R + 72) * E * (g * h).abs().sum(0)
    return {"d_x": (d, bound + rounding(d, dt) * 1.001), "d_gain": (v, vb + rounding(v, dt) * 1.001)}
