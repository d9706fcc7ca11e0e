"""The layers that a training step has before its head, as measurable cases.

A case is a plain dict; `kind` names the operator:

  linear        out = residual + dropout(act(x W^T + bias) gate) of `rows` x `width` against `outs` x `width`; `bias`, `gate`, `residual`: whether there
                is one; `pre`: z = x W^T + bias is kept for the gradients; `bits` 8: x and weight are e4m3 codes with a scale for each row
  linear_grads  the gradients of x, weight, bias and gate from that of out
  rms           sum = x + residual, y = sum gain / sqrt(mean(sum^2) + eps); `bits` 8: y in e4m3 codes with a scale for each row
  rms_grads     the gradients of sum and gain from those of y and (`residual`) of the sum's other uses
  rows8         rows in 16 or (`src` fp32) 32 bits to e4m3 codes with a scale for each row, as weights are laid out for `linear` of 8 bits
  dropout       out = residual + x m / (1 - p); the gradient is the same call without a residual

`dtype` is the 16-bit type, `drop` the probability of a dropped element, whose random numbers are a function of SEED, STEP and the element's
place alone.  With `own` false everything is computed by elementary torch operations in 32 bits.
"""
import math

import torch

own = False

SEED, STEP = 0x5EED000B, 7
EPS = 1e-5
TOP = 448.0            # largest number of the 8-bit format
PHI = 0x9E3779B97F4A7C15
PARAM_STD = 0.02
GRAD_STD = {"bf16": 1e-3, "fp16": 1.0}       # fp16 gradients carry a loss scale


def _linear(name, rows, width, outs, act="none", dtype="bf16", grads=False, bias=False, gate=False, residual=False, drop=0.0, pre=False, bits=16):
    c = dict(kind="linear_grads" if grads else "linear", rows=rows, width=width, outs=outs, act=act, dtype=dtype, bias=bias, gate=gate,
             residual=residual, drop=drop, pre=pre, bits=bits)
    return dict(c, name=name) if name else c


def _rows(name, kind, rows, width, dtype="bf16", **more):
    c = dict(kind=kind, rows=rows, width=width, dtype=dtype, **more)
    return dict(c, name=name) if name else c


def listed():
    return [
        # serving: one token through the gated product of a 7B block; reading the weight is all there is
        _linear("linear_one_token", 1, 4096, 11008, "silu", gate=True),
        # a micro-batch through the first product of a 48-block model's MLP, kept for the gradients
        _linear("linear_gpt2_xl", 8192, 1600, 6400, "gelu_tanh", bias=True, pre=True),
        # the same at 7B widths in 8 bits, as evaluation or generation of long prompts takes it
        _linear("linear8_llama_7b", 8192, 4096, 11008, "none", bits=8),
        # odd widths, as in a test model: rows at any 2-byte address; the second product of an MLP, with dropout and residual, and back
        _linear("grads_odd_width", 1531, 771, 3083, "gelu", "fp16", grads=True, bias=True, drop=0.1),
        # training at 7B widths: the gated product's gradients; the largest
        _linear("grads_llama_7b", 8192, 4096, 11008, "silu", grads=True, gate=True),
        # serving: one token's normalisation, with the residual's addition, for a product in 8 bits; a launch decides
        _rows("rms8_one_token", "rms", 1, 4096, residual=True, bits=8),
        # a micro-batch at 7B widths
        _rows("rms_grads_llama_7b", "rms_grads", 8192, 4096, residual=True),
        # the largest prompt at 13B widths, for products in 8 bits
        _rows("rms8_llama_13b", "rms", 16384, 5120, "fp16", residual=True, bits=8),
        # weights of a small product, rows of an odd width
        _rows("rows8_odd_width", "rows8", 1000, 771, src="16"),
        # master weights of a 13B product
        _rows("rows8_llama_13b", "rows8", 13824, 5120, src="32"),
        # the embedding of a short sequence; a launch decides
        _rows("dropout_short", "dropout", 48, 771, "fp16", residual=False, drop=0.1),
        # a micro-batch of the 48-block model's residual stream
        _rows("dropout_gpt2_xl", "dropout", 32768, 1600, residual=True, drop=0.1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    n = _log_int(rng, lo, hi)
    return (n + 63) // 64 * 64 if rng.random() < 0.6 else n


def draw(rng):
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    kind = rng.choice(["linear", "linear", "linear_grads", "rms", "rms_grads", "rows8", "dropout"])
    some = lambda p: rng.random() < p  # noqa: E731
    drop = rng.choice([0.0, 0.0, round(rng.uniform(0.01, 0.6), 3)])
    while kind.startswith("linear"):
        bits = rng.choice([16, 16, 8]) if kind == "linear" else 16
        c = _linear("", _log_int(rng, 1, 16384), _width(rng, 64, 13824), _width(rng, 64, 13824), rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]),
                    dtype, kind == "linear_grads", some(0.5), some(0.3), some(0.4), drop, some(0.5), bits)
        if c["rows"] * c["width"] * c["outs"] <= 8192 * 4096 * 11008:
            return c
    rows, width = _log_int(rng, 1, 32768), _width(rng, 64, 16384)
    rows = min(rows, 32768 * 5120 // width)
    if kind == "rows8":
        return _rows("", kind, rows, width, dtype, src=rng.choice(["16", "32"]))
    if kind == "dropout":
        return _rows("", kind, rows, width, dtype, residual=some(0.5), drop=drop or 0.1)
    return _rows("", kind, rows, width, dtype, residual=some(0.7), **({"bits": rng.choice([8, 16])} if kind == "rms" else {}))


# ---- inputs --------------------------------------------------------------------------------------------

class State:
    """Arrays of a case; those that it has not are None."""
    x = weight = bias = gate = residual = pre = out = x_scale = weight_scale = d_out = d_x = d_weight = d_bias = d_gate = None
    gain = sum = rstd = y = y_scale = d_y = d_sum = d_gain = codes = scale = None


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float16


def prepare(case, seed):
    s = State()
    s.case = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    normal = lambda std, *shape: torch.empty(shape, device="cuda").normal_(0.0, std, generator=gen)  # noqa: E731
    (_prepare_linear if case["kind"].startswith("linear") else _prepare_rows)(s, case, normal, _type(case))
    s.step = torch.full((1,), STEP, dtype=torch.int64, device="cuda")
    if own:
        from paper_2406_08334_amd import binding as B
        s.B = B
        kind = case["kind"]
        if kind.startswith("linear"):
            s.layer = B.linear(s.x, s.weight, s.out, bias=s.bias, gate=s.gate, residual=s.residual, pre=s.pre, act=case["act"], drop=case["drop"],
                               seed=SEED, step=s.step, x_scale=s.x_scale, weight_scale=s.weight_scale, d_out=s.d_out, d_x=s.d_x,
                               d_weight=s.d_weight, d_bias=s.d_bias, d_gate=s.d_gate)
            s.work = torch.empty(B.pt_linear_workspace(s.layer)[kind == "linear_grads"], dtype=torch.uint8, device="cuda")
        elif kind.startswith("rms"):
            s.norm = B.rms(s.x, s.y, gain=s.gain, residual=s.residual, sum=s.sum, rstd=s.rstd, y_scale=s.y_scale, eps=EPS, d_y=s.d_y,
                           d_sum=s.d_sum, d_x=s.d_x, d_gain=s.d_gain)
            s.work = torch.empty(B.pt_rms_workspace(s.norm), dtype=torch.uint8, device="cuda")
        elif kind == "rows8":
            s.rows = B.rows8(s.x, s.codes, s.scale)
        else:
            s.dropped = B.dropout(s.x, s.out, case["drop"], SEED, step=s.step, residual=s.residual)
    return s


def _prepare_linear(s, case, normal, dt):
    """Activations as a normalisation leaves them, one channel in 64 ten times as large; for the gradients what the product kept, and the
    activations of a gate's other branch."""
    R, K, N = case["rows"], case["width"], case["outs"]
    x, w = normal(1.0, R, K), normal(PARAM_STD, N, K)
    x[:, ::64] *= 10.0
    s.bias = normal(PARAM_STD, N).to(dt) if case["bias"] else None
    s.gate = normal(1.0, R, N).to(dt) if case["gate"] else None
    grads = case["kind"] == "linear_grads"
    s.residual = normal(1.0, R, N).to(dt) if case["residual"] and not grads else None
    if case["bits"] == 8:
        (s.x, s.x_scale), (s.weight, s.weight_scale) = _to8(x), _to8(w)
    else:
        s.x, s.weight = x.to(dt), w.to(dt)
    s.out = None if grads else torch.empty(R, N, dtype=dt, device="cuda")
    if grads:
        s.pre = (s.x @ s.weight.t() + (0 if s.bias is None else s.bias)).to(dt) if case["act"] != "none" or s.gate is not None else None
        s.d_out = normal(GRAD_STD[case["dtype"]], R, N).to(dt)
        s.d_x, s.d_weight = torch.empty_like(s.x), torch.empty_like(s.weight)
        s.d_bias, s.d_gate = (None if a is None else torch.empty_like(a) for a in (s.bias, s.gate))
    elif case["pre"]:
        s.pre = torch.empty(R, N, dtype=dt, device="cuda")


def _prepare_rows(s, case, normal, dt):
    """A residual stream whose rows differ in size, a branch that is added to it, gains around 1."""
    R, K, kind = case["rows"], case["width"], case["kind"]
    if kind == "rows8":
        s.x = normal(PARAM_STD, R, K).to(torch.float32 if case["src"] == "32" else dt)
        s.codes, s.scale = torch.empty(R, K, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(R, device="cuda")
        return
    size = torch.exp(normal(0.7, R, 1))
    s.x = (normal(1.0, R, K) * size).to(dt)
    if case["residual"] and kind != "rms_grads":
        s.residual = (normal(2.0, R, K) * size).to(dt)
    if kind == "dropout":
        s.out = torch.empty_like(s.x)
        return
    s.gain = (1.0 + normal(0.1, K)).to(dt)
    if kind == "rms_grads":
        s.rstd = 1.0 / torch.sqrt(s.x.float().square().mean(1) + EPS)
        s.d_y = normal(GRAD_STD[case["dtype"]], R, K).to(dt)
        s.d_sum = normal(GRAD_STD[case["dtype"]], R, K).to(dt) if case["residual"] else None
        s.d_x, s.d_gain = torch.empty_like(s.x), torch.empty_like(s.gain)
        return
    s.rstd = torch.empty(R, device="cuda")
    s.sum = torch.empty_like(s.x) if case["residual"] else None
    if case["bits"] == 8:
        s.y, s.y_scale = torch.empty(R, K, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(R, device="cuda")
    else:
        s.y = torch.empty_like(s.x)


# ---- one pass ----------------------------------------------------------------------------------------

def run(s):
    (_own if own else PLAIN[s.case["kind"]])(s)
    return {k: getattr(s, k) for k in OUTPUTS[s.case["kind"]]}


OUTPUTS = {"linear": ("out", "pre"), "linear_grads": ("d_x", "d_weight", "d_bias", "d_gate"), "rms": ("y", "y_scale", "sum", "rstd"),
           "rms_grads": ("d_x", "d_gain"), "rows8": ("codes", "scale"), "dropout": ("out",)}


def _own(s):
    kind = s.case["kind"]
    if kind == "linear":
        s.B.pt_linear_out(s.layer, s.work)
    elif kind == "linear_grads":
        s.B.pt_linear_grads(s.layer, s.work)
    elif kind == "rms":
        s.B.pt_rms_norm(s.norm)
    elif kind == "rms_grads":
        s.B.pt_rms_grads(s.norm, s.work)
    elif kind == "rows8":
        s.B.pt_rows8(s.rows)
    else:
        s.B.pt_dropout(s.dropped)


def _to8(x):
    """Rows in e4m3 codes and their scales: the largest magnitude becomes the format's largest number."""
    big = x.abs().amax(1)
    there = big >= 2.0 ** -100
    codes = x * torch.where(there, TOP / big.clamp(min=2.0 ** -100), 0.0)[:, None]
    return codes.clamp(-TOP, TOP).to(torch.float8_e4m3fn), torch.where(there, big / TOP, 0.0)


def _mix(x):
    """splitmix64's output function on 64-bit words; right shifts of signed words made logical by a mask."""
    x = (x ^ ((x >> 30) & ((1 << 34) - 1))) * _signed(0xBF58476D1CE4E5B9)
    x = (x ^ ((x >> 27) & ((1 << 37) - 1))) * _signed(0x94D049BB133111EB)
    return x ^ ((x >> 31) & ((1 << 33) - 1))


def _signed(x):
    x &= (1 << 64) - 1
    return x - (1 << 64) if x >> 63 else x


def _kept(rows, width, p, step):
    """What each element is multiplied by: 0, or 1 / (1 - p) with p in whole 65536ths.  Four elements of a row share a 64-bit word."""
    words = -(-width // 4)
    key = _mix(step * _signed(PHI) + SEED)
    z = _mix(torch.arange(1, rows * words + 1, device="cuda") * _signed(PHI) + key)
    bits = torch.stack([(z >> k) & 0xFFFF for k in (0, 16, 32, 48)], 1).view(rows, words * 4)[:, :width]
    off = min(65535, round(p * 65536))
    return torch.where(bits >= off, 65536.0 / (65536 - off), 0.0)


def _act(name, z):
    """act(z) and its derivative."""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "relu":
        return z.clamp(min=0), (z > 0).to(z.dtype)
    if name == "silu":
        f = 1 / (1 + torch.exp(-z))
        return z * f, f * (1 + z * (1 - f))
    if name == "gelu":
        f = 0.5 * torch.special.erfc(z * -math.sqrt(0.5))
        return z * f, f + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    a = math.sqrt(8 / math.pi)                   # 0.5 (1 + tanh(u)) = 1 / (1 + exp(-2 u))
    f = 1 / (1 + torch.exp(-a * (z + 0.044715 * z * z * z)))
    return z * f, f + z * f * (1 - f) * a * (1 + 3 * 0.044715 * z * z)


def _plain_linear(s):
    c = s.case
    z = s.x.float() @ s.weight.float().t()
    if s.x_scale is not None:
        z = z * s.x_scale[:, None] * s.weight_scale
    if s.bias is not None:
        z = z + s.bias.float()
    if s.pre is not None:
        s.pre = z.to(s.pre.dtype)
    y = _act(c["act"], z)[0]
    if s.gate is not None:
        y = y * s.gate.float()
    if c["drop"]:
        y = y * _kept(c["rows"], c["outs"], c["drop"], s.step)
    if s.residual is not None:
        y = y + s.residual.float()
    s.out = y.to(s.out.dtype)


def _plain_linear_grads(s):
    c, dt = s.case, s.x.dtype
    e = s.d_out.float()
    if c["drop"]:
        e = e * _kept(c["rows"], c["outs"], c["drop"], s.step)
    dz = e
    if s.pre is not None:
        y, dy = _act(c["act"], s.pre.float())
        dz = e * dy
        if s.gate is not None:
            s.d_gate = (e * y).to(dt)
            dz = dz * s.gate.float()
    s.d_x = (dz @ s.weight.float()).to(dt)
    s.d_weight = (dz.t() @ s.x.float()).to(dt)
    if s.bias is not None:
        s.d_bias = dz.sum(0).to(dt)


def _plain_rms(s):
    x = s.x.float()
    if s.residual is not None:
        x = x + s.residual.float()
        s.sum = x.to(s.x.dtype)
    s.rstd = 1.0 / torch.sqrt(x.square().mean(1) + EPS)
    y = x * s.rstd[:, None] * s.gain.float()
    if s.y_scale is None:
        s.y = y.to(s.x.dtype)
    else:
        s.y, s.y_scale = _to8(y)


def _plain_rms_grads(s):
    x, g = s.x.float() * s.rstd[:, None], s.d_y.float()
    t = g * s.gain.float()
    d = (t - x * (t * x).mean(1, keepdim=True)) * s.rstd[:, None]
    if s.d_sum is not None:
        d = d + s.d_sum.float()
    s.d_x = d.to(s.x.dtype)
    s.d_gain = (g * x).sum(0).to(s.gain.dtype)


def _plain_rows8(s):
    s.codes, s.scale = _to8(s.x.float())


def _plain_dropout(s):
    c = s.case
    y = s.x.float() * _kept(c["rows"], c["width"], c["drop"], s.step)
    if s.residual is not None:
        y = y + s.residual.float()
    s.out = y.to(s.x.dtype)


PLAIN = {"linear": _plain_linear, "linear_grads": _plain_linear_grads, "rms": _plain_rms, "rms_grads": _plain_rms_grads,
         "rows8": _plain_rows8, "dropout": _plain_dropout}


# ---- what a pass cannot do without --------------------------------------------------------------------

def work(case):
    R, K, kind = case["rows"], case["width"], case["kind"]
    if kind.startswith("linear"):
        N = case["outs"]
        if kind == "linear":
            arrays = 1 + case["gate"] + case["residual"] + case["pre"]
            return {"bytes": case["bits"] // 8 * (R + N) * K + 2 * R * N * arrays, "flops": 2 * R * N * K}
        arrays = 1 + 2 * case["gate"] + (case["act"] != "none" or case["gate"])
        return {"bytes": 4 * (R + N) * K + 2 * R * N * arrays, "flops": 4 * R * N * K}
    n = R * K
    if kind == "rms":
        return {"bytes": n * (2 + (4 if case["residual"] else 0) + case["bits"] // 8), "flops": 6 * n}
    if kind == "rms_grads":
        return {"bytes": n * (8 if case["residual"] else 6), "flops": 10 * n}
    if kind == "rows8":
        return {"bytes": n * (int(case["src"]) // 8 + 1), "flops": 2 * n}
    return {"bytes": n * (6 if case["residual"] else 4), "flops": 2 * n}


# ---- the same in 64 bits ------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _linear64, "linear_grads": _linear_grads64, "rms": _rms64, "rms_grads": _rms_grads64, "rows8": _rows64, "dropout": _dropout64}[
        case["kind"]](s, case)


def _mask64(case, width):
    """Row block by row block, in numbers of the definition: the word of elements 4 i to 4 i + 3 of row r has number r ceil(width / 4) + i."""
    if not case["drop"]:
        return 1.0
    rows, words, off = case["rows"], (width + 3) // 4, min(65535, round(case["drop"] * 65536))
    key = int(_mix(torch.tensor(_signed(SEED + STEP * PHI))))
    out = torch.zeros(rows, width, dtype=torch.float64, device="cuda")
    col = torch.arange(width, device="cuda")
    for a in range(0, rows, 2048):
        row = torch.arange(a, min(rows, a + 2048), device="cuda")[:, None]
        bits = (_mix((row * words + col // 4 + 1) * _signed(PHI) + key) >> (16 * (col % 4))) & 0xFFFF
        out[a:a + 2048] = torch.where(bits < off, 0.0, 65536.0 / (65536 - off)).double()
    return out


def _act64(name, z):
    if name == "none":
        return z
    if name == "relu":
        return torch.relu(z)
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu":
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0))
    return z * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3))


def _linear64(s, case):
    x, w = s.x.double(), s.weight.double()
    if s.x_scale is not None:
        x, w = x * s.x_scale.double()[:, None], w * s.weight_scale.double()[:, None]
    z = x @ w.t()
    if s.bias is not None:
        z += s.bias.double()
    y = _act64(case["act"], z)
    if s.gate is not None:
        y = y * s.gate.double()
    y = y * _mask64(case, case["outs"])
    if s.residual is not None:
        y = y + s.residual.double()
    return {"out": y, "pre": z if case["pre"] else None}


def _linear_grads64(s, case):
    e = s.d_out.double() * _mask64(case, case["outs"])
    d_gate = None
    if s.pre is not None:
        z = s.pre.double().requires_grad_(True)
        with torch.enable_grad():
            y = _act64(case["act"], z)
            (slope,) = torch.autograd.grad(y.sum(), z)
        if s.gate is not None:
            d_gate = e * y.detach()
            slope = slope * s.gate.double()
        e = e * slope
    return {"d_x": e @ s.weight.double(), "d_weight": e.t() @ s.x.double(), "d_bias": None if s.bias is None else e.sum(0), "d_gate": d_gate}


def _codes64(y):
    scale = y.abs().amax(1) / TOP
    return y / scale.clamp(min=1e-300)[:, None], scale


def _rms64(s, case):
    x = s.x.double() if s.residual is None else s.x.double() + s.residual.double()
    rstd = (x.square().mean(1) + EPS) ** -0.5
    y = x * rstd[:, None] * s.gain.double()
    y, scale = _codes64(y) if case["bits"] == 8 else (y, None)
    return {"y": y, "y_scale": scale, "sum": x if s.sum is not None else None, "rstd": rstd}


def _rms_grads64(s, case):
    x, g, rstd = s.x.double(), s.d_y.double(), s.rstd.double()[:, None]
    t = g * s.gain.double()
    d = rstd * t - x * rstd ** 3 * (t * x).sum(1, keepdim=True) / case["width"]
    return {"d_x": d if s.d_sum is None else d + s.d_sum.double(), "d_gain": (g * x * rstd).sum(0)}


def _rows64(s, case):
    codes, scale = _codes64(s.x.double())
    return {"codes": codes, "scale": scale}


def _dropout64(s, case):
    y = s.x.double() * _mask64(case, case["width"])
    return {"out": y if s.residual is None else y + s.residual.double()}
