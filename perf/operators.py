"""The operators that a training step has next to its chunks, as measurable cases.

A case is a plain dict; `kind` names the operator:

  head   softmax cross entropy of `rows` hidden states of `width` against a head of `vocab` rows, without keeping the logits; with
         `grad` the gradients of both as well.  `ignored`: the share of rows without a target
  adamw  one AdamW step over a list of tensors: gradient norm, clipping, update.  `bits`: width of the two states; `model` / `hidden` /
         `mlp` / `blocks` / `vocab`: the tensors; `packed`: the tensors lie back to back, at any alignment, as in one flat buffer;
         `grad32`: fp32 gradients; `plain`: no 16-bit copy of the parameters

`dtype` is the 16-bit type.  With `own` false everything is computed by elementary torch operations in 32 bits.
"""
import math

import torch

own = False

HP = dict(lr=1e-4, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1, max_norm=1.0)
STEP0 = 100            # updates applied before the measured one: moments that have settled
SIGMA = 65536.0        # loss scale of fp16 gradients
SEED = 0x5EED0008      # of the stochastic rounding of 8-bit states
GRAD_STD = 1e-3
PARAM_STD = 0.02
BLOCK = 256            # elements that share a scale
TOP = 448.0            # largest number of the 8-bit format
PHI = 0x9E3779B97F4A7C15


def listed():
    return [
        # serving: the log-probability of one token under the 48-block model's head; reading the weight is all there is
        dict(name="loss_one_row", kind="head", rows=1, width=1600, vocab=50257, dtype="bf16", grad=False, ignored=0.0),
        # a test-sized model: few rows, an odd vocabulary; launches decide
        dict(name="grad_48_rows", kind="head", rows=48, width=256, vocab=5003, dtype="fp16", grad=True, ignored=0.1),
        # evaluation over 4096 tokens at the widths of the 7B state: the loss alone
        dict(name="loss_llama_7b", kind="head", rows=4096, width=4096, vocab=32000, dtype="bf16", grad=False, ignored=0.0),
        # a micro-batch of the 48-block model
        dict(name="grad_gpt2_xl", kind="head", rows=8192, width=1600, vocab=50257, dtype="bf16", grad=True, ignored=0.0),
        # fine-tuning at 7B widths: a quarter of the rows are prompt or padding
        dict(name="grad_llama_7b", kind="head", rows=8192, width=4096, vocab=32000, dtype="bf16", grad=True, ignored=0.25),
        # odd widths: rows at any 2-byte address, no size a multiple of anything
        dict(name="grad_odd_width", kind="head", rows=1531, width=771, vocab=50257, dtype="fp16", grad=True, ignored=0.05),
        # the largest: 16384 rows at 13B widths
        dict(name="grad_llama_13b", kind="head", rows=16384, width=5120, vocab=32000, dtype="fp16", grad=True, ignored=0.0),
        # one small block of 0.8 M parameters, 12 tensors: an adapter or a test model; launches decide
        dict(name="adamw32_block_h256", kind="adamw", bits=32, model="gpt2_block", hidden=256, mlp=1024, blocks=1, vocab=0, dtype="bf16"),
        # odd widths back to back in flat buffers, as gradients come out of a bucket: 2- and 4-byte aligned tensors
        dict(name="adamw32_odd_widths", kind="adamw", bits=32, model="gpt2", hidden=771, mlp=3083, blocks=4, vocab=50257, dtype="bf16",
             packed=True),
        # 8-bit states of an 8-block model, 330 M parameters
        dict(name="adamw8_gpt2_8", kind="adamw", bits=8, model="gpt2", hidden=1600, mlp=6400, blocks=8, vocab=50257, dtype="bf16"),
        # two blocks, embedding and head at 7B widths, fp16 gradients under a loss scale
        dict(name="adamw32_llama_fp16", kind="adamw", bits=32, model="llama", hidden=4096, mlp=11008, blocks=2, vocab=32000, dtype="fp16"),
        # all 48 blocks with 8-bit states: the largest list
        dict(name="adamw8_gpt2_xl", kind="adamw", bits=8, model="gpt2", hidden=1600, mlp=6400, blocks=48, vocab=50257, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    if rng.random() < 0.55:
        while True:
            width = _log_int(rng, 64, 5120)
            if rng.random() < 0.7:
                width = (width + 31) // 32 * 32
            c = dict(kind="head", rows=_log_int(rng, 1, 16384), width=width, vocab=rng.choice([_log_int(rng, 500, 131072), 32000, 50257]),
                     dtype=dtype, grad=rng.random() < 0.7, ignored=rng.choice([0.0, 0.0, 0.1, 0.5]))
            if c["rows"] * c["width"] * c["vocab"] <= 16384 * 5120 * 32000 and 3072 not in (c["rows"], c["width"], c["vocab"]):
                return c
    most = 1_500_000_000
    target = _log_int(rng, 500_000, most)
    while True:
        model = rng.choice(["gpt2_block", "gpt2", "llama"])
        vocab = 0 if model == "gpt2_block" else rng.choice([_log_int(rng, 200, 50257), 32000, 50257])
        hidden = max(64, min(5120, int(math.sqrt(target / rng.uniform(13, 60)))))
        if rng.random() < 0.5:
            hidden = (hidden + 63) // 64 * 64
        mlp = 4 * hidden if model != "llama" else int(2.7 * hidden)
        c = dict(kind="adamw", model=model, hidden=hidden, mlp=mlp, blocks=1, vocab=vocab, dtype=dtype)
        if model != "gpt2_block":
            one, two = (sum(n for n, _ in _tensors(dict(c, blocks=b))) for b in (1, 2))
            c["blocks"] = max(1, min(48, (target - one) // (two - one) + 1))
        n = sum(n for n, _ in _tensors(c))
        if target / 4 <= n <= most and 3072 not in (hidden, mlp, 3 * hidden):
            break
    c["bits"] = rng.choice([8, 32]) if n <= 700_000_000 else 8
    if c["bits"] == 32 and rng.random() < 0.4:
        c["packed"] = True
    if rng.random() < 0.2:
        c["grad32"] = True
    if rng.random() < 0.15:
        c["plain"] = True
    return c


def _tensors(case):
    """(elements, kept out of the weight decay) of every tensor."""
    h, f, v = case["hidden"], case["mlp"], case["vocab"]
    if case["model"] == "llama":
        block = [(h * h, False)] * 4 + [(h * f, False)] * 3 + [(h, True)] * 2
        return [(v * h, False)] + block * case["blocks"] + [(h, True), (v * h, False)]
    block = [(h, True), (h, True), (3 * h * h, False), (3 * h, True), (h * h, False), (h, True), (h, True), (h, True), (h * f, False), (f, True),
             (f * h, False), (h, True)]
    if case["model"] == "gpt2_block":
        return block * case["blocks"]
    return [(v * h, False), (1024 * h, False)] + block * case["blocks"] + [(h, True), (h, True)]


# ---- inputs --------------------------------------------------------------------------------------------

class State:
    def __del__(self):
        if getattr(self, "list", None) is not None:
            self.B.pt_tensors_destroy(self.list)


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float16


def prepare(case, seed):
    s = State()
    s.case = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    (_prepare_head if case["kind"] == "head" else _prepare_adamw)(s, case, gen)
    if own:
        from paper_2406_08334_amd import binding as B
        s.B = B
        if case["kind"] == "head":
            s.head = B.head(s.hidden, s.weight, s.target, s.loss, row_scale=s.scale, d_hidden=s.d_hidden, d_weight=s.d_weight)
            s.work = torch.empty(B.pt_head_workspace(s.head)[1], dtype=torch.uint8, device="cuda")
        else:
            dt = B.PT_BF16 if case["dtype"] == "bf16" else B.PT_FP16
            s.list = B.pt_tensors_create(dt, [
                B.tensor(grad=s.g[a:a + n], master=s.w[a:a + n], param16=None if s.p is None else s.p[a:a + n], m=s.m[a:a + n], v=s.v[a:a + n],
                         m_scale=None if s.ms is None else s.ms[a // BLOCK:], v_scale=None if s.vs is None else s.vs[a // BLOCK:], no_decay=nd)
                for a, (n, nd) in zip(s.at, s.sizes)], case["bits"], None if s.sigma == 1.0 else B.pt_scaler_cfg(SIGMA, 2.0, 0.5, 1 << 30, 0), SEED)
            B.pt_tensors_set_state(s.list, STEP0, s.sigma, 0)
            s.hp = B.hparams(**HP)
    return s


def _prepare_head(s, case, gen):
    """Hidden states with a normalisation's spread that lean towards their target, some a little and some a lot; targets that repeat as
    words do.  The scale of a row is that of a mean over the rows that count, times the loss scale in fp16."""
    R, d, V = case["rows"], case["width"], case["vocab"]
    dt = _type(case)
    s.weight = torch.empty(V, d, device="cuda").normal_(0.0, PARAM_STD, generator=gen).to(dt)
    u = torch.rand(R, generator=gen, device="cuda")
    s.target = (u * u * V).long().clamp_(max=V - 1)
    lean = torch.rand(R, 1, generator=gen, device="cuda") * (12.0 / (PARAM_STD * PARAM_STD * d))
    s.hidden = (torch.randn(R, d, generator=gen, device="cuda") + lean * s.weight[s.target].float()).to(dt)
    off = torch.rand(R, generator=gen, device="cuda") < case["ignored"]
    s.target[off] = -100
    n = (s.target >= 0).sum().clamp(min=1)
    s.scale = ((SIGMA if dt == torch.float16 else 1.0) / n).float().expand(R).contiguous()
    s.loss = torch.empty(R, device="cuda")
    s.d_hidden = torch.empty_like(s.hidden) if case["grad"] else None
    s.d_weight = torch.empty_like(s.weight) if case["grad"] else None


def _prepare_adamw(s, case, gen):
    """Master weights, states and gradients of a run that has been going on.  Tensors start at multiples of BLOCK elements of flat buffers
    (zero between them), or back to back."""
    dt = _type(case)
    s.sizes = _tensors(case)
    s.at, pos = [], 0
    for n, _ in s.sizes:
        s.at.append(pos)
        pos += n if case.get("packed") else -(-n // BLOCK) * BLOCK
    s.n = pos
    full = lambda std: torch.empty(pos, device="cuda").normal_(0.0, std, generator=gen)  # noqa: E731
    s.w = full(PARAM_STD)
    s.m, s.v = full(0.3 * GRAD_STD), full(GRAD_STD)
    s.sigma = SIGMA if case["dtype"] == "fp16" and not case.get("grad32") else 1.0
    s.g = full(GRAD_STD).mul_(s.sigma).to(torch.float32 if case.get("grad32") else dt)
    if not case.get("packed"):
        real = torch.zeros(pos, dtype=torch.bool, device="cuda")
        for a, (n, _) in zip(s.at, s.sizes):
            real[a:a + n] = True
        for x in (s.w, s.m, s.v, s.g):
            x *= real
    s.ms = s.vs = None
    if case["bits"] == 8:
        s.v.abs_()
        s.ms, s.vs = (x.view(-1, BLOCK).abs().amax(1) / TOP for x in (s.m, s.v))
        s.m, s.v = ((x.view(-1, BLOCK) / k.clamp(min=1e-30)[:, None]).clamp_(-TOP, TOP).view(-1).to(torch.float8_e4m3fn)
                    for x, k in ((s.m, s.ms), (s.v, s.vs)))
    else:
        s.v.square_()
    s.p = None if case.get("plain") else s.w.to(dt)
    s.t = STEP0


# ---- one pass ----------------------------------------------------------------------------------------

def run(s):
    if s.case["kind"] == "head":
        if own:
            s.B.pt_head_loss(s.head, s.work)
        else:
            _head(s)
        return {"loss": s.loss, "d_hidden": s.d_hidden, "d_weight": s.d_weight}
    if own:
        s.B.pt_tensors_grad_sqnorm(s.list)
        s.B.pt_tensors_adamw_step(s.list, s.hp)
    else:
        _adamw(s)
    return {"w": s.w, "p": s.p, "m": s.m, "v": s.v, "m_scale": s.ms, "v_scale": s.vs}


def _head(s):
    h, w = s.hidden.float(), s.weight.float()
    there = s.target >= 0
    at = s.target.clamp(min=0)[:, None]
    z = h @ w.t()
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    lse = top + torch.log(total)
    s.loss = torch.where(there, (lse - z.gather(1, at))[:, 0], 0.0)
    if s.d_hidden is None:
        return
    g = e / total
    g.scatter_(1, at, torch.expm1(z.gather(1, at) - lse))
    g = torch.where(there[:, None], g * s.scale[:, None], 0.0)
    s.d_hidden = (g @ w).to(s.hidden.dtype)
    s.d_weight = (g.t() @ h).to(s.weight.dtype)


def _mix(x):
    """splitmix64's output function on 64-bit words; right shifts of signed words made logical by a mask."""
    x = (x ^ ((x >> 30) & ((1 << 34) - 1))) * _signed(0xBF58476D1CE4E5B9)
    x = (x ^ ((x >> 27) & ((1 << 37) - 1))) * _signed(0x94D049BB133111EB)
    return x ^ ((x >> 31) & ((1 << 33) - 1))


def _signed(x):
    x &= (1 << 64) - 1
    return x - (1 << 64) if x >> 63 else x


def _key(t):
    """The key of an update's random numbers: that of the list's seed and the update's number."""
    return int(_mix(torch.tensor(_signed((SEED + t * PHI) & ((1 << 64) - 1)))))


def _random(n, t):
    """16 random bits for each element's first state and for its second, as numbers in (0, 1): those of elements 2i and 2i + 1 lie in one
    64-bit word, a function of i alone."""
    z = _mix(torch.arange(1, n // 2 + 1, device="cuda") * _signed(PHI) + _key(t))
    part = lambda k: torch.stack(((z >> k) & 0xFFFF, (z >> (k + 32)) & 0xFFFF), 1).view(-1)  # noqa: E731
    return [(part(k).float() + 0.5) / 65536 for k in (0, 16)]


def _to8(x, u, lift):
    """Blocks of x in 8 bits: values of the format (3 bits behind the leading one down to 2^-6, steps of 2^-9 below), rounded up with the
    probability that keeps the mean, and the blocks' scales.  lift: what is not zero stays at the smallest number at least."""
    x = x.view(-1, BLOCK)
    big = x.abs().amax(1)
    there = (big >= 2.0 ** -100)[:, None]
    y = x.abs() * torch.where(there, TOP / big[:, None], 0.0)
    step = (((y.view(torch.int32) >> 23) - 127).clamp(min=-6) + 124 << 23).view(torch.float32)
    q = (torch.floor(y / step + u.view(-1, BLOCK)) * step).clamp(max=TOP)
    if lift:
        q = torch.where((x > 0) & there, q.clamp(min=2.0 ** -9), q)
    return torch.where(x < 0, -q, q).view(-1).to(torch.float8_e4m3fn), torch.where(there[:, 0], big / TOP, 0.0)


def _adamw(s):
    g = s.g.float()
    norm = torch.sqrt((g / s.sigma).square().sum())
    mult = torch.clamp(HP["max_norm"] / (norm + 1e-6), max=1.0) / s.sigma
    s.t += 1
    m, v = s.m.float(), s.v.float()
    if s.ms is not None:
        m = (m.view(-1, BLOCK) * s.ms[:, None]).view(-1)
        v = (v.view(-1, BLOCK) * s.vs[:, None]).view(-1).square()
    g = g * mult
    m = HP["beta1"] * m + (1.0 - HP["beta1"]) * g
    v = HP["beta2"] * v + (1.0 - HP["beta2"]) * g * g
    d = torch.sqrt(v) / math.sqrt(1.0 - HP["beta2"] ** s.t) + HP["eps"]
    lengths = torch.tensor([b - a for a, b in zip(s.at, s.at[1:] + [s.n])], device="cuda")
    keep = torch.tensor([1.0 if nd else 1.0 - HP["lr"] * HP["weight_decay"] for _, nd in s.sizes], device="cuda")
    s.w = s.w * torch.repeat_interleave(keep, lengths, output_size=s.n) - HP["lr"] / (1.0 - HP["beta1"] ** s.t) * m / d
    if s.p is not None:
        s.p = s.w.to(s.p.dtype)
    if s.ms is None:
        s.m, s.v = m, v
        return
    u, uv = _random(s.n, s.t)
    s.m, s.ms = _to8(m, u, False)
    s.v, s.vs = _to8(torch.sqrt(v), uv, True)


# ---- what a pass cannot do without --------------------------------------------------------------------

def work(case):
    if case["kind"] == "head":
        R, d, V = case["rows"], case["width"], case["vocab"]
        there = max(1.0, R * (1.0 - case["ignored"]))
        moved = 2 * (there + V) * d + 12 * R
        if case["grad"]:
            moved += 2 * (R + V) * d + 4 * R
        return {"bytes": moved, "flops": (6 if case["grad"] else 2) * there * d * V}
    n = sum(n for n, _ in _tensors(case))
    states = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
    return {"bytes": n * ((4 if case.get("grad32") else 2) + 8 + (0 if case.get("plain") else 2) + states), "flops": 18 * n}


# ---- the same in 64 bits ------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return _head64(s) if case["kind"] == "head" else _adamw64(s)


def _head64(s):
    """Row block by row block."""
    w = s.weight.double()
    R, V = s.hidden.shape[0], w.shape[0]
    loss = torch.zeros(R, dtype=torch.float64, device="cuda")
    dh = torch.zeros(s.hidden.shape, dtype=torch.float64, device="cuda")
    dw = torch.zeros(s.weight.shape, dtype=torch.float64, device="cuda")
    for a in range(0, R, 4096):
        rows = torch.arange(a, min(R, a + 4096), device="cuda")
        rows = rows[s.target[rows] >= 0]
        y = s.target[rows]
        h = s.hidden[rows].double()
        logp = torch.log_softmax(h @ w.t(), 1)
        loss[rows] = -logp[torch.arange(len(rows), device="cuda"), y]
        if s.d_hidden is not None:
            g = torch.exp(logp)
            g[torch.arange(len(rows), device="cuda"), y] -= 1.0
            g *= s.scale[rows].double()[:, None]
            dh[rows] = g @ w
            dw += g.t() @ h
    return {"loss": loss, "d_hidden": None if s.d_hidden is None else dh, "d_weight": None if s.d_weight is None else dw}


def _adamw64(s):
    """Slice by slice of the flat buffers."""
    sq, piece = 0.0, 1 << 26
    for a in range(0, s.n, piece):
        sq += float((s.g[a:a + piece].double() / s.sigma).square().sum())
    mult = min(1.0, HP["max_norm"] / (math.sqrt(sq) + 1e-6)) / s.sigma
    t = STEP0 + 1
    decay = torch.full((s.n,), 1.0 - HP["lr"] * HP["weight_decay"], device="cuda", dtype=torch.float64)
    for a, (n, nd) in zip(s.at, s.sizes):
        if nd:
            decay[a:a + n] = 1.0
    out = {"w": [], "m": [], "v": [], "m_scale": [], "v_scale": []}
    for a in range(0, s.n, piece):
        at = slice(a, min(s.n, a + piece))
        blocks = slice(a // BLOCK, -(-at.stop // BLOCK))
        m, v = s.m[at].double(), s.v[at].double()
        if s.ms is not None:
            m = m * s.ms[blocks].double().repeat_interleave(BLOCK)
            v = (v * s.vs[blocks].double().repeat_interleave(BLOCK)) ** 2
        g = s.g[at].double() * mult
        m = HP["beta1"] * m + (1.0 - HP["beta1"]) * g
        v = HP["beta2"] * v + (1.0 - HP["beta2"]) * g * g
        step = (m / (1.0 - HP["beta1"] ** t)) / (torch.sqrt(v / (1.0 - HP["beta2"] ** t)) + HP["eps"])
        out["w"].append(s.w[at].double() * decay[at] - HP["lr"] * step)
        if s.ms is None:
            out["m"].append(m)
            out["v"].append(v)
            continue
        word = _mix(torch.arange(a // 2 + 1, at.stop // 2 + 1, device="cuda") * _signed(PHI) + _key(t))
        for k, (name, x) in enumerate((("m", m), ("v", torch.sqrt(v)))):
            bits = torch.stack([(word >> (16 * k)) & 0xFFFF, (word >> (16 * k + 32)) & 0xFFFF], 1).reshape(-1, BLOCK)
            x = x.reshape(-1, BLOCK)
            scale = x.abs().amax(1, keepdim=True) / TOP
            y = x.abs() / scale.clamp(min=1e-200)
            _, e = torch.frexp(y.clamp(min=2.0 ** -6))
            step = torch.exp2((e - 4).double())
            q = torch.floor(y / step + (bits.double() + 0.5) / 65536) * step
            q = q.clamp(max=TOP)
            if name == "v":
                q = torch.where(y > 0, q.clamp(min=2.0 ** -9), q)
            out[name].append((q * torch.sign(x)).reshape(-1))
            out[name + "_scale"].append(scale.reshape(-1))
    out = {k: torch.cat(x) if x else None for k, x in out.items()}
    out["p"] = None if s.p is None else out["w"]
    return out
