"""Trains a small language model, embedding, head and at will a block in between, with what this package has for them:

    python -m paper_2406_08334_amd.train_head [--steps 300 --vocab 8192 --width 256 --rows 4096 --bits 8 --dtype bf16 --mlp 0 --drop 0]

A bigram model: the hidden state of a position is its token's row of the embedding, the head predicts the next token.  pt_head_loss takes
loss and gradients without the logits of all rows; its gradient of the hidden states is added up per token in fp32; a list of tensors
(pt_tensors_*) takes norm, clipping and AdamW for both, their states in 8 bits or in 32.  With --mlp N a block lies in between, of N units:
RMS norm, product with bias and gelu, product with bias, dropout and the residual, RMS norm (pt_rms_*, pt_linear_*).  Data: a Markov chain in which every token has four
successors with probabilities 0.4, 0.3, 0.2, 0.1, so the loss falls from log(vocab) towards their entropy, 1.28.  A sixteenth of the
rows has no target, as padding would.
"""
from __future__ import annotations

import argparse
import math

import torch

from . import binding as B

CHANCES = (0.4, 0.3, 0.2, 0.1)


class Block:
    """A block of an MLP before the head: hidden = h, out = norm2(h + drop(W2 gelu(W1 norm1(h) + b1) + b2)), with its gradients."""

    def __init__(self, hidden, mlp: int, drop: float, seed: int, gen):
        rows, width = hidden.shape
        dt = hidden.dtype
        like = lambda *shape: torch.empty(shape, dtype=dt, device="cuda")  # noqa: E731
        std = lambda s, *shape: torch.empty(shape, device="cuda").normal_(0.0, s, generator=gen)  # noqa: E731
        self.masters = [torch.ones(width, device="cuda"), std(width ** -0.5, mlp, width), torch.zeros(mlp, device="cuda"),
                        std(mlp ** -0.5, width, mlp), torch.zeros(width, device="cuda"), torch.ones(width, device="cuda")]
        self.no_decay = [True, False, True, False, True, True]
        self.params = [m.to(dt) for m in self.masters]
        self.grads = [torch.zeros_like(p) for p in self.params]
        g1, w1, b1, w2, b2, g2 = self.params
        d_g1, d_w1, d_b1, d_w2, d_b2, d_g2 = self.grads
        self.step = torch.zeros(1, dtype=torch.int64, device="cuda")         # of the dropout: another mask every step
        n, pre, a, s, self.out = like(rows, width), like(rows, mlp), like(rows, mlp), like(rows, width), like(rows, width)
        d_n, d_a, d_s, self.d_out, self.d_hidden = like(rows, width), like(rows, mlp), like(rows, width), like(rows, width), like(rows, width)
        rstd1, rstd2 = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        self.norm1 = B.rms(hidden, n, gain=g1, rstd=rstd1, d_y=d_n, d_sum=d_s, d_x=self.d_hidden, d_gain=d_g1)
        self.up = B.linear(n, w1, a, bias=b1, pre=pre, act="gelu", d_out=d_a, d_x=d_n, d_weight=d_w1, d_bias=d_b1)
        self.down = B.linear(a, w2, s, bias=b2, residual=hidden, drop=drop, seed=seed, step=self.step, d_out=d_s, d_x=d_a, d_weight=d_w2, d_bias=d_b2)
        self.norm2 = B.rms(s, self.out, gain=g2, rstd=rstd2, d_y=self.d_out, d_x=d_s, d_gain=d_g2)
        self.keep = [hidden, n, pre, a, s, d_n, d_a, d_s, rstd1, rstd2]
        size = max([1] + [b for x in (self.up, self.down) for b in B.pt_linear_workspace(x)] + [B.pt_rms_workspace(x) for x in (self.norm1, self.norm2)])
        self.work = torch.empty(size, dtype=torch.uint8, device="cuda")      # the calls come one after the other

    def forward(self):
        B.pt_rms_norm(self.norm1)
        B.pt_linear_out(self.up, self.work)
        B.pt_linear_out(self.down, self.work)
        B.pt_rms_norm(self.norm2)

    def backward(self):
        """From d_out to d_hidden and the parameters' gradients."""
        B.pt_rms_grads(self.norm2, self.work)
        B.pt_linear_grads(self.down, self.work)
        B.pt_linear_grads(self.up, self.work)
        B.pt_rms_grads(self.norm1, self.work)            # and what reaches the hidden states beside the block
        self.step.add_(1)


class Chain:
    """Batches of (token, next token)."""

    def __init__(self, vocab: int, seed: int):
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.vocab = vocab
        self.successors = torch.randint(0, vocab, (vocab, len(CHANCES)), generator=self.gen, device="cuda")
        self.chances = torch.tensor(CHANCES, device="cuda")

    def batch(self, rows: int):
        x = torch.randint(0, self.vocab, (rows,), generator=self.gen, device="cuda")
        y = self.successors[x, torch.multinomial(self.chances, rows, replacement=True, generator=self.gen)]
        y[::16] = -100
        return x, y


def train(steps: int = 300, vocab: int = 8192, width: int = 256, rows: int = 4096, bits: int = 8, dtype: str = "bf16", lr: float = 1e-2,
          seed: int = 0, mlp: int = 0, drop: float = 0.0, say=None):
    """-> the mean loss of every step's rows that have a target."""
    dt = torch.bfloat16 if dtype == "bf16" else torch.float16
    fp16 = dt == torch.float16
    chain = Chain(vocab, seed)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    masters = [torch.empty(vocab, width, device="cuda").normal_(0.0, std, generator=gen) for std in (1.0, 0.02)]
    embedding, head_weight = (w.to(dt) for w in masters)
    d_embedding = torch.zeros(vocab, width, device="cuda")
    d_head = torch.zeros_like(head_weight)
    hidden, d_hidden = (torch.empty(rows, width, dtype=dt, device="cuda") for _ in range(2))
    block = Block(hidden, mlp, drop, seed, gen) if mlp else None
    params, grads, no_decay = [embedding, head_weight], [d_embedding, d_head], [False, False]
    if block:
        masters, params, grads, no_decay = masters + block.masters, params + block.params, grads + block.grads, no_decay + block.no_decay
    state = torch.uint8 if bits == 8 else torch.float32
    arrays = []
    for w, p, g, plain in zip(masters, params, grads, no_decay):
        m, v = (torch.zeros(w.shape, dtype=state, device="cuda") for _ in range(2))
        scales = [torch.zeros(-(-w.numel() // 256), device="cuda") for _ in range(2)] if bits == 8 else [None, None]
        arrays.append((g, w, m, v, p, *scales, plain))
    scaler = B.pt_scaler_cfg(65536.0, 2.0, 0.5, 2000, 0) if fp16 else None
    tensors = B.pt_tensors_create(B.PT_FP16 if fp16 else B.PT_BF16, [B.tensor(*a) for a in arrays], bits, scaler, seed)
    target = torch.empty(rows, dtype=torch.int64, device="cuda")
    loss, scale = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    head = B.head(block.out if block else hidden, head_weight, target, loss, row_scale=scale, d_hidden=block.d_out if block else d_hidden, d_weight=d_head)
    if block:
        d_hidden = block.d_hidden
    workspace = torch.empty(B.pt_head_workspace(head)[1], dtype=torch.uint8, device="cuda")
    losses, loss_scale = [], 65536.0 if fp16 else 1.0
    for step in range(steps):
        x, y = chain.batch(rows)
        target.copy_(y)
        torch.index_select(embedding, 0, x, out=hidden)
        scale.copy_((loss_scale / (target >= 0).sum()).expand(rows))
        if block:
            block.forward()
        B.pt_head_loss(head, workspace)
        if block:
            block.backward()
        d_embedding.zero_().index_add_(0, x, d_hidden.float())
        B.pt_tensors_grad_sqnorm(tensors)
        B.pt_tensors_adamw_step(tensors, B.hparams(lr * min(1.0, (step + 1) / 20), 0.9, 0.95, 1e-8, 0.0, 1.0))
        losses.append(float(loss.sum() / (target >= 0).sum()))
        report = B.pt_tensors_report_read(tensors)
        loss_scale = report.loss_scale
        if say and (step % 20 == 0 or step + 1 == steps):
            say(f"step {report.step}: loss {losses[-1]:.4f}, gradient norm {report.norm:.4f}, clip {report.clip_coef:.4f}")
    B.pt_tensors_destroy(tensors)
    return losses


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("steps", 300), ("vocab", 8192), ("width", 256), ("rows", 4096), ("seed", 0)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--bits", type=int, choices=(8, 32), default=8)
    ap.add_argument("--dtype", choices=("bf16", "fp16"), default="bf16")
    ap.add_argument("--lr", type=float, default=1e-2)
    ap.add_argument("--mlp", type=int, default=0, help="units of a block between embedding and head; 0: none")
    ap.add_argument("--drop", type=float, default=0.0, help="the block's dropout")
    a = ap.parse_args()
    print(f"log(vocab) {math.log(a.vocab):.4f}, entropy of the chain {-sum(p * math.log(p) for p in CHANCES):.4f}", flush=True)
    train(**vars(a), say=lambda s: print(s, flush=True))


if __name__ == "__main__":
    main()
