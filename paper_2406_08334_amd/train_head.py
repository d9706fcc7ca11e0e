"""Trains the two largest tensors of a small language model, embedding and head, with what this package has for them:

    python -m paper_2406_08334_amd.train_head [--steps 300 --vocab 8192 --width 256 --rows 4096 --bits 8 --dtype bf16]

A bigram model: the hidden state of a position is its token's row of the embedding, the head predicts the next token.  pt_head_loss takes
loss and gradients without the logits of all rows; its gradient of the hidden states is added up per token in fp32; a list of tensors
(pt_tensors_*) takes norm, clipping and AdamW for both, their states in 8 bits or in 32.  Data: a Markov chain in which every token has four
successors with probabilities 0.4, 0.3, 0.2, 0.1, so the loss falls from log(vocab) towards their entropy, 1.28.  A sixteenth of the
rows has no target, as padding would.
"""
from __future__ import annotations

import argparse
import math

import torch

from . import binding as B

CHANCES = (0.4, 0.3, 0.2, 0.1)


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
          seed: int = 0, say=None):
    """-> the mean loss of every step's rows that have a target."""
    dt = torch.bfloat16 if dtype == "bf16" else torch.float16
    fp16 = dt == torch.float16
    chain = Chain(vocab, seed)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    masters = [torch.empty(vocab, width, device="cuda").normal_(0.0, std, generator=gen) for std in (1.0, 0.02)]
    embedding, head_weight = (w.to(dt) for w in masters)
    d_embedding = torch.zeros(vocab, width, device="cuda")
    d_head = torch.zeros_like(head_weight)
    state = torch.uint8 if bits == 8 else torch.float32
    arrays = []
    for w, p, g in zip(masters, (embedding, head_weight), (d_embedding, d_head)):
        m, v = (torch.zeros(vocab, width, dtype=state, device="cuda") for _ in range(2))
        scales = [torch.zeros(-(-w.numel() // 256), device="cuda") for _ in range(2)] if bits == 8 else [None, None]
        arrays.append((g, w, m, v, p, *scales))
    scaler = B.pt_scaler_cfg(65536.0, 2.0, 0.5, 2000, 0) if fp16 else None
    tensors = B.pt_tensors_create(B.PT_FP16 if fp16 else B.PT_BF16, [B.tensor(*a) for a in arrays], bits, scaler, seed)
    hidden, d_hidden = (torch.empty(rows, width, dtype=dt, device="cuda") for _ in range(2))
    target = torch.empty(rows, dtype=torch.int64, device="cuda")
    loss, scale = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    head = B.head(hidden, head_weight, target, loss, row_scale=scale, d_hidden=d_hidden, d_weight=d_head)
    workspace = torch.empty(B.pt_head_workspace(head)[1], dtype=torch.uint8, device="cuda")
    losses, loss_scale = [], 65536.0 if fp16 else 1.0
    for step in range(steps):
        x, y = chain.batch(rows)
        target.copy_(y)
        torch.index_select(embedding, 0, x, out=hidden)
        scale.copy_((loss_scale / (target >= 0).sum()).expand(rows))
        B.pt_head_loss(head, workspace)
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
    a = ap.parse_args()
    print(f"log(vocab) {math.log(a.vocab):.4f}, entropy of the chain {-sum(p * math.log(p) for p in CHANCES):.4f}", flush=True)
    train(**vars(a), say=lambda s: print(s, flush=True))


if __name__ == "__main__":
    main()
