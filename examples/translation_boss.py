"""Train a one-layer translation Boss on the batches the Assistant chooses, on one GPU.

The Boss is self-attention with a learned relative position bias, a residual connection, dropout on the attention probabilities and on
the layer's output, and a projection onto the vocabulary.  One step of StreamPipeline is

    screen the pool -> ordered list of sentences -> cut at the token budget        (aa_score_shrink, aa_batch_cut)
    attention -> projection -> residual + dropout -> logits                        (aa_rel_attention, aa_dropout)
    losses per sentence and their gradient                                         (aa_instance_loss_grad)
    the layer's gradients, the position table's among them                         (aa_dropout, aa_rel_attention_grad)
    update of the Boss; the losses label the sentences for the Assistant's update  (aa_assistant_step)

and nothing of it comes back to the host: the list, the number of sentences and their offsets stay on the device.  Both dropouts are
keyed by the sentence's row in the pool, so a sentence has the same masks wherever in the batch it lands, and the backward pass draws
them again instead of storing them.

The task is synthetic: a sentence's "translation" is its tokens shifted by a constant, one token to the left.

    python examples/translation_boss.py --steps 200
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_1905_03381_b200 import binding as B
from paper_1905_03381_b200 import workloads as W
from paper_1905_03381_b200.pipeline import StreamPipeline


class TranslationBoss:
    """fp32 parameters, bf16 activations, plain SGD.  `step` is the Boss's half of a StreamPipeline step."""

    def __init__(self, cfg: W.TranslationShape, indptr, tokens, lengths, heads: int = 4, dim: int = 32, buckets: int = 32,
                 distance: int = 64, p: float = 0.1, lr: float = 1.0, seed: int = 11):
        dev = tokens.device
        width = heads * dim
        self.cfg, self.indptr, self.tokens, self.lengths = cfg, indptr, tokens, lengths
        self.heads, self.dim, self.distance, self.p, self.lr, self.seed = heads, dim, distance, p, lr, seed
        self.emb = W.normal((cfg.vocab, width), 1.0, 21, torch.float32, dev)
        self.qkv = W.normal((width, 3 * width), width ** -0.5, 22, torch.float32, dev)
        self.proj = W.normal((width, width), width ** -0.5, 23, torch.float32, dev)
        self.out = W.normal((width, cfg.vocab), 0.1 * width ** -0.5, 24, torch.float32, dev)
        self.table = torch.zeros((buckets, heads), device=dev)
        self.dtable = torch.zeros_like(self.table)
        self.m = torch.zeros(1, dtype=torch.int32, device=dev)
        self.used = torch.zeros(1, dtype=torch.int32, device=dev)
        self.off = torch.zeros(cfg.n + 1, dtype=torch.int32, device=dev)
        self.slot = torch.arange(cfg.token_budget, device=dev)
        self.scratch = None
        self.history = []                       # (sum of the batch's losses, its tokens, its sentences), on the device

    def gather(self, idx):
        """Tokens and labels of the batch, one row a token; the rows past the batch's last token carry the label -1."""
        ends = self.off[1:].masked_fill(self.slot.new_ones(self.cfg.n).cumsum(0) > self.m, 2 ** 31 - 1)
        sentence = torch.searchsorted(ends, self.slot.to(torch.int32), right=True).clamp_(max=self.cfg.n - 1)
        at = self.slot - self.off[sentence]
        row = idx[sentence].long()
        length = self.lengths[row].long()
        start = self.indptr[row].long()
        live = (sentence < self.m) & (at < length)
        word = self.tokens[torch.where(live, start + at, 0)].long()
        follow = self.tokens[torch.where(live, start + (at + 1) % length.clamp(min=1), 0)].long()
        label = torch.where(live, (follow + 7) % self.cfg.vocab, -1).to(torch.int32)
        return word, label

    def step(self, t, ctx, idx, count, out_loss):
        cfg, h, d = self.cfg, self.heads, self.dim
        rows, width, dev = cfg.token_budget, h * d, self.emb.device
        ctx.aa_batch_cut(idx, count, cfg.n, self.m, self.used, lengths=self.lengths, token_budget=cfg.token_budget, out_offsets=self.off)
        count.copy_(self.m)                     # only the batch gets losses, so only the batch trains the Assistant
        off, m = self.off, self.m
        word, label = self.gather(idx)
        zeros = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16, device=dev)  # noqa: E731  rows past the batch stay zero
        qkv_w, proj, out = self.qkv.bfloat16(), self.proj.bfloat16(), self.out.bfloat16()
        probs, layer = (B.dropout_rule(self.p, self.seed, t, site, idx) for site in (0, 1))

        x = self.emb[word].bfloat16()
        qkv = x @ qkv_w
        q, k, v = (z.view(rows, h, d) for z in qkv.split(width, 1))            # views of the packed projection
        attn = B.attention(q, k, v, off, max_q=cfg.len_hi, max_k=cfg.len_hi, count_dev=m)
        bias = B.rel_bias(self.table, self.distance)
        o = zeros(rows, h, d)
        ctx.aa_rel_attention(attn, o, bias=bias, dropout=probs)
        y = zeros(rows, width)
        ctx.aa_dropout(o.view(rows, width) @ proj, layer, y, residual=x, offsets=off, count_dev=m)
        logits = y @ out

        dlogits = zeros(rows, cfg.vocab)
        ctx.aa_instance_loss_grad(B.logits_desc(logits), label, dlogits, offsets=off, count_dev=m, scale=1.0 / cfg.len_hi, out_loss=out_loss)
        dy = dlogits @ out.t()
        dz = zeros(rows, width)
        ctx.aa_dropout(dy, layer, dz, offsets=off, count_dev=m)
        do = (dz @ proj.t()).view(rows, h, d)
        dqkv = zeros(rows, 3 * width)
        dq, dk, dv = (z.view(rows, h, d) for z in dqkv.split(width, 1))
        if self.scratch is None:
            self.scratch = ctx.rel_attention_scratch(attn, bias)
        ctx.aa_rel_attention_grad(attn, do, dq, dk, dv, self.scratch, bias=bias, dropout=probs, dtable=self.dtable)
        dx = dy + dqkv @ qkv_w.t()

        self.out.sub_(self.lr * (y.t() @ dlogits))
        self.proj.sub_(self.lr * (o.view(rows, width).t() @ dz))
        self.qkv.sub_(self.lr * (x.t() @ dqkv))
        self.table.sub_(self.lr * self.dtable)
        self.emb.index_add_(0, word, dx.float(), alpha=-self.lr)
        kept = torch.arange(out_loss.numel(), device=dev) < m
        self.history.append((torch.where(kept, out_loss, 0.0).sum(), (label >= 0).sum(), m.clone()))


def train(steps: int, cfg: W.TranslationShape, depth: int = 1, device="cuda:0"):
    """Loss per token and sentences of every step."""
    indptr, col, val, lengths = cfg.csr(device)
    boss = TranslationBoss(cfg, indptr, (col % cfg.vocab).to(torch.int32), lengths)
    w, b = cfg.assistant(device)
    assistant = B.linear_assistant(w, b)
    pipe = StreamPipeline(depth, max_rows=cfg.n, max_d=cfg.buckets, capacity=cfg.n, device=device, boss_max_rows=max(cfg.n, cfg.token_budget))
    try:
        pipe.run(steps, lambda j, idx: B.csr_features(indptr, col, val, cfg.buckets, row_idx=idx), boss.step, assistant, cfg.gamma,
                 cfg.philox_seed, cfg.lr)
        torch.cuda.synchronize()
        status = pipe.device_status()
        if status != B.AA_OK:
            raise RuntimeError(B.status_string(status))
    finally:
        pipe.close()
    return [(float(loss) / max(1, int(n)), int(m)) for loss, n, m in boss.history]


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--sentences", type=int, default=2048)
    ap.add_argument("--token-budget", type=int, default=8192)
    ap.add_argument("--vocab", type=int, default=1000)
    ap.add_argument("--depth", type=int, default=1, help="screened batches that may wait for the Boss")
    args = ap.parse_args()
    cfg = W.TranslationShape(n=args.sentences, buckets=1 << 14, vocab=args.vocab, token_budget=args.token_budget)
    losses = train(args.steps, cfg, args.depth)
    every = max(1, args.steps // 10)
    for t in sorted({*range(0, args.steps, every), args.steps - 1}):
        print(f"step {t:5d}  loss per token {losses[t][0]:7.4f}  sentences in the batch {losses[t][1]}")


if __name__ == "__main__":
    main()
