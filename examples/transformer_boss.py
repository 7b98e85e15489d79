"""Train a one-layer pre-norm transformer Boss on the batches the Assistant chooses, with no product, normalisation or update left to PyTorch.

    x = embedding of the batch's tokens
    y = x + dropout(attention(norm(x)) W_o)                 (aa_layer_norm, aa_linear, aa_rel_attention, aa_dropout)
    f = y + gelu(norm(y) W_1) W_2                           (aa_layer_norm, aa_linear with activation, pre-activation and residual)
    logits = norm(f) W_v                                    (aa_instance_loss_grad for the losses and their gradient)

and back through the same layers (aa_linear_grad, aa_layer_norm_grad with the gradient of the residual connection, aa_rel_attention_grad), then one AdamW
step over all tensors (aa_adamw): fp32 parameters, bf16 copies for the products, moments in fp32 or in 8 bits.  The batch is the list that
the screening left on the device, cut at a token budget; its number of sentences and their offsets never come to the host, and token rows past
the batch are neither read nor written.

The task is the one of translation_boss.py: a sentence's tokens shifted by a constant, one token to the left.

    python examples/transformer_boss.py --steps 200 --bits 8
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import torch

from paper_1905_03381_b200 import binding as B
from paper_1905_03381_b200 import workloads as W
from paper_1905_03381_b200.pipeline import StreamPipeline
from translation_boss import TranslationBoss


class TransformerBoss(TranslationBoss):
    """`step` is the Boss's half of a StreamPipeline step; `forward` and `backward` are its parts, on any batch of ragged sentences."""

    WEIGHTS = ("qkv", "proj", "up", "down", "vocab")

    def __init__(self, cfg: W.TranslationShape, indptr, tokens, lengths, heads: int = 4, dim: int = 32, buckets: int = 32, distance: int = 64, p: float = 0.1,
                 lr: float = 2e-3, seed: int = 11, inner: int = 512, bits: int = 32, decay: float = 0.01, dtype=torch.bfloat16):
        super().__init__(cfg, indptr, tokens, lengths, heads, dim, buckets, distance, p, lr, seed)
        dev, width, self.dtype, self.width = self.emb.device, heads * dim, dtype, heads * dim
        shapes = {"qkv": (3 * width, width), "proj": (width, width), "up": (inner, width), "down": (width, inner), "vocab": (cfg.vocab, width)}
        self.param = {n: W.normal(s, s[1] ** -0.5, 30 + i, torch.float32, dev) for i, (n, s) in enumerate(shapes.items())}
        self.param["vocab"].mul_(0.1)
        self.param.update({n + "_bias": torch.zeros(shapes[n][0], device=dev) for n in self.WEIGHTS})
        for n in ("norm1", "norm2", "norm3"):
            self.param[n + "_gamma"], self.param[n + "_beta"] = torch.ones(width, device=dev), torch.zeros(width, device=dev)
        self.param.update(emb=self.emb, table=self.table)
        # gradients of weights come in the products' type, all others in fp32; the products read a copy of the weights in their type
        self.grad = {n: torch.zeros_like(t, dtype=dtype if n in self.WEIGHTS else torch.float32) for n, t in self.param.items()}
        self.grad["table"] = self.dtable
        low = dtype == torch.bfloat16
        self.copy = {n: self.param[n].to(dtype) if low else self.param[n] for n in self.WEIGHTS}
        entries = []
        for n, t in self.param.items():
            moments = B.adamw_moments8(t) if bits == 8 else {"m": torch.zeros_like(t), "v": torch.zeros_like(t)}
            entries.append(B.adamw_tensor(t, self.grad[n], copy=self.copy[n] if low and n in self.WEIGHTS else None, weight_decay=decay if n in self.WEIGHTS else 0.0, **moments))
        self.entries = entries
        self.list, self.rule = B.adamw_list(entries), B.adamw_rule(lr, 0.9, 0.98, 1e-9, seed=seed)
        self.act = None

    def buffers(self, rows):
        """What a step keeps of the forward pass, and the gradients on the way back; made once."""
        if self.act is None:
            shapes = {n: self.width for n in ("x", "a", "o", "z", "y", "c", "f", "e", "dx", "da", "do", "dz", "dy", "dc", "df", "de")}
            inner = self.param["up"].shape[0]
            shapes.update(qkv=3 * self.width, dqkv=3 * self.width, h=inner, pre=inner, dh=inner, logits=self.cfg.vocab, dlogits=self.cfg.vocab)
            self.act = {n: torch.zeros((rows, c), dtype=self.dtype, device=self.emb.device) for n, c in shapes.items()}
        return self.act

    def forward(self, ctx, word, off, m, t, idx):
        s, P, C, live = self.buffers(word.numel()), self.param, self.copy, {"offsets": off, "count_dev": m}
        rows, h, d = word.numel(), self.heads, self.dim
        self.rules = [B.dropout_rule(self.p, self.seed, t, site, idx) for site in (0, 1)] if self.p else [None, None]
        s["x"].copy_(self.emb[word])
        ctx.aa_layer_norm(s["x"], s["a"], P["norm1_gamma"], P["norm1_beta"], **live)
        ctx.aa_linear(s["a"], C["qkv"], s["qkv"], P["qkv_bias"], **live)
        q, k, v = (z.view(rows, h, d) for z in s["qkv"].split(self.width, 1))
        self.attn = B.attention(q, k, v, off, max_q=self.cfg.len_hi, max_k=self.cfg.len_hi, count_dev=m)
        self.bias = B.rel_bias(self.table, self.distance)
        ctx.aa_rel_attention(self.attn, s["o"].view(rows, h, d), bias=self.bias, dropout=self.rules[0])
        if self.p:
            ctx.aa_linear(s["o"], C["proj"], s["z"], P["proj_bias"], **live)
            ctx.aa_dropout(s["z"], self.rules[1], s["y"], residual=s["x"], offsets=off, count_dev=m)
        else:
            ctx.aa_linear(s["o"], C["proj"], s["y"], P["proj_bias"], residual=s["x"], **live)
        ctx.aa_layer_norm(s["y"], s["c"], P["norm2_gamma"], P["norm2_beta"], **live)
        ctx.aa_linear(s["c"], C["up"], s["h"], P["up_bias"], activation="gelu", pre=s["pre"], **live)
        ctx.aa_linear(s["h"], C["down"], s["f"], P["down_bias"], residual=s["y"], **live)
        ctx.aa_layer_norm(s["f"], s["e"], P["norm3_gamma"], P["norm3_beta"], **live)
        ctx.aa_linear(s["e"], C["vocab"], s["logits"], P["vocab_bias"], **live)
        return s["logits"]

    def backward(self, ctx, word, label, off, m, loss, scale):
        """Gradients of scale times the batch's mean loss into self.grad; the losses of the sentences into `loss`."""
        s, P, C, G, live = self.act, self.param, self.copy, self.grad, {"offsets": off, "count_dev": m}
        rows, h, d = word.numel(), self.heads, self.dim
        ctx.aa_instance_loss_grad(B.logits_desc(s["logits"]), label, s["dlogits"], offsets=off, count_dev=m, scale=scale, out_loss=loss)
        if self.scratch is None:
            self.scratch = {n: ctx.linear_grad_scratch(s[x], C[n], act) for n, x, act in (("qkv", "a", None), ("proj", "o", None), ("up", "c", "gelu"), ("down", "h", None), ("vocab", "e", None))}
            self.scratch.update(norm=ctx.layer_norm_grad_scratch(s["x"]), attention=ctx.rel_attention_scratch(self.attn, self.bias))

        def linear(n, x, dout, dx, **more):
            ctx.aa_linear_grad(s[x], C[n], s[dout], self.scratch[n], dx=s[dx], dw=G[n], dbias=G[n + "_bias"], **more, **live)

        def norm(n, x, dout, dx, residual=None):
            ctx.aa_layer_norm_grad(s[x], s[dout], s[dx], self.scratch["norm"], gamma=P[n + "_gamma"], residual=None if residual is None else s[residual], dgamma=G[n + "_gamma"],
                                   dbeta=G[n + "_beta"], **live)

        linear("vocab", "e", "dlogits", "de")
        norm("norm3", "f", "de", "df")
        linear("down", "h", "df", "dh")
        linear("up", "c", "dh", "dc", activation="gelu", pre=s["pre"])
        norm("norm2", "y", "dc", "dy", residual="df")
        if self.p:
            ctx.aa_dropout(s["dy"], self.rules[1], s["dz"], offsets=off, count_dev=m)
        linear("proj", "o", "dz" if self.p else "dy", "do")
        dq, dk, dv = (z.view(rows, h, d) for z in s["dqkv"].split(self.width, 1))
        ctx.aa_rel_attention_grad(self.attn, s["do"].view(rows, h, d), dq, dk, dv, self.scratch["attention"], bias=self.bias, dropout=self.rules[0], dtable=self.dtable)
        linear("qkv", "a", "dqkv", "da")
        norm("norm1", "x", "da", "dx", residual="dy")
        G["emb"].zero_().index_add_(0, word, torch.where((label >= 0)[:, None], s["dx"].float(), 0.0))

    def step(self, t, ctx, idx, count, out_loss):
        cfg = self.cfg
        ctx.aa_batch_cut(idx, count, cfg.n, self.m, self.used, lengths=self.lengths, token_budget=cfg.token_budget, out_offsets=self.off)
        count.copy_(self.m)                     # only the batch gets losses, so only the batch trains the Assistant
        word, label = self.gather(idx)
        self.forward(ctx, word, self.off, self.m, t, idx)
        self.backward(ctx, word, label, self.off, self.m, out_loss, 1.0 / cfg.len_hi)
        ctx.aa_adamw(self.list, self.rule)
        kept = torch.arange(out_loss.numel(), device=out_loss.device) < self.m
        self.history.append((torch.where(kept, out_loss, 0.0).sum(), (label >= 0).sum(), self.m.clone()))


def train(steps: int, cfg: W.TranslationShape, depth: int = 1, device="cuda:0", **options):
    """Loss per token and sentences of every step."""
    indptr, col, val, lengths = cfg.csr(device)
    boss = TransformerBoss(cfg, indptr, (col % cfg.vocab).to(torch.int32), lengths, **options)
    w, b = cfg.assistant(device)
    assistant = B.linear_assistant(w, b)
    pipe = StreamPipeline(depth, max_rows=cfg.n, max_d=cfg.buckets, capacity=cfg.n, device=device, boss_max_rows=max(cfg.n, cfg.token_budget))
    try:
        pipe.run(steps, lambda j, idx: B.csr_features(indptr, col, val, cfg.buckets, row_idx=idx), boss.step, assistant, cfg.gamma, cfg.philox_seed, cfg.lr)
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
    ap.add_argument("--bits", type=int, default=32, choices=(8, 32), help="of AdamW's moments")
    ap.add_argument("--depth", type=int, default=1, help="screened batches that may wait for the Boss")
    args = ap.parse_args()
    cfg = W.TranslationShape(n=args.sentences, buckets=1 << 14, vocab=args.vocab, token_budget=args.token_budget)
    losses = train(args.steps, cfg, args.depth, bits=args.bits)
    every = max(1, args.steps // 10)
    for t in sorted({*range(0, args.steps, every), args.steps - 1}):
        print(f"step {t:5d}  loss per token {losses[t][0]:7.4f}  sentences in the batch {losses[t][1]}")


if __name__ == "__main__":
    main()
