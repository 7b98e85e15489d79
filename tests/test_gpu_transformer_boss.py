"""Linear layers, normalisations, attention, the loss's gradient and AdamW together: the transformer Boss of the examples, its gradients against differentiated
fp64 arithmetic, its training step on screened batches."""
import importlib.util
import math
import os

import numpy as np
import pytest
import torch

import boss_reference as R
from paper_1905_03381_b200 import binding as B
from paper_1905_03381_b200 import workloads as W

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def load_example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "transformer_boss.py")
    spec = importlib.util.spec_from_file_location("transformer_boss", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def reference_loss(boss, P, word, label, lens):
    """Mean over the sentences of the summed token losses, in the type of P."""
    norm = lambda x, n: torch.nn.functional.layer_norm(x, (boss.width,), P[n + "_gamma"], P[n + "_beta"], 1e-5)  # noqa: E731
    total, at = 0.0, 0
    for n in lens:
        rows = slice(at, at + n)
        at += n
        x = P["emb"][word[rows]]
        q, k, v = (z.view(n, boss.heads, boss.dim) for z in (norm(x, "norm1") @ P["qkv"].t() + P["qkv_bias"]).split(boss.width, 1))
        bucket = torch.tensor([[R.bucket(j - i, boss.table.shape[0], boss.distance, True) for j in range(n)] for i in range(n)], device=DEV)
        score = torch.einsum("ihd,jhd->hij", q, k) / math.sqrt(boss.dim) + P["table"][bucket].permute(2, 0, 1)
        o = torch.einsum("hij,jhd->ihd", torch.softmax(score, 2), v).reshape(n, boss.width)
        y = x + o @ P["proj"].t() + P["proj_bias"]
        f = y + torch.nn.functional.gelu(norm(y, "norm2") @ P["up"].t() + P["up_bias"]) @ P["down"].t() + P["down_bias"]
        logits = norm(f, "norm3") @ P["vocab"].t() + P["vocab_bias"]
        total = total + torch.nn.functional.cross_entropy(logits, label[rows].long(), reduction="sum")
    return total / len(lens)


def make(dtype, bits=32, p=0.0):
    module = load_example()
    cfg = W.TranslationShape(n=8, buckets=64, len_lo=1, len_hi=40, vocab=50, token_budget=128)
    indptr, col, _, lengths = cfg.csr(DEV)
    return module.TransformerBoss(cfg, indptr, (col % cfg.vocab).to(torch.int32), lengths, heads=2, dim=32, inner=96, buckets=16, distance=20, p=p, bits=bits, dtype=dtype)


@pytest.mark.parametrize("dtype,bar", [(torch.float32, 2e-4), (torch.bfloat16, 6e-2)])
def test_gradients_of_the_whole_boss(dtype, bar):
    """Every gradient in the 2-norm.  fp32: a score or product is off by a few 1e-6 of its terms and passes through about ten layers: 2e-4.  bf16: about fifteen
    roundings of 2^-9 in the mean square on the way to the first layer, whose gradients are sums that cancel: 15^0.5 2^-9 = 0.8 %, times 8."""
    boss = make(dtype)
    ctx = B.AutoAssist(max_rows=128, max_d=64, device=DEV)
    lens = [7, 1, 40, 23]
    rows, rng = 128, np.random.default_rng(1)
    word = torch.tensor(rng.integers(0, 50, rows), device=DEV)
    label = torch.tensor(rng.integers(0, 50, rows), dtype=torch.int32, device=DEV)
    label[sum(lens):] = -1
    off = torch.tensor(np.concatenate([[0], np.cumsum(lens + [9])]), dtype=torch.int32, device=DEV)
    count = torch.tensor([len(lens)], dtype=torch.int32, device=DEV)          # a fifth sentence is there and not counted
    for n in ("table", "norm1_gamma", "norm2_beta", "up_bias"):
        boss.param[n].add_(W.normal(tuple(boss.param[n].shape), 0.2, 5, torch.float32, DEV))
    loss = torch.zeros(5, device=DEV)
    boss.forward(ctx, word, off, count, 0, None)
    boss.backward(ctx, word, label, off, count, loss, 1.0)
    torch.cuda.synchronize()
    assert ctx.aa_device_status() == B.AA_OK
    P = {n: (boss.copy[n] if n in boss.copy else t).double().requires_grad_() for n, t in boss.param.items()}
    want = reference_loss(boss, P, word, label, lens)
    want.backward()
    assert abs(loss[:4].mean().item() - want.item()) <= bar * want.item() and loss[4] == 0
    for n, g in boss.grad.items():
        ref = P[n].grad
        assert torch.linalg.norm(g.double() - ref) <= bar * torch.linalg.norm(ref), n
    ctx.close()


@pytest.mark.parametrize("depth,bits", [(0, 32), (1, 8)])
def test_the_training_step_runs_on_screened_batches(depth, bits):
    module = load_example()
    cfg = W.TranslationShape(n=256, buckets=1024, len_lo=8, len_hi=64, vocab=100, token_budget=1024)
    got = module.train(6, cfg, depth, heads=2, dim=32, inner=128, bits=bits)
    assert len(got) == 6 and all(math.isfinite(x) and 1024 // 64 <= m <= 1024 // 8 for x, m in got)


def test_a_captured_step_replays(tmp_path):
    """Forward, backward and update captured into one graph; replays on other tokens give what eager calls give, bit for bit."""
    lens, rows, rng = [30, 5, 40], 128, np.random.default_rng(2)
    off = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device=DEV)
    count = torch.tensor([len(lens)], dtype=torch.int32, device=DEV)
    label = torch.full((rows,), -1, dtype=torch.int32, device=DEV)
    label[:sum(lens)] = torch.tensor(rng.integers(0, 50, sum(lens)), dtype=torch.int32, device=DEV)
    words = [torch.tensor(rng.integers(0, 50, rows), device=DEV) for _ in range(3)]
    results = []
    for graph in (False, True):
        boss, stream = make(torch.bfloat16), torch.cuda.Stream(DEV)
        with torch.cuda.stream(stream):
            ctx = B.AutoAssist(max_rows=128, max_d=64, device=DEV, stream=stream)
            word, loss = words[0].clone(), torch.zeros(3, device=DEV)

            def step():
                boss.forward(ctx, word, off, count, 0, None)
                boss.backward(ctx, word, label, off, count, loss, 1.0)
                boss.rule.t = 0
                ctx.aa_adamw(boss.list, boss.rule)

            step()
            stream.synchronize()
            if graph:
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g, stream=stream):
                    step()
            for w in words[1:]:
                word.copy_(w)
                g.replay() if graph else step()
            stream.synchronize()
            assert ctx.aa_device_status() == B.AA_OK
            results.append({**{n: t.clone() for n, t in boss.param.items()}, "loss": loss.clone()})
            if graph:
                del g
            ctx.close()
    # the embedding's gradient is added up by PyTorch in no fixed order
    for n, t in results[0].items():
        assert n == "emb" or torch.equal(t, results[1][n]) or torch.allclose(t, results[1][n], rtol=1e-3, atol=1e-4), n
