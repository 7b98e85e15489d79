"""The transformer Boss's step replayed out of a graph, from the same weights as an eager one: the same bits."""
import numpy as np
import pytest
import torch

from paper_1905_03381_b200 import binding as B
from test_gpu_transformer_boss import DEV, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
def test_a_replayed_step_has_the_bits_of_an_eager_one(bits):
    """One step at a time from one state, on other tokens, other lengths and another count than at capture.  The embedding's update is left out: its gradient is added up by PyTorch in
    no fixed order.  Every step is the first (t = 1): a graph replays the t it was captured with."""
    rows, rng = 128, np.random.default_rng(2)
    boss, stream = make(torch.bfloat16, bits=bits), torch.cuda.Stream(DEV)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    with torch.cuda.stream(stream):
        ctx = B.AutoAssist(max_rows=128, max_d=64, device=DEV, stream=stream)
        word, label, off, count = torch.zeros(rows, dtype=torch.int64, device=DEV), i32([-1] * rows), i32([0] * 4), i32([0])
        loss = torch.zeros(3, device=DEV)
        state = [t for e in boss.entries for t in e._keep if t is not None] + [boss.copy[n] for n in boss.WEIGHTS]
        first = [t.clone() for t in state]

        def fill(lens, counted):
            word.copy_(torch.tensor(rng.integers(0, 50, rows), device=DEV))
            label.fill_(-1)
            n = sum(lens[:counted])
            label[:n] = i32(rng.integers(0, 50, n))
            off.copy_(i32([0, *np.cumsum(lens)]))
            count.fill_(counted)

        def restore():
            for t, f in zip(state, first):
                t.copy_(f)
            loss.zero_()

        def step():
            boss.rule.t = 0
            boss.forward(ctx, word, off, count, 0, None)
            boss.backward(ctx, word, label, off, count, loss, 1.0)
            ctx.aa_adamw(boss.list, boss.rule)

        fill([30, 5, 40], 3)
        step()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        for lens, counted in (([30, 5, 40], 3), ([1, 40, 33], 3), ([12, 40, 7], 2)):
            fill(lens, counted)
            got = []
            for go in (step, graph.replay):
                restore()
                go()
                got.append([loss.clone()] + [t.clone() for e, n in zip(boss.entries, boss.param) if n != "emb" for t in e._keep if t is not None])
            assert loss[:counted].abs().min() > 0
            for a, b in zip(*got):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        stream.synchronize()
        assert ctx.aa_device_status() == B.AA_OK
        del graph
        ctx.close()
