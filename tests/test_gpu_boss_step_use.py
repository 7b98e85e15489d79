"""Linear layers, layer normalisation and AdamW as programs use them: replayed out of captured graphs, in two contexts at once, on sizes whose tiles are shared or
left ragged.  Bars as in test_gpu_boss_step."""
import types

import numpy as np
import pytest
import torch

import boss_step_reference as S
from paper_1905_03381_b200 import binding as B
from paper_1905_03381_b200 import build
from test_gpu_boss_step import BF16, DEV, F32, HALF, c, check_grad, check_linear, close, entry, f64, i32, like, mat, norm_bars

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def aa():
    build.build()
    ctx = B.AutoAssist(max_rows=1 << 10, max_d=64, device=DEV)
    yield ctx
    torch.cuda.synchronize()
    assert ctx.aa_device_status() == B.AA_OK
    ctx.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,k,n", [(150, 65, 130), (200, 300, 701), (64, 512, 2048), (150, 501, 2001), (1000, 129, 1003), (24, 512, 512), (130, 63, 127)])
def test_linear_with_every_operand_on_ragged_tiles(aa, dtype, m, k, n):
    for act in (None, "gelu"):
        out, p, want, z, bar, pre_bar = check_linear(aa, dtype, m, k, n, act, True, True, True)
        close(out, want, bar)
        close(p, z, pre_bar)
    out, _, want, _, bar, _ = check_linear(aa, dtype, m, k, n, "relu", True, True, False, (1, 3, 5), 1)
    close(out, want, bar)


@pytest.mark.parametrize("m,k,n,pads,shift", [(70, 1024, 2056, (0, 0, 0), 0), (40, 1025, 2049, (0, 0, 0), 0), (5, 1500, 1501, (1, 3, 5), 1), (300, 1032, 2064, (0, 0, 0), 0)])
def test_gradients_of_large_fp32_weights_and_few_rows(aa, m, k, n, pads, shift):
    """Not worth copies of the weights: taken apart on the way."""
    check_grad(aa, F32, m, k, n, "silu", True, pads, shift)
    check_grad(aa, F32, m, k, n, None, False, pads, shift)


@pytest.mark.parametrize("m,k,n", [(3, 64, 40), (200, 512, 512), (700, 264, 1000)])
def test_gradients_where_dout_alone_starts_anywhere(aa, m, k, n):
    x, w, dout = mat(m, k, 1, BF16), mat(n, k, 2, BF16, std=k ** -0.5), mat(m, n, 3, BF16, 3, 1)
    for rows in (m, m // 2):
        dx, dw, db = like((m, k), BF16), like((n, k), BF16), torch.full((n,), 7.0, device=DEV)
        aa.aa_linear_grad(x, w, dout, aa.linear_grad_scratch(x, w), dx=dx, dw=dw, dbias=db, count_dev=i32([rows]))
        got, size, _ = S.linear_grad(f64(x)[:rows], f64(w), f64(dout)[:rows], None, None, None)
        close(dx[:rows], got["dx"], c(n) * size["dx"] + HALF[BF16] * np.abs(got["dx"]))
        assert torch.all(dx[rows:] == 7.0)
        close(dw, got["dw"], c(rows) * size["dw"] + HALF[BF16] * np.abs(got["dw"]))
        close(db, got["dbias"], c(rows) * size["dbias"])


class Layer:
    """A layer normalisation and a linear layer with their gradients on counted rows, and the update of the weights."""

    def __init__(self, aa, dtype, m, k, n):
        self.aa, self.dtype = aa, dtype
        self.x, self.w, self.dout = mat(m, k, 1, dtype), mat(n, k, 2, dtype, std=k ** -0.5), mat(m, n, 3, dtype)
        self.count = i32([m])
        self.h, self.dh, self.dx = (like((m, k), dtype) for _ in range(3))
        self.pre, self.out = like((m, n), dtype), like((m, n), dtype)
        self.dw, self.db = like((n, k), dtype), torch.zeros(n, device=DEV)
        self.dg, self.dbeta = torch.zeros(k, device=DEV), torch.zeros(k, device=DEV)
        self.bias = torch.zeros(n, device=DEV)
        self.s1, self.s2 = aa.linear_grad_scratch(self.h, self.w, "silu"), aa.layer_norm_grad_scratch(self.x)
        self.p, self.m, self.v = (torch.zeros(n, k, device=DEV) for _ in range(3))
        self.tensors = B.adamw_list([B.adamw_tensor(self.p, self.dw, self.m, self.v)])

    def run(self):
        aa, live = self.aa, {"count_dev": self.count}
        aa.aa_layer_norm(self.x, self.h, **live)
        aa.aa_linear(self.h, self.w, self.out, bias=self.bias, activation="silu", pre=self.pre, **live)
        aa.aa_linear_grad(self.h, self.w, self.dout, self.s1, dx=self.dh, dw=self.dw, dbias=self.db, activation="silu", pre=self.pre, **live)
        aa.aa_layer_norm_grad(self.x, self.dh, self.dx, self.s2, dgamma=self.dg, dbeta=self.dbeta, **live)
        aa.aa_adamw(self.tensors, B.adamw_rule(0.5, 0.5, 0.5, 1e-8))

    def results(self):
        r = int(self.count)
        return [t.clone() for t in (self.h[:r], self.out[:r], self.pre[:r], self.dh[:r], self.dx[:r], self.dw, self.db, self.dg, self.dbeta, self.p, self.m, self.v)]

    def check(self):
        r = int(self.count)
        h, _, inv = S.layer_norm(f64(self.x)[:r], None, None, 1e-5)
        close(self.h[:r], h, norm_bars(f64(self.x)[:r], h, inv, self.dtype) + HALF[self.dtype] * np.abs(h) + 2.0**-22 * np.abs(h))
        h = f64(self.h)[:r]
        want, z, size = S.linear(h, f64(self.w), f64(self.bias), "silu", None)
        close(self.out[:r], want, 1.13 * c(h.shape[1]) * size + 2.0**-20 * np.maximum(np.abs(z), 1.0) + HALF[self.dtype] * np.abs(want) + 2.0**-22 * np.abs(z))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,k,n", [(9, 64, 96), (300, 520, 640), (700, 515, 1001)])
def test_captured_and_replayed(dtype, m, k, n):
    """A graph whose replays take what its inputs hold then - other rows, other counts - and give the bits of calls outside of it."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = B.AutoAssist(max_rows=64, max_d=64, device=DEV, stream=stream)
        layer = Layer(ctx, dtype, m, k, n)
        layer.run()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            layer.run()
        for rows, seed in ((m, 11), (m // 2, 12), (0, 13), (1, 14)):
            layer.x.copy_(mat(m, k, seed, dtype))
            layer.dout.copy_(mat(m, n, seed + 100, dtype))
            layer.count.fill_(rows)
            got = []
            for go in (graph.replay, layer.run):
                for t in (layer.p, layer.m, layer.v):
                    t.zero_()
                go()
                got.append(layer.results())
            assert all(torch.equal(a, b) for a, b in zip(*got))
            layer.check()
            if rows == 0:
                assert not got[0][5].any() and not got[0][6].any() and not got[0][7].any() and torch.all(layer.p == 0)
        stream.synchronize()
        assert ctx.aa_device_status() == B.AA_OK
        ctx.close()


def test_two_contexts_at_once():
    """Two contexts on streams of their own, whose launches overlap: each gives what it gives alone."""
    pairs = []
    for seed, (dtype, m, k, n) in enumerate([(BF16, 2000, 512, 1024), (F32, 700, 515, 1001)]):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            ctx = B.AutoAssist(max_rows=64, max_d=64, device=DEV, stream=stream)
            layer = Layer(ctx, dtype, m, k, n)
            layer.run()
            stream.synchronize()
            alone = layer.results()
        pairs.append((stream, ctx, layer, alone))
    torch.cuda.synchronize()
    for _ in range(5):
        for stream, _, layer, _ in pairs:
            with torch.cuda.stream(stream):
                for t in (layer.p, layer.m, layer.v):
                    t.zero_()
                layer.run()
    torch.cuda.synchronize()
    for stream, ctx, layer, alone in pairs:
        with torch.cuda.stream(stream):
            assert all(torch.equal(a, b) for a, b in zip(layer.results(), alone))
        assert ctx.aa_device_status() == B.AA_OK
        ctx.close()


def test_tensors_of_another_device_are_refused(aa):
    x, w, out = mat(4, 8, 1, F32), mat(8, 8, 2, F32), like((4, 8), F32)
    s1, s2 = aa.linear_grad_scratch(x, w), aa.layer_norm_grad_scratch(x)
    e = entry(16, 1, F32, 32, False, 0.0)
    keep, aa.workspace = aa.workspace, types.SimpleNamespace(device=torch.device("cuda:1"))
    try:
        for bad in (lambda: aa.aa_linear(x, w, out), lambda: aa.aa_linear_grad(x, w, out, s1, dx=like((4, 8), F32)), lambda: aa.aa_layer_norm(x, out),
                    lambda: aa.aa_layer_norm_grad(x, out, like((4, 8), F32), s2), lambda: aa.aa_adamw(B.adamw_list([e]), B.adamw_rule(0.1))):
            with pytest.raises(TypeError, match="cuda:1"):
                bad()
    finally:
        aa.workspace = keep
