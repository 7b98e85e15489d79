"""The 64-bit reference of linear layers, layer normalisation and AdamW, pinned on differences and on PyTorch's float64 forms."""
import numpy as np
import pytest
import torch
import torch.nn.functional as F

import boss_step_reference as S


def rand(*shape, seed=0):
    return np.random.default_rng([seed, *shape]).standard_normal(shape)


@pytest.mark.parametrize("name", [None, "relu", "gelu", "silu"])
def test_linear_and_its_gradient(name):
    x, w, b, res, dout = rand(7, 5), rand(4, 5, seed=1), rand(4, seed=2), rand(7, 4, seed=3), rand(7, 4, seed=4)
    tx, tw, tb = (torch.tensor(t, requires_grad=True) for t in (x, w, b))
    z = F.linear(tx, tw, tb)
    y = {None: lambda t: t, "relu": F.relu, "gelu": F.gelu, "silu": F.silu}[name](z) + torch.tensor(res)
    out, pre, size = S.linear(x, w, b, name, res)
    assert np.allclose(out, y.detach(), rtol=1e-12, atol=1e-12) and np.allclose(pre, z.detach(), rtol=1e-12) and np.all(size >= np.abs(pre))
    y.backward(torch.tensor(dout))
    got, _, _ = S.linear_grad(x, w, dout, name, pre, None)
    for k, t in (("dx", tx), ("dw", tw), ("dbias", tb)):
        assert np.allclose(got[k], t.grad, rtol=1e-11, atol=1e-12)
    step = 1e-6                                              # and against differences
    for i in range(5):
        e = np.zeros_like(x)
        e[2, i] = step
        d = (S.linear(x + e, w, b, name, res)[0] - S.linear(x - e, w, b, name, res)[0]) / (2 * step)
        assert abs((d * dout).sum() - got["dx"][2, i]) < 1e-7


@pytest.mark.parametrize("affine", [True, False])
def test_layer_norm_and_its_gradient(affine):
    x, g, b, dout = rand(6, 9), rand(9, seed=1), rand(9, seed=2), rand(6, 9, seed=3)
    tx, tg, tb = (torch.tensor(t, requires_grad=True) for t in (x, g, b))
    y = F.layer_norm(tx, (9,), tg if affine else None, tb if affine else None, 1e-3)
    y.backward(torch.tensor(dout))
    out, _, _ = S.layer_norm(x, g if affine else None, b if affine else None, 1e-3)
    got, _, _, _ = S.layer_norm_grad(x, g if affine else None, 1e-3, dout, None)
    assert np.allclose(out, y.detach(), rtol=1e-12, atol=1e-12) and np.allclose(got["dx"], tx.grad, rtol=1e-10, atol=1e-12)
    if affine:
        assert np.allclose(got["dgamma"], tg.grad, rtol=1e-11, atol=1e-12) and np.allclose(got["dbeta"], tb.grad, rtol=1e-11, atol=1e-12)


def test_adamw_is_torch_adamw():
    p, m, v = rand(50), np.zeros(50), np.zeros(50)
    t = torch.tensor(p, requires_grad=True)
    opt = torch.optim.AdamW([t], lr=0.03, betas=(0.9, 0.98), eps=1e-6, weight_decay=0.1)
    for step in range(1, 6):
        g = rand(50, seed=step)
        t.grad = torch.tensor(g)
        opt.step()
        p, m, v = S.adamw(p, g, m, v, {"lr": 0.03, "beta1": 0.9, "beta2": 0.98, "eps": 1e-6, "t": step}, 0.1)
        assert np.allclose(p, t.detach(), rtol=1e-12, atol=1e-13)


def test_e4m3_table_and_codes():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(S.e4m3_values(), want, equal_nan=True)
    x = rand(700).astype(np.float32)
    for root in (False, True):
        a = np.abs(x) if root else x
        lo, byte, units, step = S.to_codes(a, np.zeros(700, dtype=np.int64), root)
        hi, _, _, _ = S.to_codes(a, np.full(700, 65535), root)
        table = want[np.isfinite(want)]
        assert np.all(np.isin(lo, table)) and np.all(np.isin(hi, table)) and byte.dtype == np.uint8
        tops = np.array([units[i:i + 256].max() for i in range(0, 700, 256)])
        assert np.all((tops >= 128) & (tops < 256))
        assert np.all(np.abs(np.abs(lo) - units) <= step) and np.all(np.abs(np.abs(hi) - units) <= step)


def test_random_rounding_is_without_bias():
    u = np.arange(65536)
    for x in (0.3, 1.06, 100.7, 2.0**-8 + 1e-4):
        a = np.full(65536, x, dtype=np.float32)
        a[0::256] = 200.0                                     # the blocks' largest: units are the numbers themselves
        keep = np.arange(65536) % 256 != 0
        m, _, _, step = S.to_codes(a, u, False)
        assert abs(m[keep].mean() - x) < 2.0**-13 * step[keep].max() + 0.004 * step[keep].max()
        r, _, _, step = S.to_codes(a, u, True)
        assert abs((r[keep] ** 2).mean() - x * x) < 0.005 * 2 * x * step[keep].max()
