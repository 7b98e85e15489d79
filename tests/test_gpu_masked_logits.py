"""Losses and their gradient where logits are finite but very large: classes masked by a finite value, rows shifted as a whole.

A row's softmax depends on differences of its logits only, which fp32 holds exactly where they matter; so the bars are those of ordinary logits.
  gradient : |G - G_ref| <= 1e-5 g p + 2^-22 g [c = y], plus 2^-8 |G_ref| for bf16 (as for ordinary logits);
  losses   : 1e-4 as everywhere, plus 2^-22 |f| where the label itself is masked (one subtraction and one addition, each rounded to 2^-24).
Widths reach every kernel: a row in a few lanes, in a warp, in a small CTA, in a shared-memory ring, swept by a CTA, at any alignment.
"""
import numpy as np
import pytest
import torch

import boss_reference as R
from paper_1905_03381_b200 import binding as B
from paper_1905_03381_b200 import build, workloads as W

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
WIDTHS = [10, 100, 1000, 3001, 9000, 32000, 70000]


@pytest.fixture(scope="module")
def aa():
    build.build()
    ctx = B.AutoAssist(max_rows=1 << 12, max_d=64, device=DEV)
    yield ctx
    torch.cuda.synchronize()
    assert ctx.aa_device_status() == B.AA_OK
    ctx.close()


def f64(t):
    return t.detach().double().cpu().numpy()


def masked_rows(cols, dtype, value):
    """Logits and labels: all but the first few classes masked, every other group of 32 classes masked, all masked, one class left, none left but the label."""
    x = W.normal((6, cols), 3.0, cols, dtype, DEV)
    c = torch.arange(cols, device=DEV)
    x[0, 4:] = value
    x[1, (c // 4) % 2 == 1] = value
    x[2] = value                                     # nothing but masked classes: uniform
    x[3, c != cols - 1] = value
    x[4, 2:] = value
    labels = np.array([1, 0, cols // 2, cols - 1, cols - 1, cols // 3], dtype=np.int32)      # row 4's label is a masked class
    return x, labels


def shifted_rows(cols, dtype, shift):
    x = (W.normal((4, cols), 3.0, cols + 1, F32, DEV) + shift).to(dtype)
    return x, np.array([0, cols - 1, cols // 2, 1], dtype=np.int32)


def check_losses(got, x, y):
    x = f64(x)
    top = x.max(axis=1)                              # differences first: 1e20 + log(10) is 1e20 in 64 bits too
    want = np.log(np.exp(x - top[:, None]).sum(axis=1)) + (top - x[np.arange(len(y)), y])
    assert np.all(np.abs(f64(got) - want) <= 1e-4 + 2.0**-22 * np.abs(want)), (f64(got), want)


def check_gradient(aa, x, y, dtype):
    rows = len(y)
    w = np.linspace(0.5, 2.0, rows).astype(np.float32)
    grad, loss = torch.full(x.shape, 7.0, dtype=dtype, device=DEV), torch.full((rows,), 7.0, device=DEV)
    labels = torch.tensor(y, device=DEV)
    aa.aa_instance_loss_grad(B.logits_desc(x), labels, grad, weight=torch.tensor(w, device=DEV), mean=False, out_loss=loss)
    torch.cuda.synchronize()
    g = w.astype(np.float64)
    want = R.loss_grad(f64(x), y, g)
    onehot = np.zeros_like(want)
    onehot[np.arange(rows), y] = 1.0
    bar = 1e-5 * np.abs(want + onehot * g[:, None]) + 2.0**-22 * g[:, None] * onehot + (2.0**-8 * np.abs(want) if dtype == BF16 else 0.0) + 1e-37
    assert np.all(np.abs(f64(grad) - want) <= bar)
    check_losses(loss, x, y)


VALUES = [-1e4, -1e9, -1e10, -1e20, -1e30, "lowest"]
SHIFTS = [3e3, 1e5, -1e7, 1e10, -1e20, -1e30, 3e38]


def value_of(value, dtype):
    return torch.finfo(dtype).min if value == "lowest" else value


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", WIDTHS)
def test_loss_gradient_of_classes_masked_by_a_finite_value(aa, dtype, cols):
    for value in VALUES:
        check_gradient(aa, *masked_rows(cols, dtype, value_of(value, dtype)), dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", WIDTHS)
def test_loss_gradient_of_shifted_rows(aa, dtype, cols):
    for shift in SHIFTS:
        check_gradient(aa, *shifted_rows(cols, dtype, shift), dtype)


def check_instance_losses(aa, x, y):
    rows, labels = len(y), torch.tensor(y, device=DEV)
    out = torch.full((rows,), 7.0, device=DEV)
    aa.aa_instance_loss(B.logits_desc(x), labels, out)
    check_losses(out, x, y)
    order = np.random.default_rng(rows).permutation(rows).astype(np.int32)
    listed = torch.full((rows,), 7.0, device=DEV)
    aa.aa_instance_loss_rows(B.logits_desc(x), labels, torch.tensor(order, device=DEV), listed)
    check_losses(listed, x[torch.tensor(order, device=DEV).long()], y[order])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", WIDTHS)
def test_instance_loss_of_classes_masked_by_a_finite_value(aa, dtype, cols):
    for value in VALUES:
        check_instance_losses(aa, *masked_rows(cols, dtype, value_of(value, dtype)))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", WIDTHS)
def test_instance_loss_of_shifted_rows(aa, dtype, cols):
    for shift in SHIFTS:
        check_instance_losses(aa, *shifted_rows(cols, dtype, shift))


def test_instance_loss_of_rows_of_nothing_but_infinities_stays_undefined(aa):
    """As before: no class left is NaN, a class of +inf is NaN, a label of -inf is +inf."""
    for cols in WIDTHS:
        x = W.normal((3, cols), 1.0, 5, F32, DEV)
        x[0] = -float("inf")
        x[1, 0] = float("inf")
        x[2, 1] = -float("inf")
        out = torch.empty(3, device=DEV)
        aa.aa_instance_loss(B.logits_desc(x), torch.tensor([0, 1, 1], dtype=torch.int32, device=DEV), out)
        got = f64(out)
        assert np.isnan(got[0]) and np.isnan(got[1]) and np.isposinf(got[2])
