"""Pins of the fp64 reference of the Boss's training operators, and the host-side checks of their entry points.  No GPU needed."""
import ctypes
import math

import boss_reference as R
import numpy as np
import pytest
import torch

from oracle import aa_oracle as O
from paper_1905_03381_b200 import binding as B
from paper_1905_03381_b200 import build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return B.lib()


def test_philox_words_agree_with_the_oracles_draw():
    ids = np.array([0, 1, 77, 2**31, 2**33 + 5], dtype=np.uint64)
    w0 = R.philox(ids & R.MASK, ids >> np.uint64(32), 9, 0, 1234, 0)[0]
    assert np.allclose((w0 >> np.uint64(8)).astype(np.float64) / 2**24, O.uniform(1234, 9, ids.astype(np.int64)), rtol=0, atol=0)


def test_draws_are_uniform_and_streams_are_apart():
    key = R.instance_key(3, 4, 5)
    u = R.draws(key, np.arange(40000), 1).reshape(-1)
    n = u.size
    assert abs(u.mean() - 32767.5) < 5 * 65536 / math.sqrt(12 * n)
    counts = np.bincount(u >> 8, minlength=256)
    chi = ((counts - n / 256) ** 2 / (n / 256)).sum()
    assert abs(chi - 255) < 6 * math.sqrt(2 * 255)
    for other in (R.draws(key, np.arange(40000), 2), R.draws(R.instance_key(3, 4, 6), np.arange(40000), 1), R.draws(R.instance_key(3, 5, 5), np.arange(40000), 1)):
        c = np.corrcoef(u, other.reshape(-1))[0, 1]
        assert abs(c) < 6 / math.sqrt(n)


def test_dropout_factor_does_not_depend_on_where_an_instance_sits():
    a = R.dropout_factor(5, 37, 0.3, 1, 2, 3, 99)
    assert a.shape == (5, 37) and set(np.unique(a)) == {0.0, 65536.0 / (65536 - R.threshold(0.3))}
    # more rows of the same instance only add rows
    assert np.array_equal(R.dropout_factor(9, 37, 0.3, 1, 2, 3, 99)[:5], a)


@pytest.mark.parametrize("buckets,distance,both", [(32, 128, True), (32, 128, False), (20, 50, True), (4, 3, True), (3, 7, False), (256, 2048, True), (128, 1000, False),
                                                   (64, 17, True)])
def test_buckets_of_the_library_and_their_shape(lib, buckets, distance, both):
    t = ctypes.c_void_p(0)
    b = B.aa_rel_bias()
    b.buckets, b.max_distance, b.bidirectional, b.table = buckets, distance, int(both), t
    nb = buckets // 2 if both else buckets
    last = -1
    for n in sorted({*range(0, 300), distance - 1, distance, distance + 1, 5000, 2**40}):
        want = R.bucket(-n, buckets, distance, both)
        assert lib.aa_rel_bucket(ctypes.byref(b), -n) == want
        assert lib.aa_rel_bucket(ctypes.byref(b), n) == R.bucket(n, buckets, distance, both)
        assert want >= last
        last = want
    assert R.bucket(-distance, buckets, distance, both) == nb - 1
    assert R.bucket(-(nb // 2), buckets, distance, both) >= nb // 2


def test_bucket_boundaries_at_powers_are_exact():
    # 8 (128 / 8)^(k / 8) is an integer at every even k: 8, 16, 32, 64
    for k, n in ((8, 8), (10, 16), (12, 32), (14, 64)):
        assert R.bucket(-n, 32, 128, True) == k and R.bucket(-n + 1, 32, 128, True) == k - 1


def test_malformed_bias_descriptors(lib):
    for buckets, distance, both in ((0, 5, 0), (31, 128, 1), (1, 5, 0), (2, 5, 1), (32, 8, 1), (32, 4096, 1), (129, 500, 0), (258, 500, 1)):
        b = B.aa_rel_bias()
        b.buckets, b.max_distance, b.bidirectional = buckets, distance, both
        assert lib.aa_rel_bucket(ctypes.byref(b), 1) == -1
    assert lib.aa_rel_bucket(None, 0) == -1


def test_loss_gradient_is_the_losses_difference():
    rng = np.random.default_rng(0)
    x, y, w = rng.normal(size=(6, 9)) * 2, np.array([0, 3, -1, 8, 2, 2]), rng.uniform(0.5, 2, 6)
    g = R.loss_grad(x, y, w)
    f = lambda z: (R.row_losses(z, y) * w)[y >= 0].sum()  # noqa: E731
    eps = 1e-5
    for r in range(6):
        for c in range(9):
            d = np.zeros_like(x)
            d[r, c] = eps
            assert abs((f(x + d) - f(x - d)) / (2 * eps) - g[r, c]) < 1e-8
    lt = torch.tensor(x, requires_grad=True)
    (torch.nn.functional.cross_entropy(lt, torch.tensor(y), ignore_index=-1, reduction="none") * torch.tensor(w)).sum().backward()
    assert np.allclose(lt.grad.numpy(), g, atol=1e-14)


@pytest.mark.parametrize("lq,lk,causal,both", [(5, 5, True, False), (4, 7, True, True), (6, 3, True, True), (5, 6, False, True), (1, 6, True, False)])
def test_attention_gradients_are_differences_of_the_output(lq, lk, causal, both):
    rng = np.random.default_rng(lq * 10 + lk)
    h, hk, d = 4, 2, 3
    q, k, v = rng.normal(size=(lq, h, d)), rng.normal(size=(lk, hk, d)), rng.normal(size=(lk, hk, d))
    table, dout = rng.normal(size=(8, h)), rng.normal(size=(lq, h, d))
    factor = R.attention_factor(h, lq, lk, 0.25, 1, 2, 3, 4)
    kw = dict(scale=0.7, causal=causal, distance=5, bidirectional=both, factor=factor)
    got = R.attention_sequence(q, k, v, table=table, dout=dout, **kw)
    args = {"q": q, "k": k, "v": v, "table": table}
    eps = 1e-5
    for name in args:
        num = np.zeros_like(args[name])
        for at in np.ndindex(*num.shape):
            out = []
            for sign in (1, -1):
                moved = {n: x.copy() for n, x in args.items()}
                moved[name][at] += sign * eps
                out.append((R.attention_sequence(moved["q"], moved["k"], moved["v"], table=moved["table"], **kw)["out"] * dout).sum())
            num[at] = (out[0] - out[1]) / (2 * eps)
        assert np.max(np.abs(num - got["d" + name])) < 1e-8


def test_null_arguments_are_refused(lib):
    assert lib.aa_dropout(None, None, None, None, 0, None, None, None) == B.AA_ERR_INVALID_ARG
    assert lib.aa_instance_loss_grad(None, None, None, None, 0, None, None, 1.0, 0, None, None) == B.AA_ERR_INVALID_ARG
    assert lib.aa_rel_attention(None, None, None, None, None) == B.AA_ERR_INVALID_ARG
    assert lib.aa_rel_attention_scratch_bytes(None, None, None) == B.AA_ERR_INVALID_ARG
    assert lib.aa_rel_attention_grad(None, None, None, None, None, None, None, None, None, None, 0) == B.AA_ERR_INVALID_ARG


def test_struct_sizes_match_the_header(lib, tmp_path):
    import os
    import subprocess

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "t.c"
    src.write_text('#include "autoassist.h"\n' + "".join(
        f'_Static_assert(sizeof({n}) == {ctypes.sizeof(getattr(B, n))}, "{n}");\n' for n in ("aa_rows", "aa_dropout_rule", "aa_tokens", "aa_attn", "aa_rel_bias"))
        + "int main(void) { return 0; }\n")
    subprocess.check_call(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(root, "include"), "-c", str(src), "-o", str(tmp_path / "t.o")])
