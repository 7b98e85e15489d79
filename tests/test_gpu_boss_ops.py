"""The operators that train the Boss on a generated batch, against their fp64 reference: instance-keyed dropout, the gradient of the
instance loss, and ragged attention with a learned relative position bias.

Bars (derived from the formats, fixed before any run):
  dropout   : zeros exactly where the reference drops; else |y - y_ref| <= 2^-22 (|scale x| + |res|), plus 2^-8 |y_ref| for the one rounding to bf16.
  loss grad : arguments of the exponential reach ~64 (ulp 2^-17, halved, times ln 2) and the sum carries the same: |G - G_ref| <= 1e-5 g p + 2^-22 g [c = y],
              plus 2^-8 |G_ref| for bf16; losses: 1e-4 a row as everywhere.
  attention : 3e-5 of the sum of absolute terms in fp32 (score errors of a few 1e-6 in the exponent, accumulation);
              bf16: operands of the second products are rounded to bf16 (2^-8 of each term at most) and the result once more (2^-8): 2^-7 of the absolute
              terms + 2^-8 of the result; the bias table's gradient is never rounded below fp32 and keeps the fp32 bar.
"""
import numpy as np
import pytest
import torch

import boss_reference as R
from oracle import aa_oracle as O
from paper_1905_03381_b200 import binding as B
from paper_1905_03381_b200 import build, workloads as W

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def aa():
    build.build()
    ctx = B.AutoAssist(max_rows=1 << 16, max_d=64, device=DEV)
    yield ctx
    torch.cuda.synchronize()
    assert ctx.aa_device_status() == B.AA_OK
    ctx.close()


def f64(t):
    return t.detach().double().cpu().numpy()


def offs(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device=DEV)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


# ------------------------------------------------------------------------------------------------------------------ dropout

def padded(shape, pad, std, seed, dtype):
    return W.normal((shape[0], shape[1] + pad), std, seed, dtype, DEV)[:, :shape[1]]


def check_dropout(y, x, res, factor, dtype):
    want = f64(x) * factor + (0 if res is None else f64(res))
    bar = 2.0**-22 * (np.abs(f64(x) * factor) + (0 if res is None else np.abs(f64(res)))) + (2.0**-8 * np.abs(want) if dtype == BF16 else 0.0)
    got = f64(y)
    assert np.all(np.abs(got - want) <= bar)
    if res is None:
        assert np.array_equal(got == 0, (factor == 0) | (f64(x) == 0))
    else:
        assert np.array_equal(got[factor == 0], f64(res)[factor == 0])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols,pad,p,residual", [(1, 1, 0, 0.5, False), (3, 7, 0, 0.1, True), (1, 8, 0, 0.9, True), (5, 65, 0, 0.3, True), (33, 129, 7, 0.5, False),
                                                      (40, 64, 0, 0.1, True), (17, 512, 0, 0.1, True), (9, 1000, 24, 0.2, True), (70, 1001, 0, 0.5, False), (2, 5003, 5, 0.1, True),
                                                      (2500, 24, 0, 0.25, True), (4, 40, 0, 0.0, True)])
def test_dropout_of_rows(aa, dtype, rows, cols, pad, p, residual):
    x, res = padded((rows, cols), pad, 1.0, 1 + rows, dtype), padded((rows, cols), 2 * pad, 1.0, 2 + rows, dtype) if residual else None
    ids = np.random.default_rng(rows).integers(0, 2**31 - 1, rows)
    out = torch.full((rows, cols), 7.0, dtype=dtype, device=DEV)
    seed, step, site, base = 2**63 + 11, 2**40 + 3, 5, 2**33
    aa.aa_dropout(x, B.dropout_rule(p, seed, step, site, i32(ids), base), out, residual=res)
    factor = np.concatenate([R.dropout_factor(1, cols, p, seed, step, site, base + int(i)) for i in ids])
    check_dropout(out, x, res, factor, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [16, 130, 512])
def test_dropout_of_ragged_sentences_and_its_backward(aa, dtype, cols):
    lens = [3, 0, 1, 17, 0, 0, 40, 2, 300, 1]
    off, n = offs(lens), sum(lens)
    x = W.normal((n, cols), 1.0, 3, dtype, DEV)
    rule = B.dropout_rule(0.3, 9, 8, 7, i32(np.arange(10) * 5 + 2))
    factor = np.concatenate([R.dropout_factor(m, cols, 0.3, 9, 8, 7, 5 * s + 2) for s, m in enumerate(lens)])
    res, out = W.normal((n, cols), 1.0, 4, dtype, DEV), torch.empty_like(x)
    aa.aa_dropout(x, rule, out, residual=res, offsets=off)
    check_dropout(out, x, res, factor, dtype)
    g = W.normal((n, cols), 1.0, 5, dtype, DEV)
    inplace = g.clone()
    aa.aa_dropout(inplace, rule, inplace, offsets=off)          # backward, in place
    check_dropout(inplace, g, None, factor, dtype)


def test_dropout_follows_the_instance_not_the_slot_and_respects_the_device_count(aa):
    x = W.normal((50, 96), 1.0, 6, F32, DEV)
    ids = np.random.default_rng(1).permutation(1000)[:50]
    out, moved = torch.full_like(x, 9.0), torch.full_like(x, 9.0)
    order = np.random.default_rng(2).permutation(50)
    count = i32([33])
    aa.aa_dropout(x, B.dropout_rule(0.5, 1, 2, 3, i32(ids)), out)
    aa.aa_dropout(x[torch.tensor(order, device=DEV)].contiguous(), B.dropout_rule(0.5, 1, 2, 3, i32(ids[order])), moved, count_dev=count)
    o, m = f64(out), f64(moved)
    assert np.array_equal(o[order][:33], m[:33]) and np.all(m[33:] == 9.0)
    # token rows of sentences past the device count and in no sentence stay as they are; a count beyond the list is the list's length
    off = i32([2, 5, 5, 30])
    for c, last in ((2, 5), (0, 2), (-4, 2), (99, 30)):
        out.fill_(9.0)
        aa.aa_dropout(x, B.dropout_rule(0.5, 1, 2), out, offsets=off, count_dev=i32([c]))
        touched = (f64(out) != 9.0).any(axis=1)
        assert touched[2:last].all() and not touched[:2].any() and not touched[last:].any()


def test_dropped_infinities_are_zero(aa):
    x = torch.full((4, 256), float("inf"), device=DEV)
    x[1] = float("nan")
    out = torch.empty_like(x)
    aa.aa_dropout(x, B.dropout_rule(0.5, 1, 2), out)
    factor = np.concatenate([R.dropout_factor(1, 256, 0.5, 1, 2, 0, r) for r in range(4)])
    assert np.array_equal(f64(out) == 0, factor == 0)


def test_dropout_refusals_and_latched_offsets(aa):
    x = torch.zeros((4, 16), device=DEV)
    rule = B.dropout_rule(0.5, 1, 2)
    for bad in (lambda: aa.aa_dropout(x, B.dropout_rule(1.0, 1, 2), x), lambda: aa.aa_dropout(x, B.dropout_rule(-0.1, 1, 2), x),
                lambda: aa.aa_dropout(x, B.dropout_rule(float("nan"), 1, 2), x),
                lambda: aa.aa_dropout(x, rule, torch.zeros((4, 15), device=DEV)), lambda: aa.aa_dropout(x, rule, torch.zeros((4, 16), dtype=BF16, device=DEV)),
                lambda: aa.aa_dropout(x, rule, x, residual=torch.zeros((3, 16), device=DEV))):
        with pytest.raises(B.AutoAssistError) as e:
            bad()
        assert e.value.status == B.AA_ERR_INVALID_ARG
    buf = torch.zeros(100, device=DEV)
    with pytest.raises(B.AutoAssistError):
        aa.aa_dropout(buf[:64].view(4, 16), rule, buf[8:72].view(4, 16))          # shifted overlap
    aa.aa_dropout(x, rule, x, offsets=i32([0, 3, 2, 4]))
    torch.cuda.synchronize()
    assert aa.aa_device_status() == B.AA_ERR_BAD_INDEX
    aa.aa_dropout(torch.zeros((0, 16), device=DEV), rule, torch.zeros((0, 16), device=DEV))
    assert aa.aa_device_status() == B.AA_OK


# ------------------------------------------------------------------------------------------------------------ loss gradient

def check_loss(x, y, factor, grad, dtype):
    xs, g = f64(x), np.where(y >= 0, factor, 0.0)
    want = R.loss_grad(xs, y, factor)
    prob = want.copy()
    onehot = np.zeros_like(prob)
    onehot[np.arange(len(y)), np.maximum(y, 0)] = (y >= 0).astype(float)
    prob = np.abs(want + onehot * g[:, None])
    bar = 1e-5 * prob + 2.0**-22 * np.abs(g)[:, None] * onehot + (2.0**-8 * np.abs(want) if dtype == BF16 else 0.0) + 1e-37
    assert np.all(np.abs(f64(grad) - want) <= bar)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (5, 2, 0), (300, 10, 0), (77, 100, 0), (33, 101, 0), (64, 1000, 8), (9, 1003, 3), (12, 4096, 0), (7, 8190, 1), (5, 32000, 0), (3, 40001, 0),
                                           (2, 70000, 8), (3, 131071, 0)])
def test_loss_gradient_of_rows(aa, dtype, rows, cols, pad):
    x = padded((rows, cols), pad, 3.0, 10 + cols, dtype)
    rng = np.random.default_rng(cols)
    y = rng.integers(0, cols, rows).astype(np.int32)
    y[rng.random(rows) < 0.2] = -1
    w = rng.uniform(0.5, 4.0, rows).astype(np.float32)
    grad, loss = torch.full((rows, cols), 7.0, dtype=dtype, device=DEV), torch.full((rows,), 7.0, device=DEV)
    aa.aa_instance_loss_grad(B.logits_desc(x), i32(y), grad, weight=torch.tensor(w, device=DEV), scale=0.5, mean=True, out_loss=loss)
    check_loss(x, y, 0.5 * w.astype(np.float64) / rows, grad, dtype)
    same = torch.empty_like(loss)
    aa.aa_instance_loss(B.logits_desc(x), i32(y), same)
    assert np.max(np.abs(f64(loss) - R.row_losses(f64(x), y))) <= 1e-4 and np.max(np.abs(f64(loss) - f64(same))) <= 1e-4
    # in place, sum, no weights
    z = x.clone() if pad == 0 else torch.empty((rows, cols + pad), dtype=dtype, device=DEV)[:, :cols].copy_(x)
    aa.aa_instance_loss_grad(B.logits_desc(z), i32(y), z, mean=False, scale=2.0)
    check_loss(x, y, np.full(rows, 2.0), z, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [60, 3001, 33000])
def test_loss_gradient_of_sentences(aa, dtype, cols):
    lens = [4, 0, 9, 1, 0, 23, 2]
    off, n = offs(lens), sum(lens) + 3          # three rows in no sentence
    x, rng = W.normal((n, cols), 3.0, 20, dtype, DEV), np.random.default_rng(4)
    y = rng.integers(0, cols, n).astype(np.int32)
    y[[1, 6]] = -1
    w = rng.uniform(0.5, 4.0, 7).astype(np.float32)
    for count, m in ((None, 7), (6, 6), (3, 3), (0, 0)):
        grad, loss = torch.full((n, cols), 7.0, dtype=dtype, device=DEV), torch.full((7,), -5.0, device=DEV)
        aa.aa_instance_loss_grad(B.logits_desc(x), i32(y), grad, offsets=off, weight=torch.tensor(w, device=DEV), out_loss=loss,
                                 count_dev=None if count is None else i32([count]))
        end = sum(lens[:m])
        inst = np.repeat(np.arange(7), lens)[:end]
        assert np.all(f64(grad)[end:] == 7.0) and np.all(f64(loss)[m:] == -5.0)
        if end:
            check_loss(x[:end], y[:end], w.astype(np.float64)[inst] / m, grad[:end], dtype)
            sums = np.zeros(m)
            np.add.at(sums, inst, R.row_losses(f64(x), y)[:end])
            assert np.all(np.abs(f64(loss)[:m] - sums) <= 1e-4 * np.maximum(1, lens[:m]))


def test_loss_gradient_masked_classes_and_bad_labels(aa):
    x = W.normal((6, 300), 3.0, 30, F32, DEV)
    x[0, 5:] = -float("inf")                       # masked classes
    x[1, :] = torch.finfo(F32).min                 # the type's lowest value everywhere: uniform
    x[2, 7] = 3.0e38
    y = np.array([2, 3, 7, 299, -1, 1], dtype=np.int32)
    grad = torch.empty_like(x)
    aa.aa_instance_loss_grad(B.logits_desc(x), i32(y), grad, mean=False)
    check_loss(x, y, np.ones(6), grad, F32)
    assert np.allclose(f64(grad)[1], np.where(np.arange(300) == 3, 1 / 300 - 1, 1 / 300), rtol=1e-5, atol=0)
    y[3] = 300
    aa.aa_instance_loss_grad(B.logits_desc(x), i32(y), grad, mean=False)
    torch.cuda.synchronize()
    assert aa.aa_device_status() == B.AA_ERR_BAD_INDEX and np.all(f64(grad)[3] == 0)


def test_loss_gradient_device_count_of_rows(aa):
    x, y = W.normal((90, 40), 3.0, 31, BF16, DEV), np.random.default_rng(7).integers(0, 40, 90).astype(np.int32)
    grad, loss = torch.full((90, 40), 7.0, dtype=BF16, device=DEV), torch.full((90,), 7.0, device=DEV)
    aa.aa_instance_loss_grad(B.logits_desc(x), i32(y), grad, count_dev=i32([31]), out_loss=loss)
    check_loss(x[:31], y[:31], np.full(31, 1 / 31), grad[:31], BF16)
    assert np.all(f64(grad)[31:] == 7.0) and np.all(f64(loss)[31:] == 7.0)


def test_loss_gradient_refusals(aa):
    x, y = torch.zeros((4, 8), device=DEV), i32([0, 1, 2, 3])
    for grad in (torch.zeros((4, 7), device=DEV), torch.zeros((3, 8), device=DEV), torch.zeros((4, 8), dtype=BF16, device=DEV)):
        with pytest.raises(B.AutoAssistError) as e:
            aa.aa_instance_loss_grad(B.logits_desc(x), y, grad)
        assert e.value.status == B.AA_ERR_INVALID_ARG
    small = B.AutoAssist(max_rows=2, max_d=8, device=DEV)
    with pytest.raises(B.AutoAssistError) as e:
        small.aa_instance_loss_grad(B.logits_desc(x), y, x.clone(), offsets=i32([0, 4]), out_loss=torch.zeros(1, device=DEV))
    assert e.value.status == B.AA_ERR_WORKSPACE
    small.close()


# ---------------------------------------------------------------------------------------------------------------- attention

def run_attention(aa, lq, lk, heads, kv, dim, dtype, causal, table, distance, both, p, scale=None, packed=False, head_major=False, ids=None, count=None, train=True, values=1.0):
    nq, nk = sum(lq), sum(lk)
    if packed:
        buf = W.normal((max(nq, 1), heads + 2 * kv, dim), 1.0, 41, dtype, DEV)[:nq]
        q, k, v = buf[:, :heads], buf[:, heads:heads + kv], buf[:, heads + kv:]
    elif head_major:
        q, k, v = (W.normal((h, n, dim), 1.0, 42 + i, dtype, DEV).transpose(0, 1) for i, (h, n) in enumerate(((heads, nq), (kv, nk), (kv, nk))))
    else:
        q, k, v = (W.normal((n, h, dim), values if i < 2 else 1.0, 42 + i, dtype, DEV) for i, (h, n) in enumerate(((heads, nq), (kv, nk), (kv, nk))))
    ids = np.arange(len(lq)) * 3 + 1 if ids is None else ids
    attn = B.attention(q, k, v, offs(lq), offs(lk), max(lq, default=0), max(lk, default=0), scale=scale, causal=causal, count_dev=count)
    bias = None if table is None else B.rel_bias(table, distance, both)
    drop = B.dropout_rule(p, 77, 5, 2, i32(ids), 100) if p else None
    empty = lambda t: torch.full(t.shape, 7.0, dtype=dtype, device=DEV) if not head_major else torch.full((t.shape[1], t.shape[0], dim), 7.0, dtype=dtype, device=DEV).transpose(0, 1)  # noqa: E731
    got = {"out": empty(q)}
    aa.aa_rel_attention(attn, got["out"], bias=bias, dropout=drop)
    dout = None
    if train:
        dout = W.normal((nq, heads, dim), 1.0, 45, dtype, DEV)
        got.update(dq=empty(q), dk=empty(k), dv=empty(v))
        if table is not None:
            got["dtable"] = torch.full_like(table, 7.0)
        aa.aa_rel_attention_grad(attn, dout, got["dq"], got["dk"], got["dv"], aa.rel_attention_scratch(attn, bias), bias=bias, dropout=drop, dtable=got.get("dtable"))
    torch.cuda.synchronize()
    return q, k, v, dout, ids, {n: f64(t) for n, t in got.items()}


def check_attention(aa, lq, lk, heads, kv, dim, dtype, causal, buckets=16, distance=40, both=True, p=0.0, scale=None, **kw):
    table = None if buckets == 0 else W.normal((buckets, heads), 0.5, 40, F32, DEV)
    q, k, v, dout, ids, got = run_attention(aa, lq, lk, heads, kv, dim, dtype, causal, table, distance, both, p, scale=scale, **kw)
    s = dim ** -0.5 if scale is None else scale
    want = {n: np.zeros_like(got[n]) for n in got}
    bars = {n: np.zeros_like(got[n]) for n in got}
    qo, ko = np.concatenate([[0], np.cumsum(lq)]), np.concatenate([[0], np.cumsum(lk)])
    tb = None if table is None else f64(table)
    for n in range(len(lq)):
        a, b = slice(qo[n], qo[n + 1]), slice(ko[n], ko[n + 1])
        factor = R.attention_factor(heads, lq[n], lk[n], p, 77, 5, 2, 100 + int(ids[n])) if p else None
        ref = R.attention_sequence(f64(q[a]), f64(k[b]), f64(v[b]), s, causal, tb, distance, both, factor, None if dout is None else f64(dout[a]))
        for name, at in (("out", a), ("dq", a), ("dk", b), ("dv", b)):
            if name in got:
                want[name][at], bars[name][at] = ref[name], ref[name + "_abs"]
        if "dtable" in got:
            want["dtable"] += ref["dtable"]
            bars["dtable"] += ref["dtable_abs"]
    for name in got:
        rounded = dtype == BF16 and name != "dtable"
        bar = (2.0**-7 if rounded else 3e-5) * bars[name] + (2.0**-8 * np.abs(want[name]) if rounded else 0.0)
        err = np.abs(got[name] - want[name])
        assert np.all(err <= bar), (name, float(np.max(err / (bar + 1e-30))), int((err > bar).sum()))
    return got


RAGGED = [5, 1, 0, 33, 64, 17, 130, 2]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads,kv,dim,causal,both,buckets,p", [
    (2, 2, 64, False, True, 16, 0.0), (4, 2, 64, True, False, 16, 0.2), (4, 1, 32, True, True, 32, 0.0), (2, 2, 128, False, False, 20, 0.3), (3, 3, 40, False, True, 8, 0.1),
    (1, 1, 8, True, False, 4, 0.5), (2, 1, 96, False, True, 0, 0.1), (5, 5, 24, True, True, 64, 0.0), (2, 2, 7, False, True, 16, 0.1), (2, 1, 200, True, False, 16, 0.1)])
def test_attention_of_ragged_sentences(aa, dtype, heads, kv, dim, causal, both, buckets, p):
    check_attention(aa, RAGGED, RAGGED, heads, kv, dim, dtype, causal, buckets=buckets, both=both, p=p)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lq,lk", [([1], [1]), ([1, 1, 1], [300, 1, 65]), ([7, 70, 3, 0, 2], [3, 64, 0, 9, 200]), ([129], [31]), ([64, 65], [64, 129]), ([200], [200])])
def test_attention_of_unequal_lengths(aa, dtype, causal, lq, lk):
    got = check_attention(aa, lq, lk, 4, 2, 64, dtype, causal, both=not causal, p=0.1)
    if causal and lq == [129]:
        assert np.all(got["out"][:98] == 0) and np.all(got["dq"][:98] == 0)      # positions before the first key


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim", [64, 128, 72])
def test_attention_longer_than_the_bias_reaches(aa, dtype, dim):
    check_attention(aa, [700, 515], [700, 515], 2, 1, dim, dtype, True, both=False, p=0.1)
    check_attention(aa, [600], [600], 2, 2, dim, dtype, False, both=True, distance=60)
    check_attention(aa, [400], [400], 1, 1, dim, dtype, False, both=False, distance=900, buckets=128)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_one_new_token_over_long_contexts(aa, dtype):
    for lk in ([1, 4001, 63, 64, 65, 2048], [20000]):
        check_attention(aa, [1] * len(lk), lk, 8, 2, 64, dtype, True, both=False, p=0.0, train=False)
        check_attention(aa, [1] * len(lk), lk, 4, 4, 128, dtype, False, both=True, p=0.1, train=False)
    check_attention(aa, [3, 1, 9], [3000, 0, 5000], 6, 2, 128, dtype, True, both=True, p=0.1, train=False)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_strides(aa, dtype):
    check_attention(aa, [40, 9, 70], [40, 9, 70], 4, 2, 64, dtype, True, packed=True, p=0.1)
    check_attention(aa, [40, 9, 70], [40, 9, 70], 3, 3, 36, dtype, False, packed=True)           # odd strides
    check_attention(aa, [40, 9, 70], [40, 9, 70], 4, 2, 64, dtype, False, head_major=True, p=0.1)


def test_attention_one_key_has_no_score_gradient(aa):
    """A softmax over one key is constant: dq, dk and the table's gradient are exactly zero."""
    for dtype in (F32, BF16):
        got = check_attention(aa, [1] * 9, [1] * 9, 2, 2, 64, dtype, True, p=0.3)
        assert not got["dq"].any() and not got["dk"].any() and not got["dtable"].any()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_large_scores(aa, dtype):
    # scores of a few hundred: the softmax is nearly one-hot.  fp32 products of 64 terms of size ~400 are off by ~1e-4 in the exponent,
    # so the bars of this case are looser in that proportion; what matters is that nothing overflows
    q, k, v, dout, ids, got = run_attention(aa, [90], [90], 2, 2, 64, dtype, False, W.normal((16, 2), 0.5, 40, F32, DEV), 40, True, 0.0, scale=1.0, values=6.0)
    ref = R.attention_sequence(f64(q), f64(k), f64(v), 1.0, False, f64(W.normal((16, 2), 0.5, 40, F32, DEV)), 40, True, None, f64(dout))
    for name in got:
        assert np.all(np.abs(got[name] - ref[name]) <= (1e-2 if name != "dtable" and dtype == BF16 else 2e-3) * (ref[name + "_abs"] + np.abs(ref[name])) + 1e-6)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("low", [-float("inf"), torch.finfo(F32).min, -1e30])
def test_attention_bias_as_a_mask(aa, dtype, low):
    """Buckets whose bias is the lowest value: masked where other keys are left, uniform where nothing else is; -inf leaves such rows empty."""
    heads, lens = 2, [50, 1, 3]
    n = sum(lens)
    table = torch.zeros((4, heads), device=DEV)
    table[0, 0] = low                    # one direction, distance 0 (and the later keys): the query's own position is masked, row 0 sees nothing else
    q, k = torch.zeros((n, heads, 64), dtype=dtype, device=DEV), torch.zeros((n, heads, 64), dtype=dtype, device=DEV)
    v = W.normal((n, heads, 64), 1.0, 3, dtype, DEV)
    attn, bias = B.attention(q, k, v, offs(lens), causal=True), B.rel_bias(table, 9, False)
    out, dq, dk, dv, dt = torch.full_like(q, 7.0), torch.full_like(q, 7.0), torch.full_like(k, 7.0), torch.full_like(v, 7.0), torch.full_like(table, 7.0)
    aa.aa_rel_attention(attn, out, bias=bias)
    dout = W.normal((n, heads, 64), 1.0, 4, dtype, DEV)
    aa.aa_rel_attention_grad(attn, dout, dq, dk, dv, aa.rel_attention_scratch(attn, bias), bias=bias, dtable=dt)
    torch.cuda.synchronize()
    a = 0
    for m in lens:
        vs, o = f64(v[a:a + m, 0]), f64(out[a:a + m, 0])
        first = np.zeros(64) if low == -float("inf") else vs[0]
        assert np.allclose(o[0], first, atol=1e-2)
        for i in range(1, m):
            assert np.allclose(o[i], vs[:i].mean(axis=0), atol=2e-2)
        a += m
    for t in (out, dq, dk, dv, dt):
        assert torch.isfinite(t).all()
    assert not dt[0, 0].item()


def test_attention_ignores_what_lies_outside_of_a_sequence(aa):
    """Tokens behind the counted sequences hold NaN and infinities; nothing of them reaches the result and their rows stay as they are."""
    lens = [30, 70, 20]
    for dtype in (F32, BF16):
        clean = check_attention(aa, lens, lens, 2, 1, 64, dtype, False, p=0.1)
        n = sum(lens)
        q, k, v = (torch.cat([W.normal((n, h, 64), 1.0, 42 + i, dtype, DEV), torch.full((80, h, 64), float("nan") if i else float("inf"), dtype=dtype, device=DEV)])
                   for i, h in enumerate((2, 1, 1)))
        off = i32(list(np.concatenate([[0], np.cumsum(lens), [n + 80]])))
        table = W.normal((16, 2), 0.5, 40, F32, DEV)
        attn, bias = B.attention(q, k, v, off, max_q=100, max_k=100, count_dev=i32([3])), B.rel_bias(table, 40)
        drop = B.dropout_rule(0.1, 77, 5, 2, i32([1, 4, 7, 10]), 100)
        out = torch.full_like(q, 7.0)
        aa.aa_rel_attention(attn, out, bias=bias, dropout=drop)
        dout = torch.cat([W.normal((n, 2, 64), 1.0, 45, dtype, DEV), torch.full((80, 2, 64), float("nan"), dtype=dtype, device=DEV)])
        dq, dk, dv, dt = torch.full_like(q, 7.0), torch.full_like(k, 7.0), torch.full_like(v, 7.0), torch.empty_like(table)
        aa.aa_rel_attention_grad(attn, dout, dq, dk, dv, aa.rel_attention_scratch(attn, bias), bias=bias, dropout=drop, dtable=dt)
        for name, t in (("out", out), ("dq", dq), ("dk", dk), ("dv", dv)):
            assert np.array_equal(f64(t)[:n], clean[name]) and np.all(f64(t)[n:] == 7.0)
        # how pairs are shared between the partial sums may depend on the number of sequences: equal up to the order of additions
        assert np.allclose(f64(dt), clean["dtable"], rtol=1e-4, atol=1e-4)


def test_attention_is_reproducible_and_follows_its_stream(aa):
    lens = [100, 3, 257, 64]
    table = W.normal((32, 4), 0.5, 40, F32, DEV)
    runs = [run_attention(aa, lens, lens, 4, 2, 64, BF16, True, table, 128, False, 0.1)[-1] for _ in range(2)]
    for name in runs[0]:
        assert np.array_equal(runs[0][name], runs[1][name])
    side = torch.cuda.Stream(DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        other = B.AutoAssist(max_rows=16, max_d=16, device=DEV, stream=side)
        third = run_attention(other, lens, lens, 4, 2, 64, BF16, True, table, 128, False, 0.1)[-1]
    other.close()
    for name in runs[0]:
        assert np.array_equal(runs[0][name], third[name])


def test_attention_gradient_against_differences(aa):
    """Central differences of the fp32 forward call along random directions, step 2^-6: truncation ~1e-4 of the second order's scale, rounding ~1e-4."""
    lens, heads, kv, dim = [6, 20], 4, 2, 16
    table = W.normal((16, heads), 0.5, 40, F32, DEV)
    q, k, v, dout, ids, got = run_attention(aa, lens, lens, heads, kv, dim, F32, True, table, 10, False, 0.2)
    drop = B.dropout_rule(0.2, 77, 5, 2, i32(ids), 100)

    def objective(q, k, v, table):
        out = torch.empty_like(q)
        aa.aa_rel_attention(B.attention(q, k, v, offs(lens), causal=True), out, bias=B.rel_bias(table, 10, False), dropout=drop)
        return float((out.double() * dout.double()).sum())

    args = {"q": q, "k": k, "v": v, "table": table}
    eps = 2.0**-6
    for n, name in enumerate(args):
        d = W.normal(tuple(args[name].shape), 1.0, 60 + n, F32, DEV)
        d = d / d.norm()
        up, down = (objective(**{**args, name: (args[name] + sign * eps * d).contiguous()}) for sign in (1, -1))
        want = (up - down) / (2 * eps)
        assert abs((f64(d) * got["d" + name]).sum() - want) <= 2e-3 * (1 + abs(want))


def test_attention_refusals_and_latched_offsets(aa):
    q, k = torch.zeros((10, 4, 16), device=DEV), torch.zeros((10, 2, 16), device=DEV)
    off = i32([0, 4, 10])
    out = torch.full_like(q, 7.0)
    table = torch.zeros((16, 4), device=DEV)

    def status(**kw):
        a = B.attention(q, k, k, off)
        for n, x in kw.items():
            setattr(a, n, x)
        with pytest.raises(B.AutoAssistError) as e:
            aa.aa_rel_attention(a, out)
        return e.value.status

    assert status(kv_heads=3) == status(heads=0) == status(head_dim=0) == status(dtype=5) == status(n_seq=-1) == status(max_q=-1) == B.AA_ERR_INVALID_ARG
    assert status(scale=float("nan")) == status(q_offsets=None) == B.AA_ERR_INVALID_ARG
    wide = torch.zeros((4, 1, 264), device=DEV)
    with pytest.raises(B.AutoAssistError) as e:
        aa.aa_rel_attention(B.attention(wide, wide, wide, i32([0, 4])), torch.zeros_like(wide))
    assert e.value.status == B.AA_ERR_UNSUPPORTED
    attn = B.attention(q, k, k, off)
    with pytest.raises(B.AutoAssistError) as e:
        aa.aa_rel_attention(attn, out, bias=B.rel_bias(torch.zeros((15, 4), device=DEV), 40))
    assert e.value.status == B.AA_ERR_INVALID_ARG
    for bad in (lambda: aa.aa_rel_attention(attn, out, bias=B.rel_bias(torch.zeros((16, 3), device=DEV), 40)), lambda: aa.aa_rel_attention(attn, out[:9]),
                lambda: aa.aa_rel_attention_grad(attn, out, out.clone(), k.clone(), k.clone(), torch.empty(1 << 20, dtype=torch.uint8, device=DEV), dtable=table),
                lambda: B.attention(q, k.to(BF16), k.to(BF16), off), lambda: B.attention(q, k, k, off, i32([0, 10]))):
        with pytest.raises(TypeError):
            bad()
    shared = torch.zeros((10, 1, 16), device=DEV).expand(10, 2, 16)          # dk with overlapping heads
    with pytest.raises(B.AutoAssistError) as e:
        aa.aa_rel_attention_grad(attn, out, torch.empty_like(q), shared, k.clone(), aa.rel_attention_scratch(attn))
    assert e.value.status == B.AA_ERR_INVALID_ARG
    with pytest.raises(B.AutoAssistError) as e:
        aa.aa_rel_attention_grad(attn, out, torch.empty_like(q), k.clone(), k.clone(), torch.empty(512, dtype=torch.uint8, device=DEV))
    assert e.value.status == B.AA_ERR_WORKSPACE
    # sequences that break the bounds are skipped and latched, the others are evaluated
    for offsets, bound in ((i32([0, 4, 10]), 5), (i32([0, 4, 11]), 20), (i32([0, 4, 2]), 20)):
        out.fill_(7.0)
        aa.aa_rel_attention(B.attention(q, k, k, offsets, max_q=bound, max_k=bound), out)
        torch.cuda.synchronize()
        assert aa.aa_device_status() == B.AA_ERR_BAD_INDEX
        assert torch.all(out[:4] == 0) and torch.all(out[4:] == 7.0)
    # nothing to do
    none = torch.zeros((0, 4, 16), device=DEV)
    aa.aa_rel_attention(B.attention(none, none, none, i32([0])), none)
    dt = torch.full((16, 4), 7.0, device=DEV)
    a0 = B.attention(none, none, none, i32([0, 0]))
    aa.aa_rel_attention_grad(a0, none, none, none, none, aa.rel_attention_scratch(a0, B.rel_bias(table, 40)), bias=B.rel_bias(table, 40), dtable=dt)
    assert not dt.any() and aa.aa_device_status() == B.AA_OK


# ---------------------------------------------------------------------------------------------------- the operators together

def test_screened_batch_through_every_operator(aa):
    """Screen a pool, cut the batch, train-step operators on it with device counts only; against the reference on the same batch."""
    cfg = W.TranslationShape(n=256, buckets=4096, len_lo=3, len_hi=40, vocab=500, token_budget=600)
    indptr, col, val, lengths = cfg.csr(DEV)
    idx, cnt = torch.zeros(256, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    aa2 = B.AutoAssist(max_rows=2048, max_d=4096, device=DEV)
    w, b = W.linear_assistant(4096, 2, DEV)
    aa2.aa_score_shrink(B.csr_features(indptr, col, val, 4096), B.linear_assistant(w, b), 0.2, 1, 0, idx, cnt)
    m, used, off = (torch.zeros(k, dtype=torch.int32, device=DEV) for k in (1, 1, 257))
    aa2.aa_batch_cut(idx, cnt, 256, m, used, lengths=lengths, token_budget=cfg.token_budget, out_offsets=off)
    rows, h, d = cfg.token_budget, 2, 32
    x = W.normal((rows, h * d), 1.0, 1, F32, DEV)
    rule = lambda site: B.dropout_rule(0.1, 3, 0, site, idx)  # noqa: E731
    table = W.normal((32, h), 0.5, 2, F32, DEV)
    t3 = lambda t: t.view(rows, h, d)  # noqa: E731
    attn = B.attention(t3(x), t3(x), t3(x), off, max_q=40, max_k=40, count_dev=m)
    o, y = torch.zeros_like(x), torch.zeros_like(x)
    aa2.aa_rel_attention(attn, t3(o), bias=B.rel_bias(table, 20), dropout=rule(0))
    aa2.aa_dropout(o, rule(1), y, residual=x, offsets=off, count_dev=m)
    proj = W.normal((h * d, cfg.vocab), 0.2, 3, F32, DEV)
    logits = y @ proj
    labels = W.randint(0, cfg.vocab, (rows,), 4, DEV)
    g, loss = torch.zeros_like(logits), torch.zeros(256, device=DEV)
    aa2.aa_instance_loss_grad(B.logits_desc(logits), labels, g, offsets=off, count_dev=m, out_loss=loss)
    torch.cuda.synchronize()
    assert aa2.aa_device_status() == B.AA_OK
    aa2.close()
    M = int(m.item())
    ends = f64(off).astype(int)[:M + 1]
    assert 5 < M < 256 and ends[M] <= rows
    xs, want = f64(x), np.zeros((rows, h * d))
    for s in range(M):
        sl, ident = slice(ends[s], ends[s + 1]), int(idx[s].item())
        n = ends[s + 1] - ends[s]
        q = xs[sl].reshape(n, h, d)
        a = R.attention_sequence(q, q, q, d ** -0.5, False, f64(table), 20, True, R.attention_factor(h, n, n, 0.1, 3, 0, 0, ident))["out"].reshape(n, h * d)
        want[sl] = xs[sl] + a * R.dropout_factor(n, h * d, 0.1, 3, 0, 1, ident)
    T = ends[M]
    assert np.max(np.abs(f64(y)[:T] - want[:T])) <= 1e-4 and not f64(y)[T:].any()
    ref_logits = f64(logits)[:T]
    f = R.row_losses(ref_logits, f64(labels).astype(int)[:T])
    inst = np.repeat(np.arange(M), np.diff(ends))
    sums = np.bincount(inst, f, M)
    assert np.all(np.abs(f64(loss)[:M] - sums) <= 1e-4 * np.maximum(1, np.diff(ends)))
    check_loss(logits[:T], f64(labels).astype(int)[:T], np.full(T, 1.0 / M), g[:T], F32)
    assert not f64(g)[T:].any() and O is not None
