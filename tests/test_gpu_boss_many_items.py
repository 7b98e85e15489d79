"""The Boss operators on batches that give every resident CTA, warp or sub-warp several items, so that what is carried from one item to the next
(ring stages and their phases, prefetched operands, running instances, partial sums of the table's gradient) is compared with the fp64 reference.
Bars as for the small cases."""
import numpy as np
import pytest
import torch

import boss_reference as R
from paper_1905_03381_b200 import binding as B
from paper_1905_03381_b200 import build, workloads as W
from test_gpu_boss_ops import check_attention, check_dropout, check_loss, f64, i32, offs

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


def sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


# ---- gradient of the instance loss: rows of 16..64 KB go through one persistent CTA an SM, up to six stages each

@pytest.mark.parametrize("dtype,rows,cols,pad", [(BF16, 1500, 8200, 0), (BF16, 1203, 8203, 0), (F32, 1300, 4200, 0), (F32, 1100, 4202, 1), (BF16, 950, 32000, 0)])
def test_loss_gradient_of_many_long_rows(aa, dtype, rows, cols, pad):
    assert rows > 6 * sms() and 1024 < (cols * (2 if dtype == BF16 else 4) + 15) // 16 <= 4096
    rng = np.random.default_rng(cols)
    x = W.normal((rows, cols + pad), 3.0, cols, dtype, DEV)[:, :cols]
    x[5, 7:] = -1e30
    y = rng.integers(0, cols, rows).astype(np.int32)
    y[rng.random(rows) < 0.2] = -1
    y[40:60] = -1                                               # a run of padding rows
    lens = []
    while sum(lens) < rows:
        lens += [0, 0, 0] if rng.random() < 0.2 else [int(rng.integers(1, 20))]
    lens[-1] -= sum(lens) - rows
    n = len(lens)
    w = rng.uniform(0.5, 4.0, n).astype(np.float32)
    inst = np.repeat(np.arange(n), lens)
    losses = R.row_losses(f64(x), y)
    for count in (None, n - n // 4):
        m = n if count is None else count
        end = int(sum(lens[:m]))
        grad, loss = torch.full((rows, cols + pad), 7.0, dtype=dtype, device=DEV)[:, :cols], torch.full((n,), -5.0, device=DEV)
        aa.aa_instance_loss_grad(B.logits_desc(x), i32(y), grad, offsets=offs(lens), weight=torch.tensor(w, device=DEV), out_loss=loss,
                                 count_dev=None if count is None else i32([count]))
        check_loss(x[:end], y[:end], w.astype(np.float64)[inst[:end]] / m, grad[:end], dtype)
        assert torch.all(grad[end:] == 7.0) and torch.all(loss[m:] == -5.0)
        sums = np.bincount(inst[:end], losses[:end], m)
        assert np.all(np.abs(f64(loss)[:m] - sums) <= 1e-4 * np.maximum(1, lens[:m]) + 2.0**-22 * np.abs(sums))
    z = torch.empty((rows, cols + pad), dtype=dtype, device=DEV)[:, :cols].copy_(x)
    aa.aa_instance_loss_grad(B.logits_desc(z), i32(y), z, mean=False)        # in place, a row an instance
    check_loss(x, y, np.ones(rows), z, dtype)


# ---- dropout: a sub-warp walks a run of rows, from instance to instance

@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols,lanes", [(30000, 512, 32), (30011, 130, 32), (21000, 1001, 32), (80000, 104, 8), (80003, 99, 8), (320000, 24, 2)])
def test_dropout_of_many_sentences(aa, dtype, rows, cols, lanes):
    assert rows > 8 * sms() * 256 // lanes                      # more rows than sub-warps that can be resident
    rng = np.random.default_rng(rows)
    lens = np.where(rng.random(rows) < 0.4, 0, rng.integers(1, 40, rows))
    lens = lens[:int(np.searchsorted(np.cumsum(lens), rows))]
    lens[100:140] = 0                                           # a long run of empty ones
    n, used = len(lens), int(lens.sum())
    assert rows - 4000 < used <= rows
    ids = rng.permutation(4 * n)[:n].astype(np.int64)
    seed, step, site = 2**40 + 9, 3, 6
    x, res = W.normal((rows, cols), 1.0, 3, dtype, DEV), W.normal((rows, cols), 1.0, 4, dtype, DEV)
    key = R.philox(ids & 0xFFFFFFFF, ids >> 32, step, 0, seed & 0xFFFFFFFF, seed >> 32)[2:]
    inst = np.repeat(np.arange(n), lens)
    start = np.concatenate([[0], np.cumsum(lens)])
    groups = -(-cols // 8)
    block = (np.arange(used) - start[inst])[:, None] * groups + np.arange(groups)[None, :]
    t = R.threshold(0.3)
    factor = (R.draws([k[inst][:, None] for k in key], block, site).reshape(used, groups * 8)[:, :cols] >= t) * (65536.0 / (65536 - t))
    for count in (None, n // 2):
        end = used if count is None else int(start[count])
        out = torch.full_like(x, 7.0)
        aa.aa_dropout(x, B.dropout_rule(0.3, seed, step, site, i32(ids)), out, residual=res, offsets=i32(start), count_dev=None if count is None else i32([count]))
        check_dropout(out[:end], x[:end], res[:end], factor[:end], dtype)
        assert torch.all(out[end:] == 7.0)
    aa.aa_dropout(x, B.dropout_rule(0.3, seed, step, site, i32(ids)), res, offsets=i32(start))
    check_dropout(res[:used], x[:used], None, factor, dtype)


# ---- attention of sentences: a CTA takes sentence after sentence, 32 candidates looked up at a time

def sentence_lengths(n, seed, long_share):
    """Runs of equal and of unequal lengths, empty sides among them."""
    rng = np.random.default_rng(seed)
    lk = np.where(rng.random(n) < long_share, rng.integers(65, 129, n), rng.integers(0, 41, n))
    lq = np.where((np.arange(n) // 50) % 2 == 0, lk, np.where(lk > 64, rng.integers(0, 129, n), rng.integers(0, 65, n)))
    return [int(v) for v in lq], [int(v) for v in lk]


@pytest.mark.parametrize("dtype,heads,kv,dim,n,long_share,causal", [
    (BF16, 16, 16, 64, 950, 0.2, True), (BF16, 16, 16, 32, 950, 0.2, False), (BF16, 32, 16, 64, 900, 0.15, True), (BF16, 12, 12, 128, 500, 0.0, False),
    (BF16, 24, 12, 128, 420, 0.0, True), (F32, 16, 16, 24, 300, 0.2, True)])
def test_attention_of_many_sentences(aa, dtype, heads, kv, dim, n, long_share, causal):
    lq, lk = sentence_lengths(n, heads + dim, long_share)
    # candidates of one CTA of a class that keeps an SM to itself: more than a warp looks up at once (fp32: more query tiles than CTAs)
    assert dtype == F32 or n > 32 * (sms() // kv)
    check_attention(aa, lq, lk, heads, kv, dim, dtype, causal, buckets=16, distance=40, both=not causal, p=0.1)


def test_attention_of_sixteen_heads_on_one_key_head(aa):
    """The diagonal sums of so many heads do not fit beside a sentence's tiles: every sentence takes the tiles of the long ones in the backward pass."""
    lens = [5, 1, 0, 33, 64, 17, 130, 2] * 3
    check_attention(aa, lens, lens, 16, 1, 64, BF16, True, buckets=16, distance=40, both=False, p=0.1)


# ---- attention of long sequences: the rows kernel walks query tiles, the keys kernel the tiles of every head of a group

# a wider bias leaves room for fewer stages and operand pairs: at a width of 128 two pairs up to a reach of about 125, three stages up to about 825
@pytest.mark.parametrize("dim,causal,distance", [(64, True, 40), (64, True, 2000), (128, False, 40), (128, True, 40), (128, True, 300), (128, False, 300),
                                                 (128, True, 2000), (72, False, 2000)])
def test_attention_of_several_long_sequences(aa, dim, causal, distance):
    lq, lk = [520, 300, 128, 600, 1, 256, 333], [520, 450, 300, 600, 500, 100, 0]
    tiles = sum((x + 127) // 128 for x in lq)
    assert tiles > 1.5 * (sms() // 16)
    check_attention(aa, lq, lk, 16, 4, dim, BF16, causal, buckets=32, distance=distance, both=not causal, p=0.1)


# ---- few new tokens: as many sequences as fill the GPU without a split of the context

@pytest.mark.parametrize("p", [0.0, 0.2])
def test_new_tokens_of_many_sequences(aa, p):
    rng = np.random.default_rng(3)
    lk = [int(v) for v in rng.integers(0, 400, 300)]
    assert len(lk) * 4 > 8 * sms() // 2
    check_attention(aa, [1] * 300, lk, 8, 4, 64, BF16, True, both=False, p=p, train=False)
