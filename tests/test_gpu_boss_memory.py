"""What the Boss operators accept as memory of their operands: views of one packed array, the operand itself where the call says so, no overlap."""
import numpy as np
import pytest
import torch

from paper_1905_03381_b200 import binding as B
from paper_1905_03381_b200 import build, workloads as W

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def aa():
    build.build()
    ctx = B.AutoAssist(max_rows=1 << 12, max_d=64, device=DEV)
    yield ctx
    torch.cuda.synchronize()
    assert ctx.aa_device_status() == B.AA_OK
    ctx.close()


def offs(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device=DEV)


def refused(call):
    with pytest.raises(B.AutoAssistError) as e:
        call()
    assert e.value.status == B.AA_ERR_INVALID_ARG


# ---- attention

def problem(dtype, lens, heads=4, kv=2, dim=64):
    n = sum(lens)
    q, k, v, g = (W.normal((n, h, dim), 1.0, 50 + i, dtype, DEV) for i, h in enumerate((heads, kv, kv, heads)))
    return q, k, v, g, B.attention(q, k, v, offs(lens), max_q=max(lens), max_k=max(lens), causal=True)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lens", [[9, 40, 3], [300, 20]])
def test_attention_output_may_be_the_queries_themselves_and_no_other_operand(aa, dtype, lens):
    q, k, v, g, attn = problem(dtype, lens)
    want = torch.empty_like(q)
    aa.aa_rel_attention(attn, want)
    aa.aa_rel_attention(attn, q)
    assert torch.equal(q, want)
    q, k, v, g, attn = problem(dtype, lens, kv=4)
    for out in (k, v):
        refused(lambda: aa.aa_rel_attention(attn, out))
    flat = torch.zeros(q.numel() + 64, dtype=dtype, device=DEV)
    shifted = B.attention(flat[:-64].view(q.shape), k, v, offs(lens), causal=True)
    refused(lambda: aa.aa_rel_attention(shifted, flat[64:].view(q.shape)))           # one head further on


def test_one_new_token_over_its_own_queries(aa):
    q, kv = W.normal((3, 8, 64), 1.0, 1, BF16, DEV), W.normal((900, 2, 2, 64), 1.0, 2, BF16, DEV)
    attn = B.attention(q, kv[:, 0], kv[:, 1], offs([1, 1, 1]), offs([700, 150, 50]), 1, 700)
    want = torch.empty_like(q)
    aa.aa_rel_attention(attn, want)
    aa.aa_rel_attention(attn, q)
    assert torch.equal(q, want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lens", [[9, 40, 3], [300, 20]])
def test_attention_gradients_overlap_nothing(aa, dtype, lens):
    q, k, v, g, attn = problem(dtype, lens, kv=4)
    scratch = aa.rel_attention_scratch(attn)
    fresh = lambda: [torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)]  # noqa: E731
    for at in range(3):
        for other in (q, k, v, g):
            grads = fresh()
            grads[at] = other
            refused(lambda: aa.aa_rel_attention_grad(attn, g, *grads, scratch))
    grads = fresh()
    for at in range(3):
        twice = list(grads)
        twice[at] = grads[at - 1]
        refused(lambda: aa.aa_rel_attention_grad(attn, g, *twice, scratch))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lens", [[9, 40, 3], [300, 20], [1]])
@pytest.mark.parametrize("head_major", [False, True])
def test_gradients_as_views_of_one_packed_array(aa, dtype, lens, head_major):
    """q, k, v, dout, out and the gradients interleaved in one array: nothing overlaps, nothing is refused."""
    heads, kv, dim, n = 4, 2, 64, sum(lens)
    q, k, v, g, attn = problem(dtype, lens)
    out, dq, dk, dv = torch.empty_like(q), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    aa.aa_rel_attention(attn, out)
    aa.aa_rel_attention_grad(attn, g, dq, dk, dv, aa.rel_attention_scratch(attn))
    sizes = [heads, kv, kv, heads, heads, heads, kv, kv]
    buf = torch.zeros((sum(sizes), n, dim) if head_major else (n, sum(sizes), dim), dtype=dtype, device=DEV)
    views = [x.transpose(0, 1) for x in buf.split(sizes, 0)] if head_major else buf.split(sizes, 1)
    for view, x in zip(views, (q, k, v, g)):
        view.copy_(x)
    packed = B.attention(*views[:3], offs(lens), max_q=max(lens), max_k=max(lens), causal=True)
    aa.aa_rel_attention(packed, views[4])
    aa.aa_rel_attention_grad(packed, views[3], *views[5:], aa.rel_attention_scratch(packed))
    torch.cuda.synchronize()
    for view, x in zip(views[4:], (out, dq, dk, dv)):
        assert torch.equal(view, x)


# ---- matrices

@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [64, 100, 1001])
def test_rows_as_column_slices_of_one_matrix(aa, dtype, cols):
    """Operands side by side in one matrix do not overlap."""
    buf = W.normal((37, 4 * cols), 1.0, 3, dtype, DEV)
    x, res, out, grad = buf.split(cols, 1)
    rule = B.dropout_rule(0.3, 1, 2)
    want = torch.empty((37, cols), dtype=dtype, device=DEV)
    aa.aa_dropout(x.contiguous(), rule, want, residual=res.contiguous())
    aa.aa_dropout(x, rule, out, residual=res)
    assert torch.allclose(out.float(), want.float(), rtol=2.0**-7 if dtype == BF16 else 2.0**-21, atol=0)
    y = W.randint(0, cols, (37,), 4, DEV)
    aa.aa_instance_loss_grad(B.logits_desc(x.contiguous()), y, want)
    aa.aa_instance_loss_grad(B.logits_desc(x), y, grad)
    assert torch.allclose(grad.float(), want.float(), rtol=1e-2 if dtype == BF16 else 1e-5, atol=1e-7)
    # columns in common are an overlap, whatever their number
    wide = torch.zeros((37, 2 * cols - 1), dtype=dtype, device=DEV)
    refused(lambda: aa.aa_dropout(wide[:, :cols], rule, wide[:, cols - 1:]))
    refused(lambda: aa.aa_instance_loss_grad(B.logits_desc(wide[:, :cols]), y, wide[:, cols - 1:]))


# ---- lists

def test_lists_shorter_than_what_is_read_or_written_are_refused(aa):
    x, n = torch.zeros((6, 16), device=DEV), 6
    i32 = lambda n: torch.zeros(n, dtype=torch.int32, device=DEV)  # noqa: E731
    f32 = lambda n: torch.zeros(n, device=DEV)  # noqa: E731
    rule = lambda n: B.dropout_rule(0.5, 1, 2, row_idx=i32(n))  # noqa: E731
    off = offs([2, 4])
    logits = B.logits_desc(x)
    q = torch.zeros((6, 2, 16), device=DEV)
    attn = B.attention(q, q, q, off)
    many = B.logits_desc(x[:5])
    many.rows = 6
    for bad in (
            lambda: aa.aa_dropout(x, rule(n - 1), x), lambda: aa.aa_dropout(x, rule(1), x, offsets=off), lambda: aa.aa_dropout(x, rule(3), x, offsets=off, n_seg=3),
            lambda: aa.aa_dropout(x, rule(n), x, count_dev=i32(0)),
            lambda: aa.aa_instance_loss_grad(logits, i32(n - 1), x), lambda: aa.aa_instance_loss_grad(logits, i32(n), x, weight=f32(n - 1)),
            lambda: aa.aa_instance_loss_grad(logits, i32(n), x, out_loss=f32(n - 1)), lambda: aa.aa_instance_loss_grad(logits, i32(n), x, offsets=off, n_seg=3),
            lambda: aa.aa_instance_loss_grad(logits, i32(n), x, offsets=off, weight=f32(1)), lambda: aa.aa_instance_loss_grad(logits, i32(n), x, offsets=off, out_loss=f32(1)),
            lambda: aa.aa_instance_loss_grad(logits, i32(n), x, count_dev=i32(0)), lambda: aa.aa_instance_loss_grad(many, i32(n), x),
            lambda: B.attention(q, q, q, off, n_seq=3), lambda: B.attention(q, q, q, off, i32(2), n_seq=2), lambda: B.attention(q, q, q, off, count_dev=i32(0)),
            lambda: aa.aa_rel_attention(attn, torch.empty_like(q), dropout=rule(1)),
            lambda: aa.aa_rel_attention_grad(attn, q.clone(), q.clone(), q.clone(), q.clone(), aa.rel_attention_scratch(attn), dropout=rule(1))):
        with pytest.raises(TypeError):
            bad()
    # exactly as long as needed, and longer
    aa.aa_dropout(x, rule(2), x, offsets=off)
    aa.aa_dropout(x, rule(9), x, offsets=off, n_seg=1)
    aa.aa_instance_loss_grad(logits, i32(n), x, offsets=off, weight=f32(2), out_loss=f32(2))
    aa.aa_rel_attention(B.attention(q, q, q, off, n_seq=1), torch.empty_like(q), dropout=rule(1))
    torch.cuda.synchronize()
    assert aa.aa_device_status() == B.AA_OK


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_sequences_that_break_a_bound_of_zero_are_latched(aa, dtype):
    """A bound of no token at all is a bound like any other: sequences beyond it are skipped and reported."""
    q, k, v, g, _ = problem(dtype, [4, 6])
    table = torch.zeros((16, 4), device=DEV)
    none = torch.zeros((0, 4, 64), dtype=dtype, device=DEV)
    for attn in (B.attention(q, k, v, offs([4, 6]), max_q=0, max_k=6), B.attention(none, k, v, offs([4, 6]), max_k=6)):
        out = torch.full_like(q, 7.0) if attn._keep[0] is q else none
        aa.aa_rel_attention(attn, out, bias=B.rel_bias(table, 40))
        torch.cuda.synchronize()
        assert aa.aa_device_status() == B.AA_ERR_BAD_INDEX and torch.all(out == 7.0)
    attn, bias = B.attention(q, k, v, offs([4, 6]), max_q=0, max_k=0), B.rel_bias(table, 40)
    dq, dk, dv, dt = torch.full_like(q, 7.0), torch.full_like(k, 7.0), torch.full_like(v, 7.0), torch.full_like(table, 7.0)
    aa.aa_rel_attention_grad(attn, g, dq, dk, dv, aa.rel_attention_scratch(attn, bias), bias=bias, dtable=dt)
    torch.cuda.synchronize()
    assert aa.aa_device_status() == B.AA_ERR_BAD_INDEX and all(torch.all(t == 7.0) for t in (dq, dk, dv)) and not dt.any()
    # empty sequences keep to it
    attn = B.attention(q, k, v, offs([0, 0]), max_q=0, max_k=0)
    aa.aa_rel_attention(attn, dq, bias=bias)
    aa.aa_rel_attention_grad(attn, g, dq, dk, dv, aa.rel_attention_scratch(attn, bias), bias=bias, dtable=dt)
    torch.cuda.synchronize()
    assert aa.aa_device_status() == B.AA_OK and all(torch.all(t == 7.0) for t in (dq, dk, dv)) and not dt.any()
