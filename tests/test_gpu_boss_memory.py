"""What the Boss operators accept as memory of their operands: views of one packed array, the operand itself where the call says so, no overlap."""
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


def refused(call):
    with pytest.raises(B.AutoAssistError) as e:
        call()
    assert e.value.status == B.AA_ERR_INVALID_ARG


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
