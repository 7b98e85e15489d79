"""Host-side refusals of the Boss operators that need no GPU: the calls end before anything is enqueued."""
import ctypes

import pytest
import torch

from paper_1905_03381_b200 import binding as B
from paper_1905_03381_b200 import build

# the descriptors below hold no real addresses, so no call may get as far as a device
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="refusals are looked at where nothing can run")


@pytest.fixture(scope="module")
def lib():
    build.build()
    return B.lib()


def matrix(rows, cols):
    return B.aa_rows(1 << 20, B.AA_BF16, 0, rows, cols, cols)


def test_dropout_of_rows_whose_column_numbers_do_not_fit(lib):
    """A lane's column number may pass the row's end by a unit of the kernel; it has to stay below 2^31."""
    ctx = ctypes.create_string_buffer(1 << 16)
    rule = B.aa_dropout_rule()
    rule.p = 0.5

    def status(cols):
        m = matrix(1, cols)
        return lib.aa_dropout(ctx, ctypes.byref(m), ctypes.byref(rule), None, 0, None, None, ctypes.byref(m))

    for cols in (2**31 - 16, 2**31 - 600, 2**31 - 1023):
        assert status(cols) == B.AA_ERR_UNSUPPORTED
    assert status(2**31) == status(0) == B.AA_ERR_INVALID_ARG
    assert status(2**31 - 1024) not in (B.AA_ERR_UNSUPPORTED, B.AA_ERR_INVALID_ARG)


def test_kernels_that_start_early_read_what_the_call_before_may_write_by_ordinary_loads():
    """Every kernel of the Boss operators may start while the launch before it still runs and waits for it on the device.  Loads of the read-only path
    are defined for memory that nothing writes while the kernel lives, and may be moved above that wait; the lists, counts, offsets, weights and row
    statistics that the launch before may have written have to be read by ordinary loads."""
    import glob
    import os
    import re

    files = [os.path.join(build.CSRC, f) for f in ("boss_common.cuh", "dropout.cu", "instance_loss_grad.cu")] + glob.glob(os.path.join(build.CSRC, "rel_attention*"))
    assert len(files) >= 11
    for path in files:
        for n, line in enumerate(open(path), 1):
            code = line.split("//")[0]
            assert not re.search(r"__ldg\(|\.nc\b|__restrict__", code), f"{os.path.basename(path)}:{n}: {line.strip()}"
