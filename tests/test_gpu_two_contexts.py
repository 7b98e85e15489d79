"""Two library contexts on two host threads, each with a stream of its own."""
import ctypes
import subprocess
import threading

import pytest
import torch

from paper_1905_03381_b200 import binding as B
from paper_1905_03381_b200 import build, workloads as W

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

# The calls come from a loop in C: two threads that take turns with the interpreter hardly ever meet inside the library.
LOOP = """
#include "autoassist.h"
int repeat(aa_ctx* ctx, const aa_attn* attn, const aa_rel_bias* bias, const aa_tokens* out, const aa_logits* logits, const int32_t* labels, const aa_rows* grad, int n) {
    for (int i = 0; i < n; ++i) {
        int st = aa_rel_attention(ctx, attn, bias, 0, out);
        if (st == AA_OK) st = aa_instance_loss_grad(ctx, logits, labels, 0, 0, 0, 0, 1.0f, AA_REDUCE_MEAN, 0, grad);
        if (st != AA_OK) return 100 * i + st;
    }
    return 0;
}
"""


def test_calls_of_different_shared_memory_sizes_do_not_refuse_each_other(tmp_path):
    """The same kernels, needing little shared memory on one thread and much on the other (a far-reaching bias; longer rows)."""
    lib = build.build()
    (tmp_path / "loop.c").write_text(LOOP)
    subprocess.check_call(["gcc", "-shared", "-fPIC", "-I", build.INCLUDE, "-o", str(tmp_path / "loop.so"), str(tmp_path / "loop.c"), lib])
    B.lib()
    repeat = ctypes.CDLL(str(tmp_path / "loop.so")).repeat
    off = torch.tensor([0, 5, 9], dtype=torch.int32, device=DEV)
    q = W.normal((9, 1, 64), 1.0, 1, torch.float32, DEV)
    table = W.normal((64, 1), 0.5, 2, torch.float32, DEV)
    label = torch.tensor([3, 4], dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    got, start = {}, threading.Barrier(2)

    def work(name, bias, cols):
        stream = torch.cuda.Stream(DEV)
        ctx = B.AutoAssist(max_rows=16, max_d=16, device=DEV, stream=stream)
        with torch.cuda.stream(stream):
            logits = W.normal((2, cols), 1.0, 3, torch.bfloat16, DEV)
            out, grad = torch.empty_like(q), torch.empty_like(logits)
        attn, desc = B.attention(q, q, q, off), B.logits_desc(logits)
        tokens, rows = B._tokens(out, "out"), B.rows_desc(grad)
        start.wait()
        got[name] = repeat(ctx._ctx, ctypes.byref(attn), None if bias is None else ctypes.byref(bias), ctypes.byref(tokens), ctypes.byref(desc),
                           ctypes.c_void_p(label.data_ptr()), ctypes.byref(rows), 20000)
        stream.synchronize()
        ctx.close()

    threads = [threading.Thread(target=work, args=a) for a in (("little", None, 8200), ("much", B.rel_bias(table, 2048), 32000))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert got == {"little": 0, "much": 0}
