"""Linear layers and layer normalisation at sizes that fill the GPU - tiles of pairs of CTAs, several of them one after the other, contractions cut or summed in runs,
several rows a group of threads - against fp64 on the GPU.  Bars as in test_gpu_boss_step, and for the longest sums:
  bf16 sums: the matrix units round towards zero once in 16 terms, by half a step on average (2^-24 of the sum so far, which is half of the run's on average); runs of
             16,384 terms are added up in fp32.  So 1,024 2^-24 / 2 = 2^-15 of the sum of absolute terms, and 2^-24 of it for each run.
"""
import pytest
import torch

from paper_1905_03381_b200 import binding as B
from paper_1905_03381_b200 import build
from test_gpu_boss_step import BF16, DEV, HALF

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def aa():
    build.build()
    ctx = B.AutoAssist(max_rows=1 << 10, max_d=64, device=DEV)
    yield ctx
    torch.cuda.synchronize()
    assert ctx.aa_device_status() == B.AA_OK
    ctx.close()


def random(shape, seed, dtype=BF16, std=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV).mul_(std).to(dtype)


def below(got, bar):
    off = got.double().abs() - bar
    assert torch.all(off <= 0), f"off by {got.double().abs().max():.3e}, {off.max():.3e} above the bar"


def cancelling(rows, cols, seed, minus):
    """Numbers of [1, 2), then the same again (minus: with their signs turned)."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    half = (1.0 + torch.rand((rows // 2, cols), generator=g, device=DEV)).to(BF16)
    return torch.cat([half, -half if minus else half])


def test_weights_gradients_of_many_tokens_keep_their_sums(aa):
    """Sums over 196,608 tokens whose second half takes back the first: every output is 0, and what it is off by has nowhere to hide."""
    tokens, n = 196_608, 2304                                     # 81 tiles of a pair: whole ones, and some that are cut
    x, dout = cancelling(tokens, n, 1, False), cancelling(tokens, n, 2, True)
    w = torch.zeros((n, n), dtype=BF16, device=DEV)
    dw, db = torch.empty_like(w), torch.empty(n, device=DEV)
    aa.aa_linear_grad(x, w, dout, aa.linear_grad_scratch(x, w), dw=dw, dbias=db)
    half = tokens // 2
    size = 2.0 * (x[:half].float().t() @ dout[:half].float()).t().double()
    below(dw, (2.0**-15 + tokens / 16384 * 2.0**-24) * size)
    # dbias: eight tokens at a time in fp32, rounded to nearest, of which a thread has every 32nd token
    below(db, tokens / 8 * 2.0**-24 * 2.0 * dout[:half].double().sum(0))


def test_long_contractions_keep_their_sums(aa):
    """The same along the inputs of a layer, forward and in dx."""
    k = 131_072
    x = cancelling(k, 2048, 3, True).t().contiguous()
    w = cancelling(k, 1100, 4, False).t().contiguous()
    out = torch.empty((2048, 1100), dtype=BF16, device=DEV)
    aa.aa_linear(x, w, out)
    size = 2.0 * (x[:, :k // 2].float() @ w[:, :k // 2].float().t()).double()
    below(out, (2.0**-15 + 2.0**-19) * size)                      # runs of 256 terms
    dout, w = cancelling(k, 1100, 5, True).t().contiguous(), cancelling(k, 2048, 6, False)
    x = torch.zeros((1100, 2048), dtype=BF16, device=DEV)
    dx = torch.empty_like(x)
    aa.aa_linear_grad(x, w, dout, aa.linear_grad_scratch(x, w), dx=dx)
    size = 2.0 * (dout[:, :k // 2].float() @ w[:k // 2].float()).double()
    below(dx, (2.0**-15 + k / 16384 * 2.0**-24) * size)
