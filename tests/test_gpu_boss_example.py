"""The example that trains a small Boss through the operators, end to end on the GPU."""
import importlib.util
import os

import pytest
import torch

from paper_1905_03381_b200 import workloads as W

pytestmark = pytest.mark.gpu


def load_example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "translation_boss.py")
    spec = importlib.util.spec_from_file_location("translation_boss", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("depth", [0, 1])
def test_the_boss_learns_on_screened_batches(depth):
    """From log(vocab) a token at the start, the loss must fall by at least a fifth; every batch keeps to the token budget."""
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    cfg = W.TranslationShape(n=512, buckets=4096, len_lo=8, len_hi=64, vocab=100, token_budget=2048)
    got = load_example().train(80, cfg, depth)
    first, last = got[0][0], sum(x for x, _ in got[-5:]) / 5
    assert abs(first - torch.log(torch.tensor(100.0)).item()) < 0.5
    assert last < 0.8 * first, (first, last)
    assert all(2048 // 64 <= m <= 2048 // 8 for _, m in got)
