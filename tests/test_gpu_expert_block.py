"""The sparse feed-forward block of the example, forward and backward, at a training and a decoding size."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("expert_block", os.path.join(ROOT, "examples", "expert_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("tokens,d,f,experts,topk", [(300, 256, 136, 8, 2), (5, 128, 64, 16, 4), (129, 264, 100, 4, 3)])
def test_block(example, tokens, d, f, experts, topk):
    block = example.ExpertBlock(tokens, d, f, experts, topk)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x, dout = (torch.randn(tokens, d, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    forward, worst = example.check(block, x, dout)
    # Three bf16 roundings forward (h, out; x itself is exact), four backward (dY, dH, dZ, result): each at most
    # 2^-8 of its value and independent, so 2^-8 * sqrt(4) with a factor of two to spare.
    assert forward < 2 ** -6 and worst < 2 ** -6, (forward, worst)
