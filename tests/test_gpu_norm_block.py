"""The example's block: norm, linear layers and their gradients in a run, and the same block in 4 bits, stage by stage."""
import importlib.util
import os

import pytest
import torch

from feed_forward_util import assert_close, device_ok
from fp4_util import linear64, quantized64, unpacked, values_of
from norm_util import check_backward, check_forward
from paper_2505_01637_b200 import binding as mb

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF = torch.bfloat16


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("norm_block", os.path.join(ROOT, "examples", "norm_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def inputs(tokens, d):
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    return [torch.randn(tokens, d, generator=g, device="cuda").to(BF) for _ in range(2)]


@pytest.mark.parametrize("tokens,d,f", [(300, 256, 136), (5, 128, 64), (129, 264, 100), (700, 520, 1024)])
def test_training(example, tokens, d, f):
    block = example.NormBlock(tokens, d, f)
    x, dout = inputs(tokens, d)
    forward, worst = example.check(block, x, dout)
    # Three bf16 roundings forward (n, h, out), four backward (dH, dZ, dN, result): each at most 2^-8 of its value and
    # independent, so 2^-8 * sqrt(4) with a factor of two to spare.
    assert forward < 2 ** -6 and worst < 2 ** -6, (forward, worst)
    check_forward(x, block.gamma, block.beta, example.EPS, False, block.n, block.mean, block.rstd)
    check_backward(x, block.gamma, block.mean, block.rstd, block.dn, dout, False, block.dx, block.dgamma, block.dbeta)


def decoded(t):
    q = torch.cat([t.q, torch.full((64,), 0xEE, dtype=torch.uint8, device="cuda")])
    s = torch.cat([t.scales, torch.full((64,), 0xEE, dtype=torch.uint8, device="cuda")])
    return unpacked(q, s, t.fmt, t.rows, t.parts, t.k)


@pytest.mark.parametrize("fmt", [mb.MORELLO_MXFP4, mb.MORELLO_NVFP4])
@pytest.mark.parametrize("tokens,d,f", [(1, 256, 136), (12, 520, 1000), (300, 256, 520), (129, 264, 100)])
def test_serving_in_four_bits(example, tokens, d, f, fmt):
    block = example.NormBlock(tokens, d, f, fmt=fmt)
    x, _ = inputs(tokens, d)
    block.quantize_weights()
    graph = torch.cuda.CUDAGraph()
    block.serve(x)
    eager = block.out.clone()
    with torch.cuda.graph(graph):
        block.serve(x)
    block.out.fill_(0)
    graph.replay()
    torch.cuda.synchronize()
    device_ok()
    assert torch.equal(block.out, eager)
    # Every stage from what the one before it left.
    check_forward(x, block.gamma, block.beta, example.EPS, False, block.n, block.mean, block.rstd)
    values = []
    for t, of in ((block.n4, block.n), (block.w1_4, block.w1.t()), (block.h4, block.h), (block.w2_4, block.w2.t())):
        codes, byte = decoded(t)
        want, want_byte = quantized64(of, fmt)
        assert torch.equal(byte, want_byte)
        values.append(values_of(codes, byte, fmt))
        assert torch.equal(values[-1], values_of(want, want_byte, fmt))
    n, w1, h, w2 = values
    assert_close(block.h, *linear64(n, w1, None, None, None, "silu", True, d, False), "h")
    assert_close(block.out, *linear64(h, w2, None, None, x, "none", False, f, False), "out")
