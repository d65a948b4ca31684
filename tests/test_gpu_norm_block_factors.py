"""The example's block in 4 bits with a factor for every tensor: what the quantisation loses does not grow with the layer.

For Gaussian values in blocks of 16 that are scaled so that the largest of a block is 6 s: it is 2.08 deviations on average, so
a deviation is 2.9 s.  The grid's steps are 1/2 below 2 s (0.69 deviations, 51 % of the values), 1 below 4 s (33 %) and 2
above (16 %), an error's mean square is step^2 / 12 there: 0.011 + 0.027 + 0.055 = 0.093 s^2, 0.106 of a deviation.  Scales are
off by 2^-4 at most, which moves the steps by as much: at most 0.113, and 0.115 leaves a part in fifty for the sample."""
import importlib.util
import math
import os

import pytest
import torch

from feed_forward_util import assert_close, device_ok
from fp4_util import linear64, quantized64, unpacked, values_of
from paper_2505_01637_b200 import binding as mb

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF = torch.bfloat16
NV, MX = mb.MORELLO_NVFP4, mb.MORELLO_MXFP4
LOSS = 0.115


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("norm_block", os.path.join(ROOT, "examples", "norm_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def rows(tokens, d):
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    return torch.randn(tokens, d, generator=g, device="cuda").to(BF)


def read_back(t):
    y = torch.empty(t.rows, t.k, device="cuda")
    alpha = None if t.mult is None else 1 / t.mult
    mb.morello_fp4_dequantize(t.fmt, 1, t.rows, t.parts, t.k, t.q, t.scales, alpha, y)
    return y.double()


def loss(got, want):
    return float((got.double() - want.double()).norm() / want.double().norm())


@pytest.mark.parametrize("tokens,d,f", [(64, 256, 2048), (16, 256, 65536), (4, 4096, 16384)])
def test_loss_of_the_weights_and_of_the_block(example, tokens, d, f):
    block, x = example.NormBlock(tokens, d, f), rows(tokens, d)
    full = block.forward(x).clone()
    block.quantize_weights(x)
    low = block.serve(x)
    device_ok()
    assert loss(read_back(block.w1_4), block.w1.t()) <= LOSS
    assert loss(read_back(block.w2_4), block.w2.t()) <= LOSS
    # z loses sqrt(2) LOSS; h = silu(g) u of Gaussian g and u has mean square 0.356, its change silu'(g) u dg + silu(g) du
    # (0.379 + 0.356) dz^2 (means of silu^2 and silu'^2 over a unit Gaussian: 0.356, 0.379); h and W2 lose LOSS each again (h is
    # no Gaussian: 0.09 for drawn g and u).
    z = math.sqrt(2) * LOSS
    bound = math.sqrt((0.379 + 0.356) / 0.356 * z * z + 2 * LOSS ** 2)
    change = full.double() - x.double()
    assert float((low.double() - full.double()).norm() / change.norm()) <= bound


@pytest.mark.parametrize("fmt", [NV, MX])
@pytest.mark.parametrize("tokens,d,f", [(12, 520, 1000), (300, 256, 520)])
def test_stages_with_factors(example, tokens, d, f, fmt):
    block, x = example.NormBlock(tokens, d, f, fmt=fmt), rows(tokens, d)
    block.quantize_weights(x)
    assert (block.alpha1 is None) == (fmt == MX) and (block.n4.mult is None) == (fmt == MX)
    block.serve(x)
    device_ok()
    values = []
    for t, of in ((block.n4, block.n), (block.w1_4, block.w1.t()), (block.h4, block.h), (block.w2_4, block.w2.t())):
        guard = torch.full((64,), 0xEE, dtype=torch.uint8, device="cuda")
        codes, byte = unpacked(torch.cat([t.q, guard]), torch.cat([t.scales, guard]), fmt, t.rows, t.parts, t.k)
        want, want_byte = quantized64(of, fmt, t.mult)
        assert torch.equal(byte, want_byte)
        values.append(values_of(codes, byte, fmt))
        assert torch.equal(values[-1], values_of(want, want_byte, fmt))
    n, w1, h, w2 = values
    assert_close(block.h, *linear64(n, w1, block.alpha1, None, None, "silu", True, d, False), "h")
    assert_close(block.out, *linear64(h, w2, block.alpha2, None, x, "none", False, f, False), "out")


def test_new_weights_under_a_captured_pass(example):
    block, x = example.NormBlock(9, 264, 520), rows(9, 264)
    block.quantize_weights(x)
    graph = torch.cuda.CUDAGraph()
    block.serve(x)
    with torch.cuda.graph(graph):
        block.serve(x)
    block.w1.mul_(8)
    block.w2.mul_(0.01)
    block.quantize_weights(x)
    want = block.serve(x).clone()
    block.out.fill_(0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(block.out, want)
