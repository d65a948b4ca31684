"""The logits' gradient where a token names an expert more than once: the places' terms are added up."""
import pytest
import torch

from feed_forward_util import assert_close, gen
from paper_2505_01637_b200 import binding as mb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,experts,topk", [(1, 4, 2), (50, 8, 4), (300, 64, 6), (40, 300, 32), (20, 1024, 8)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_repeated_experts(tokens, experts, topk, score, renorm, kind):
    g = gen(tokens + experts)
    x = torch.randn(tokens, experts, generator=g, device="cuda").to(kind)
    idx = torch.randint(0, min(experts, topk), (tokens, topk), generator=g, device="cuda", dtype=torch.int32)
    idx[0, :2] = experts - 1
    skip = torch.rand(tokens, topk, generator=g, device="cuda") < 0.1
    skip[0] = False
    idx[skip] = -1
    dw = torch.randn(tokens, topk, generator=g, device="cuda")
    dx = torch.full_like(x, float("nan"))
    mb.morello_route_backward(0 if score == "softmax" else 1, renorm, 1.5, kind == torch.float32, tokens, experts, topk, x, idx, dw, dx)
    x64 = x.double().requires_grad_(True)
    p = torch.softmax(x64, 1) if score == "softmax" else torch.sigmoid(x64)
    w = torch.where(idx >= 0, torch.gather(p, 1, idx.long().clamp(min=0)), torch.zeros((), dtype=torch.float64, device="cuda"))
    if renorm:
        w = w / w.sum(1, keepdim=True).clamp(min=1e-300)
    (want,) = torch.autograd.grad(w, x64, 1.5 * dw.double())
    # topk terms of at most 1.5 |dw| each, in f32
    bound = 1e-5 * (1.5 * dw.double().abs().sum(1, keepdim=True) + 1e-3)
    assert_close(dx, want, bound.expand_as(want))
