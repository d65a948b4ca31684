"""f32 outputs on few rows whose contraction is longer than the tensor memory's accumulators hold in parts of 512."""
import pytest
import torch

from feed_forward_util import device_ok, gen, plan_of
from paper_2505_01637_b200 import binding as mb

pytestmark = pytest.mark.gpu

# A part of 512 elements is 32 truncating additions of at most 2^-23 of the largest partial sum each, all one way:
# 32 * 2^-23 = 3.8e-6 at the worst; the parts' sum to nearest leaves a few 2^-24.
LIMIT = 3.9e-6


def bf16(g, *shape, scale=1.0):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.bfloat16) * scale


def off(got, want):
    return float((got - want).norm() / want.norm())


# Strips of columns that fill the device, so that the contraction is not cut into slices.
@pytest.mark.parametrize("m,k,n,gated,colmajor", [(64, 32768, 19072, False, False), (64, 32768, 9536, True, False), (49, 16400, 19100, False, True),
                                                  (40, 32768, 9530, True, True), (64, 2112, 19072, False, False),
                                                  (16, 32832, 19072, False, False)])
def test_uncut(m, k, n, gated, colmajor):
    g = gen(m + k)
    wide = 2 * n if gated else n
    x, w = bf16(g, m, k), bf16(g, *((wide, k) if colmajor else (k, wide)), scale=k ** -0.5)
    y = torch.full((m, n), float("nan"), device="cuda")
    mb.morello_linear(0, gated, 1, colmajor, m, k, n, x, w, None, None, y)
    device_ok()
    x64 = x.double()
    z = torch.empty(m, wide, dtype=torch.float64, device="cuda")
    for c in range(0, wide, 2048):
        part = w[c:c + 2048].double().t() if colmajor else w[:, c:c + 2048].double()
        z[:, c:c + 2048] = x64 @ part
    want = z[:, :n] * z[:, n:] if gated else z
    assert off(y, want) <= LIMIT * (2 ** 0.5 if gated else 1)


@pytest.mark.parametrize("m,k,n", [(64, 65536, 640), (33, 40000, 300)])
def test_cut_into_slices(m, k, n):
    g = gen(m)
    x, w = bf16(g, m, k), bf16(g, k, n, scale=k ** -0.5)
    y, z = torch.empty(m, n, device="cuda"), torch.empty(m, n, device="cuda", dtype=torch.bfloat16)
    mb.morello_linear(0, 0, 1, 0, m, k, n, x, w, None, None, y, z)
    device_ok()
    want = x.double() @ w.double()
    assert off(y, want) <= LIMIT
    assert off(z.double(), want) <= 2 ** -8


@pytest.mark.parametrize("how", ["spread", "one"])
def test_experts(how):
    """Experts of several row chunks among them, whose accumulators are used again."""
    t, topk, e, k, n = 64, 2, 8, 16384, 2560
    g = gen(4)
    idx = torch.full((t, topk), 3, dtype=torch.int32, device="cuda")
    if how == "spread":
        idx = torch.argsort(torch.rand(t, e, generator=g, device="cuda"), 1)[:, :topk].to(torch.int32).contiguous()
    plan, parts = plan_of(idx, e)
    x, w = bf16(g, t, k), bf16(g, e, k, n, scale=k ** -0.5)
    y = torch.empty(parts["row_src"].numel(), n, device="cuda")
    mb.morello_expert_linear(0, 0, 1, 0, 1, t, topk, e, k, n, plan, x, w, None, y)
    device_ok()
    for expert in range(e):
        first, count = int(parts["offsets"][expert]), int(parts["counts"][expert])
        if count:
            token = parts["row_src"][first:first + count].long() // topk
            assert off(y[first:first + count], x[token].double() @ w[expert].double()) <= LIMIT
