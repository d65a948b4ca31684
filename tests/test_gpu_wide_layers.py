"""Gradients of layers with more columns than one dimension of a grid has strips of 256 for."""
import pytest
import torch

from feed_forward_util import ACTS, BF16, TINY, assert_close, device_ok, dz64, gen
from paper_2505_01637_b200 import binding as mb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [65535 * 256 + 264, 65535 * 256 + 513])
@pytest.mark.parametrize("act,gated", [("relu", False), ("none", True)])
def test_backward(n, act, gated):
    m, k = 2, 2
    g = gen(n)
    wide = 2 * n if gated else n

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.bfloat16)

    x, w, z, dy = randn(m, k), randn(k, wide), randn(m, wide), randn(m, n)
    dx, dw, db = torch.full_like(x, float("nan")), torch.full_like(w, float("nan")), torch.full((wide,), float("nan"), device="cuda")
    mb.morello_linear_backward(ACTS[act], gated, 0, 0, 0, m, k, n, x, w, z, dy, dx, dw, db)
    device_ok()
    dz, edz = dz64(z.double(), dy.double(), act, gated)
    eprod = edz + BF16 * (dz.abs() + edz)
    assert_close(db, dz.sum(0), edz.sum(0) + 1e-5 * dz.abs().sum(0) + TINY, "db")
    x64 = x.double()
    assert_close(dw, x64.t() @ dz, x64.abs().t() @ eprod + 1e-5 * (x64.abs().t() @ dz.abs()) + TINY, "dW")
    w64 = w.double()
    assert_close(dx, dz @ w64.t(), eprod @ w64.abs().t() + 1e-5 * (dz.abs() @ w64.abs().t()) + TINY, "dX")
