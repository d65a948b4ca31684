"""Norms in place, where a block's next rows are on their way while others are written: Y over X, dX over R."""
import pytest
import torch

from norm_util import check_backward, check_forward, gen, norm64
from paper_2505_01637_b200 import binding as mb

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
# blocks with several groups of rows, teams of less than a warp, rows off 8 columns, rows past the ring
SHAPES = [(20000, 64), (9000, 57), (70, 129), (5000, 333), (4001, 2047), (3000, 2048), (1500, 4096), (801, 8192), (700, 16383),
          (600, 16384), (400, 20001)]


def placed(values, off):
    """(buffer, view): the values `off` elements past a 16-byte boundary, 16 sevens and more on either side."""
    whole = torch.full((16 + off + values.numel() + 16,), 7.0, dtype=values.dtype, device="cuda")
    view = whole[16 + off:16 + off + values.numel()].view(values.shape)
    view.copy_(values)
    return whole, view


def untouched(whole, view, off):
    return bool(torch.all(whole[:16 + off] == 7) and torch.all(whole[16 + off + view.numel():] == 7))


@pytest.mark.parametrize("off", [0, 1, 3])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("m,n", SHAPES)
def test_forward(m, n, rms, off):
    g = gen(m + n)
    x = (torch.randn(m, n, generator=g, device="cuda") + 0.3).to(BF)
    gamma, beta = (1 + 0.3 * torch.randn(2, n, generator=g, device="cuda")).to(BF)
    whole, y = placed(x, off)
    mean, rstd = torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
    mb.morello_layer_norm(int(rms), 0, m, n, 1e-5, y, gamma, beta, y, None if rms else mean, rstd)
    check_forward(x, gamma, beta, 1e-5, rms, y, None if rms else mean, rstd)
    assert untouched(whole, y, off)


@pytest.mark.parametrize("off", [0, 1])
@pytest.mark.parametrize("kind", [BF, F32])
@pytest.mark.parametrize("m,n", SHAPES)
def test_backward(m, n, kind, off):
    g = gen(m * 3 + n)
    x, r = (torch.randn(m, n, generator=g, device="cuda").to(kind) for _ in range(2))
    dy, gamma = torch.randn(m, n, generator=g, device="cuda").to(BF), torch.randn(n, generator=g, device="cuda").to(BF)
    mean, rstd, _, _ = norm64(x, None, None, 1e-5, False)
    mean, rstd = mean[:, 0].float(), rstd[:, 0].float()
    whole, dx = placed(r, off)
    mb.morello_layer_norm_backward(0, int(kind == F32), 0, m, n, x, gamma, mean, rstd, dy, dx, dx, None, None)
    check_backward(x, gamma, mean, rstd, dy, r, False, dx, None, None)
    assert untouched(whole, dx, off)
