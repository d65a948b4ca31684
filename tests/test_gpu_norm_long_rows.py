"""Norms of rows of millions of columns: the statistics and the gradients' sums keep what a chain of f32 additions would lose.

The bounds are those of the shorter rows: a thread's sums begin anew every 32 columns and are joined in 64 bits, so an
f32 mean of values v is within 2^-17 of mean |v| at any length."""
import pytest
import torch

from norm_util import check_backward, check_forward, forward, gen, norm64
from paper_2505_01637_b200 import binding as mb

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def backward(x, gamma, dy, rms, dx_only=True):
    m, n = x.shape
    mean, rstd, _, _ = norm64(x, None, None, 1e-5, rms)
    mean, rstd = (None if rms else mean[:, 0].float()), rstd[:, 0].float()
    dx = torch.full_like(x, float("nan"))
    dg, db = (None, None) if dx_only else (torch.full((n,), float("nan"), device="cuda") for _ in range(2))
    mb.morello_layer_norm_backward(int(rms), int(x.dtype == F32), 0, m, n, x, gamma, mean, rstd, dy, None, dx, dg, db)
    check_backward(x, gamma, mean, rstd, dy, None, rms, dx, dg, db)


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("n", [1 << 24, (1 << 22) + 3])
def test_rows_of_equal_terms(n, rms):
    # Every addition of a chain of these rounds the same way.
    x = torch.full((2, n), 1.1, device="cuda")
    x[1, ::2] = -1.1
    y, mean, rstd = forward(x, None, None, 1e-5, rms)
    if rms:
        check_forward(x, None, None, 1e-5, rms, y, mean, rstd)
    else:      # the first row's variance is what rounding leaves
        check_forward(x[1:], None, None, 1e-5, rms, y[1:], mean[1:], rstd[1:])
    gamma, dy = (torch.full(s, 1.1, device="cuda").to(BF) for s in ((n,), (2, n)))
    backward(torch.randn(2, n, generator=gen(n), device="cuda"), gamma, dy, rms)
    if rms:
        backward(x, gamma, dy, rms)


@pytest.mark.parametrize("kind", [BF, F32])
@pytest.mark.parametrize("m,n", [(3, (1 << 20) + 1), (1, (1 << 23) + 8), (5, 32768), (5, 32769), (200, 65601)])
def test_random_rows(m, n, kind):
    g = gen(n)
    x = (torch.randn(m, n, generator=g, device="cuda") * 1.7 + 0.3).to(kind)
    gamma, beta = (0.3 * torch.randn(2, n, generator=g, device="cuda") + 1).to(BF)
    dy = (torch.randn(m, n, generator=g, device="cuda") + 0.5).to(BF)
    for rms in (False, True):
        y, mean, rstd = forward(x, gamma, beta, 1e-5, rms)
        check_forward(x, gamma, beta, 1e-5, rms, y, mean, rstd)
        backward(x, gamma, dy, rms, dx_only=False)
