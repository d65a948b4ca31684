"""dgamma and dbeta of many rows, under the bound that the kernel's order of additions gives.

A block is 512 threads in teams of a row each, one block to an SM, and a thread adds up its columns through all its block's
rows; then the teams' sums are added in a row, and the blocks' by eight warps, each its share in a row, and the eight.  Every addition and the three
roundings of a term (difference, factor, product) are off by 2^-24 at most of the sum of the terms' magnitudes."""
import pytest
import torch

from norm_util import gen
from paper_2505_01637_b200 import binding as mb

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def teams(n):
    threads = 8 if n <= 64 else 16 if n <= 128 else 32
    while threads < 512 and n > 16 * threads:
        threads *= 2
    return 512 // threads


@pytest.mark.parametrize("kind", [BF, F32])
@pytest.mark.parametrize("equal", [False, True])
@pytest.mark.parametrize("m,n", [(100000, 4104), (60001, 8191), (40000, 16384), (300000, 1000), (3000000, 8), (2000003, 33)])
def test_many_rows(m, n, equal, kind):
    g = gen(m)
    x = torch.empty(m, n, dtype=kind, device="cuda")
    dy = torch.empty(m, n, dtype=BF, device="cuda")
    if equal:      # every addition of a chain rounds the same way
        x.fill_(1.1)
        dy.fill_(0.3)
    else:
        x.normal_(generator=g)
        dy.normal_(generator=g)
    mean, rstd = torch.full((m,), 0.1, device="cuda"), torch.full((m,), 1.3, device="cuda")
    dgamma, dbeta = torch.full((n,), float("nan"), device="cuda"), torch.full((n,), float("nan"), device="cuda")
    mb.morello_layer_norm_backward(0, int(kind == F32), 0, m, n, x, None, mean, rstd, dy, None, None, dgamma, dbeta)
    sums = torch.zeros(4, n, dtype=torch.float64, device="cuda")
    for at in range(0, m, 20000):
        d = dy[at:at + 20000].double()
        t = (x[at:at + 20000].double() - mean[0].double()) * rstd[0].double() * d
        sums += torch.stack([t.sum(0), t.abs().sum(0), d.sum(0), d.abs().sum(0)])
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    rows = -(-(-(-m // teams(n))) // sms)
    bound = (rows + teams(n) + (-(-sms // 8)) + 8 + 3) * 2.0 ** -24
    assert torch.all((dgamma.double() - sums[0]).abs() <= bound * sums[1])
    assert torch.all((dbeta.double() - sums[2]).abs() <= bound * sums[3])


@pytest.mark.parametrize("value", [1.1, 0.7])
@pytest.mark.parametrize("m,n", [(1 << 29, 1), (1 << 27, 8)])
def test_no_chain_grows_with_the_rows(m, n, value):
    # A block takes 2048 groups of rows at most; equal terms, so that every addition of a chain rounds the same way.
    x = torch.full((m, n), value, device="cuda")
    dy = torch.full((m, n), 0.3, dtype=BF, device="cuda")
    mean, rstd = torch.full((m,), 0.1, device="cuda"), torch.full((m,), 1.3, device="cuda")
    dgamma, dbeta = torch.full((n,), float("nan"), device="cuda"), torch.full((n,), float("nan"), device="cuda")
    need = mb.morello_layer_norm_backward_workspace_bytes(m, n)
    ws = torch.full((need + 64,), 0xAB, dtype=torch.uint8, device="cuda")
    mb.morello_layer_norm_backward(0, 1, 0, m, n, x, None, mean, rstd, dy, None, None, dgamma, dbeta, ws, need)
    assert torch.all(ws[need:] == 0xAB)
    d = float(dy[0, 0])
    t = (float(x[0, 0]) - float(mean[0])) * float(rstd[0]) * d
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    parts = -(-(-(-m // teams(n))) // (2048 * sms)) * sms
    bound = (2048 + -(-parts // 8) + teams(n) + 8 + 3) * 2.0 ** -24
    assert torch.all((dgamma.double() - m * t).abs() <= bound * m * abs(t)), float(dgamma[0]) / (m * t) - 1
    assert torch.all((dbeta.double() - m * d).abs() <= bound * m * d), float(dbeta[0]) / (m * d) - 1
