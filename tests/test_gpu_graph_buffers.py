"""Graphs captured on the library's own buffers stay valid when later calls make the buffers grow.  A process of its own: the
buffers have to begin small."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SCRIPT = """
import torch
from paper_2505_01637_b200 import binding as mb

def bf16(*shape, scale=1.0):
    return (torch.randn(*shape, device="cuda") * scale).to(torch.bfloat16)

torch.manual_seed(0)
mb.morello_device_limits()
m, k, n = 150, 1001, 67                       # rows off 16-byte boundaries: padded copies in the scratch
x, w, y = bf16(m, k), bf16(k, n, scale=k ** -0.5), torch.zeros(m, n, device="cuda", dtype=torch.bfloat16)
A, B, C = (torch.randint(-4, 5, s, device="cuda").float() for s in ((64, 96), (96, 40), (64, 40)))

def layer():
    mb.morello_linear(0, 0, 0, 0, m, k, n, x, w, None, None, y)

def product():                                # its terms are in a buffer of their own
    mb.morello_matmul_f32(1, 64, 96, 40, A, B, C)

def check():
    want = x.double() @ w.double()
    bound = 1e-5 * (x.double().abs() @ w.double().abs()) + 1e-6 + 2.0 ** -8 * want.abs()
    assert bool(((y.double() - want).abs() <= bound).all())
    assert torch.equal(C, A @ B)              # integers

graphs = []
for call in (layer, product):
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    graphs.append(g)
check()
mb.morello_linear(0, 0, 0, 0, 20000, 1001, 67, bf16(20000, 1001), w, None, None, torch.empty(20000, n, device="cuda", dtype=torch.bfloat16))
mb.morello_matmul_f32(1, 2048, 2048, 2048, *(torch.ones(2048, 2048, device="cuda") for _ in range(3)))
torch.cuda.synchronize()
# Memory that was given back would be handed out again here.
fill = [torch.full((size,), float("nan"), device="cuda") for size in [1 << 18] * 64 + [1 << 21] * 16]
for _ in range(2):
    x.copy_(bf16(m, k))
    A.copy_(torch.randint(-4, 5, (64, 96), device="cuda").float())
    y.zero_(), C.zero_()
    for g in graphs:
        g.replay()
    torch.cuda.synchronize()
    check()
assert all(bool(f.isnan().all()) for f in fill)
assert mb.morello_read_device_status()[0] == mb.MORELLO_OK
print("graphs ok")
"""


def test_graphs_survive_growth():
    r = subprocess.run([sys.executable, "-c", SCRIPT], cwd=ROOT, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and "graphs ok" in r.stdout, r.stdout + r.stderr
