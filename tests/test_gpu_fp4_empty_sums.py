"""Products of 4-bit tensors without a contraction, Y = act(bias) + R, in every kernel form: few rows, tiles of single blocks,
gated tiles; by the TMA engine and past it.  No accumulator is awaited there, and none may be announced."""
import pytest
import torch

from feed_forward_util import assert_close, device_ok, gen, misaligned
from fp4_util import MX, NV, linear64
from paper_2505_01637_b200 import binding as mb

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
ACTS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("m,n", [(1, 24), (16, 333), (17, 264), (200, 1000), (129, 257), (3000, 2056)])
def test_empty_sums(m, n, f32, gated):
    g = gen(m + n)
    wide = 2 * n if gated else n
    bias = torch.randn(wide, generator=g, device="cuda").to(BF)
    alpha = torch.tensor([0.5], device="cuda")
    nothing = torch.zeros(m, 0, dtype=torch.float64, device="cuda"), torch.zeros(wide, 0, dtype=torch.float64, device="cuda")
    for fmt, act, off in ((MX, "relu", False), (NV, "gelu", True), (NV, "none", False)):
        move = misaligned if off else (lambda t: t)
        r = move(torch.randn(m, n, generator=g, device="cuda").to(BF))
        y = move(torch.full((m, n), float("nan"), dtype=F32 if f32 else BF, device="cuda"))
        for _ in range(3):      # one behind the other: what a call leaves behind would meet the next one's blocks
            mb.morello_fp4_linear(fmt, ACTS[act], int(gated), int(f32), m, 0, n, None, None, None, None, alpha, bias, r, y)
        device_ok()
        want, bound = linear64(*nothing, alpha, bias, r, act, gated, 0, f32)
        assert_close(y, want, bound, "y")
