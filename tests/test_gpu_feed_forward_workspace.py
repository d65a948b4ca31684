"""The operators within a caller's workspace of exactly the reported size: nothing behind it is touched, one byte less is
refused, and the results are those of the library's own scratch."""
import pytest
import torch

from feed_forward_util import ACTS, device_ok, gen, plan_of, randn
from paper_2505_01637_b200 import binding as mb
from test_gpu_experts import routed

pytestmark = pytest.mark.gpu

TAIL = 4096


def check(need, call, outs):
    """call(workspace, bytes) fills outs."""
    call(None, 0)
    device_ok()
    want = [o.clone() for o in outs]
    for o in outs:
        o.fill_(float("nan"))
    buf = torch.full((need + TAIL,), 0xA5, device="cuda", dtype=torch.uint8)
    buf[:need] = 0xFF            # every bf16 and f32 of it a NaN
    call(buf, need)
    device_ok()
    assert bool((buf[need:] == 0xA5).all())
    for o, w in zip(outs, want):
        bits = torch.int32 if o.dtype == torch.float32 else torch.int16
        assert torch.equal(o.view(bits), w.view(bits))
    if need:
        with pytest.raises(mb.MorelloError) as e:
            call(buf, need - 1)
        assert e.value.status == mb.MORELLO_ERR_WORKSPACE


@pytest.mark.parametrize("m,k,n", [(1, 63, 65), (6, 100, 60), (64, 101, 67), (90, 100, 60), (333, 257, 129), (200, 64, 72)])
@pytest.mark.parametrize("gated,colmajor", [(False, False), (True, False), (False, True), (True, True)])
def test_linear(m, k, n, gated, colmajor):
    g = gen(m + k)
    wide = 2 * n if gated else n
    x, w = randn(g, m, k), randn(g, *((wide, k) if colmajor else (k, wide)), scale=0.1)
    y, z = torch.full((m, n), float("nan"), device="cuda", dtype=torch.bfloat16), torch.full((m, wide), float("nan"), device="cuda", dtype=torch.bfloat16)
    check(mb.morello_linear_workspace_bytes(gated, colmajor, m, k, n),
          lambda ws, size: mb.morello_linear(ACTS["gelu"], gated, 0, colmajor, m, k, n, x, w, None, None, y, z, ws, size), [y, z])


@pytest.mark.parametrize("m,k,n", [(1, 63, 65), (64, 101, 67), (90, 100, 60), (333, 257, 129), (200, 64, 72), (1100, 72, 40)])
@pytest.mark.parametrize("act,gated,colmajor,f32", [("none", False, False, False), ("gelu", False, True, False), ("silu", True, False, True),
                                                    ("silu", True, True, False)])
def test_linear_backward(m, k, n, act, gated, colmajor, f32):
    g = gen(m + k)
    wide = 2 * n if gated else n
    x, w, z, dy = randn(g, m, k), randn(g, *((wide, k) if colmajor else (k, wide)), scale=0.1), randn(g, m, wide), randn(g, m, n)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w, dtype=torch.float32 if f32 else torch.bfloat16), torch.empty(wide, device="cuda")
    check(mb.morello_linear_backward_workspace_bytes(ACTS[act], gated, colmajor, m, k, n),
          lambda ws, size: mb.morello_linear_backward(ACTS[act], gated, f32, 0, colmajor, m, k, n, x, w, z, dy, dx, dw, db, ws, size),
          [dx, dw, db])


EXPERTS = [(1, 2, 4, 33, 35), (64, 2, 4, 63, 65), (65, 2, 5, 63, 65), (150, 2, 3, 100, 100), (300, 3, 7, 72, 136)]


@pytest.mark.parametrize("t,topk,e,k,n", EXPERTS)
@pytest.mark.parametrize("gated,colmajor,gather", [(False, False, False), (True, False, True), (True, True, True), (False, True, False)])
def test_experts(t, topk, e, k, n, gated, colmajor, gather):
    g = gen(t + k)
    plan, parts = plan_of(routed(g, t, topk, e, "dropped"), e)
    rows, wide = parts["row_src"].numel(), 2 * n if gated else n
    w = randn(g, e, *((wide, k) if colmajor else (k, wide)), scale=0.1)
    x, z, dy = randn(g, t if gather else rows, k), randn(g, rows, wide), randn(g, rows, n)
    holds = (parts["row_src"] >= 0)[:, None]
    if not gather:
        x = x * holds
    z, dy = z * holds, dy * holds
    y, kept = torch.zeros(rows, n, device="cuda", dtype=torch.bfloat16), torch.zeros(rows, wide, device="cuda", dtype=torch.bfloat16)
    dx, dw, db = torch.zeros_like(x), torch.empty_like(w), torch.empty(e, wide, device="cuda")
    live = parts["row_src"] >= 0

    def forward(ws, size):
        mb.morello_expert_linear(ACTS["silu"], gated, 0, colmajor, gather, t, topk, e, k, n, plan, x, w, None, y, kept, ws, size)
        y[~live] = 0             # rows without a pair may be left alone
        kept[~live] = 0

    def backward(ws, size):
        mb.morello_expert_linear_backward(ACTS["silu"], gated, 0, 0, colmajor, gather, t, topk, e, k, n, plan, x, w, z, dy, dx, dw, db, ws,
                                          size)
        if not gather:
            dx[~live] = 0

    check(mb.morello_expert_linear_workspace_bytes(gated, colmajor, gather, t, topk, e, k, n), forward, [y, kept])
    check(mb.morello_expert_linear_backward_workspace_bytes(ACTS["silu"], gated, colmajor, gather, t, topk, e, k, n), backward, [dx, dw, db])
