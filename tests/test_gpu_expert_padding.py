"""Rows of the experts' layout that hold no pair: up to the next multiple of 16 they are finite, further on anything, and
neither reaches a gradient, whatever way the operands take to the products."""
import pytest
import torch

from feed_forward_util import ACTS, BF16, TINY, assert_close, device_ok, dz64, gen, misaligned, plan_of, randn
from paper_2505_01637_b200 import binding as mb
from test_gpu_experts import routed, rows_of

pytestmark = pytest.mark.gpu


def run(t, topk, e, k, n, act="none", gated=False, colmajor=False, gather=False, shift=(), f32=False, how="spread"):
    g = gen(t + 3 * k + n)
    plan, parts = plan_of(routed(g, t, topk, e, how), e)
    rows, wide = parts["row_src"].numel(), 2 * n if gated else n
    live_rows = int(parts["offsets"][-1])
    w = randn(g, e, *((wide, k) if colmajor else (k, wide)), scale=k ** -0.5)
    x, z, dy = randn(g, t if gather else rows, k), randn(g, rows, wide), randn(g, rows, n)
    any_row = torch.ones(rows, dtype=torch.bool, device="cuda")
    for _, first, count, _ in rows_of(parts, e):
        any_row[first:first + (count + 15) // 16 * 16] = False
    finite = (parts["row_src"] < 0) & ~any_row
    for v in (z, dy) if gather else (x, z, dy):
        v[finite] = 100.0
        v[any_row] = float("nan")
    kind = torch.float32 if f32 else torch.bfloat16
    dx = torch.full(x.shape, float("nan"), device="cuda", dtype=torch.bfloat16)
    dw = torch.full(w.shape, float("nan"), device="cuda", dtype=kind)
    db = torch.full((e, wide), float("nan"), device="cuda")
    if "x" in shift:
        x = misaligned(x)
    if "dy" in shift:
        dy = misaligned(dy)
    mb.morello_expert_linear_backward(ACTS[act], gated, f32, 0, colmajor, gather, t, topk, e, k, n, plan, x, w, z, dy, dx, dw, db)
    device_ok()
    want_dx = torch.zeros(t if gather else rows, k, dtype=torch.float64, device="cuda")
    bound_dx = torch.zeros_like(want_dx)
    rounded = 0 if act == "none" and not gated else BF16
    held = torch.zeros(e, dtype=torch.bool, device="cuda")
    for expert, first, count, pairs in rows_of(parts, e):
        held[expert] = True
        span = slice(first, first + count)
        dz, edz = dz64(z[span].double(), dy[span].double(), act, gated)
        eprod = edz + rounded * (dz.abs() + edz)
        w64 = w[expert].double()
        w64 = w64.t() if colmajor else w64
        at = pairs // topk if gather else torch.arange(first, first + count, device="cuda")
        one = dz @ w64.t()
        want_dx.index_add_(0, at, one)
        bound_dx.index_add_(0, at, eprod @ w64.abs().t() + 1e-5 * (dz.abs() @ w64.abs().t()) + TINY + 1e-6 * one.abs())
        x64 = (x[pairs // topk] if gather else x[span]).double()
        assert_close(dw[expert].t() if colmajor else dw[expert], x64.t() @ dz,
                     x64.abs().t() @ eprod + 1e-5 * (x64.abs().t() @ dz.abs()) + TINY, "dW of expert %d, %d rows" % (expert, count))
        assert_close(db[expert], dz.sum(0), edz.sum(0) + 1e-5 * dz.abs().sum(0) + TINY, "db")
    assert bool((dw[~held] == 0).all()) and bool((db[~held] == 0).all())
    if gather:
        assert_close(dx, want_dx, bound_dx, "dX")
    else:
        pairs_rows = parts["row_src"] >= 0
        assert_close(dx[pairs_rows], want_dx[pairs_rows], bound_dx[pairs_rows], "dX")
        assert bool((dx[finite] == 0).all()) and bool(dx[live_rows:].isnan().all())


# One row, fewer than 16, counts of every remainder, several blocks an expert; outputs of one tile and of many.
SIZES = [(1, 1, 1, 64, 64), (9, 2, 4, 72, 136), (64, 2, 5, 136, 72), (130, 2, 3, 264, 520), (700, 2, 40, 72, 136), (900, 2, 4, 520, 264),
         (300, 3, 300, 64, 72)]


@pytest.mark.parametrize("t,topk,e,k,n", SIZES)
@pytest.mark.parametrize("colmajor", [False, True])
@pytest.mark.parametrize("shift", [(), ("dy",), ("x",), ("x", "dy")])
def test_plain_product(t, topk, e, k, n, colmajor, shift):
    run(t, topk, e, k, n, colmajor=colmajor, shift=shift)


@pytest.mark.parametrize("t,topk,e,k,n", SIZES)
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("how", ["one", "dropped"])
def test_uneven_experts(t, topk, e, k, n, f32, how):
    run(t, topk, e, k, n, f32=f32, how=how)


@pytest.mark.parametrize("t,topk,e,k,n", [(64, 2, 5, 136, 72), (700, 2, 40, 72, 136), (130, 2, 3, 100, 68)])
@pytest.mark.parametrize("act,gated,gather", [("none", False, True), ("gelu", False, False), ("silu", True, False), ("silu", True, True)])
def test_other_ways(t, topk, e, k, n, act, gated, gather):
    run(t, topk, e, k, n, act=act, gated=gated, gather=gather)


def test_all_remainders():
    """Experts of 1, 2, ... 70 rows."""
    counts = list(range(1, 71))
    t, k, n = sum(counts), 136, 264
    idx = torch.cat([torch.full((c,), i, dtype=torch.int32) for i, c in enumerate(counts)])
    idx = idx[torch.randperm(t, generator=torch.Generator().manual_seed(3))].view(t, 1).cuda()
    e = len(counts)
    plan, parts = plan_of(idx, e)
    g = gen(9)
    rows = parts["row_src"].numel()
    x, w, dy = randn(g, rows, k), randn(g, e, k, n, scale=0.1), randn(g, rows, n)
    for v in (x, dy):
        v[parts["row_src"] < 0] = 50.0
    dw = torch.empty(e, k, n, device="cuda", dtype=torch.bfloat16)
    mb.morello_expert_linear_backward(0, 0, 0, 0, 0, 0, t, 1, e, k, n, plan, x, w, None, dy, None, dw, None)
    device_ok()
    for expert, first, count, _ in rows_of(parts, e):
        x64, d64 = x[first:first + count].double(), dy[first:first + count].double()
        assert_close(dw[expert], x64.t() @ d64, 1e-5 * (x64.abs().t() @ d64.abs()) + TINY, "dW of %d rows" % count)
