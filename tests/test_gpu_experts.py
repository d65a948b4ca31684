"""The experts' products, their gradients and the weighted sum against the definition in 64 bits."""
import pytest
import torch

from feed_forward_util import (ACTS, BF16, TINY, assert_close, device_ok, dz64, forward64, gen, misaligned, plan_of,
                               randn)
from paper_2505_01637_b200 import binding as mb

pytestmark = pytest.mark.gpu


def routed(g, t, topk, e, how):
    if how == "one":          # every token to the same expert
        return torch.full((t, topk), e - 1, dtype=torch.int32, device="cuda")
    idx = torch.argsort(torch.rand(t, e, generator=g, device="cuda") + torch.linspace(0, 1, e, device="cuda"), 1)
    idx = idx[:, :topk].to(torch.int32).contiguous()
    if how == "dropped":
        idx[torch.rand(t, topk, generator=g, device="cuda") < 0.4] = -1
        idx[-1] = -1          # a token without any expert
    return idx


def rows_of(parts, e):
    """(expert, first row, row count, pairs) of every expert that has rows."""
    offsets, counts = parts["offsets"].tolist(), parts["counts"].tolist()
    for x in range(e):
        if counts[x]:
            first = offsets[x]
            yield x, first, counts[x], parts["row_src"][first:first + counts[x]].long()


SIZES = [(1, 1, 1, 64, 64), (1, 4, 8, 128, 72), (4, 2, 16, 256, 136), (16, 4, 4, 72, 264), (64, 2, 3, 128, 128),
         (65, 2, 5, 136, 72), (200, 3, 6, 264, 200), (700, 2, 4, 128, 264), (40, 1, 64, 64, 64)]
ODD = [(3, 2, 4, 33, 35), (90, 2, 4, 63, 65), (150, 2, 3, 100, 100)]


@pytest.mark.parametrize("t,topk,e,k,n", SIZES + ODD)
@pytest.mark.parametrize("gated,colmajor,gather", [(False, False, False), (True, False, True), (True, True, True), (False, True, True),
                                                   (True, True, False)])
@pytest.mark.parametrize("how", ["spread", "dropped", "one"])
def test_forward(t, topk, e, k, n, gated, colmajor, gather, how):
    g = gen(t + k)
    idx = routed(g, t, topk, e, how)
    plan, parts = plan_of(idx, e)
    rows, wide = parts["row_src"].numel(), 2 * n if gated else n
    live_rows = int(parts["offsets"][-1])
    w = randn(g, e, *((wide, k) if colmajor else (k, wide)), scale=k ** -0.5)
    b = randn(g, e, wide, scale=0.5)
    src = parts["row_src"]
    x = randn(g, t if gather else rows, k)
    if not gather:
        x = x * (src >= 0)[:, None]
        x[live_rows:] = float("nan")
    y = torch.full((rows, n), float("nan"), device="cuda", dtype=torch.bfloat16)
    z = torch.full((rows, wide), float("nan"), device="cuda", dtype=torch.bfloat16)
    mb.morello_expert_linear(ACTS["silu"], gated, 0, colmajor, gather, t, topk, e, k, n, plan, x, w, b, y, z)
    device_ok()
    for expert, first, count, pairs in rows_of(parts, e):
        x64 = (x[pairs // topk] if gather else x[first:first + count]).double()
        w64 = w[expert].double()
        want, bound, z64, ez = forward64(x64, w64.t() if colmajor else w64, b[expert].double(), None, "silu", gated)
        assert_close(y[first:first + count], want, bound, "Y of expert %d" % expert)
        assert_close(z[first:first + count], z64, ez, "Z of expert %d" % expert)
    padding = torch.zeros(rows, dtype=torch.bool, device="cuda")       # up to the next multiple of 16
    for expert, first, count, _ in rows_of(parts, e):
        padding[first + count:first + (count + 15) // 16 * 16] = True
    assert bool((src[padding] < 0).all()) and bool((y[padding] == 0).all()) and bool((z[padding] == 0).all())
    assert bool(y[live_rows:].isnan().all()) and bool(z[live_rows:].isnan().all())      # not touched


@pytest.mark.parametrize("t", [8, 130])
def test_forward_f32_and_misaligned(t):
    g = gen(4)
    topk, e, k, n = 2, 4, 72, 136
    plan, parts = plan_of(routed(g, t, topk, e, "spread"), e)
    x, w = misaligned(randn(g, t, k)), misaligned(randn(g, e, k, n, scale=0.1))
    y = misaligned(torch.zeros(parts["row_src"].numel(), n, device="cuda"))
    mb.morello_expert_linear(ACTS["none"], 0, 1, 0, 1, t, topk, e, k, n, plan, x, w, None, y)
    device_ok()
    for expert, first, count, pairs in rows_of(parts, e):
        want, bound, _, _ = forward64(x[pairs // topk].double(), w[expert].double(), None, None, "none", False)
        assert_close(y[first:first + count], want, bound)


@pytest.mark.parametrize("t,topk,e,k,n", [(1, 2, 4, 64, 64), (30, 2, 4, 72, 136), (200, 2, 5, 136, 72), (700, 2, 4, 64, 128),
                                          (90, 2, 4, 63, 65), (100, 3, 40, 72, 72)])
@pytest.mark.parametrize("gated,colmajor,gather", [(False, False, False), (True, False, True), (True, True, True), (False, True, False)])
@pytest.mark.parametrize("how", ["spread", "dropped", "one"])
def test_backward(t, topk, e, k, n, gated, colmajor, gather, how):
    run_backward(t, topk, e, k, n, gated, colmajor, gather, how, "silu" if gated else "gelu", False)


@pytest.mark.parametrize("act,gated", [("none", False), ("none", True)])
def test_accumulated_gradients(act, gated):
    run_backward(150, 2, 6, 72, 136, gated, False, True, "spread", act, True)


def run_backward(t, topk, e, k, n, gated, colmajor, gather, how, act, accumulate):
    g = gen(t + n)
    idx = routed(g, t, topk, e, how)
    plan, parts = plan_of(idx, e)
    rows, wide = parts["row_src"].numel(), 2 * n if gated else n
    live_rows = int(parts["offsets"][-1])
    holds = (parts["row_src"] >= 0)[:, None]
    w = randn(g, e, *((wide, k) if colmajor else (k, wide)), scale=k ** -0.5)
    x = randn(g, t if gather else rows, k)
    z, dy = randn(g, rows, wide) * holds, randn(g, rows, n) * holds
    free = torch.ones(rows, dtype=torch.bool, device="cuda")           # rows that may hold anything
    for _, first, count, _ in rows_of(parts, e):
        free[first:first + (count + 15) // 16 * 16] = False
    for v in (z, dy) if gather else (x.mul_(holds), z, dy):
        v[free] = float("nan")
    kind = torch.float32 if accumulate else torch.bfloat16
    dx = torch.full(x.shape, float("nan"), device="cuda", dtype=torch.bfloat16)
    dw = torch.full(w.shape, 0.25 if accumulate else float("nan"), device="cuda", dtype=kind)
    db = torch.full((e, wide), 0.5 if accumulate else float("nan"), device="cuda")
    mb.morello_expert_linear_backward(ACTS[act], gated, accumulate, accumulate, colmajor, gather, t, topk, e, k, n, plan, x, w, z,
                                      dy, dx, dw, db)
    device_ok()
    want_dx = torch.zeros(t if gather else rows, k, dtype=torch.float64, device="cuda")
    bound_dx = torch.zeros_like(want_dx)
    seen = set()
    rounded = 0 if act == "none" and not gated else BF16
    for expert, first, count, pairs in rows_of(parts, e):
        seen.add(expert)
        span = slice(first, first + count)
        dz, edz = dz64(z[span].double(), dy[span].double(), act, gated)
        eprod = edz + rounded * (dz.abs() + edz)
        w64 = w[expert].double()
        w64 = w64.t() if colmajor else w64
        one = dz @ w64.t()
        bound = eprod @ w64.abs().t() + 1e-5 * (dz.abs() @ w64.abs().t()) + TINY
        at = pairs // topk if gather else torch.arange(first, first + count, device="cuda")
        want_dx.index_add_(0, at, one)
        bound_dx.index_add_(0, at, bound + 1e-6 * one.abs())
        x64 = (x[pairs // topk] if gather else x[span]).double()
        want = x64.t() @ dz + (0.25 if accumulate else 0)
        bound = x64.abs().t() @ eprod + 1e-5 * (x64.abs().t() @ dz.abs()) + TINY
        assert_close(dw[expert].t() if colmajor else dw[expert], want, bound, "dW of expert %d" % expert)
        assert_close(db[expert], dz.sum(0) + (0.5 if accumulate else 0), edz.sum(0) + 1e-5 * dz.abs().sum(0) + TINY, "db")
    for expert in range(e):
        if expert not in seen:
            assert bool((dw[expert] == (0.25 if accumulate else 0)).all()) and bool((db[expert] == (0.5 if accumulate else 0)).all())
    if gather:
        assert_close(dx, want_dx, bound_dx, "dX")
    else:
        assert_close(dx[~free], want_dx[~free], bound_dx[~free], "dX")
        assert bool(dx[live_rows:].isnan().all())


@pytest.mark.parametrize("t,topk,e,n", [(1, 1, 1, 8), (5, 2, 4, 72), (100, 3, 8, 264), (33, 8, 64, 65), (4, 32, 40, 16)])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("how", ["spread", "dropped"])
def test_combine(t, topk, e, n, f32, how):
    g = gen(n)
    idx = routed(g, t, topk, e, how)
    plan, parts = plan_of(idx, e)
    rows, live_rows = parts["row_src"].numel(), int(parts["offsets"][-1])
    y = torch.randn(rows, n, generator=g, device="cuda").to(torch.float32 if f32 else torch.bfloat16)
    w = torch.rand(t, topk, generator=g, device="cuda")
    r = randn(g, t, n)
    slot = parts["slot"].view(t, topk).long()
    picked = y.double()[slot.clamp(min=0)] * (slot >= 0)[..., None]
    for weights, resid in ((w, r), (None, None)):
        out = torch.full((t, n), float("nan"), device="cuda", dtype=torch.bfloat16)
        mb.morello_expert_combine(f32, t, topk, e, n, plan, weights, y, resid, out)
        terms = picked * (1.0 if weights is None else weights.double()[..., None])
        want = terms.sum(1) + (0 if resid is None else resid.double())
        assert_close(out, want, 1e-6 * (terms.abs().sum(1) + 4) + TINY)
    dout = randn(g, t, n)
    dy = torch.full((rows, n), float("nan"), device="cuda", dtype=torch.bfloat16)
    dw = torch.full((t, topk), float("nan"), device="cuda")
    mb.morello_expert_combine_backward(f32, t, topk, e, n, plan, w, y, dout, dy, dw)
    d64 = dout.double()
    want = (picked * d64[:, None]).sum(-1)
    bound = 1e-6 * (picked.abs() * d64.abs()[:, None]).sum(-1) * 8 + TINY
    assert_close(dw, want, bound)
    want = torch.zeros(rows, n, dtype=torch.float64, device="cuda")
    live = slot >= 0
    want[slot[live]] = (d64[:, None] * w.double()[..., None])[live]
    assert_close(dy[:live_rows], want[:live_rows], TINY * want[:live_rows].abs())
    assert bool(dy[live_rows:].isnan().all())


def test_no_tokens():
    plan = torch.zeros(mb.morello_expert_plan_words(0, 2, 3), dtype=torch.int32, device="cuda")
    mb.morello_expert_plan(0, 2, 3, None, plan)
    dw = torch.full((3, 8, 8), 5.0, device="cuda", dtype=torch.bfloat16)
    db = torch.full((3, 8), 5.0, device="cuda")
    mb.morello_expert_linear(0, 0, 0, 0, 1, 0, 2, 3, 8, 8, plan, None, None, None, None)
    mb.morello_expert_combine(0, 0, 2, 3, 8, plan, None, None, None, None)
    mb.morello_expert_linear_backward(0, 0, 0, 0, 0, 1, 0, 2, 3, 8, 8, plan, None, None, None, None, None, dw, db)
    torch.cuda.synchronize()
    assert bool((dw == 0).all()) and bool((db == 0).all())
