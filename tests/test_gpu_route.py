"""Routing to experts, its gradient and the row plan against plain definitions."""
import math

import pytest
import torch

from feed_forward_util import BF16, gen, plan_of
from paper_2505_01637_b200 import binding as mb

pytestmark = pytest.mark.gpu
SCORES = {"softmax": 0, "sigmoid": 1}


def best(key, count):
    """Indices of the `count` largest entries of a list, ties to the lowest index, NaN below everything."""
    order = sorted(range(len(key)), key=lambda e: (-(key[e] if key[e] == key[e] else -math.inf),
                                                   0 if key[e] == key[e] else 1, e))
    return order[:count]


def choose_keys(key, score, groups, topk_groups, topk):
    """The definition on f32 keys, token by token, on the CPU."""
    key = key.cpu()
    out = []
    for row in key:
        allowed = list(range(len(row)))
        if groups > 1:
            per = len(row) // groups
            rank = []
            for g in range(groups):
                top = torch.sort(row[g * per:(g + 1) * per], descending=True).values
                rank.append(float(top[0] + top[1]) if score == "sigmoid" and per > 1 else float(top[0]))
            keep = set(best(rank, topk_groups))
            allowed = [e for e in allowed if e // per in keep]
        values = row.tolist()
        out.append([allowed[i] for i in best([values[e] for e in allowed], topk)])
    return torch.tensor(out, dtype=torch.int64)


def weights64(x, idx, score, renorm, scale):
    x = x.double()
    p = torch.sigmoid(x) if score == "sigmoid" else torch.softmax(x, 1)
    w = torch.gather(p, 1, idx)
    if renorm:
        w = w / w.sum(1, keepdim=True)
    return w * scale


def call(x, bias, score, renorm, scale, topk, groups=1, topk_groups=1):
    t, e = x.shape
    idx = torch.full((t, topk), -5, dtype=torch.int32, device="cuda")
    w = torch.full((t, topk), float("nan"), device="cuda")
    mb.morello_route(SCORES[score], renorm, scale, x.dtype == torch.float32, t, e, topk, groups, topk_groups, x, bias, idx, w)
    return idx, w


# Values on a grid of 1/8: ties are frequent, and sigmoid keys of different logits stay apart.
@pytest.mark.parametrize("t,e,topk,groups,topk_groups", [
    (1, 1, 1, 1, 1), (3, 8, 2, 1, 1), (7, 33, 5, 1, 1), (64, 64, 8, 8, 3), (50, 128, 4, 4, 2), (9, 256, 8, 8, 4),
    (40, 257, 32, 1, 1), (5, 1024, 32, 32, 5), (17, 60, 6, 6, 1), (12, 16, 16, 1, 1), (4, 24, 3, 24, 3)])
@pytest.mark.parametrize("score,renorm", [("softmax", False), ("softmax", True), ("sigmoid", False), ("sigmoid", True)])
@pytest.mark.parametrize("bf16", [False, True])
def test_choice_and_weights(t, e, topk, groups, topk_groups, score, renorm, bf16):
    g = gen(t + e)
    x = torch.round(torch.randn(t, e, generator=g, device="cuda") * 8) / 8
    x = x.to(torch.bfloat16 if bf16 else torch.float32)
    for bias in (None, torch.round(torch.randn(e, generator=g, device="cuda") * 4) / 16):
        idx, w = call(x, bias, score, renorm, 2.5, topk, groups, topk_groups)
        # sigmoid keys on the device's own 32-bit scores: the choice is defined on them
        s = 1 / (1 + torch.exp(-x.float())) if score == "sigmoid" else x.float()
        want = choose_keys(s if bias is None else s + bias, score, groups, topk_groups, topk)
        assert torch.equal(idx.cpu().long(), want)
        exact = weights64(x, want.cuda(), score, renorm, 2.5)
        assert bool(((w.double() - exact).abs() <= 2e-6 * exact).all())


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
def test_masked_rows(score, renorm):
    """-inf logits weigh nothing; a row of nothing else has weights of zero and the lowest indices; NaN keys lose."""
    x = torch.full((4, 40), -math.inf, device="cuda")
    x[1, 30] = 1.0
    x[2] = torch.finfo(torch.float32).min
    x[3] = 0.5
    x[3, 0] = float("nan")
    idx, w = call(x, None, score, renorm, 1.0, 3)
    idx, w = idx.cpu(), w.cpu()
    assert idx[0].tolist() == [0, 1, 2] and w[0].tolist() == [0, 0, 0]
    assert idx[1].tolist() == [30, 0, 1] and w[1, 1:].tolist() == [0, 0] and float(w[1, 0]) > 0.7
    if renorm:
        assert float(w[1, 0]) == 1.0
    assert idx[2].tolist() == [0, 1, 2] and not bool(w[2].isnan().any())
    assert idx[3].tolist() == [1, 2, 3]


@pytest.mark.parametrize("t,e,topk", [(1, 1, 1), (5, 8, 2), (33, 64, 8), (20, 257, 5), (3, 1024, 32)])
@pytest.mark.parametrize("score,renorm", [("softmax", False), ("softmax", True), ("sigmoid", False), ("sigmoid", True)])
@pytest.mark.parametrize("bf16", [False, True])
def test_gradient(t, e, topk, score, renorm, bf16):
    g = gen(t * e)
    x = torch.randn(t, e, generator=g, device="cuda").to(torch.bfloat16 if bf16 else torch.float32)
    idx, _ = call(x, None, score, renorm, 1.5, topk)
    dw = torch.randn(t, topk, generator=g, device="cuda")
    dx = torch.full((t, e), float("nan"), device="cuda", dtype=x.dtype)
    mb.morello_route_backward(SCORES[score], renorm, 1.5, not bf16, t, e, topk, x, idx, dw, dx)
    leaf = x.double().requires_grad_(True)
    want = torch.autograd.grad(weights64(leaf, idx.long(), score, renorm, 1.5), leaf, dw.double())[0]
    scale = 1.5 * dw.double().abs().amax(1, keepdim=True)
    bound = 4e-6 * scale + (BF16 * want.abs() if bf16 else 0)
    assert bool(((dx.double() - want).abs() <= bound).all())


@pytest.mark.parametrize("score,renorm", [("softmax", False), ("softmax", True), ("sigmoid", True), ("sigmoid", False)])
def test_gradient_against_differences(score, renorm):
    t, e, topk = 4, 16, 3
    g = gen(2)
    x = torch.randn(t, e, generator=g, device="cuda")
    idx, _ = call(x, None, score, renorm, 1.0, topk)
    dw = torch.randn(t, topk, generator=g, device="cuda")
    dx = torch.empty_like(x)
    mb.morello_route_backward(SCORES[score], renorm, 1.0, 1, t, e, topk, x, idx, dw, dx)
    step = 2.0 ** -7
    for place in [(0, int(idx[0, 0])), (1, int(idx[1, 2])), (2, 5)]:
        value = []
        for sign in (1, -1):
            moved = x.clone()
            moved[place] += sign * step
            again, w = call(moved, None, score, renorm, 1.0, topk)
            assert torch.equal(again.sort(1).values, idx.sort(1).values)
            order = torch.argsort(again, 1).gather(1, torch.argsort(torch.argsort(idx, 1), 1))
            value.append(float((w.gather(1, order).double() * dw.double()).sum()))
        # difference error: step^2 / 6 of a third derivative below 1, and 2e-7 * weights / step
        assert abs((value[0] - value[1]) / (2 * step) - float(dx[place])) <= 3e-4


@pytest.mark.parametrize("t,topk,e", [(1, 1, 1), (3, 2, 4), (1, 8, 64), (100, 4, 8), (700, 3, 33), (2500, 2, 16), (5000, 8, 256),
                                      (64, 32, 1024)])
@pytest.mark.parametrize("drop", [False, True])
def test_plan(t, topk, e, drop):
    g = gen(t)
    idx = torch.randint(0, e, (t, topk), generator=g, device="cuda", dtype=torch.int32)
    idx = torch.minimum(idx, torch.randint(0, e, (t, topk), generator=g, device="cuda", dtype=torch.int32))
    if drop:
        idx[torch.rand(t, topk, generator=g, device="cuda") < 0.3] = -1
        idx[0, 0] = e + 7
    _, got = plan_of(idx, e)
    got = {k: v.cpu() for k, v in got.items()}
    flat = idx.cpu().reshape(-1).tolist()
    rows = got["row_src"].numel()
    src, block, slot, offsets, counts = [-1] * rows, [-1] * (rows // 128), [-1] * len(flat), [], []
    at = 0
    for expert in range(e):
        pairs = [i for i, v in enumerate(flat) if v == expert]
        offsets.append(at)
        counts.append(len(pairs))
        for j, i in enumerate(pairs):
            src[at + j] = i
            slot[i] = at + j
        for b in range((len(pairs) + 127) // 128):
            block[at // 128 + b] = expert
        at += (len(pairs) + 127) // 128 * 128
    offsets.append(at)
    assert at <= rows
    assert got["row_src"].tolist() == src and got["block_expert"].tolist() == block
    assert got["offsets"].tolist() == offsets and got["counts"].tolist() == counts and got["slot"].tolist() == slot


def test_plan_of_nothing():
    plan = torch.full((mb.morello_expert_plan_words(0, 2, 5),), 9, dtype=torch.int32, device="cuda")
    mb.morello_expert_plan(0, 2, 5, None, plan)
    assert plan.cpu().tolist() == [0] * 6 + [0] * 5
