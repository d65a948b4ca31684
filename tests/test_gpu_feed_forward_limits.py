"""The feed-forward operators at their limits: long contractions in f32, outputs past 2^31 elements, large plans,
independent streams, captured graphs."""
import pytest
import torch

from feed_forward_util import ACTS, assert_close, device_ok, forward64, gen, plan_of, randn
from paper_2505_01637_b200 import binding as mb

pytestmark = pytest.mark.gpu


# A part of 512 elements is 32 truncating additions of at most 2^-23 of the largest partial sum each, all one way:
# 32 * 2^-23 = 3.8e-6 at the worst, whatever the length; without parts 8192 elements would be 9e-6.  The parts and
# the exact 64-bit sums leave a few 2^-24.
@pytest.mark.parametrize("m,k,n,gated,colmajor", [(1, 8192, 200, False, False), (20, 8192, 72, True, True), (64, 4096, 256, False, True),
                                                  (200, 8192, 264, False, False), (150, 4096, 100, True, False), (130, 2048, 33, False, False)])
def test_long_contractions_in_f32(m, k, n, gated, colmajor):
    g = gen(k + m)
    wide = 2 * n if gated else n
    x, w = randn(g, m, k), randn(g, *((wide, k) if colmajor else (k, wide)), scale=k ** -0.5)
    y = torch.empty(m, n, device="cuda")
    mb.morello_linear(0, gated, 1, colmajor, m, k, n, x, w, None, None, y)
    device_ok()
    want = forward64(x.double(), (w.t() if colmajor else w).double(), None, None, "none", gated)[0]
    limit = 3.9e-6 * (2 ** 0.5 if gated else 1)
    assert float((y - want).norm() / want.norm()) <= limit


def test_long_weight_gradients_in_f32():
    m, k, n = 8192, 72, 136
    g = gen(1)
    x, dy = randn(g, m, k), randn(g, m, n)
    dw, db = torch.empty(k, n, device="cuda"), torch.empty(n, device="cuda")
    mb.morello_linear_backward(0, 0, 1, 0, 0, m, k, n, x, x, None, dy, None, dw, db)
    want = x.double().t() @ dy.double()
    assert float((dw - want).norm() / want.norm()) <= 3.9e-6
    # column sums: f32 additions to nearest of at most 8192 terms in a tree of depth below 64
    want = dy.double().sum(0)
    assert bool(((db - want).abs() <= 64 * 2 ** -24 * dy.double().abs().sum(0)).all())


@pytest.mark.parametrize("n", [33000, 33003])
def test_output_past_2_31_elements(n):
    """The last rows and columns of an output of more than 2^31 elements, through both ways out of the kernel."""
    m, k = 65600, 64
    assert m * n > 2 ** 31
    g = gen(2)
    x, w, b = randn(g, m, k), randn(g, k, n, scale=0.125), randn(g, n)
    y = torch.empty(m, n, device="cuda", dtype=torch.bfloat16)
    mb.morello_linear(ACTS["relu"], 0, 0, 0, m, k, n, x, w, b, None, y)
    device_ok()
    for rows in (slice(0, 40), slice(m - 150, m)):
        want, bound, _, _ = forward64(x[rows].double(), w.double(), b.double(), None, "relu", False)
        assert_close(y[rows], want, bound)
    del y
    torch.cuda.empty_cache()


def test_plan_of_many_chunks():
    """More chunks than one block adds up by itself."""
    t, topk, e = 70000, 4, 100
    idx = torch.randint(0, e, (t, topk), generator=gen(3), device="cuda", dtype=torch.int32)
    _, got = plan_of(idx, e)
    flat = idx.reshape(-1).long()
    order = torch.sort(flat, stable=True).indices
    counts = torch.bincount(flat, minlength=e)
    ends = torch.cumsum((counts + 127) // 128 * 128, 0)
    starts = ends - (counts + 127) // 128 * 128
    at = starts[flat[order]] + torch.arange(t * topk, device="cuda") - (torch.cumsum(counts, 0) - counts)[flat[order]]
    slot = torch.empty_like(at)
    slot[order] = at
    src = torch.full((got["row_src"].numel(),), -1, dtype=torch.long, device="cuda")
    src[at] = order
    assert torch.equal(got["slot"].long(), slot) and torch.equal(got["row_src"].long(), src)
    assert torch.equal(got["counts"].long(), counts) and torch.equal(got["offsets"][1:].long(), ends)
    block = torch.searchsorted(ends, torch.arange(got["block_expert"].numel(), device="cuda") * 128, right=True)
    block[block == e] = -1
    assert torch.equal(got["block_expert"].long(), block)


def test_many_experts_fall_back_to_single_blocks():
    """More experts than a CTA pair can look up."""
    t, topk, e, k, n = 3000, 2, 300, 64, 72
    idx = torch.randint(0, e, (t, topk), generator=gen(4), device="cuda", dtype=torch.int32)
    idx[:1500, 0] = 7
    plan, parts = plan_of(idx, e)
    g = gen(5)
    x, w = randn(g, t, k), randn(g, e, k, n, scale=0.125)
    y = torch.empty(parts["row_src"].numel(), n, device="cuda", dtype=torch.bfloat16)
    mb.morello_expert_linear(0, 0, 0, 0, 1, t, topk, e, k, n, plan, x, w, None, y)
    device_ok()
    for expert in (0, 7, 150, 299):
        first, count = int(parts["offsets"][expert]), int(parts["counts"][expert])
        if count == 0:
            continue
        token = parts["row_src"][first:first + count].long() // topk
        want, bound, _, _ = forward64(x[token].double(), w[expert].double(), None, None, "none", False)
        assert_close(y[first:first + count], want, bound)


def test_two_streams_with_their_own_workspaces():
    """Two chains of odd-sized layers, which need copies, at the same time."""
    m, k, n = 150, 101, 67
    need = mb.morello_linear_workspace_bytes(0, 0, m, k, n)
    g = gen(6)
    chains = []
    for _ in range(2):
        x, w = randn(g, m, k), randn(g, k, n, scale=0.1)
        chains.append((torch.cuda.Stream(), x, w, torch.empty(m, n, device="cuda", dtype=torch.bfloat16),
                       torch.empty(need, device="cuda", dtype=torch.uint8)))
    torch.cuda.synchronize()
    for _ in range(30):
        for s, x, w, y, ws in chains:
            mb.morello_linear(ACTS["silu"], 0, 0, 0, m, k, n, x, w, None, None, y, None, ws, need, s)
    torch.cuda.synchronize()
    for _, x, w, y, _ in chains:
        want, bound, _, _ = forward64(x.double(), w.double(), None, None, "silu", False)
        assert_close(y, want, bound)


@pytest.mark.parametrize("t", [6, 100])
def test_routed_block_in_a_graph(t):
    """Routing, plan, both products and the sum replayed on new logits: nothing of the first run is kept."""
    topk, e, d = 2, 8, 64
    g = gen(7)
    logits, x = torch.randn(t, e, generator=g, device="cuda"), randn(g, t, d)
    w1, w2 = randn(g, e, d, d, scale=0.125), randn(g, e, d, d, scale=0.125)
    idx, weights = torch.empty(t, topk, dtype=torch.int32, device="cuda"), torch.empty(t, topk, device="cuda")
    plan = torch.empty(mb.morello_expert_plan_words(t, topk, e), dtype=torch.int32, device="cuda")
    rows = mb.morello_expert_plan_rows(t, topk, e)
    h = torch.empty(rows, d, device="cuda", dtype=torch.bfloat16)
    y, out = torch.empty(rows, d, device="cuda"), torch.empty(t, d, device="cuda", dtype=torch.bfloat16)

    def block():
        mb.morello_route(0, 1, 1.0, 1, t, e, topk, 1, 1, logits, None, idx, weights)
        mb.morello_expert_plan(t, topk, e, idx, plan)
        mb.morello_expert_linear(ACTS["silu"], 0, 0, 0, 1, t, topk, e, d, d, plan, x, w1, None, h)
        mb.morello_expert_linear(0, 0, 1, 0, 0, t, topk, e, d, d, plan, h, w2, None, y)
        mb.morello_expert_combine(1, t, topk, e, d, plan, weights, y, x, out)

    block()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block()
    logits.copy_(torch.randn(t, e, generator=g, device="cuda"))
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    device_ok()
    top, want_idx = torch.topk(logits, topk, dim=1)
    assert torch.equal(idx.long(), want_idx)
    hidden = torch.einsum("td,tkde->tke", x.double(), w1.double()[want_idx])
    hidden = hidden * torch.sigmoid(hidden)
    want = torch.einsum("tke,tkef->tkf", hidden, w2.double()[want_idx])
    want = x.double() + (want * torch.softmax(top.double(), 1)[..., None]).sum(1)
    # h and out are rounded to bf16: 2^-8 of each term of the sums of 64
    bound = 2 ** -8 * torch.einsum("tke,tkef->tkf", hidden.abs(), w2.double().abs()[want_idx]).sum(1) + 1e-4
    assert_close(out, want, bound)
