"""A sparse feed-forward block, forward and backward, on the library's operators.

    python examples/expert_block.py [--tokens 1024] [--d 1024] [--f 512] [--experts 16] [--topk 2]

For tokens x [T][d] (bf16), a router and E experts with gated first and plain second weights:

    logits = x Wr                               morello_linear (f32 output)
    idx, w = route(logits)                      morello_route, morello_expert_plan
    h      = silu(x W1g) * (x W1u), by expert   morello_expert_linear, rows gathered from the tokens
    y      = h W2, by expert                    morello_expert_linear
    out    = x + sum of a token's w * y         morello_expert_combine

and the gradients of everything from d(out).  The forward result is compared with a plain computation in 64 bits, the
gradients with central differences of the loss along random directions, also in 64 bits with the same experts chosen."""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2505_01637_b200 import binding as mb  # noqa: E402


class ExpertBlock:
    """Weights, buffers and the two passes for a fixed number of tokens."""

    def __init__(self, tokens, d, f, experts, topk, seed=0):
        self.t, self.d, self.f, self.e, self.k = tokens, d, f, experts, topk
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def weight(*shape):
            return (torch.randn(*shape, generator=g, device="cuda") / math.sqrt(shape[-2])).to(torch.bfloat16)

        self.wr, self.w1, self.w2 = weight(d, experts), weight(experts, d, 2 * f), weight(experts, f, d)
        bf, f32, i32 = torch.bfloat16, torch.float32, torch.int32
        rows = mb.morello_expert_plan_rows(tokens, topk, experts)

        def empty(*shape, dtype=bf):
            return torch.empty(*shape, dtype=dtype, device="cuda")

        self.logits, self.weights = empty(tokens, experts, dtype=f32), empty(tokens, topk, dtype=f32)
        self.idx = empty(tokens, topk, dtype=i32)
        self.plan = empty(mb.morello_expert_plan_words(tokens, topk, experts), dtype=i32)
        self.z, self.h, self.y, self.out = empty(rows, 2 * f), empty(rows, f), empty(rows, d, dtype=f32), empty(tokens, d)
        # gradients
        self.dy, self.dh, self.dx, self.dxr = empty(rows, d), empty(rows, f), empty(tokens, d), empty(tokens, d)
        self.dweights, self.dlogits = empty(tokens, topk, dtype=f32), empty(tokens, experts, dtype=f32)
        self.dwr, self.dw1, self.dw2 = (torch.empty_like(w) for w in (self.wr, self.w1, self.w2))

    def forward(self, x):
        t, d, f, e, k = self.t, self.d, self.f, self.e, self.k
        mb.morello_linear(mb.MORELLO_ACT_NONE, 0, mb.MORELLO_F32, 0, t, d, e, x, self.wr, None, None, self.logits)
        mb.morello_route(mb.MORELLO_SCORE_SOFTMAX, 1, 1.0, mb.MORELLO_F32, t, e, k, 1, 1, self.logits, None, self.idx, self.weights)
        mb.morello_expert_plan(t, k, e, self.idx, self.plan)
        mb.morello_expert_linear(mb.MORELLO_ACT_SILU, 1, mb.MORELLO_BF16, 0, 1, t, k, e, d, f, self.plan, x, self.w1, None,
                                 self.h, self.z)
        mb.morello_expert_linear(mb.MORELLO_ACT_NONE, 0, mb.MORELLO_F32, 0, 0, t, k, e, f, d, self.plan, self.h, self.w2, None,
                                 self.y)
        mb.morello_expert_combine(mb.MORELLO_F32, t, k, e, d, self.plan, self.weights, self.y, x, self.out)
        return self.out

    def backward(self, x, dout):
        """Gradients of the weights and of x (dx: through the experts and the router; the residual's is dout itself)."""
        t, d, f, e, k = self.t, self.d, self.f, self.e, self.k
        mb.morello_expert_combine_backward(mb.MORELLO_F32, t, k, e, d, self.plan, self.weights, self.y, dout, self.dy, self.dweights)
        mb.morello_expert_linear_backward(mb.MORELLO_ACT_NONE, 0, mb.MORELLO_BF16, 0, 0, 0, t, k, e, f, d, self.plan, self.h, self.w2,
                                          None, self.dy, self.dh, self.dw2, None)
        mb.morello_expert_linear_backward(mb.MORELLO_ACT_SILU, 1, mb.MORELLO_BF16, 0, 0, 1, t, k, e, d, f, self.plan, x, self.w1,
                                          self.z, self.dh, self.dx, self.dw1, None)
        mb.morello_route_backward(mb.MORELLO_SCORE_SOFTMAX, 1, 1.0, mb.MORELLO_F32, t, e, k, self.logits, self.idx, self.dweights,
                                  self.dlogits)
        # The router's product: its output gradient as bf16, like every product's operands.
        mb.morello_linear_backward(mb.MORELLO_ACT_NONE, 0, mb.MORELLO_BF16, 0, 0, t, d, e, x, self.wr, None,
                                   self.dlogits.to(torch.bfloat16), self.dxr, self.dwr, None)
        return self.dx, self.dxr, self.dwr, self.dw1, self.dw2


def plain64(x, wr, w1, w2, idx):
    """out - x in 64 bits, with the experts of idx."""
    idx = idx.long()
    w = torch.softmax(torch.gather(x @ wr, 1, idx), 1)
    out = torch.zeros_like(x)
    for e in range(w1.shape[0]):
        token, place = (idx == e).nonzero(as_tuple=True)
        gate, up = (x[token] @ w1[e]).chunk(2, 1)
        out.index_add_(0, token, (torch.nn.functional.silu(gate) * up) @ w2[e] * w[token, place][:, None])
    return out


def check(block, x, dout, seed=1):
    """(relative error of the forward pass, largest relative error of the gradients along random directions)"""
    out = block.forward(x).double()
    grads = block.backward(x, dout)
    args = [v.double() for v in (x, block.wr, block.w1, block.w2)]
    want = args[0] + plain64(*args, block.idx)
    forward = float((out - want).norm() / (want - args[0]).norm())
    # d(loss)/d(x, wr, w1, w2) for loss = <dout, out>, the residual left out
    mine = [grads[0].double() + grads[1].double(), grads[2].double(), grads[3].double(), grads[4].double()]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    worst = 0.0
    for i in range(4):
        # along the gradient itself plus noise, so that the derivative is not near zero
        way = mine[i] / mine[i].norm() + torch.randn(args[i].shape, generator=g, device="cuda", dtype=torch.float64) / args[i].numel() ** 0.5
        step = 1e-4
        ends = []
        for sign in (1, -1):
            moved = list(args)
            moved[i] = args[i] + sign * step * way
            ends.append(float((plain64(*moved, block.idx) * dout.double()).sum()))
        diff, grad = (ends[0] - ends[1]) / (2 * step), float((mine[i] * way).sum())
        worst = max(worst, abs(diff - grad) / abs(diff))
    return forward, worst


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("tokens", 1024), ("d", 1024), ("f", 512), ("experts", 16), ("topk", 2)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args(argv)
    block = ExpertBlock(a.tokens, a.d, a.f, a.experts, a.topk)
    g = torch.Generator(device="cuda")
    g.manual_seed(7)
    x, dout = ((torch.randn(a.tokens, a.d, generator=g, device="cuda")).to(torch.bfloat16) for _ in range(2))
    forward, worst = check(block, x, dout)
    status, detail = mb.morello_read_device_status()
    assert status == mb.MORELLO_OK, (status, hex(detail))
    print("forward: relative error %.2e; gradients against differences: %.2e" % (forward, worst))
    for name, call in (("forward", lambda: block.forward(x)), ("backward", lambda: block.backward(x, dout))):
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        for _ in range(5):
            call()
        begin.record()
        for _ in range(20):
            call()
        end.record()
        torch.cuda.synchronize()
        print("%s: %.1f us" % (name, begin.elapsed_time(end) / 20 * 1e3))
    # bf16 activations, weights and gradients: every rounding is within 2^-9 of its value on average
    return 0 if forward < 1e-2 and worst < 2e-2 else 1


if __name__ == "__main__":
    sys.exit(main())
