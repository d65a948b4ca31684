"""A feed-forward block with its norm: trained in bf16, served in 4 bits, on the library's operators.

    python examples/norm_block.py [--tokens 1024] [--d 1024] [--f 2048]

For rows x [T][d] (bf16):

    n   = layer norm of x                       morello_layer_norm
    h   = silu(n W1g) * (n W1u)                 morello_linear, gated; Z kept
    out = x + h W2                              morello_linear with residual

and the gradients of x, gamma, beta, W1 and W2 from d(out): morello_linear_backward twice, then
morello_layer_norm_backward, which adds the residual's gradient.  For serving the same weights are quantised once, and n and h
as they come:

    n, h -> 4 bits                              morello_fp4_quantize
    both products                               morello_fp4_linear

Blocks of 16 have scales in e4m3, which loses bits below 2^-6: the weights of a wide layer, 1 / sqrt(f), would be there.  So
each tensor gets a factor that puts its largest scale near the top of e4m3's range, the weights' from the weights, the
activations' from sample rows; the inverse of both goes into the product's alpha.  (Blocks of 32 have powers of two and
need none.)

The forward result is compared with a plain computation in 64 bits, the gradients with central differences of the loss
along random directions, also in 64 bits, and the 4-bit result with the bf16 one."""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2505_01637_b200 import binding as mb  # noqa: E402

BF, F32, U8 = torch.bfloat16, torch.float32, torch.uint8
EPS = 1e-5


def kept(there, value):
    """value, in the memory that an earlier one had: captured passes read it there."""
    return value if there is None else there.copy_(value)


class Fp4:
    """A 4-bit tensor of the library: its two buffers, and what is needed to fill them."""

    def __init__(self, rows, k, fmt=mb.MORELLO_NVFP4, parts=1):
        self.rows, self.k, self.fmt, self.parts = rows, k, fmt, parts
        self.q = torch.empty(mb.morello_fp4_bytes(rows, k), dtype=U8, device="cuda")
        self.scales = torch.empty(mb.morello_fp4_scale_bytes(fmt, rows, parts, k), dtype=U8, device="cuda")
        self.mult = None        # the tensor's factor, one f32 on the device

    def fit(self, x, room=1.0):
        """A factor for tensors whose largest magnitude is up to `room` times that of x."""
        if self.fmt == mb.MORELLO_NVFP4:
            self.mult = kept(self.mult, (448 * 6 / (room * x.float().abs().amax().clamp(min=1e-30))).reshape(1))
        return self

    def quantize(self, x, layout=mb.MORELLO_W_COLMAJOR):
        mb.morello_fp4_quantize(self.fmt, int(x.dtype == F32), layout, self.rows, self.parts, self.k, x, self.mult, self.q,
                                self.scales)
        return self


def alpha_of(there, x, w):
    """What takes two tensors' factors out of their product again."""
    return None if x.mult is None or w.mult is None else kept(there, 1 / (x.mult * w.mult))


class NormBlock:
    """Weights, buffers and the passes for a fixed number of rows."""

    def __init__(self, tokens, d, f, seed=0, fmt=mb.MORELLO_NVFP4):
        self.t, self.d, self.f, self.fmt = tokens, d, f, fmt
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def weight(*shape):
            return (torch.randn(*shape, generator=g, device="cuda") / math.sqrt(shape[0])).to(BF)

        self.gamma = (1 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(BF)
        self.beta = (0.1 * torch.randn(d, generator=g, device="cuda")).to(BF)
        self.w1, self.w2 = weight(d, 2 * f), weight(f, d)

        def empty(*shape, dtype=BF):
            return torch.empty(*shape, dtype=dtype, device="cuda")

        self.n, self.mean, self.rstd = empty(tokens, d), empty(tokens, dtype=F32), empty(tokens, dtype=F32)
        self.z, self.h, self.out = empty(tokens, 2 * f), empty(tokens, f), empty(tokens, d)
        # gradients
        self.dh, self.dn, self.dx = empty(tokens, f), empty(tokens, d), empty(tokens, d)
        self.dgamma, self.dbeta = empty(d, dtype=F32), empty(d, dtype=F32)
        self.dw1, self.dw2 = torch.empty_like(self.w1), torch.empty_like(self.w2)
        # 4 bits
        self.n4, self.h4 = Fp4(tokens, d, fmt), Fp4(tokens, f, fmt)
        self.w1_4, self.w2_4 = Fp4(2 * f, d, fmt, parts=2), Fp4(d, f, fmt)
        self.alpha1 = self.alpha2 = None

    def norm(self, x):
        mb.morello_layer_norm(0, mb.MORELLO_BF16, self.t, self.d, EPS, x, self.gamma, self.beta, self.n, self.mean, self.rstd)

    def forward(self, x):
        t, d, f = self.t, self.d, self.f
        self.norm(x)
        mb.morello_linear(mb.MORELLO_ACT_SILU, 1, mb.MORELLO_BF16, 0, t, d, f, self.n, self.w1, None, None, self.h, self.z)
        mb.morello_linear(mb.MORELLO_ACT_NONE, 0, mb.MORELLO_BF16, 0, t, f, d, self.h, self.w2, None, x, self.out)
        return self.out

    def backward(self, x, dout):
        """Gradients of x, gamma, beta and the weights."""
        t, d, f = self.t, self.d, self.f
        mb.morello_linear_backward(mb.MORELLO_ACT_NONE, 0, mb.MORELLO_BF16, 0, 0, t, f, d, self.h, self.w2, None, dout, self.dh,
                                   self.dw2, None)
        mb.morello_linear_backward(mb.MORELLO_ACT_SILU, 1, mb.MORELLO_BF16, 0, 0, t, d, f, self.n, self.w1, self.z, self.dh,
                                   self.dn, self.dw1, None)
        mb.morello_layer_norm_backward(0, mb.MORELLO_BF16, 0, t, d, x, self.gamma, self.mean, self.rstd, self.dn, dout, self.dx,
                                       self.dgamma, self.dbeta)
        return self.dx, self.dgamma, self.dbeta, self.dw1, self.dw2

    def quantize_weights(self, sample=None):
        """The weights to 4 bits.  sample: rows of x, from whose bf16 pass the activations' factors are taken (with room for
        four times as much: beyond that, magnitudes are cut off); None: every tensor without a factor."""
        if sample is not None:
            self.forward(sample)
            self.n4.fit(self.n, 4.0)
            self.h4.fit(self.h, 4.0)
            self.w1_4.fit(self.w1)
            self.w2_4.fit(self.w2)
            self.alpha1 = alpha_of(self.alpha1, self.n4, self.w1_4)
            self.alpha2 = alpha_of(self.alpha2, self.h4, self.w2_4)
        self.w1_4.quantize(self.w1, mb.MORELLO_W_ROWMAJOR)
        self.w2_4.quantize(self.w2, mb.MORELLO_W_ROWMAJOR)

    def serve(self, x):
        """The forward pass in 4 bits; quantize_weights() has been called."""
        t, d, f = self.t, self.d, self.f
        self.norm(x)
        n, h = self.n4.quantize(self.n), self.h4
        mb.morello_fp4_linear(self.fmt, mb.MORELLO_ACT_SILU, 1, mb.MORELLO_BF16, t, d, f, n.q, n.scales, self.w1_4.q, self.w1_4.scales,
                              self.alpha1, None, None, self.h)
        h.quantize(self.h)
        mb.morello_fp4_linear(self.fmt, mb.MORELLO_ACT_NONE, 0, mb.MORELLO_BF16, t, f, d, h.q, h.scales, self.w2_4.q, self.w2_4.scales,
                              self.alpha2, None, x, self.out)
        return self.out


def forward64(x, gamma, beta, w1, w2):
    mean = x.mean(1, keepdim=True)
    n = (x - mean) / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + EPS) * gamma + beta
    gate, up = (n @ w1).chunk(2, dim=1)
    return x + (torch.nn.functional.silu(gate) * up) @ w2


def check(block, x, dout):
    """(error of the forward result, worst error of a gradient along a random direction), relative."""
    at = [v.double() for v in (x, block.gamma, block.beta, block.w1, block.w2)]
    want = forward64(*at)
    out = block.forward(x).clone()
    grads = block.backward(x, dout)
    worst = 0.0
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    for i, grad in enumerate(grads):
        # Along the gradient's own direction a little off it: the slope is as large as it gets.
        way = grad.double() / grad.double().norm() + torch.randn(grad.shape, generator=g, device="cuda").double() / grad.numel() ** 0.5
        step = 1e-4
        up, down = list(at), list(at)
        up[i], down[i] = at[i] + step * way, at[i] - step * way
        slope = float((((forward64(*up) - forward64(*down)) * dout.double()).sum()) / (2 * step))
        mine = float((grad.double() * way).sum())
        worst = max(worst, abs(mine - slope) / abs(slope))
    return float((out.double() - want).norm() / (want - at[0]).norm()), worst


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--tokens", type=int, default=1024)
    ap.add_argument("--d", type=int, default=1024)
    ap.add_argument("--f", type=int, default=2048)
    args = ap.parse_args()
    block = NormBlock(args.tokens, args.d, args.f)
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    x, dout = (torch.randn(args.tokens, args.d, generator=g, device="cuda").to(BF) for _ in range(2))
    forward, worst = check(block, x, dout)
    full = block.forward(x).clone()
    block.quantize_weights(x)
    low = block.serve(x)
    change = (full.double() - x.double()).norm()
    print("forward error %.2e, worst gradient error %.2e, 4 bits against bf16 %.2e (of the block's own part)" %
          (forward, worst, float((low.double() - full.double()).norm() / change)))
    status, detail = mb.morello_read_device_status()
    assert status == mb.MORELLO_OK, (status, hex(detail))


if __name__ == "__main__":
    main()
