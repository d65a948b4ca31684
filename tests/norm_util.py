"""64-bit definitions of the norms and the error bounds the tests hold them to.

The bounds are derived, not fitted.  A thread adds at most 32 numbers in a row and the joins are trees or rows of at most
32, so an f32 mean of values v is within 2^-17 (128 roundings of 2^-24) of mean |v|; differences, factors and the root add a few
roundings more, which the same 2^-17 covers.  A bf16 result is within 2^-8 of its value, an f32 one within 2^-24."""
import torch

from paper_2505_01637_b200 import binding as mb

F32 = 2.0 ** -17
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def misaligned(t):
    """The same values at an address that is off a 16-byte boundary by one element."""
    flat = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)
    flat[1:] = t.reshape(-1)
    return flat[1:].view(t.shape)


def norm64(x, gamma, beta, eps, rms):
    x = x.double()
    mean = torch.zeros_like(x[:, :1]) if rms else x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + eps)
    h = (x - mean) * rstd
    y = h if gamma is None else h * gamma.double()
    return mean, rstd, h, y if beta is None else y + beta.double()


def check_forward(x, gamma, beta, eps, rms, y, mean, rstd):
    m64, r64, h, want = norm64(x, gamma, beta, eps, rms)
    g = torch.ones_like(h[:1]) if gamma is None else gamma.double()[None]
    b = torch.zeros_like(g) if beta is None else beta.double()[None]
    # the mean is off by F32 of the differences, about F32 / rstd, which the factor rstd gamma carries to y
    tol = ROUND[torch.bfloat16] * want.abs() + F32 * ((h * g).abs() + g.abs() + b.abs()) + 1e-30
    assert torch.all((y.double() - want).abs() <= tol), float(((y.double() - want).abs() / tol).max())
    if rstd is not None:
        assert torch.all((rstd.double() - r64[:, 0]).abs() <= F32 * r64[:, 0])
    if mean is not None and not rms:
        spread = (x.double() - m64).abs().mean(1)
        assert torch.all((mean.double() - m64[:, 0]).abs() <= 2.0 ** -23 * m64[:, 0].abs() + F32 * spread + 1e-30)


def check_backward(x, gamma, mean, rstd, dy, r, rms, dx, dgamma, dbeta, base_g=None, base_b=None):
    m = x.shape[0]
    mu = 0.0 if rms else mean.double()[:, None]
    rs = rstd.double()[:, None]
    h = (x.double() - mu) * rs
    g = dy.double() if gamma is None else dy.double() * gamma.double()
    mg = 0.0 if rms else g.mean(1, keepdim=True)
    gh = (g * h).mean(1, keepdim=True)
    if dx is not None:
        want = rs * (g - mg - h * gh)
        tol = F32 * rs * (g.abs() + (0 if rms else g.abs().mean(1, keepdim=True)) + h.abs() * (g * h).abs().mean(1, keepdim=True))
        if r is not None:
            want = want + r.double()
            tol = tol + 2.0 ** -23 * r.double().abs()
        tol = tol + ROUND[dx.dtype] * want.abs() + 1e-30
        assert torch.all((dx.double() - want).abs() <= tol), float(((dx.double() - want).abs() / tol).max())
    # Sums over rows: at most m / 296 + 1 of them in a thread, then 8 or 32 of a block, 37 of a warp and 8 in order.
    steps = (m / 296 + 128) * 2.0 ** -24
    for got, terms, base in ((dgamma, dy.double() * h, base_g), (dbeta, dy.double(), base_b)):
        if got is None:
            continue
        want = terms.sum(0) + (0 if base is None else base.double())
        tol = steps * (terms.abs().sum(0) + (0 if base is None else base.double().abs())) + 1e-30
        assert torch.all((got.double() - want).abs() <= tol), float(((got.double() - want).abs() / tol).max())


def forward(x, gamma, beta, eps, rms, keep=True):
    m, n = x.shape
    y = torch.full((m, n), float("nan"), device="cuda", dtype=torch.bfloat16)
    mean = torch.full((m,), float("nan"), device="cuda") if keep and not rms else None
    rstd = torch.full((m,), float("nan"), device="cuda") if keep else None
    mb.morello_layer_norm(int(rms), int(x.dtype == torch.float32), m, n, eps, x, gamma, beta, y, mean, rstd)
    return y, mean, rstd
