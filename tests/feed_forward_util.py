"""64-bit definitions of the feed-forward operators and the error bounds the tests hold them to.

The bounds are derived, not fitted.  A product's f32 sum is within 1e-5 * sum|x w| + 1e-6 (the library's own rule);
an activation has a slope of at most 1.13 and an f32 evaluation error of at most 4e-6 * (1 + |z|); a bf16 result is
within 2^-8 of its value (half a unit in the last place of an 8-bit significand), BF16 below."""
import math

import torch

from paper_2505_01637_b200 import binding as mb

BF16 = 2.0 ** -8
TINY = 1e-6
ACTS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(torch.bfloat16)


def misaligned(t):
    """The same values at an address that is off a 16-byte boundary by one element."""
    flat = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)
    flat[1:] = t.reshape(-1)
    return flat[1:].view(t.shape)


def act64(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def slope64(z, act):
    if act == "none":
        return torch.ones_like(z)
    if act == "relu":
        return (z > 0).double()
    with torch.enable_grad():
        z = z.clone().requires_grad_(True)
        return torch.autograd.grad(act64(z, act).sum(), z)[0]


def split(z, gated):
    n = z.shape[-1] // 2
    return (z[..., :n], z[..., n:]) if gated else (z, None)


def forward64(x, w, bias, r, act, gated):
    """(y, bound of y before its rounding, z, bound of z); x [m][k], w [k][w] in 64 bits."""
    z = x @ w
    ez = 1e-5 * (x.abs() @ w.abs()) + TINY
    if bias is not None:
        z = z + bias
        ez = ez + 1e-6 * bias.abs()
    a, b = split(z, gated)
    ea, eb = split(ez, gated)
    y = act64(a, act)
    ey = 1.13 * ea + (0 if act == "none" else 4e-6 * (1 + a.abs()))
    if gated:
        y, ey = y * b, ey * b.abs() + y.abs() * eb + ey * eb
    if r is not None:
        y = y + r
        ey = ey + 1e-6 * r.abs()
    return y, ey, z, ez


def dz64(z, dy, act, gated):
    """(dz, bound of its f32 evaluation)"""
    a, b = split(z, gated)
    s = slope64(a, act)
    es = 0 if act in ("none", "relu") else 1e-5 * (1 + a.abs())
    if not gated:
        return dy * s, dy.abs() * es + TINY * dy.abs()
    v = act64(a, act)
    return (torch.cat([dy * b * s, dy * v], -1),
            torch.cat([(dy * b).abs() * (es + TINY), dy.abs() * 4e-6 * (1 + a.abs())], -1))


def assert_close(got, want, bound, what=""):
    """|got - want| <= bound, element by element; bf16 results may be rounded besides."""
    got64 = got.double()
    if got.dtype == torch.bfloat16:
        bound = bound + BF16 * (want.abs() + bound)
    err = (got64 - want).abs()
    bad = ~(err <= bound)
    if bool(bad.any()):
        at = tuple(int(v) for v in bad.nonzero()[0])
        raise AssertionError("%s: %d of %d elements off; first at %s: got %r want %r bound %r" % (
            what, int(bad.sum()), got.numel(), at, float(got64[at]), float(want[at]), float(bound[at])))


def device_ok():
    status, detail = mb.morello_read_device_status()
    assert status == mb.MORELLO_OK, (status, hex(detail))


def plan_of(idx, experts):
    """The plan buffer of idx [T][K] from the library, and its sections."""
    t, k = idx.shape
    plan = torch.full((mb.morello_expert_plan_words(t, k, experts),), 12345, dtype=torch.int32, device="cuda")
    mb.morello_expert_plan(t, k, experts, idx, plan)
    return plan, sections(plan, t, k, experts)


def sections(plan, t, k, experts):
    rows = mb.morello_expert_plan_rows(t, k, experts)
    sizes = [rows, rows // 128, experts + 1, experts, t * k]
    sizes.append(plan.numel() - sum(sizes))
    parts = torch.split(plan, sizes)
    return dict(zip(["row_src", "block_expert", "offsets", "counts", "slot"], parts))
