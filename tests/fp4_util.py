"""4-bit tensors in the library's layout, and their definition in 64 bits."""
import torch

from feed_forward_util import act64, split
from paper_2505_01637_b200 import binding as mb

MX, NV = mb.MORELLO_MXFP4, mb.MORELLO_NVFP4
BLOCK = {MX: 32, NV: 16}
E2M1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
POWERS = torch.tensor([2.0 ** e for e in range(-127, 128)], dtype=torch.float64)


def e4m3_values():
    """The 127 values of e4m3 without a sign, in order."""
    return torch.tensor([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127],
                        dtype=torch.float64)


def nearest(v, grid):
    """Index of the member of a sorted grid nearest to v, ties to even, the last one beyond its end."""
    grid = grid.to(v.device)
    middle = (grid[:-1] + grid[1:]) / 2
    place = torch.bucketize(v.contiguous(), middle)
    tie = (place < len(middle)) & (v == middle[place.clamp(max=len(middle) - 1)]) & (place % 2 == 1)
    return place + tie.long()


def quantized64(x, fmt, mult=None):
    """(codes [rows][k], scale bytes [rows][blocks]) of finite x [rows][k]."""
    if mult is not None:
        x = x.float() * mult.float()
    x = x.double()
    rows, k = x.shape
    block = BLOCK[fmt]
    blocks = (k + block - 1) // block
    padded = torch.zeros(rows, blocks * block, dtype=torch.float64, device=x.device)
    padded[:, :k] = x
    g = padded.view(rows, blocks, block)
    amax = g.abs().amax(2)
    if fmt == MX:
        byte = (torch.bucketize(amax, POWERS.to(x.device), right=True) - 3).clamp(min=0)      # floor(log2) - 2, plus 127
        scale = POWERS.to(x.device)[byte]
    else:
        byte = nearest(amax / 6, e4m3_values())
        scale = e4m3_values().to(x.device)[byte]
    v = torch.where(scale[..., None] > 0, g / scale[..., None], torch.zeros_like(g))
    codes = nearest(v.abs(), E2M1) + 8 * torch.signbit(v).long()
    return codes.view(rows, -1)[:, :k], byte


def values_of(codes, byte, fmt):
    """64-bit values; a NaN byte makes its block NaN."""
    block = BLOCK[fmt]
    e = E2M1.to(codes.device)
    v = torch.where(codes >= 8, -e[codes % 8], e[codes % 8])
    if fmt == MX:
        scale = torch.where(byte == 255, float("nan"), POWERS.to(codes.device)[byte.clamp(max=254)])
    else:
        scale = torch.where(byte == 127, float("nan"), e4m3_values().to(codes.device)[byte.clamp(max=126)])
    return v * scale.repeat_interleave(block, 1)[:, :codes.shape[1]]


def buffers(fmt, rows, parts, k, fill=0xEE):
    """Buffers for a tensor of the reported sizes, with a guard of 64 bytes behind each."""
    q = torch.full((mb.morello_fp4_bytes(rows, k) + 64,), fill, dtype=torch.uint8, device="cuda")
    s = torch.full((mb.morello_fp4_scale_bytes(fmt, rows, parts, k) + 64,), fill, dtype=torch.uint8, device="cuda")
    return q, s


def unpacked(q, scales, fmt, rows, parts, k):
    """(codes, scale bytes) from buffers(); checks their padding and guards."""
    pitch, block = (k + 31) // 32 * 16, BLOCK[fmt]
    each, blocks = rows // parts, (k + block - 1) // block
    down, across = (each + 127) // 128, (blocks + 3) // 4
    assert torch.all(q[rows * pitch:] == 0xEE) and torch.all(scales[parts * down * across * 512:] == 0xEE)
    b = q[:rows * pitch].view(rows, pitch).long()
    codes = torch.stack([b & 15, b >> 4], 2).view(rows, -1)
    assert torch.all(codes[:, k:] == 0)
    s = scales[:parts * down * across * 512].view(parts, down, across, 32, 4, 4).permute(0, 1, 4, 3, 2, 5)
    s = s.reshape(parts, down * 128, across * 4).long()
    assert torch.all(s[:, each:] == 0) and torch.all(s[:, :, blocks:] == 0)
    return codes[:, :k], s[:, :each, :blocks].reshape(rows, blocks)


def packed(codes, byte, fmt, parts=1):
    """Buffers from codes and scale bytes, without the library."""
    rows, k = codes.shape
    pitch, each, blocks = (k + 31) // 32 * 16, rows // parts, byte.shape[1]
    down, across = (each + 127) // 128, (blocks + 3) // 4
    full = torch.zeros(rows, 2 * pitch, dtype=torch.uint8, device=codes.device)
    full[:, :k] = codes.to(torch.uint8)
    q = (full[:, 0::2] + 16 * full[:, 1::2]).contiguous()
    s = torch.zeros(parts, down * 128, across * 4, dtype=torch.uint8, device=codes.device)
    s[:, :each, :blocks] = byte.view(parts, each, blocks).to(torch.uint8)
    return q, s.view(parts, down, 4, 32, across, 4).permute(0, 1, 4, 3, 2, 5).contiguous()


def linear64(x, w, alpha, bias, r, act, gated, k, parted):
    """(y, bound before its rounding) of the product of 64-bit values x [m][k], w [wide][k].

    Products are exact.  The tensor cores add 64 of them a step by truncation, at most 2^-23 of the terms' sum each
    time, twice a step (inside it and to the accumulator); parted: the sums of 16 steps, added to nearest."""
    steps = (k + 63) // 64
    each = 2.0 ** -23 * (2 * min(steps, 16) + (steps + 15) // 16 if parted else 2 * steps) + 2.0 ** -22
    z, ez = x @ w.t(), each * (x.abs() @ w.abs().t())
    if alpha is not None:
        z, ez = z * alpha.double(), (ez + 2.0 ** -24 * z.abs()) * alpha.double().abs()
    if bias is not None:
        z = z + bias.double()
        ez = ez + 2.0 ** -24 * z.abs()
    a, b = split(z, gated)
    ea, eb = split(ez, gated)
    y = act64(a, act)
    ey = 1.13 * ea + (0 if act == "none" else 4e-6 * (1 + a.abs()))
    if gated:
        y, ey = y * b, ey * b.abs() + y.abs() * eb + ey * eb + 2.0 ** -24 * (y * b).abs()
    if r is not None:
        y = y + r.double()
    return y, ey + 2.0 ** -23 * (y.abs() + (0 if r is None else r.double().abs()))
