"""Quantisation to 4-bit blocks and reading back: every code and scale byte against the definition."""
import pytest
import torch

from feed_forward_util import gen, misaligned
from fp4_util import BLOCK, E2M1, MX, NV, buffers, e4m3_values, packed, quantized64, unpacked, values_of
from paper_2505_01637_b200 import binding as mb

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
SHAPES = [(1, 1, 1), (1, 1, 2048), (3, 1, 17), (16, 1, 2047), (130, 1, 96), (128, 1, 256), (64, 2, 100), (257, 1, 520),
          (6, 3, 33), (300, 2, 1000), (1, 1, 31), (2, 2, 16)]


def quantize(x, fmt, rowmajor=False, parts=1, mult=None):
    """x [rows][k] through the library, given in the other layout where asked: (q, scales)."""
    rows, k = x.shape
    q, s = buffers(fmt, rows, parts, k)
    data = x
    if rowmajor:
        data = x.t().contiguous() if x.storage_offset() == 0 else misaligned(x.t().contiguous())
    mb.morello_fp4_quantize(fmt, int(x.dtype == F32), 0 if rowmajor else 1, rows, parts, k, data, mult, q, s)
    return q, s


def check(x, fmt, rowmajor=False, parts=1, mult=None):
    rows, k = x.shape
    q, s = quantize(x, fmt, rowmajor, parts, mult)
    codes, byte = unpacked(q, s, fmt, rows, parts, k)
    want, want_byte = quantized64(x, fmt, mult)
    assert torch.equal(byte, want_byte), int((byte != want_byte).sum())
    same = (codes == want) | ((codes % 8 == 0) & (want % 8 == 0))          # a zero may have either sign
    assert bool(same.all()), int((~same).sum())
    return q, s, codes, byte


@pytest.mark.parametrize("scaled", [False, True])
@pytest.mark.parametrize("rowmajor", [False, True])
@pytest.mark.parametrize("kind", [BF, F32])
@pytest.mark.parametrize("fmt", [MX, NV])
@pytest.mark.parametrize("rows,parts,k", SHAPES)
def test_quantize_and_read_back(rows, parts, k, fmt, kind, rowmajor, scaled):
    g = gen(rows * 7 + k)
    x = (torch.randn(rows, k, generator=g, device="cuda") * torch.exp(2 * torch.randn(rows, 1, generator=g, device="cuda"))).to(kind)
    mult = torch.tensor([3.7], device="cuda") if scaled else None
    q, s, codes, byte = check(x, fmt, rowmajor, parts, mult)
    want = values_of(codes, byte, fmt)
    alpha = torch.tensor([0.37], device="cuda")
    for out in (BF, F32):
        y = torch.full((rows, k), 9.0, dtype=out, device="cuda")
        mb.morello_fp4_dequantize(fmt, int(out == F32), rows, parts, k, q, s, None, y)
        assert torch.equal(y.double(), want)
        mb.morello_fp4_dequantize(fmt, int(out == F32), rows, parts, k, q, s, alpha, y)
        step = 2.0 ** -23 + (2.0 ** -8 if out == BF else 0)
        assert torch.all((y.double() - want * alpha.double()).abs() <= step * (want * alpha.double()).abs())


@pytest.mark.parametrize("rowmajor", [False, True])
@pytest.mark.parametrize("kind", [BF, F32])
@pytest.mark.parametrize("fmt", [MX, NV])
def test_unaligned(fmt, kind, rowmajor):
    g = gen(5)
    x = misaligned(torch.randn(70, 264, generator=g, device="cuda").to(kind))
    q, s, codes, byte = check(x, fmt, rowmajor)
    y = misaligned(torch.zeros(70, 264, dtype=kind, device="cuda"))
    mb.morello_fp4_dequantize(fmt, int(kind == F32), 70, 1, 264, q, s, None, y)
    assert torch.equal(y.double(), values_of(codes, byte, fmt))


@pytest.mark.parametrize("kind", [BF, F32])
def test_ties_of_every_scale(kind):
    # Midpoints of the 4-bit values times every e4m3 scale, one ulp beside them too.  The block's 6 s fixes its scale.
    eight = e4m3_values()[1:].float()
    middle = ((E2M1[:-1] + E2M1[1:]) / 2).float()
    tie = eight[:, None] * middle[None]
    size = 2 ** 16 if kind == BF else 1
    bits = tie.view(torch.int32)
    x = torch.stack([tie, (bits + size).view(F32), (bits - size).view(F32)], 2).reshape(len(eight), -1)
    x = torch.cat([x[:, :15], 6 * eight[:, None], x[:, 6:], 6 * eight[:, None]], 1)           # two blocks, 6 s in each
    x = torch.cat([x, -x], 0).cuda().to(kind)
    assert x.shape[1] == 32
    for mult in (None, torch.ones(1, device="cuda")):
        for rowmajor in (False, True):
            _, _, _, byte = check(x, NV, rowmajor, mult=mult)
            assert torch.equal(byte[:, 0], torch.arange(1, 127, device="cuda").repeat(2))


@pytest.mark.parametrize("fmt", [MX, NV])
def test_border_of_the_scale(fmt):
    # Largest magnitudes beside and on the borders between two scales.
    if fmt == MX:
        edge = torch.tensor([2.0 ** e for e in range(-140, 128)], dtype=torch.float32)
    else:
        v = e4m3_values()
        edge = (6 * torch.cat([(v[:-1] + v[1:]) / 2, v[1:]])).float()
    bits = edge.view(torch.int32)
    amax = torch.cat([edge, (bits + 1).view(F32), (bits - 1).view(F32)])
    x = torch.zeros(len(amax), BLOCK[fmt])
    x[:, 3] = amax
    x[:, 5] = -amax / 3
    for rowmajor in (False, True):
        check(x.cuda(), fmt, rowmajor)


@pytest.mark.parametrize("rowmajor", [False, True])
@pytest.mark.parametrize("kind", [BF, F32])
@pytest.mark.parametrize("fmt", [MX, NV])
def test_extremes(fmt, kind, rowmajor):
    x = torch.randn(8, 64, generator=gen(1), device="cuda")
    x[0] = 0.0
    x[1] = 1e-42                     # subnormal
    x[2, :40] = 3e38
    x[3, 20] = float("nan")
    x[4, 50] = float("-inf")
    x[5] = 2.0 ** -126
    x[6, 1:] = 0.0
    x = x.to(kind)
    bad = torch.zeros(8, 64, dtype=torch.bool, device="cuda")
    bad[3, 20 // BLOCK[fmt] * BLOCK[fmt]:][:BLOCK[fmt]] = True
    bad[4, 50 // BLOCK[fmt] * BLOCK[fmt]:][:BLOCK[fmt]] = True
    q, s = quantize(x, fmt, rowmajor)
    y = torch.zeros(8, 64, device="cuda")
    mb.morello_fp4_dequantize(fmt, 1, 8, 1, 64, q, s, None, y)
    assert torch.equal(torch.isnan(y), bad)
    codes, byte = quantized64(torch.where(bad, torch.zeros_like(x), x), fmt)
    want = values_of(codes, byte, fmt)
    assert torch.equal(y.double()[~bad], want[~bad])


def test_values_of_every_code_and_byte():
    for fmt, most in ((MX, 256), (NV, 128)):
        byte = torch.arange(most, device="cuda").view(-1, 1)
        codes = torch.arange(16, device="cuda").repeat(most, BLOCK[fmt] // 16)
        q, s = packed(codes, byte, fmt)
        for out in (BF, F32):
            y = torch.zeros(most, BLOCK[fmt], dtype=out, device="cuda")
            mb.morello_fp4_dequantize(fmt, int(out == F32), most, 1, BLOCK[fmt], q, s, None, y)
            want = values_of(codes, byte, fmt)
            # the largest values of the largest power of two are past f32's end
            want = torch.where(want.abs() >= 2.0 ** 128, want * float("inf"), want)
            assert torch.equal(torch.isnan(y), torch.isnan(want))
            assert torch.equal(torch.nan_to_num(y.double(), 0.0), torch.nan_to_num(want.to(torch.float64), 0.0))


def test_empty_stream_and_graph():
    x = torch.zeros(0, 64, device="cuda", dtype=BF)
    q, s = buffers(MX, 0, 1, 64)
    mb.morello_fp4_quantize(MX, 0, 1, 0, 1, 64, x, None, q, s)
    mb.morello_fp4_quantize(MX, 0, 1, 5, 1, 0, x, None, q, s)
    mb.morello_fp4_dequantize(MX, 0, 5, 1, 0, q, s, None, x)
    assert torch.all(q == 0xEE) and torch.all(s == 0xEE)
    x = torch.randn(200, 300, generator=gen(2), device="cuda").to(BF)
    q, s = buffers(NV, 200, 2, 300)
    y = torch.empty_like(x)

    def both(stream=None):
        mb.morello_fp4_quantize(NV, 0, 1, 200, 2, 300, x, None, q, s, stream=stream)
        mb.morello_fp4_dequantize(NV, 0, 200, 2, 300, q, s, None, y, stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    both(side)
    side.synchronize()
    assert torch.equal(y.double(), values_of(*quantized64(x, NV), NV))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    x.mul_(-1.75)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y.double(), values_of(*quantized64(x, NV), NV))


@pytest.mark.parametrize("off", [0, 1, 2, 4])
@pytest.mark.parametrize("rows,k", [(1, 1), (2, 255), (33, 256), (130, 257), (40, 258), (3, 511), (129, 513), (64, 1028), (5, 2047)])
def test_nothing_beside_the_tensors(rows, k, off):
    # Y, Q and the scales lie in larger buffers whose other bytes stay as they are.
    x = torch.randn(rows, k, generator=gen(k), device="cuda").to(BF)
    nq, ns = mb.morello_fp4_bytes(rows, k), mb.morello_fp4_scale_bytes(NV, rows, 1, k)
    guarded = torch.full((32 + nq + 32 + ns + 32,), 0x5A, dtype=torch.uint8, device="cuda")
    ns0 = 32 + nq + (-nq) % 16
    q, s = guarded[32:32 + nq], guarded[ns0:ns0 + ns]
    mb.morello_fp4_quantize(NV, 0, 1, rows, 1, k, x, None, q, s)
    beside = torch.ones_like(guarded, dtype=torch.bool)
    beside[32:32 + nq] = False
    beside[ns0:ns0 + ns] = False
    assert torch.all(guarded[beside] == 0x5A)
    want = values_of(*quantized64(x, NV), NV)
    for out in (BF, F32):
        whole = torch.full((16 + rows * k + 16,), 9.0, dtype=out, device="cuda")
        y = whole[8 + off:8 + off + rows * k].view(rows, k)
        mb.morello_fp4_dequantize(NV, int(out == F32), rows, 1, k, q, s, None, y)
        assert torch.equal(y.double(), want)
        assert torch.all(whole[:8 + off] == 9.0) and torch.all(whole[8 + off + rows * k:] == 9.0)


@pytest.mark.parametrize("rowmajor,rows,k", [(False, 2100000, 16), (False, 530000, 4100), (True, 3, 16800000), (True, 2200000, 1000)])
def test_long_tensors(rowmajor, rows, k):
    # More groups of rows, or pieces of a row, than a grid has, and elements past 2^31: the last ones as by themselves.
    x = torch.empty(k if rowmajor else rows, rows if rowmajor else k, dtype=BF, device="cuda")
    x.normal_(generator=gen(3))
    q, s = buffers(MX, rows, 1, k)
    mb.morello_fp4_quantize(MX, 0, int(not rowmajor), rows, 1, k, x, None, q, s)
    last = min(rows, 200 + rows % 128)              # from an atom's first row on, or all of them
    few = 64 * 128 if rows < 200 else k
    part = (x[-few:, -last:].t() if rowmajor else x[-last:]).contiguous()
    q2, s2 = quantize(part, MX)
    pitch, pitch2 = (k + 31) // 32 * 16, (few + 31) // 32 * 16
    assert torch.equal(q[:rows * pitch].view(rows, pitch)[-last:, -pitch2:], q2[:last * pitch2].view(last, pitch2))
    y = torch.empty(rows, k, dtype=BF, device="cuda")
    mb.morello_fp4_dequantize(MX, 0, rows, 1, k, q, s, None, y)
    y2 = torch.empty(last, few, dtype=BF, device="cuda")
    mb.morello_fp4_dequantize(MX, 0, last, 1, few, q2, s2, None, y2)
    assert torch.equal(y[-last:, -few:], y2)
