"""Products of 4-bit tensors against the 64-bit definition."""
import pytest
import torch

from feed_forward_util import assert_close, device_ok, gen, misaligned
from fp4_util import BLOCK, MX, NV, linear64, packed, values_of
from paper_2505_01637_b200 import binding as mb

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
ACTS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}


def tensor(g, rows, k, fmt, parts=1):
    """Random codes and scales: (q, scales, 64-bit values of about 1)."""
    blocks = (k + BLOCK[fmt] - 1) // BLOCK[fmt]
    codes = torch.randint(0, 16, (rows, k), generator=g, device="cuda")
    near = (127 - 3, 127 + 2) if fmt == MX else (8 * 4, 8 * 8)
    byte = torch.randint(*near, (rows, blocks), generator=g, device="cuda")
    q, s = packed(codes, byte, fmt, parts)
    return q, s, values_of(codes, byte, fmt)


def run(m, k, n, fmt, act="none", gated=False, bias=False, residual=False, f32=False, scaled=False, seed=0, off=False):
    g = gen(seed + m * 3 + n * 5 + k)
    wide = 2 * n if gated else n
    xq, xs, x = tensor(g, m, k, fmt)
    wq, ws, w = tensor(g, wide, k, fmt, 2 if gated else 1)
    w_scale = (torch.tensor([1.0 / (3 * max(1, k) ** 0.5)], device="cuda"))
    alpha = w_scale if scaled else None
    move = misaligned if off else (lambda t: t)
    b = move(torch.randn(wide, generator=g, device="cuda").to(BF)) if bias else None
    r = move(torch.randn(m, n, generator=g, device="cuda").to(BF)) if residual else None
    guard = torch.full((m * n + 16,), 77.0, dtype=F32 if f32 else BF, device="cuda")
    y = (guard[1:] if off else guard)[:m * n].view(m, n)
    mb.morello_fp4_linear(fmt, ACTS[act], int(gated), int(f32), m, k, n, xq, xs, wq, ws, alpha, b, r, y)
    device_ok()
    want, bound = linear64(x, w, alpha, b, r, act, gated, k, f32)
    assert_close(y, want, bound, "y")
    assert torch.all(guard[m * n + int(off):] == 77) and (not off or guard[0] == 77)
    again = torch.empty_like(y)
    mb.morello_fp4_linear(fmt, ACTS[act], int(gated), int(f32), m, k, n, xq, xs, wq, ws, alpha, b, r, again)
    assert torch.equal(y, again)


SHAPES = [(1, 32, 8), (1, 2048, 256), (5, 16, 40), (16, 1000, 136), (33, 256, 64), (64, 4096, 512), (65, 512, 128), (100, 300, 72),
          (128, 1, 128), (129, 2047, 2049), (200, 640, 1000), (333, 2047, 333), (1000, 1024, 520), (257, 64, 1)]


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("fmt", [MX, NV])
@pytest.mark.parametrize("m,k,n", SHAPES)
def test_plain(m, k, n, fmt, f32):
    run(m, k, n, fmt, f32=f32, scaled=True)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("m,k,n", [(3, 96, 200), (40, 512, 72), (150, 1024, 264), (70, 257, 129), (300, 512, 1032)])
def test_epilogues(m, k, n, act, gated):
    run(m, k, n, NV if m % 2 else MX, act, gated, bias=True, residual=True, scaled=True)
    run(m, k, n, MX if m % 2 else NV, act, gated, bias=True, f32=True, scaled=True)
    run(m, k, n, NV, act, gated, residual=True, scaled=True, off=True)


@pytest.mark.parametrize("fmt", [MX, NV])
@pytest.mark.parametrize("m,k,n", [(1, 2048, 8192), (16, 2048, 4096), (64, 8192, 1024), (2048, 512, 2048), (700, 4096, 3000)])
def test_large(m, k, n, fmt):
    run(m, k, n, fmt, "silu", n >= 4096, scaled=True)
    run(m, k, n, fmt, "gelu", False, True, True, True, True)


@pytest.mark.parametrize("fmt", [MX, NV])
@pytest.mark.parametrize("m", [1, 7, 8, 9, 16, 17, 31, 32, 33, 48, 63, 64])
def test_few_rows(m, fmt):
    # one slice, a cluster of every size, slices of different lengths, parts of f32 sums in a slice
    for k, n in ((200, 2000), (768, 333), (2048, 520), (2400, 128), (4096, 19000), (16384, 250)):
        run(m, k, n, fmt, "silu", m % 2 == 0 and n < 9000, True, m % 3 == 0, k > 4096 or m % 5 == 0, True)


@pytest.mark.parametrize("fmt", [MX, NV])
@pytest.mark.parametrize("m,k,n", [(1, 300, 40), (20, 1000, 130), (140, 2048, 390), (520, 700, 512)])
def test_whole_numbers_exactly(m, k, n, fmt):
    # Codes of whole numbers, scales 1 and 2: every sum is a whole number below 2^24.
    g = gen(k)
    whole = torch.tensor([0, 2, 4, 5, 6, 10, 12, 13], device="cuda")      # 0, 1, 2, 3, 4, -1, -2, -3

    def make(rows):
        codes = whole[torch.randint(0, 8, (rows, k), generator=g, device="cuda")]
        one = 127 if fmt == MX else 8 * 7
        byte = one + (1 if fmt == MX else 8) * torch.randint(0, 2, (rows, (k + BLOCK[fmt] - 1) // BLOCK[fmt]), generator=g, device="cuda")
        return (*packed(codes, byte, fmt), values_of(codes, byte, fmt))

    xq, xs, x = make(m)
    wq, ws, w = make(n)
    y = torch.empty(m, n, device="cuda")
    mb.morello_fp4_linear(fmt, 0, 0, 1, m, k, n, xq, xs, wq, ws, None, None, None, y)
    assert torch.equal(y.double(), x @ w.t())


@pytest.mark.parametrize("m", [3, 40, 200])
@pytest.mark.parametrize("fmt", [MX, NV])
def test_scale_of_every_row_and_block(m, fmt):
    # All elements 1, every scale its own: a scale taken from another row, block or part shows.
    k, n = 544, 300
    g = gen(m)
    for gated in (False, True):
        wide = 2 * n if gated else n

        def make(rows, parts):
            blocks = (k + BLOCK[fmt] - 1) // BLOCK[fmt]
            codes = torch.full((rows, k), 2, device="cuda")
            low, high = (120, 134) if fmt == MX else (8, 120)
            byte = torch.randint(low, high, (rows, blocks), generator=g, device="cuda")
            return (*packed(codes, byte, fmt, parts), values_of(codes, byte, fmt))

        xq, xs, x = make(m, 1)
        wq, ws, w = make(wide, 2 if gated else 1)
        y = torch.empty(m, n, device="cuda")
        mb.morello_fp4_linear(fmt, 0, int(gated), 1, m, k, n, xq, xs, wq, ws, None, None, None, y)
        want, bound = linear64(x, w, None, None, None, "none", gated, k, True)
        assert_close(y, want, bound)


@pytest.mark.parametrize("m", [2, 70])
@pytest.mark.parametrize("fmt", [MX, NV])
def test_nan_scale_reaches_its_results_alone(m, fmt):
    g = gen(9)
    k, n = 96, 40
    _, _, x = tensor(g, m, k, fmt)
    codes = torch.randint(0, 8, (m, k), generator=g, device="cuda")
    byte = torch.full((m, k // BLOCK[fmt]), 127 if fmt == MX else 56, device="cuda")
    byte[1, 1] = 255 if fmt == MX else 127
    xq, xs = packed(codes, byte, fmt)
    wq, ws, w = tensor(g, n, k, fmt)
    y = torch.empty(m, n, device="cuda", dtype=BF)
    mb.morello_fp4_linear(fmt, 0, 0, 0, m, k, n, xq, xs, wq, ws, None, None, None, y)
    nan = torch.isnan(y)
    assert bool(nan[1].all()) and not bool(nan[0].any()) and not bool(nan[2:].any())


def test_empty_sums_and_residual_in_place():
    b = torch.randn(24, generator=gen(1), device="cuda").to(BF)
    r = torch.randn(5, 24, generator=gen(2), device="cuda").to(BF)
    y = torch.empty_like(r)
    for m in (5, 1):
        mb.morello_fp4_linear(NV, ACTS["relu"], 0, 0, m, 0, 24, None, None, None, None, None, b, r, y)
        want = torch.relu(b.double()) + r.double()[:m]
        assert torch.all((y[:m].double() - want).abs() <= 2.0 ** -8 * want.abs())
    y.fill_(3.0)
    mb.morello_fp4_linear(NV, 0, 0, 0, 0, 64, 24, None, None, None, None, None, None, None, None)
    mb.morello_fp4_linear(NV, 0, 0, 0, 5, 64, 0, None, None, None, None, None, None, None, None)
    assert torch.all(y == 3)
    g = gen(4)
    for m in (9, 150):
        xq, xs, x = tensor(g, m, 128, MX)
        wq, ws, w = tensor(g, 264, 128, MX)
        r = torch.randn(m, 264, generator=g, device="cuda").to(BF)
        y = r.clone()
        mb.morello_fp4_linear(MX, 0, 0, 0, m, 128, 264, xq, xs, wq, ws, None, None, y, y)
        want, bound = linear64(x, w, None, None, r, "none", False, 128, False)
        assert_close(y, want, bound)


@pytest.mark.parametrize("m", [4, 180])
def test_stream_and_graph(m):
    g = gen(m)
    k, n = 512, 320
    xq, xs, x = tensor(g, m, k, NV)
    wq, ws, w = tensor(g, 2 * n, k, NV, 2)
    y = torch.empty(m, n, device="cuda", dtype=BF)

    def call(stream=None):
        mb.morello_fp4_linear(NV, ACTS["silu"], 1, 0, m, k, n, xq, xs, wq, ws, None, None, None, y, stream=stream)

    def check(x):
        want, bound = linear64(x, w, None, None, None, "silu", True, k, False)
        assert_close(y, want, bound)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(side)
    side.synchronize()
    check(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    q2, s2, x2 = tensor(gen(77), m, k, NV)
    xq.copy_(q2)
    xs.copy_(s2)
    graph.replay()
    torch.cuda.synchronize()
    check(x2)


@pytest.mark.parametrize("n", [4096, 4001])
def test_elements_past_two_to_the_31(n):
    m, k = 540000, 32
    g = gen(n)
    xq, xs, x = tensor(g, m, k, MX)
    wq, ws, w = tensor(g, n, k, MX)
    y = torch.full((m, n), 77.0, dtype=BF, device="cuda")
    mb.morello_fp4_linear(MX, 0, 0, 0, m, k, n, xq, xs, wq, ws, None, None, None, y)
    device_ok()
    for at in (slice(0, 300), slice(m - 300, m)):
        want, bound = linear64(x[at], w, None, None, None, "none", False, k, False)
        assert_close(y[at], want, bound, "y")
