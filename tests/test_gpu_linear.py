"""Linear layers with their epilogue and their gradients against the definition in 64 bits."""
import itertools

import pytest
import torch

from feed_forward_util import (ACTS, BF16, TINY, assert_close, device_ok, dz64, forward64, gen, misaligned, randn)
from paper_2505_01637_b200 import binding as mb

pytestmark = pytest.mark.gpu


def weights(g, k, wide, colmajor):
    w = randn(g, *((wide, k) if colmajor else (k, wide)), scale=max(k, 1) ** -0.5)
    return w, (w.t() if colmajor else w).double()


def run_linear(m, k, n, act="none", gated=False, colmajor=False, bias=True, residual=True, keep_z=True, f32=False, seed=0,
               shift=False):
    g = gen(seed + m + 3 * k + 7 * n)
    wide = 2 * n if gated else n
    x = randn(g, m, k)
    w, w64 = weights(g, k, wide, colmajor)
    b = randn(g, wide, scale=0.5) if bias else None
    r = randn(g, m, n) if residual else None
    y = torch.full((m, n), float("nan"), device="cuda", dtype=torch.float32 if f32 else torch.bfloat16)
    z = torch.full((m, wide), float("nan"), device="cuda", dtype=torch.bfloat16) if keep_z else None
    if shift:
        x, w, y = misaligned(x), misaligned(w), misaligned(y)
        b, r, z = (None if v is None else misaligned(v) for v in (b, r, z))
    mb.morello_linear(ACTS[act], gated, f32, colmajor, m, k, n, x, w, b, r, y, z)
    device_ok()
    want, bound, z64, ez = forward64(x.double(), w64, None if b is None else b.double(),
                                     None if r is None else r.double(), act, gated)
    assert_close(y, want, bound, "Y")
    if keep_z:
        assert_close(z, z64, ez, "Z")


@pytest.mark.parametrize("m,k,n", [(1, 64, 64), (1, 2048, 512), (2, 8, 8), (3, 1000, 136), (16, 512, 1024), (17, 4096, 128),
                                   (33, 256, 264), (64, 1024, 512), (65, 128, 128), (128, 64, 256), (129, 192, 264),
                                   (300, 520, 648), (512, 1024, 1024), (1025, 256, 520)])
@pytest.mark.parametrize("gated,colmajor", [(False, False), (False, True), (True, False), (True, True)])
def test_sizes(m, k, n, gated, colmajor):
    run_linear(m, k, n, "silu", gated, colmajor)


@pytest.mark.parametrize("m,k,n", [(1, 1, 1), (1, 7, 5), (5, 63, 65), (70, 33, 31), (130, 257, 259), (1, 2047, 513),
                                   (200, 100, 100), (256, 1001, 512), (256, 512, 1001)])
@pytest.mark.parametrize("gated,colmajor", [(False, False), (False, True), (True, False), (True, True)])
def test_odd_sizes(m, k, n, gated, colmajor):
    run_linear(m, k, n, "gelu", gated, colmajor)


@pytest.mark.parametrize("act,gated,f32", list(itertools.product(ACTS, [False, True], [False, True])))
@pytest.mark.parametrize("m", [5, 150])
def test_activations_and_types(act, gated, f32, m):
    run_linear(m, 136, 72, act, gated, False, True, True, True, f32)


@pytest.mark.parametrize("bias,residual,keep_z", list(itertools.product([False, True], repeat=3)))
@pytest.mark.parametrize("m", [20, 140])
def test_optional_tensors(bias, residual, keep_z, m):
    run_linear(m, 72, 200, "gelu", False, False, bias, residual, keep_z)


@pytest.mark.parametrize("m,k,n,gated", [(4, 128, 128, False), (200, 128, 136, True), (40, 72, 264, True)])
@pytest.mark.parametrize("colmajor", [False, True])
def test_misaligned_tensors(m, k, n, gated, colmajor):
    run_linear(m, k, n, "silu", gated, colmajor, shift=True)


@pytest.mark.parametrize("m,n,gated", [(1, 24, False), (70, 130, True), (200, 64, False)])
def test_empty_sum(m, n, gated):
    run_linear(m, 0, n, "gelu", gated, False)


@pytest.mark.parametrize("m,k,n", [(0, 8, 8), (4, 8, 0), (0, 0, 0)])
def test_nothing_to_do(m, k, n):
    y = torch.full((8, 8), 7.0, device="cuda", dtype=torch.bfloat16)
    x = torch.ones(64, 64, device="cuda", dtype=torch.bfloat16)
    mb.morello_linear(0, 0, 0, 0, m, k, n, x, x, None, None, y)
    assert bool((y == 7).all())


@pytest.mark.parametrize("m", [3, 100])
def test_residual_in_place(m):
    g = gen(5)
    x, w, y = randn(g, m, 64), randn(g, 64, 72, scale=0.125), randn(g, m, 72)
    want, bound, _, _ = forward64(x.double(), w.double(), None, y.double(), "relu", False)
    mb.morello_linear(ACTS["relu"], 0, 0, 0, m, 64, 72, x, w, None, y, y)
    assert_close(y, want, bound)


@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("m", [4, 80])
def test_extreme_values(act, m):
    """Large and infinite z: the activations' limits; NaN stays in its own row."""
    k = n = 64
    x = torch.zeros(m, k, device="cuda", dtype=torch.bfloat16)
    w = torch.eye(k, device="cuda", dtype=torch.bfloat16)
    inf = float("inf")
    x[0, 0], x[1, 1], x[2, 2], x[3, 3] = 3e38, -3e38, 200.0, -200.0
    y = torch.empty(m, n, device="cuda", dtype=torch.float32)
    bias = torch.zeros(n, device="cuda", dtype=torch.bfloat16)
    bias[5], bias[6], bias[7] = inf, -inf, float("nan")
    mb.morello_linear(ACTS[act], 0, 1, 0, m, k, n, x, w, bias, None, y)
    y = y.cpu()
    assert y[0, 0] == x[0, 0].float().cpu() and y[2, 2] == 200.0
    assert y[1, 1] == 0 and y[3, 3] == 0
    assert bool((y[:, 5] == inf).all()) and bool((y[:, 6] == 0).all()) and bool(y[:, 7].isnan().all())
    assert not bool(y[:, 8:].isnan().any())


@pytest.mark.parametrize("m", [7, 333])
def test_repeated_calls_give_the_same_bits(m):
    g = gen(11)
    x, w = randn(g, m, 520), randn(g, 520, 264)
    ys = []
    for _ in range(3):
        y = torch.empty(m, 264, device="cuda", dtype=torch.bfloat16)
        mb.morello_linear(ACTS["silu"], 0, 0, 0, m, 520, 264, x, w, None, None, y)
        ys.append(y)
    assert torch.equal(ys[0], ys[1]) and torch.equal(ys[0], ys[2])


@pytest.mark.parametrize("m,k,n,gated", [(6, 100, 60, True), (90, 100, 60, True), (90, 104, 64, False)])
def test_own_stream_and_workspace(m, k, n, gated):
    g = gen(3)
    wide = 2 * n if gated else n
    need = mb.morello_linear_workspace_bytes(gated, 0, m, k, n)
    ws = torch.empty(max(need, 16), device="cuda", dtype=torch.uint8)
    guard = torch.full((64,), 77, device="cuda", dtype=torch.uint8)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        x, w = randn(g, m, k), randn(g, k, wide, scale=0.1)
        y = torch.empty(m, n, device="cuda", dtype=torch.bfloat16)
        mb.morello_linear(ACTS["gelu"], gated, 0, 0, m, k, n, x, w, None, None, y, None, ws, need, s)
    s.synchronize()
    want, bound, _, _ = forward64(x.double(), w.double(), None, None, "gelu", gated)
    assert_close(y, want, bound)
    assert bool((guard == 77).all())
    if need:
        with pytest.raises(mb.MorelloError) as e:
            mb.morello_linear(0, gated, 0, 0, m, k, n, x, w, None, None, y, None, ws, need - 1)
        assert e.value.status == mb.MORELLO_ERR_WORKSPACE


def test_captured_in_a_graph():
    g = gen(8)
    m, k, n = 96, 256, 128
    x, w = randn(g, m, k), randn(g, k, n, scale=0.06)
    y = torch.zeros(m, n, device="cuda", dtype=torch.bfloat16)
    mb.morello_linear(ACTS["silu"], 0, 0, 0, m, k, n, x, w, None, None, y)
    torch.cuda.synchronize()
    first = y.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mb.morello_linear(ACTS["silu"], 0, 0, 0, m, k, n, x, w, None, None, y)
    x.mul_(2)
    y.zero_()
    graph.replay()
    torch.cuda.synchronize()
    want, bound, _, _ = forward64(x.double(), w.double(), None, None, "silu", False)
    assert_close(y, want, bound)
    assert not torch.equal(y, first)


# --- gradients ---------------------------------------------------------------------------------------

def run_backward(m, k, n, act="gelu", gated=False, colmajor=False, bias=True, grad_f32=False, accumulate=False, seed=0,
                 shift=False, want_dx=True, want_dw=True):
    g = gen(seed + 5 * m + 3 * k + n)
    wide = 2 * n if gated else n
    x, dy, z = randn(g, m, k), randn(g, m, n), randn(g, m, wide)
    w, w64 = weights(g, k, wide, colmajor)
    kind = torch.float32 if grad_f32 else torch.bfloat16
    dx = torch.full((m, k), float("nan"), device="cuda", dtype=torch.bfloat16) if want_dx else None
    dw = torch.full(w.shape, 0.25 if accumulate else float("nan"), device="cuda", dtype=kind) if want_dw else None
    db = torch.full((wide,), 0.5 if accumulate else float("nan"), device="cuda") if bias else None
    if shift:
        x, dy, z, w = (misaligned(v) for v in (x, dy, z, w))
        dx, dw = misaligned(dx), misaligned(dw)
    mb.morello_linear_backward(ACTS[act], gated, grad_f32, accumulate, colmajor, m, k, n, x, w, z, dy, dx, dw, db)
    device_ok()
    dz, edz = dz64(z.double(), dy.double(), act, gated)
    # dz is rounded to bf16 for the products.
    rounded = 0 if act == "none" and not gated else BF16
    eprod = edz + rounded * (dz.abs() + edz)
    if want_dx:
        want = dz @ w64.t()
        assert_close(dx, want, eprod @ w64.abs().t() + 1e-5 * (dz.abs() @ w64.abs().t()) + TINY, "dX")
    x64 = x.double()
    if want_dw:
        want = x64.t() @ dz
        bound = x64.abs().t() @ eprod + 1e-5 * (x64.abs().t() @ dz.abs()) + TINY
        if accumulate:
            want, bound = want + 0.25, bound + 1e-6
        assert_close(dw.t() if colmajor else dw, want, bound, "dW")
    if bias:
        want = dz.sum(0) + (0.5 if accumulate else 0.0)
        assert_close(db, want, edz.sum(0) + 1e-5 * dz.abs().sum(0) + TINY, "db")


@pytest.mark.parametrize("m,k,n", [(1, 64, 64), (5, 128, 72), (64, 256, 136), (65, 72, 200), (256, 512, 264), (1000, 136, 520),
                                   (333, 640, 256)])
@pytest.mark.parametrize("gated,colmajor", [(False, False), (False, True), (True, False), (True, True)])
def test_gradients(m, k, n, gated, colmajor):
    run_backward(m, k, n, "silu", gated, colmajor)


@pytest.mark.parametrize("m,k,n", [(1, 1, 1), (3, 7, 5), (66, 63, 65), (129, 100, 259), (200, 257, 100)])
@pytest.mark.parametrize("gated,colmajor", [(False, False), (False, True), (True, False), (True, True)])
def test_gradients_of_odd_sizes(m, k, n, gated, colmajor):
    run_backward(m, k, n, "gelu", gated, colmajor)


@pytest.mark.parametrize("act,gated", list(itertools.product(ACTS, [False, True])))
def test_gradients_of_activations(act, gated):
    run_backward(150, 136, 72, act, gated, grad_f32=True)


@pytest.mark.parametrize("act,gated,colmajor", [("none", False, False), ("none", False, True), ("silu", True, False)])
def test_accumulated_gradients(act, gated, colmajor):
    run_backward(130, 72, 136, act, gated, colmajor, grad_f32=True, accumulate=True)


@pytest.mark.parametrize("want_dx,want_dw,bias", [(True, False, False), (False, True, False), (False, False, True)])
@pytest.mark.parametrize("act", ["none", "gelu"])
def test_only_some_gradients(want_dx, want_dw, bias, act):
    run_backward(100, 72, 136, act, bias=bias, want_dx=want_dx, want_dw=want_dw)


@pytest.mark.parametrize("gated,colmajor", [(False, True), (True, False)])
def test_gradients_of_misaligned_tensors(gated, colmajor):
    run_backward(140, 72, 136, "silu", gated, colmajor, shift=True)


@pytest.mark.parametrize("m,k,n", [(0, 8, 16), (4, 8, 0), (4, 0, 16)])
def test_gradients_of_empty_sums(m, k, n):
    x = torch.ones(4, 16, device="cuda", dtype=torch.bfloat16)
    dx, dw = (torch.full((64, 64), 3.0, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    db = torch.full((64,), 3.0, device="cuda")
    mb.morello_linear_backward(0, 0, 0, 0, 0, m, k, n, x, x, None, x, dx, dw, db)
    torch.cuda.synchronize()
    assert bool((dx.view(-1)[:m * k] == 0).all()) and bool((dx.view(-1)[m * k:] == 3).all())
    assert bool((dw.view(-1)[:k * n] == 0).all()) and bool((dw.view(-1)[k * n:] == 3).all())
    if m == 0:
        assert bool((db[:n] == 0).all())
    else:
        assert bool((db[:n] == m).all())
    assert bool((db[n:] == 3).all())


@pytest.mark.parametrize("act,gated", [("gelu", False), ("silu", True), ("gelu_tanh", False)])
def test_gradient_against_differences(act, gated):
    """Directional derivatives of the library's own forward pass (f32 output, central differences)."""
    m, k, n = 24, 64, 40
    g = gen(21)
    wide = 2 * n if gated else n
    x, w, b = randn(g, m, k), randn(g, k, wide, scale=0.125), randn(g, wide, scale=0.3)
    dy = randn(g, m, n)
    z = torch.empty(m, wide, device="cuda", dtype=torch.bfloat16)
    y = torch.empty(m, n, device="cuda", dtype=torch.float32)

    def value(x, w, b):
        mb.morello_linear(ACTS[act], gated, 1, 0, m, k, n, x, w, b, None, y)
        return (y.double() * dy.double()).sum()

    mb.morello_linear(ACTS[act], gated, 1, 0, m, k, n, x, w, b, None, y, z)
    dx = torch.empty_like(x)
    dw = torch.empty(k, wide, device="cuda", dtype=torch.float32)
    db = torch.empty(wide, device="cuda", dtype=torch.float32)
    mb.morello_linear_backward(ACTS[act], gated, 1, 0, 0, m, k, n, x, w, z, dy, dx, dw, db)
    # Steps that are exact in bf16: a change of +-2^-3 in a few places, whose differences have an error of
    # the third derivative, at most 2^-6 / 6 * |f'''| of the sum of the places' terms; 3 % holds it and the
    # bf16 roundings of z and dz.
    for which, at in [("x", (3, 5)), ("w", (7, 9)), ("b", (11,))]:
        step = 0.125
        moved = []
        for sign in (1, -1):
            t = {"x": x.clone(), "w": w.clone(), "b": b.clone()}
            t[which][at] = 0.0
            base = float({"x": x, "w": w, "b": b}[which][at])
            t[which][at] = base + sign * step
            moved.append((float(t[which][at]), float(value(**t))))
        diff = (moved[0][1] - moved[1][1]) / (moved[0][0] - moved[1][0])
        grad = float({"x": dx, "w": dw, "b": db}[which][at])
        assert abs(diff - grad) <= 0.03 * abs(diff) + 0.1, (which, diff, grad)
