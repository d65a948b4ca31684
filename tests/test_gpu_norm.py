"""Layer norm, forward and backward, against its 64-bit definition."""
import pytest
import torch

from norm_util import check_backward, check_forward, forward, gen, misaligned, norm64

pytestmark = pytest.mark.gpu
mb = pytest.importorskip("paper_2505_01637_b200.binding")

BF, F32 = torch.bfloat16, torch.float32
# every team size, whole and ragged rows, rows past the registers, odd lengths
SHAPES = [(1, 1), (1, 2), (3, 7), (17, 64), (9, 256), (70, 264), (5, 512), (33, 1024), (2, 1025), (7, 1032), (300, 2048),
          (1, 2048), (333, 2047), (40, 4096), (2, 4097), (3, 4104), (5, 8192), (2, 8191), (2, 8200), (3, 16384), (2, 16383),
          (2, 16392), (3, 20001), (1500, 128)]


def make(m, n, kind, seed, mean=0.3):
    g = gen(seed)
    x = (torch.randn(m, n, generator=g, device="cuda") * 1.7 + mean).to(kind)
    gamma = (1 + 0.3 * torch.randn(n, generator=g, device="cuda")).to(BF)
    beta = (0.3 * torch.randn(n, generator=g, device="cuda")).to(BF)
    dy = torch.randn(m, n, generator=g, device="cuda").to(BF)
    r = torch.randn(m, n, generator=g, device="cuda").to(kind)
    return x, gamma, beta, dy, r


@pytest.mark.parametrize("kind", [BF, F32])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("m,n", SHAPES)
def test_forward(m, n, rms, kind):
    x, gamma, beta, _, _ = make(m, n, kind, m + n)
    y, mean, rstd = forward(x, gamma, beta, 1e-5, rms)
    check_forward(x, gamma, beta, 1e-5, rms, y, mean, rstd)
    again, _, _ = forward(x, gamma, beta, 1e-5, rms, keep=False)
    assert torch.equal(y, again)
    y, _, _ = forward(x, None, None, 1e-6, rms)
    check_forward(x, None, None, 1e-6, rms, y, None, None)


@pytest.mark.parametrize("kind", [BF, F32])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("m,n", SHAPES)
def test_backward(m, n, rms, kind):
    x, gamma, _, dy, r = make(m, n, kind, m * 3 + n)
    mean64, rstd64, _, _ = norm64(x, None, None, 1e-5, rms)
    mean, rstd = (None if rms else mean64[:, 0].float()), rstd64[:, 0].float()
    code = int(kind == F32)
    dx = torch.full_like(x, float("nan"))
    dgamma, dbeta = torch.full((n,), float("nan"), device="cuda"), torch.full((n,), float("nan"), device="cuda")
    mb.morello_layer_norm_backward(int(rms), code, 0, m, n, x, gamma, mean, rstd, dy, r, dx, dgamma, dbeta)
    check_backward(x, gamma, mean, rstd, dy, r, rms, dx, dgamma, dbeta)
    # one at a time: the same bits
    only = torch.full_like(x, float("nan"))
    mb.morello_layer_norm_backward(int(rms), code, 0, m, n, x, gamma, mean, rstd, dy, r, only, None, None)
    assert torch.equal(only, dx)
    for want in (0, 1):
        one = [None, None]
        one[want] = torch.full((n,), float("nan"), device="cuda")
        mb.morello_layer_norm_backward(int(rms), code, 0, m, n, x, gamma, mean, rstd, dy, None, None, one[0], one[1])
        assert torch.equal(one[want], (dgamma, dbeta)[want])
    # added to what is there; dX over R; no gamma
    base_g, base_b = dy[0].float().clone(), dy[-1].float().clone()
    got_g, got_b, over = base_g.clone(), base_b.clone(), r.clone()
    mb.morello_layer_norm_backward(int(rms), code, 1, m, n, x, None, mean, rstd, dy, over, over, got_g, got_b)
    check_backward(x, None, mean, rstd, dy, r, rms, over, got_g, got_b, base_g, base_b)


@pytest.mark.parametrize("kind", [BF, F32])
@pytest.mark.parametrize("m,n", [(20000, 64), (9001, 256), (5000, 520), (2503, 1024), (1701, 2048), (1303, 4096), (799, 8192),
                                 (601, 16384), (700, 12008), (4000, 2056), (20000, 7), (5000, 333), (4001, 2047), (799, 8191),
                                 (600, 12001), (3000, 1)])
def test_batches(m, n, kind):
    # many rows to a block, the last ones a part of a group
    for rms in (False, True):
        test_forward(m, n, rms, kind)
        test_backward(m, n, rms, kind)


@pytest.mark.parametrize("n", [8, 9, 16, 57, 63, 64, 65, 72, 120, 121, 127, 128, 129, 136])
def test_short_rows(n):
    # the heads' rows: several to a warp, groups that end inside one
    for m in (1, 3, 65, 9473):
        for rms in (False, True):
            test_forward(m, n, rms, BF)
            test_backward(m, n, rms, BF)


@pytest.mark.parametrize("kind", [BF, F32])
@pytest.mark.parametrize("m,n", [(5, 256), (5, 2048), (5, 8192), (5, 16384), (5, 3), (17, 1), (40, 1), (100, 5), (1500, 7), (2000, 264),
                                 (700, 2048)])
def test_unaligned_tensors(m, n, kind):
    x, gamma, beta, dy, r = (misaligned(t) for t in make(m, n, kind, n))
    y = misaligned(torch.zeros(m, n, device="cuda", dtype=BF))
    mb.morello_layer_norm(0, int(kind == F32), m, n, 1e-5, x, gamma, beta, y)
    check_forward(x, gamma, beta, 1e-5, False, y, None, None)
    mean, rstd, _, _ = norm64(x, None, None, 1e-5, False)
    mean, rstd = mean[:, 0].float(), rstd[:, 0].float()
    dx, dg = misaligned(torch.zeros_like(x)), misaligned(torch.zeros(n, device="cuda"))
    mb.morello_layer_norm_backward(0, int(kind == F32), 0, m, n, x, gamma, mean, rstd, dy, r, dx, dg, None)
    check_backward(x, gamma, mean, rstd, dy, r, False, dx, dg, None)


def test_in_place_and_neighbours_untouched():
    x, gamma, beta, _, _ = make(37, 520, BF, 5)
    guarded = torch.full((39, 520), 7.0, device="cuda", dtype=BF)
    guarded[1:38] = x
    mb.morello_layer_norm(0, 0, 37, 520, 1e-5, guarded[1:38], gamma, beta, guarded[1:38])
    check_forward(x, gamma, beta, 1e-5, False, guarded[1:38], None, None)
    assert torch.all(guarded[0] == 7) and torch.all(guarded[38] == 7)


@pytest.mark.parametrize("n", [96, 2048, 2047, 8192, 16384, 20000])
def test_mean_far_from_zero(n):
    # Differences of about 1 around 30000: the mean alone is off by 2^-10 in f32.
    x, gamma, beta, _, _ = make(4, n, F32, n, mean=30000.0)
    y, mean, rstd = forward(x, gamma, beta, 1e-5, False)
    check_forward(x, gamma, beta, 1e-5, False, y, mean, rstd)


@pytest.mark.parametrize("n", [64, 2047, 4096, 20000])
def test_rows_of_one_value_and_extremes(n):
    x = torch.randn(6, n, generator=gen(n), device="cuda")
    x[0] = 0.0
    x[1] = 3.0
    x[2] = 1e-20                # squares below the smallest number: eps decides
    x[3, 0] = float("nan")
    x[4, n - 1] = float("inf")
    gamma, beta = torch.ones(n, device="cuda", dtype=BF), torch.full((n,), 0.5, device="cuda", dtype=BF)
    y, mean, rstd = forward(x, gamma, beta, 1e-5, False)
    assert torch.all(y[0] == 0.5) and torch.all((y[1:3].double() - 0.5).abs() <= 2.0 ** -8)
    assert torch.isnan(y[3:5]).all() and torch.isnan(rstd[3:5]).all()
    check_forward(x[5:], gamma, beta, 1e-5, False, y[5:], mean[5:], rstd[5:])


def test_gradient_agrees_with_differences():
    m, n = 6, 40
    x, gamma, beta, dy, _ = make(m, n, F32, 11)
    for rms in (False, True):
        mean, rstd, _, _ = norm64(x, None, None, 1e-5, rms)
        mean, rstd = mean[:, 0].float(), rstd[:, 0].float()
        dx = torch.empty_like(x)
        dg, db = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        mb.morello_layer_norm_backward(int(rms), 1, 0, m, n, x, gamma, None if rms else mean, rstd, dy, None, dx, dg, db)

        def loss(x, gamma, beta):
            return float((norm64(x, gamma, beta, 1e-5, rms)[3] * dy.double()).sum())

        g = gen(3)
        for what, grad, base in ((0, dx, x), (1, dg, gamma), (2, db, beta)):
            way = torch.randn(base.shape, generator=g, device="cuda", dtype=torch.float64)
            step = 1e-5
            at = [t.double() for t in (x, gamma, beta)]
            up, down = list(at), list(at)
            up[what], down[what] = at[what] + step * way, at[what] - step * way
            slope = (loss(*up) - loss(*down)) / (2 * step)
            # central differences: third derivatives times step^2 and 2^-52 / step, both below 1e-8 of the terms
            size = float((grad.double() * way).abs().sum())
            assert abs(slope - float((grad.double() * way).sum())) <= 1e-5 * size


@pytest.mark.parametrize("m", [0, 1])
def test_empty(m):
    n = 24
    x = torch.zeros(m, n, device="cuda", dtype=BF)
    dg = torch.full((n,), 5.0, device="cuda")
    db = dg.clone()
    if m == 0:
        mb.morello_layer_norm(0, 0, 0, n, 1e-5, x, None, None, x)
        mb.morello_layer_norm_backward(0, 0, 1, 0, n, None, None, None, None, None, None, None, dg, db)
        assert torch.all(dg == 5) and torch.all(db == 5)
        mb.morello_layer_norm_backward(0, 0, 0, 0, n, None, None, None, None, None, None, None, dg, db)
        assert torch.all(dg == 0) and torch.all(db == 0)
    else:
        mb.morello_layer_norm(0, 0, 1, 0, 1e-5, None, None, None, None)
        mb.morello_layer_norm_backward(0, 0, 0, 1, 0, None, None, None, None, None, None, None, None, None)


def test_workspace_stream_and_graph():
    m, n = 515, 1160
    x, gamma, beta, dy, r = make(m, n, BF, 2)
    mean, rstd, _, _ = norm64(x, None, None, 1e-5, False)
    mean, rstd = mean[:, 0].float(), rstd[:, 0].float()
    need = mb.morello_layer_norm_backward_workspace_bytes(m, n)
    ws = torch.full((need + 64,), 0xAB, device="cuda", dtype=torch.uint8)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    dg, db = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")

    def both(stream=None):
        mb.morello_layer_norm(0, 0, m, n, 1e-5, x, gamma, beta, y, stream=stream)
        mb.morello_layer_norm_backward(0, 0, 0, m, n, x, gamma, mean, rstd, dy, r, dx, dg, db, ws, need, stream=stream)

    def check():
        check_forward(x, gamma, beta, 1e-5, False, y, None, None)
        check_backward(x, gamma, mean, rstd, dy, r, False, dx, dg, db)
        assert torch.all(ws[need:] == 0xAB)

    with pytest.raises(mb.MorelloError) as e:
        mb.morello_layer_norm_backward(0, 0, 0, m, n, x, gamma, mean, rstd, dy, r, dx, dg, db, ws, need - 1)
    assert e.value.status == mb.MORELLO_ERR_WORKSPACE
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    both(side)
    side.synchronize()
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for seed in (21, 22):
        fresh = make(m, n, BF, seed)
        for old, new in zip((x, gamma, beta, dy, r), fresh):
            old.copy_(new)
        m64, r64, _, _ = norm64(x, None, None, 1e-5, False)
        mean.copy_(m64[:, 0])
        rstd.copy_(r64[:, 0])
        graph.replay()
        torch.cuda.synchronize()
        check()


@pytest.mark.parametrize("n", [16384, 16383])
def test_elements_past_two_to_the_31(n):
    m = 140000
    g = gen(n)
    x = torch.empty(m, n, device="cuda", dtype=BF).normal_(generator=g)
    gamma = (1 + 0.3 * torch.randn(n, generator=g, device="cuda")).to(BF)
    y, mean, rstd = forward(x, gamma, None, 1e-5, False)
    for at in (slice(0, 3), slice(m - 3, m)):
        check_forward(x[at], gamma, None, 1e-5, False, y[at], mean[at], rstd[at])
    dy = y.normal_(generator=g)
    dx = torch.full_like(x, float("nan"))
    mb.morello_layer_norm_backward(0, 0, 0, m, n, x, gamma, mean, rstd, dy, None, dx, None, None)
    for at in (slice(0, 3), slice(m - 3, m)):
        check_backward(x[at], gamma, mean[at], rstd[at], dy[at], None, False, dx[at], None, None)


@pytest.mark.parametrize("kind", [BF, F32])
@pytest.mark.parametrize("m,n", [(300, 20001), (1, 20000), (129, 16392), (300, 16384), (700, 64), (77, 63), (9, 8191), (1100, 16383), (149, 4096)])
def test_workspace_of_the_reported_size(m, n, kind):
    x, gamma, _, dy, r = make(m, n, kind, m)
    mean, rstd, _, _ = norm64(x, None, None, 1e-5, False)
    mean, rstd = mean[:, 0].float(), rstd[:, 0].float()
    need = mb.morello_layer_norm_backward_workspace_bytes(m, n)
    ws = torch.full((need + 64,), 0xAB, device="cuda", dtype=torch.uint8)
    dx = torch.full_like(x, float("nan"))
    dg, db = torch.full((n,), float("nan"), device="cuda"), torch.full((n,), float("nan"), device="cuda")
    for move in (lambda t: t, misaligned):
        mb.morello_layer_norm_backward(0, int(kind == F32), 0, m, n, move(x), gamma, mean, rstd, move(dy), r, dx, dg, db, ws, need)
        check_backward(x, gamma, mean, rstd, dy, r, False, dx, dg, db)
        assert torch.all(ws[need:] == 0xAB)
