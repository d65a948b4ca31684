"""Refusals and size functions of the feed-forward entry points: none of them needs a device."""
import pytest

P = 4096      # an aligned stand-in address: every call below is refused before it is looked at


@pytest.fixture(scope="module")
def mb():
    from paper_2505_01637_b200 import build
    build.build()
    from paper_2505_01637_b200 import binding
    binding.lib()
    return binding


def refused(mb, status, fn, *args):
    with pytest.raises(mb.MorelloError) as e:
        getattr(mb, fn)(*args, stream=0)
    assert e.value.status == status, e.value


def test_linear_refusals(mb):
    arg, shape, null, off = (mb.MORELLO_ERR_INVALID_ARGUMENT, mb.MORELLO_ERR_INVALID_SHAPE, mb.MORELLO_ERR_NULL_POINTER,
                             mb.MORELLO_ERR_MISALIGNED)

    def fw(status, act=0, gated=0, y_type=0, layout=0, m=2, k=8, n=8, X=P, W=P, b=None, R=None, Y=P, Z=None, ws=None, wsb=0):
        refused(mb, status, "morello_linear", act, gated, y_type, layout, m, k, n, X, W, b, R, Y, Z, ws, wsb)

    fw(arg, act=5)
    fw(arg, act=-1)
    fw(arg, gated=2)
    fw(arg, y_type=2)
    fw(arg, layout=7)
    fw(shape, m=-1)
    fw(shape, n=1 << 31)
    fw(shape, n=(1 << 30) + 1, gated=1)
    fw(shape, m=1 << 30, k=1 << 30, n=1 << 30)
    fw(null, X=None)
    fw(null, W=None)
    fw(null, Y=None)
    fw(off, X=P + 1)
    fw(off, b=P + 1)
    fw(off, R=P + 1)
    fw(off, Z=P + 1)
    fw(off, Y=P + 2, y_type=1)
    fw(off, ws=P + 8, wsb=64)

    def bw(status, act=0, gated=0, kind=0, acc=0, layout=0, m=2, k=8, n=8, X=P, W=P, Z=P, dY=P, dX=P, dW=P, db=P):
        refused(mb, status, "morello_linear_backward", act, gated, kind, acc, layout, m, k, n, X, W, Z, dY, dX, dW, db)

    bw(arg, acc=1)                 # bf16 gradients do not accumulate
    bw(arg, acc=2, kind=1)
    bw(arg, kind=3)
    bw(arg, act=9)
    bw(shape, k=-4)
    bw(null, Z=None, act=2)
    bw(null, Z=None, gated=1)
    bw(null, dY=None)
    bw(null, W=None)
    bw(null, X=None)
    bw(off, dW=P + 2, kind=1)
    bw(off, db=P + 2)


def test_route_and_plan_refusals(mb):
    arg, shape, null, off = (mb.MORELLO_ERR_INVALID_ARGUMENT, mb.MORELLO_ERR_INVALID_SHAPE, mb.MORELLO_ERR_NULL_POINTER,
                             mb.MORELLO_ERR_MISALIGNED)

    def route(status, score=0, renorm=0, kind=1, t=4, e=16, k=2, g=1, tg=1, x=P, b=None, idx=P, w=P):
        refused(mb, status, "morello_route", score, renorm, 1.0, kind, t, e, k, g, tg, x, b, idx, w)

    route(arg, score=2)
    route(arg, renorm=-1)
    route(arg, kind=2)
    route(shape, t=-1)
    route(shape, e=0)
    route(shape, e=1025)
    route(shape, k=0)
    route(shape, k=33, e=64)
    route(shape, k=17)                   # more than the experts
    route(shape, g=3)                    # does not divide the experts
    route(shape, g=4, tg=5)
    route(shape, g=4, tg=1, k=5)         # more than the groups that stay hold
    route(shape, g=0)
    route(shape, g=64, e=128, tg=2)
    route(null, x=None)
    route(null, idx=None)
    route(null, w=None)
    route(off, x=P + 2)
    route(off, b=P + 2)
    refused(mb, shape, "morello_route_backward", 0, 0, 1.0, 1, 4, 8, 9, P, P, P, P)
    refused(mb, null, "morello_route_backward", 0, 0, 1.0, 1, 4, 8, 2, P, P, P, None)
    refused(mb, shape, "morello_expert_plan", -1, 2, 4, P, P)
    refused(mb, shape, "morello_expert_plan", 1 << 30, 2, 4, P, P)
    refused(mb, null, "morello_expert_plan", 4, 2, 4, None, P)
    refused(mb, null, "morello_expert_plan", 4, 2, 4, P, None)
    refused(mb, off, "morello_expert_plan", 4, 2, 4, P, P + 2)


def test_expert_refusals(mb):
    arg, shape, null = mb.MORELLO_ERR_INVALID_ARGUMENT, mb.MORELLO_ERR_INVALID_SHAPE, mb.MORELLO_ERR_NULL_POINTER

    def fw(status, act=0, gated=0, y_type=0, layout=0, gather=0, t=4, kk=2, e=4, k=8, n=8, plan=P, X=P, W=P, Y=P):
        refused(mb, status, "morello_expert_linear", act, gated, y_type, layout, gather, t, kk, e, k, n, plan, X, W, None, Y)

    fw(arg, act=6)
    fw(arg, gather=2)
    fw(arg, layout=2)
    fw(shape, t=-2)
    fw(shape, kk=33)
    fw(shape, e=2000)
    fw(shape, k=-1)
    fw(shape, t=1 << 26, k=1 << 30, n=1 << 30)
    fw(null, plan=None)
    fw(null, X=None)
    fw(null, Y=None)
    refused(mb, arg, "morello_expert_linear_backward", 0, 0, 0, 1, 0, 0, 4, 2, 4, 8, 8, P, P, P, P, P, P, P, P)
    refused(mb, null, "morello_expert_linear_backward", 4, 0, 0, 0, 0, 0, 4, 2, 4, 8, 8, P, P, P, None, P, P, P, P)
    refused(mb, arg, "morello_expert_combine", 2, 4, 2, 4, 8, P, P, P, P, P)
    refused(mb, null, "morello_expert_combine", 0, 4, 2, 4, 8, P, P, None, P, P)
    refused(mb, null, "morello_expert_combine_backward", 0, 4, 2, 4, 8, P, P, None, P, P, P)


def test_sizes(mb):
    rows, words = mb.morello_expert_plan_rows, mb.morello_expert_plan_words
    assert rows(0, 4, 8) == 0 and rows(1, 1, 8) == 128 and rows(4, 4, 64) == 2048
    assert rows(4096, 4, 32) == (4096 * 4 + 127 * 32) // 128 * 128
    assert rows(100, 1, 1) == 128 and rows(129, 1, 1) == 256
    assert words(4, 4, 64) == 2048 + 16 + 65 + 64 + 16 + 64
    assert rows(-1, 1, 1) == words(1, 0, 1) == rows(1, 1, 5000) == -1
    # no copy where the tensor cores' loads can address the tensors
    assert mb.morello_linear_workspace_bytes(0, 0, 100, 64, 64) == 0
    assert mb.morello_linear_workspace_bytes(1, 1, 100, 64, 63) == 0         # column-major: n is not a row length
    assert mb.morello_linear_workspace_bytes(0, 0, 2, 63, 64) == 256          # X alone: its rows, 64 long
    assert mb.morello_linear_workspace_bytes(0, 0, 2, 64, 63) == 64 * 64 * 2  # W alone
    assert mb.morello_linear_workspace_bytes(1, 0, 2, 64, 63) == 64 * 128 * 2
    assert mb.morello_linear_workspace_bytes(0, 0, 2, -1, 64) == 0
    assert mb.morello_linear_backward_workspace_bytes(4, 0, 0, 100, 64, 64) >= 100 * 64 * 2
    assert mb.morello_expert_linear_workspace_bytes(0, 0, 0, 16, 2, 4, 64, 64) == 0
