"""Refusals and size functions of the norms' entry points: none of them needs a device."""
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


def test_forward_refusals(mb):
    arg, shape, null, off = (mb.MORELLO_ERR_INVALID_ARGUMENT, mb.MORELLO_ERR_INVALID_SHAPE, mb.MORELLO_ERR_NULL_POINTER,
                             mb.MORELLO_ERR_MISALIGNED)

    def fw(status, rms=0, kind=0, m=2, n=8, eps=1e-5, X=P, g=P, b=P, Y=P, mean=P, rstd=P):
        refused(mb, status, "morello_layer_norm", rms, kind, m, n, eps, X, g, b, Y, mean, rstd)

    fw(arg, rms=2)
    fw(arg, kind=-1)
    fw(arg, kind=2)
    fw(arg, eps=-1e-9)
    fw(arg, eps=float("nan"))
    fw(shape, m=-1)
    fw(shape, n=1 << 31)
    fw(null, X=None)
    fw(null, Y=None)
    fw(off, X=P + 1)
    fw(off, X=P + 2, kind=1)
    fw(off, g=P + 1)
    fw(off, b=P + 1)
    fw(off, Y=P + 1)
    fw(off, mean=P + 2)
    fw(off, rstd=P + 2)


def test_backward_refusals(mb):
    arg, shape, null, off = (mb.MORELLO_ERR_INVALID_ARGUMENT, mb.MORELLO_ERR_INVALID_SHAPE, mb.MORELLO_ERR_NULL_POINTER,
                             mb.MORELLO_ERR_MISALIGNED)

    def bw(status, rms=0, kind=0, acc=0, m=2, n=8, X=P, g=P, mean=P, rstd=P, dY=P, R=P, dX=P, dg=P, db=P, ws=None, wsb=0):
        refused(mb, status, "morello_layer_norm_backward", rms, kind, acc, m, n, X, g, mean, rstd, dY, R, dX, dg, db, ws, wsb)

    bw(arg, rms=-1)
    bw(arg, kind=3)
    bw(arg, acc=2)
    bw(shape, m=-5)
    bw(shape, n=-5)
    bw(null, X=None)
    bw(null, mean=None)
    bw(null, rstd=None)
    bw(null, rstd=None, rms=1)
    bw(null, dY=None)
    bw(off, dX=P + 1)
    bw(off, R=P + 2, kind=1)
    bw(off, dg=P + 1)
    bw(off, db=P + 2)
    bw(off, ws=P + 8, wsb=64)


def test_workspace_sizes(mb):
    size = mb.morello_layer_norm_backward_workspace_bytes
    assert size(0, 64) == 0 and size(64, 0) == 0 and size(-1, 8) == 0
    assert size(1, 64) == 2 * 64 * 4
    assert size(1 << 20, 4096) == 296 * 2 * 4096 * 4        # bounded by the blocks, not by the rows
