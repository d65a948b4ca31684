"""Refusals and size functions of the 4-bit entry points: none of them needs a device."""
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


def statuses(mb):
    return mb.MORELLO_ERR_INVALID_ARGUMENT, mb.MORELLO_ERR_INVALID_SHAPE, mb.MORELLO_ERR_NULL_POINTER, mb.MORELLO_ERR_MISALIGNED


def test_quantize_refusals(mb):
    arg, shape, null, off = statuses(mb)

    def call(status, fmt=0, kind=0, layout=1, rows=4, parts=1, k=32, X=P, mult=P, Q=P, S=P):
        refused(mb, status, "morello_fp4_quantize", fmt, kind, layout, rows, parts, k, X, mult, Q, S)

    call(arg, fmt=2)
    call(arg, fmt=-1)
    call(arg, kind=2)
    call(arg, layout=2)
    call(shape, rows=-1)
    call(shape, k=-1)
    call(shape, parts=0)
    call(shape, rows=5, parts=2)
    call(shape, rows=1 << 31)
    call(null, X=None)
    call(null, Q=None)
    call(null, S=None)
    call(off, X=P + 1)
    call(off, X=P + 2, kind=1)
    call(off, mult=P + 2)
    call(off, Q=P + 8)
    call(off, S=P + 8)

    def back(status, fmt=0, kind=0, rows=4, parts=1, k=32, Q=P, S=P, alpha=P, Y=P):
        refused(mb, status, "morello_fp4_dequantize", fmt, kind, rows, parts, k, Q, S, alpha, Y)

    back(arg, fmt=2)
    back(arg, kind=-1)
    back(shape, rows=3, parts=2)
    back(null, Q=None)
    back(null, S=None)
    back(null, Y=None)
    back(off, Q=P + 4)
    back(off, S=P + 4)
    back(off, alpha=P + 1)
    back(off, Y=P + 1)
    back(off, Y=P + 2, kind=1)


def test_linear_refusals(mb):
    arg, shape, null, off = statuses(mb)

    def call(status, fmt=0, act=0, gated=0, y_type=0, m=2, k=32, n=8, X=P, Xs=P, W=P, Ws=P, alpha=P, b=P, R=P, Y=P):
        refused(mb, status, "morello_fp4_linear", fmt, act, gated, y_type, m, k, n, X, Xs, W, Ws, alpha, b, R, Y)

    call(arg, fmt=2)
    call(arg, act=5)
    call(arg, act=-1)
    call(arg, gated=2)
    call(arg, y_type=2)
    call(shape, m=-1)
    call(shape, k=-1)
    call(shape, n=1 << 31)
    call(shape, n=1 << 30, gated=1)
    for name in ("X", "Xs", "W", "Ws", "Y"):
        call(null, **{name: None})
    for name in ("X", "Xs", "W", "Ws"):
        call(off, **{name: P + 8})
    call(off, alpha=P + 2)
    call(off, b=P + 1)
    call(off, R=P + 1)
    call(off, Y=P + 1)
    call(off, Y=P + 2, y_type=1)


def test_sizes(mb):
    assert mb.morello_fp4_bytes(3, 1) == 3 * 16 and mb.morello_fp4_bytes(3, 33) == 3 * 32 and mb.morello_fp4_bytes(0, 64) == 0
    assert mb.morello_fp4_bytes(-1, 8) == -1 and mb.morello_fp4_bytes(8, -1) == -1
    size = mb.morello_fp4_scale_bytes
    assert size(mb.MORELLO_MXFP4, 1, 1, 1) == 512 and size(mb.MORELLO_MXFP4, 129, 1, 129) == 4 * 512
    assert size(mb.MORELLO_NVFP4, 128, 1, 64) == 512 and size(mb.MORELLO_NVFP4, 128, 1, 65) == 1024
    assert size(mb.MORELLO_NVFP4, 256, 2, 64) == 1024 and size(mb.MORELLO_NVFP4, 130, 2, 64) == 1024
    assert size(mb.MORELLO_NVFP4, 129, 2, 64) == -1 and size(2, 128, 1, 64) == -1 and size(0, 8, 0, 64) == -1
