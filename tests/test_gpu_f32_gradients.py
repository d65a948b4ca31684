"""f32 weight gradients over more rows than one run of sums takes, with the input gradient in the same call: the launch is
summed in parts, and both outputs are held to the bounds of the shorter ones."""
import pytest

import test_gpu_experts
import test_gpu_linear

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,k,n", [(1025, 64, 72), (1100, 264, 136), (2048, 136, 264), (4096, 72, 64), (1500, 1024, 520)])
@pytest.mark.parametrize("colmajor", [False, True])
@pytest.mark.parametrize("act,gated,accumulate", [("none", False, False), ("none", False, True), ("gelu", False, False),
                                                  ("silu", True, True)])
def test_dense(m, k, n, colmajor, act, gated, accumulate):
    test_gpu_linear.run_backward(m, k, n, act, gated, colmajor, grad_f32=True, accumulate=accumulate)


@pytest.mark.parametrize("m,k,n,shift", [(1100, 100, 72, False), (1100, 72, 100, False), (1300, 72, 136, True)])
def test_dense_that_the_tma_engine_cannot_address(m, k, n, shift):
    test_gpu_linear.run_backward(m, k, n, "silu", False, False, grad_f32=True, shift=shift)


@pytest.mark.parametrize("want_dx,want_dw,bias", [(True, True, False), (False, True, True), (True, False, True)])
def test_dense_some(want_dx, want_dw, bias):
    test_gpu_linear.run_backward(1100, 136, 72, "gelu", grad_f32=True, bias=bias, want_dx=want_dx, want_dw=want_dw)


@pytest.mark.parametrize("t,topk,e,k,n", [(300, 2, 6, 72, 136), (700, 2, 4, 136, 72), (100, 2, 16, 64, 264), (2100, 1, 2, 264, 64)])
@pytest.mark.parametrize("colmajor", [False, True])
@pytest.mark.parametrize("act,gated,gather", [("none", False, False), ("silu", True, False), ("silu", True, True)])
def test_experts(t, topk, e, k, n, colmajor, act, gated, gather):
    test_gpu_experts.run_backward(t, topk, e, k, n, gated, colmajor, gather, "spread", act, True)
