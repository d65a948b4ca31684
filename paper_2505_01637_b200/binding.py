"""Python binding of the C ABI (``include/morello.h``): argument marshalling only.

Every function has the name and argument order of its C counterpart.  Tensor
arguments may be torch CUDA tensors (their ``data_ptr()`` is passed) or plain
integer device addresses; ``stream`` may be a ``torch.cuda.Stream``, an integer
``cudaStream_t`` or None (torch's current stream when torch is loaded and CUDA is
up, else the default stream).  Status codes other than MORELLO_OK raise
``MorelloError``.  There is no fallback: if the shared library has not been
built, importing this module's functions raises."""
from __future__ import annotations

import ctypes
import os
import sys

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmorello.so")

MORELLO_OK = 0
MORELLO_ERR_INVALID_SHAPE = 1
MORELLO_ERR_NULL_POINTER = 2
MORELLO_ERR_MISALIGNED = 3
MORELLO_ERR_UNSUPPORTED_DEVICE = 4
MORELLO_ERR_WORKSPACE = 5
MORELLO_ERR_CUDA = 6
MORELLO_ERR_DEVICE_TIMEOUT = 7
MORELLO_ERR_UNSUPPORTED_PATH = 8
MORELLO_ERR_INVALID_ARGUMENT = 9

MORELLO_PATH_AUTO = -1
MORELLO_PATH_SKINNY = 0
MORELLO_PATH_TCGEN05 = 1

MORELLO_ACT_NONE, MORELLO_ACT_RELU, MORELLO_ACT_GELU, MORELLO_ACT_GELU_TANH, MORELLO_ACT_SILU = range(5)
MORELLO_BF16, MORELLO_F32 = 0, 1
MORELLO_W_ROWMAJOR, MORELLO_W_COLMAJOR = 0, 1
MORELLO_SCORE_SOFTMAX, MORELLO_SCORE_SIGMOID = 0, 1
MORELLO_MXFP4, MORELLO_NVFP4 = 0, 1

_i64, _vp, _int, _sz = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t

# name -> (restype, argtypes); mirrors include/morello.h declaration by declaration
SIGNATURES = {
    "morello_matmul_accum": (_int, [_i64, _i64, _i64, _i64, _vp, _vp, _vp, _vp]),
    "morello_matmul": (_int, [_i64, _i64, _i64, _i64, _vp, _vp, _vp, _vp]),
    "morello_matmul_forced": (_int, [_int, _int, _i64, _i64, _i64, _i64, _vp, _vp, _vp,
                                     _vp, _sz, _vp]),
    "morello_matmul_accum_f32": (_int, [_i64, _i64, _i64, _i64, _vp, _vp, _vp, _vp]),
    "morello_matmul_f32": (_int, [_i64, _i64, _i64, _i64, _vp, _vp, _vp, _vp]),
    "morello_matmul_accum_colmajor_b": (_int, [_int, _i64, _i64, _i64, _i64, _vp, _vp, _vp, _vp]),
    "morello_matmul_accum_packed_b": (_int, [_int, _i64, _i64, _i64, _i64, _vp, _vp, _vp, _vp]),
    "morello_selftest_wait_timeout": (_int, [ctypes.c_uint32, _vp]),
    "morello_matmul_colmajor_b": (_int, [_int, _i64, _i64, _i64, _i64, _vp, _vp, _vp, _vp]),
    "morello_matmul_packed_b": (_int, [_int, _i64, _i64, _i64, _i64, _vp, _vp, _vp, _vp]),
    "morello_workspace_bytes": (_sz, [_i64, _i64, _i64, _i64]),
    "morello_matmul_accum_ws": (_int, [_i64, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _sz, _vp]),
    "morello_matmul_accum_host": (_int, [_i64, _i64, _i64, _i64, _vp, _vp, _vp]),
    "morello_matmul_accum_noalloc": (_int, [_int, _i64, _i64, _i64, _i64, _vp, _vp, _vp, _vp]),
    "morello_noalloc_scratch_limit": (_sz, []),
    "morello_select_path": (_int, [_i64, _i64, _i64, _i64]),
    "morello_describe_route": (_int, [_i64, _i64, _i64, _i64, ctypes.c_char_p, _sz]),
    "morello_selftest_per_device_once": (_int, [_int, _int]),
    "morello_matmul_accum_forced": (_int, [_int, _int, _i64, _i64, _i64, _i64, _vp, _vp, _vp,
                                           _vp, _sz, _vp]),
    "morello_workspace_bytes_forced": (_sz, [_int, _int, _i64, _i64, _i64, _i64]),
    "morello_linear": (_int, [_int] * 4 + [_i64] * 3 + [_vp] * 7 + [_sz, _vp]),
    "morello_linear_workspace_bytes": (_sz, [_int] * 2 + [_i64] * 3),
    "morello_linear_backward": (_int, [_int] * 5 + [_i64] * 3 + [_vp] * 8 + [_sz, _vp]),
    "morello_linear_backward_workspace_bytes": (_sz, [_int] * 3 + [_i64] * 3),
    "morello_route": (_int, [_int, _int, ctypes.c_float, _int] + [_i64] * 5 + [_vp] * 5),
    "morello_route_backward": (_int, [_int, _int, ctypes.c_float, _int] + [_i64] * 3 + [_vp] * 5),
    "morello_expert_plan_rows": (_i64, [_i64] * 3),
    "morello_expert_plan_words": (_i64, [_i64] * 3),
    "morello_expert_plan": (_int, [_i64] * 3 + [_vp] * 3),
    "morello_expert_linear": (_int, [_int] * 5 + [_i64] * 5 + [_vp] * 7 + [_sz, _vp]),
    "morello_expert_linear_workspace_bytes": (_sz, [_int] * 3 + [_i64] * 5),
    "morello_expert_linear_backward": (_int, [_int] * 6 + [_i64] * 5 + [_vp] * 9 + [_sz, _vp]),
    "morello_expert_linear_backward_workspace_bytes": (_sz, [_int] * 4 + [_i64] * 5),
    "morello_expert_combine": (_int, [_int] + [_i64] * 4 + [_vp] * 6),
    "morello_expert_combine_backward": (_int, [_int] + [_i64] * 4 + [_vp] * 7),
    "morello_layer_norm": (_int, [_int] * 2 + [_i64] * 2 + [ctypes.c_float] + [_vp] * 7),
    "morello_layer_norm_backward": (_int, [_int] * 3 + [_i64] * 2 + [_vp] * 10 + [_sz, _vp]),
    "morello_layer_norm_backward_workspace_bytes": (_sz, [_i64] * 2),
    "morello_fp4_bytes": (_i64, [_i64] * 2),
    "morello_fp4_scale_bytes": (_i64, [_int] + [_i64] * 3),
    "morello_fp4_quantize": (_int, [_int] * 3 + [_i64] * 3 + [_vp] * 5),
    "morello_fp4_dequantize": (_int, [_int] * 2 + [_i64] * 3 + [_vp] * 5),
    "morello_fp4_linear": (_int, [_int] * 4 + [_i64] * 3 + [_vp] * 9),
    "morello_read_device_status": (_int, [_vp, ctypes.POINTER(ctypes.c_uint32)]),
    "morello_device_limits": (_int, [ctypes.POINTER(ctypes.c_int), ctypes.POINTER(ctypes.c_int)]),
    "morello_launch_count": (ctypes.c_uint64, []),
    "morello_last_cuda_error": (_int, []),
    "morello_status_string": (ctypes.c_char_p, [_int]),
    "morello_version": (ctypes.c_char_p, []),
}


class MorelloError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = int(status)
        msg = lib().morello_status_string(self.status).decode()
        if self.status == MORELLO_ERR_CUDA:
            msg += " [cudaError %d]" % lib().morello_last_cuda_error()
        super().__init__("%s: %s (status %d)" % (where, msg, self.status))


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded shared library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(
                "%s is missing: build it with `python -m paper_2505_01637_b200.build` "
                "(there is no fallback implementation)" % LIB_PATH)
        handle = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype, fn.argtypes = res, args
        _lib = handle
    return _lib


def _addr(x):
    if x is None:
        return None
    if type(x) is int:
        return x or None
    try:
        return x.data_ptr() or None
    except AttributeError:
        pass
    if hasattr(x, "ctypes"):          # numpy array (host entry point)
        return x.ctypes.data or None
    if isinstance(x, int):
        return x or None
    raise TypeError("expected a tensor, an array or an integer address, got %r" % type(x))


_raw_stream = _device = None          # torch's own calls, once it has set the GPU up


def _stream(stream):
    if stream is None:
        return _raw_stream(_device()) or None if _raw_stream is not None else _torch_stream()
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream or None


def _torch_stream():
    global _raw_stream, _device
    torch = sys.modules.get("torch")
    if torch is None or not (torch.cuda.is_initialized() or torch.cuda.is_available()):
        return None
    # The raw handle of the current device's current stream, where torch has the calls for it: building a Stream
    # object, and the wrappers around these, cost microseconds, as much as a small call's launch.
    now = torch.cuda.current_stream().cuda_stream or None
    raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
    if raw is not None and device is not None:
        _raw_stream, _device = raw, device
    return now


def _check(status: int, where: str) -> None:
    if status != MORELLO_OK:
        raise MorelloError(status, where)


def morello_matmul_accum(b, m, k, n, A, B, C, stream=None) -> None:
    _check(lib().morello_matmul_accum(b, m, k, n, _addr(A), _addr(B), _addr(C), _stream(stream)),
           "morello_matmul_accum")


def morello_matmul(b, m, k, n, A, B, C, stream=None) -> None:
    """C = A x B (C's prior contents are not read)."""
    _check(lib().morello_matmul(b, m, k, n, _addr(A), _addr(B), _addr(C), _stream(stream)),
           "morello_matmul")


def morello_matmul_forced(path, split_k, b, m, k, n, A, B, C, workspace=None,
                          workspace_bytes=0, stream=None) -> None:
    _check(lib().morello_matmul_forced(path, split_k, b, m, k, n, _addr(A), _addr(B), _addr(C),
                                       _addr(workspace), workspace_bytes, _stream(stream)),
           "morello_matmul_forced")


def morello_matmul_accum_f32(b, m, k, n, A, B, C, stream=None) -> None:
    """C += A x B with float32 A and B (split into bf16 terms inside the library)."""
    _check(lib().morello_matmul_accum_f32(b, m, k, n, _addr(A), _addr(B), _addr(C), _stream(stream)),
           "morello_matmul_accum_f32")


def morello_matmul_f32(b, m, k, n, A, B, C, stream=None) -> None:
    """C = A x B with float32 A and B (C is not read)."""
    _check(lib().morello_matmul_f32(b, m, k, n, _addr(A), _addr(B), _addr(C), _stream(stream)),
           "morello_matmul_f32")


def morello_matmul_accum_colmajor_b(tile, b, m, k, n, A, Bt, C, stream=None) -> None:
    """C += A x B with B given column-major: Bt[b][n][k]."""
    _check(lib().morello_matmul_accum_colmajor_b(tile, b, m, k, n, _addr(A), _addr(Bt), _addr(C),
                                                 _stream(stream)),
           "morello_matmul_accum_colmajor_b")


def morello_matmul_accum_packed_b(strip, b, m, k, n, A, Bp, C, stream=None) -> None:
    """C += A x B with B packed in strips of `strip` columns: Bp[b][ceil(n/strip)][k][strip]."""
    _check(lib().morello_matmul_accum_packed_b(strip, b, m, k, n, _addr(A), _addr(Bp), _addr(C),
                                               _stream(stream)),
           "morello_matmul_accum_packed_b")


def morello_matmul_colmajor_b(tile, b, m, k, n, A, Bt, C, stream=None) -> None:
    """C = A x B with B given column-major (C is not read)."""
    _check(lib().morello_matmul_colmajor_b(tile, b, m, k, n, _addr(A), _addr(Bt), _addr(C), _stream(stream)),
           "morello_matmul_colmajor_b")


def morello_matmul_packed_b(strip, b, m, k, n, A, Bp, C, stream=None) -> None:
    """C = A x B with B packed in strips of `strip` columns (C is not read)."""
    _check(lib().morello_matmul_packed_b(strip, b, m, k, n, _addr(A), _addr(Bp), _addr(C), _stream(stream)),
           "morello_matmul_packed_b")


def morello_workspace_bytes(b, m, k, n) -> int:
    return int(lib().morello_workspace_bytes(b, m, k, n))


def morello_matmul_accum_ws(b, m, k, n, A, B, C, workspace, workspace_bytes, stream=None) -> None:
    _check(lib().morello_matmul_accum_ws(b, m, k, n, _addr(A), _addr(B), _addr(C),
                                         _addr(workspace), workspace_bytes, _stream(stream)),
           "morello_matmul_accum_ws")


def morello_matmul_accum_host(b, m, k, n, A_host, B_host, C_host) -> None:
    _check(lib().morello_matmul_accum_host(b, m, k, n, _addr(A_host), _addr(B_host), _addr(C_host)),
           "morello_matmul_accum_host")


def morello_matmul_accum_noalloc(split_k, b, m, k, n, A, B, C, stream=None) -> None:
    """Allocation-free variant: partial sums live in a fixed array inside the library."""
    _check(lib().morello_matmul_accum_noalloc(split_k, b, m, k, n, _addr(A), _addr(B), _addr(C),
                                              _stream(stream)),
           "morello_matmul_accum_noalloc")


def morello_noalloc_scratch_limit() -> int:
    return int(lib().morello_noalloc_scratch_limit())


def morello_select_path(b, m, k, n) -> int:
    return int(lib().morello_select_path(b, m, k, n))


def morello_describe_route(b, m, k, n) -> str:
    """One line naming the kernel, tile and k slices the selector picks for this shape."""
    buf = ctypes.create_string_buffer(512)
    _check(lib().morello_describe_route(b, m, k, n, buf, len(buf)), "morello_describe_route")
    return buf.value.decode()


def morello_selftest_per_device_once(devices, calls_per_device) -> int:
    return int(lib().morello_selftest_per_device_once(devices, calls_per_device))


def morello_matmul_accum_forced(path, split_k, b, m, k, n, A, B, C, workspace=None,
                                workspace_bytes=0, stream=None) -> None:
    _check(lib().morello_matmul_accum_forced(path, split_k, b, m, k, n, _addr(A), _addr(B),
                                             _addr(C), _addr(workspace), workspace_bytes,
                                             _stream(stream)),
           "morello_matmul_accum_forced")


def morello_workspace_bytes_forced(path, split_k, b, m, k, n) -> int:
    return int(lib().morello_workspace_bytes_forced(path, split_k, b, m, k, n))


def morello_linear(act, gated, y_type, w_layout, m, k, n, X, W, bias, R, Y, Z=None, workspace=None,
                   workspace_bytes=0, stream=None) -> None:
    """Y = act(X W + bias) + R, or gated act(X Wg + bg) * (X Wu + bu) + R; bias, R and Z may be None."""
    _check(lib().morello_linear(act, gated, y_type, w_layout, m, k, n, _addr(X), _addr(W), _addr(bias), _addr(R),
                                _addr(Y), _addr(Z), _addr(workspace), workspace_bytes, _stream(stream)),
           "morello_linear")


def morello_linear_workspace_bytes(gated, w_layout, m, k, n) -> int:
    return int(lib().morello_linear_workspace_bytes(gated, w_layout, m, k, n))


def morello_linear_backward(act, gated, grad_type, accumulate, w_layout, m, k, n, X, W, Z, dY, dX, dW, dbias,
                            workspace=None, workspace_bytes=0, stream=None) -> None:
    """Gradients of morello_linear; dX, dW and dbias may be None."""
    _check(lib().morello_linear_backward(act, gated, grad_type, accumulate, w_layout, m, k, n, _addr(X), _addr(W),
                                         _addr(Z), _addr(dY), _addr(dX), _addr(dW), _addr(dbias), _addr(workspace),
                                         workspace_bytes, _stream(stream)),
           "morello_linear_backward")


def morello_linear_backward_workspace_bytes(act, gated, w_layout, m, k, n) -> int:
    return int(lib().morello_linear_backward_workspace_bytes(act, gated, w_layout, m, k, n))


def morello_route(score, renorm, scale, logits_type, tokens, experts, topk, groups, topk_groups, logits, bias, idx,
                  weights, stream=None) -> None:
    """Chooses every token's experts and their weights; bias may be None."""
    _check(lib().morello_route(score, renorm, scale, logits_type, tokens, experts, topk, groups, topk_groups,
                               _addr(logits), _addr(bias), _addr(idx), _addr(weights), _stream(stream)),
           "morello_route")


def morello_route_backward(score, renorm, scale, logits_type, tokens, experts, topk, logits, idx, dweights, dlogits,
                           stream=None) -> None:
    _check(lib().morello_route_backward(score, renorm, scale, logits_type, tokens, experts, topk, _addr(logits),
                                        _addr(idx), _addr(dweights), _addr(dlogits), _stream(stream)),
           "morello_route_backward")


def morello_expert_plan_rows(tokens, topk, experts) -> int:
    return int(lib().morello_expert_plan_rows(tokens, topk, experts))


def morello_expert_plan_words(tokens, topk, experts) -> int:
    return int(lib().morello_expert_plan_words(tokens, topk, experts))


def morello_expert_plan(tokens, topk, experts, idx, plan, stream=None) -> None:
    """Sorts the routed pairs by expert; plan is an int32 buffer of morello_expert_plan_words() words."""
    _check(lib().morello_expert_plan(tokens, topk, experts, _addr(idx), _addr(plan), _stream(stream)),
           "morello_expert_plan")


def morello_expert_linear(act, gated, y_type, w_layout, gather, tokens, topk, experts, k, n, plan, X, W, bias, Y,
                          Z=None, workspace=None, workspace_bytes=0, stream=None) -> None:
    """morello_linear with the weights of every row's expert, rows in the plan's layout."""
    _check(lib().morello_expert_linear(act, gated, y_type, w_layout, gather, tokens, topk, experts, k, n, _addr(plan),
                                       _addr(X), _addr(W), _addr(bias), _addr(Y), _addr(Z), _addr(workspace),
                                       workspace_bytes, _stream(stream)),
           "morello_expert_linear")


def morello_expert_linear_workspace_bytes(gated, w_layout, gather, tokens, topk, experts, k, n) -> int:
    return int(lib().morello_expert_linear_workspace_bytes(gated, w_layout, gather, tokens, topk, experts, k, n))


def morello_expert_linear_backward(act, gated, grad_type, accumulate, w_layout, gather, tokens, topk, experts, k, n,
                                   plan, X, W, Z, dY, dX, dW, dbias, workspace=None, workspace_bytes=0,
                                   stream=None) -> None:
    """Gradients of morello_expert_linear; dX, dW and dbias may be None."""
    _check(lib().morello_expert_linear_backward(act, gated, grad_type, accumulate, w_layout, gather, tokens, topk,
                                                experts, k, n, _addr(plan), _addr(X), _addr(W), _addr(Z), _addr(dY),
                                                _addr(dX), _addr(dW), _addr(dbias), _addr(workspace),
                                                workspace_bytes, _stream(stream)),
           "morello_expert_linear_backward")


def morello_expert_linear_backward_workspace_bytes(act, gated, w_layout, gather, tokens, topk, experts, k, n) -> int:
    return int(lib().morello_expert_linear_backward_workspace_bytes(act, gated, w_layout, gather, tokens, topk,
                                                                    experts, k, n))


def morello_expert_combine(y_type, tokens, topk, experts, n, plan, weights, Y, R, out, stream=None) -> None:
    """out[t] = R[t] + sum_j weights[t][j] * Y[slot[t][j]]; weights and R may be None."""
    _check(lib().morello_expert_combine(y_type, tokens, topk, experts, n, _addr(plan), _addr(weights), _addr(Y),
                                        _addr(R), _addr(out), _stream(stream)),
           "morello_expert_combine")


def morello_expert_combine_backward(y_type, tokens, topk, experts, n, plan, weights, Y, dout, dY, dweights,
                                    stream=None) -> None:
    """Gradients of morello_expert_combine; dY and dweights may be None."""
    _check(lib().morello_expert_combine_backward(y_type, tokens, topk, experts, n, _addr(plan), _addr(weights),
                                                 _addr(Y), _addr(dout), _addr(dY), _addr(dweights), _stream(stream)),
           "morello_expert_combine_backward")


def morello_selftest_wait_timeout(limit_ms, stream=None) -> None:
    """Makes one bounded device-side wait run out on purpose (see the header); raises unless it
    gave up as designed.  The device status word is set afterwards."""
    _check(lib().morello_selftest_wait_timeout(limit_ms, _stream(stream)), "morello_selftest_wait_timeout")


def morello_layer_norm(rms, x_type, m, n, eps, X, gamma, beta, Y, mean=None, rstd=None, stream=None) -> None:
    """Y = (X - mean) * rstd * gamma + beta of every row; gamma, beta, mean and rstd may be None."""
    _check(lib().morello_layer_norm(rms, x_type, m, n, eps, _addr(X), _addr(gamma), _addr(beta), _addr(Y), _addr(mean),
                                    _addr(rstd), _stream(stream)),
           "morello_layer_norm")


def morello_layer_norm_backward(rms, x_type, accumulate, m, n, X, gamma, mean, rstd, dY, R, dX, dgamma, dbeta,
                                workspace=None, workspace_bytes=0, stream=None) -> None:
    """Gradients of morello_layer_norm; gamma, R, dX, dgamma and dbeta may be None (with rms: mean too)."""
    _check(lib().morello_layer_norm_backward(rms, x_type, accumulate, m, n, _addr(X), _addr(gamma), _addr(mean),
                                             _addr(rstd), _addr(dY), _addr(R), _addr(dX), _addr(dgamma), _addr(dbeta),
                                             _addr(workspace), workspace_bytes, _stream(stream)),
           "morello_layer_norm_backward")


def morello_layer_norm_backward_workspace_bytes(m, n) -> int:
    return int(lib().morello_layer_norm_backward_workspace_bytes(m, n))


def morello_fp4_bytes(rows, k) -> int:
    return int(lib().morello_fp4_bytes(rows, k))


def morello_fp4_scale_bytes(format, rows, parts, k) -> int:
    return int(lib().morello_fp4_scale_bytes(format, rows, parts, k))


def morello_fp4_quantize(format, x_type, x_layout, rows, parts, k, X, mult, Q, scales, stream=None) -> None:
    """X (times the one f32 at mult, if any) to 4-bit blocks along k with a scale each."""
    _check(lib().morello_fp4_quantize(format, x_type, x_layout, rows, parts, k, _addr(X), _addr(mult), _addr(Q),
                                      _addr(scales), _stream(stream)),
           "morello_fp4_quantize")


def morello_fp4_dequantize(format, y_type, rows, parts, k, Q, scales, alpha, Y, stream=None) -> None:
    """Y[rows][k] = the values of a 4-bit tensor (times the one f32 at alpha, if any)."""
    _check(lib().morello_fp4_dequantize(format, y_type, rows, parts, k, _addr(Q), _addr(scales), _addr(alpha), _addr(Y),
                                        _stream(stream)),
           "morello_fp4_dequantize")


def morello_fp4_linear(format, act, gated, y_type, m, k, n, X, X_scales, W, W_scales, alpha, bias, R, Y,
                       stream=None) -> None:
    """morello_linear on 4-bit X and W: z = alpha * (X W) + bias; alpha, bias and R may be None."""
    _check(lib().morello_fp4_linear(format, act, gated, y_type, m, k, n, _addr(X), _addr(X_scales), _addr(W),
                                    _addr(W_scales), _addr(alpha), _addr(bias), _addr(R), _addr(Y), _stream(stream)),
           "morello_fp4_linear")


def morello_read_device_status(stream=None):
    """Returns (status, detail) after synchronising the stream; does not raise."""
    detail = ctypes.c_uint32(0)
    st = lib().morello_read_device_status(_stream(stream), ctypes.byref(detail))
    return int(st), int(detail.value)


def morello_device_limits():
    """(SMs, two-CTA clusters the device holds at once) of the current device."""
    sms, pairs = ctypes.c_int(0), ctypes.c_int(0)
    _check(lib().morello_device_limits(ctypes.byref(sms), ctypes.byref(pairs)), "morello_device_limits")
    return int(sms.value), int(pairs.value)


def morello_launch_count() -> int:
    return int(lib().morello_launch_count())


def morello_last_cuda_error() -> int:
    return int(lib().morello_last_cuda_error())


def morello_status_string(status: int) -> str:
    return lib().morello_status_string(int(status)).decode()


def morello_version() -> str:
    return lib().morello_version().decode()
