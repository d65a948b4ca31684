// C entry point of the product of 4-bit tensors.
#include "../../include/morello.h"
#include "activation.cuh"
#include "fp4.h"

namespace morello {
namespace {

constexpr int64_t kMaxExtent = (1ll << 31) - 1024;   // tile coordinates are ints

bool aligned(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

}  // namespace
}  // namespace morello

using namespace morello;

#pragma GCC visibility push(default)
extern "C" {

int morello_fp4_linear(int format, int act, int gated, int y_type, int64_t m, int64_t k, int64_t n, const void* X,
                       const void* X_scales, const void* W, const void* W_scales, const float* alpha, const void* bias,
                       const void* R, void* Y, void* stream) {
  if (format < 0 || format > 1 || act < 0 || act >= kActCount || gated < 0 || gated > 1 || y_type < 0 || y_type > 1)
    return MORELLO_ERR_INVALID_ARGUMENT;
  if (m < 0 || k < 0 || n < 0 || m > kMaxExtent || k > kMaxExtent || n > (gated ? kMaxExtent / 2 : kMaxExtent))
    return MORELLO_ERR_INVALID_SHAPE;
  const bool empty = m == 0 || n == 0, y_f32 = y_type == MORELLO_F32;
  if (!empty && (!Y || (k > 0 && (!X || !X_scales || !W || !W_scales)))) return MORELLO_ERR_NULL_POINTER;
  if (!aligned(X, 16) || !aligned(X_scales, 16) || !aligned(W, 16) || !aligned(W_scales, 16) || !aligned(alpha, 4) ||
      !aligned(bias, 2) || !aligned(R, 2) || !aligned(Y, y_f32 ? 4 : 2))
    return MORELLO_ERR_MISALIGNED;
  DeviceInfo dev;
  void* none = nullptr;
  int rc;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if ((rc = operator_workspace(0, nullptr, 0, s, &none, &dev)) != MORELLO_OK || empty) return rc;
  Fp4Call c;
  c.nv = format == MORELLO_NVFP4;
  c.m = m;
  c.n = n;
  c.k = k;
  c.X = X;
  c.X_scales = X_scales;
  c.W = W;
  c.W_scales = W_scales;
  c.alpha = alpha;
  c.epi.act = act;
  c.epi.gated = gated != 0;
  c.epi.out_f32 = y_f32;
  c.epi.bias = static_cast<const uint16_t*>(bias);
  c.epi.residual = static_cast<const uint16_t*>(R);
  c.epi.Y = Y;
  uint64_t launches = 0;
  const cudaError_t e = m <= kFp4FewRows ? fp4_rows_launch(dev, c, s, &launches) : fp4_tile_launch(dev, c, s, &launches);
  count_launches(launches);
  return e == cudaSuccess ? MORELLO_OK : record_cuda_error(e);
}

}  // extern "C"
#pragma GCC visibility pop
