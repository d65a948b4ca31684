// Eight bf16 elements of a row at a time, whatever the row's alignment.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "activation.cuh"

namespace morello {

// Elements per access that rows of `cols` elements from p on allow: 8, 4, 2 or 1.
inline int access_width(int64_t cols, const void* p) {
  for (int w = 8; w > 1; w /= 2)
    if (cols % w == 0 && reinterpret_cast<uintptr_t>(p) % (2 * w) == 0) return w;
  return 1;
}

// Eight elements from src on, of which `cols` exist, in accesses of `width` elements.
__device__ __forceinline__ uint4 load8_raw(const uint16_t* src, int width, int64_t cols) {
  if (cols >= 8) {
    if (width == 8) return *reinterpret_cast<const uint4*>(src);
    if (width == 4) {
      const uint2 a = reinterpret_cast<const uint2*>(src)[0], b = reinterpret_cast<const uint2*>(src)[1];
      return make_uint4(a.x, a.y, b.x, b.y);
    }
    // Rows of odd length start on 4-byte boundaries and off them in turn.
    if (width == 2 || (reinterpret_cast<uintptr_t>(src) & 2u) == 0) {
      const uint32_t* q = reinterpret_cast<const uint32_t*>(src);
      return make_uint4(q[0], q[1], q[2], q[3]);
    }
    const uint32_t first = src[0], last = src[7];
    const uint32_t* q = reinterpret_cast<const uint32_t*>(src + 1);
    const uint32_t a = q[0], b = q[1], c = q[2];
    return make_uint4(first | (a << 16), (a >> 16) | (b << 16), (b >> 16) | (c << 16), (c >> 16) | (last << 16));
  }
  uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t v = e < cols ? (uint32_t)src[e] : 0u;
    w[e >> 1] |= v << ((e & 1) * 16);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8_raw(uint16_t* dst, int width, int64_t cols, const uint4& w) {
  if (cols >= 8 && width == 8) {
    *reinterpret_cast<uint4*>(dst) = w;
  } else if (cols >= 8 && width == 4) {
    reinterpret_cast<uint2*>(dst)[0] = make_uint2(w.x, w.y);
    reinterpret_cast<uint2*>(dst)[1] = make_uint2(w.z, w.w);
  } else if (cols >= 8 && width == 2) {
    uint32_t* q = reinterpret_cast<uint32_t*>(dst);
    q[0] = w.x; q[1] = w.y; q[2] = w.z; q[3] = w.w;
  } else {
    const uint32_t q[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < cols) dst[e] = (uint16_t)(q[e >> 1] >> ((e & 1) * 16));
  }
}
__device__ __forceinline__ void unpack8(const uint4& w, float (&v)[8]) {
  v[0] = bf16_low(w.x); v[1] = bf16_high(w.x); v[2] = bf16_low(w.y); v[3] = bf16_high(w.y);
  v[4] = bf16_low(w.z); v[5] = bf16_high(w.z); v[6] = bf16_low(w.w); v[7] = bf16_high(w.w);
}
__device__ __forceinline__ uint4 pack8(const float (&v)[8]) {
  return make_uint4(bf16_pack(v[0], v[1]), bf16_pack(v[2], v[3]), bf16_pack(v[4], v[5]), bf16_pack(v[6], v[7]));
}

}  // namespace morello
