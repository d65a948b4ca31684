// What the tile kernels' epilogues share: a thread holds 32 columns of one row, a warp a block of 32 rows x 32 columns that
// goes through shared memory.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "activation.cuh"
#include "sm100.cuh"

namespace morello {

using sm100::st_shared_v4;
using sm100::tmem_ld_32x32;

template <int kAct>
__device__ __forceinline__ void act32(float (&v)[32]) {
#pragma unroll
  for (int e = 0; e < 32; ++e) v[e] = act_value<kAct>(v[e]);
}
__device__ __forceinline__ void act32_by(int act, float (&v)[32]) {
  if (act == kActNone) return;
  if (act == kActRelu) act32<kActRelu>(v);
  else if (act == kActGelu) act32<kActGelu>(v);
  else if (act == kActGeluTanh) act32<kActGeluTanh>(v);
  else act32<kActSilu>(v);
}
// A thread's 32 columns to its row of a 32 x 32 block: bf16 in the 64-byte swizzle (the row's 16-byte chunk
// j sits at chunk j ^ ((row / 2) % 4)), f32 in the 128-byte one (chunk j at j ^ (row % 8)).
__device__ __forceinline__ void put_row16(uint32_t block, int lane, const float (&v)[32]) {
  const uint32_t at = block + (uint32_t)lane * 64u, sw = (uint32_t)(lane >> 1) & 3u;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    st_shared_v4(at + (((uint32_t)j ^ sw) << 4), bf16_pack(v[8 * j], v[8 * j + 1]), bf16_pack(v[8 * j + 2], v[8 * j + 3]),
                 bf16_pack(v[8 * j + 4], v[8 * j + 5]), bf16_pack(v[8 * j + 6], v[8 * j + 7]));
}
__device__ __forceinline__ void put_row32(uint32_t block, int lane, const float (&v)[32]) {
  const uint32_t at = block + (uint32_t)lane * 128u, sw = (uint32_t)(lane & 7);
#pragma unroll
  for (int j = 0; j < 8; ++j)
    st_shared_v4(at + (((uint32_t)j ^ sw) << 4), __float_as_uint(v[4 * j]), __float_as_uint(v[4 * j + 1]),
                 __float_as_uint(v[4 * j + 2]), __float_as_uint(v[4 * j + 3]));
}
// Starts the load of 32 columns of sums; tmem_ld_wait() completes it.
__device__ __forceinline__ void start_sums32(uint32_t taddr, bool empty, uint32_t (&r)[32]) {
  if (!empty) {
    tmem_ld_32x32(taddr, r);
  } else {
#pragma unroll
    for (int e = 0; e < 32; ++e) r[e] = 0u;
  }
}
__device__ __forceinline__ void add_octet(const uint4& w, float* v) {
  v[0] += bf16_low(w.x); v[1] += bf16_high(w.x); v[2] += bf16_low(w.y); v[3] += bf16_high(w.y);
  v[4] += bf16_low(w.z); v[5] += bf16_high(w.z); v[6] += bf16_low(w.w); v[7] += bf16_high(w.w);
}
__device__ __forceinline__ void add_bias32(const uint16_t* bias, int cols, bool octets, float (&v)[32]) {
  if (octets) {        // cols % 8 == 0, 16-byte-aligned
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (8 * j < cols) add_octet(reinterpret_cast<const uint4*>(bias)[j], v + 8 * j);
  } else {
#pragma unroll
    for (int j = 0; j < 32; ++j)
      if (j < cols) v[j] += bf16_value(bias[j]);
  }
}

// Where the TMA engine cannot address a tensor (n % 8 != 0, odd addresses) its 32 x 32 blocks move between shared
// and global memory a row at a time, a lane to a column: 64 or 128 contiguous bytes an access.
struct PlainBlock {
  int64_t at;        // the block's first element, this lane's column
  int64_t pitch;
  int rows;          // of the block that exist; 0 for a lane past the last column
};
__device__ __forceinline__ uint32_t place16(uint32_t block, int row, int lane) {
  return block + (uint32_t)row * 64u + ((((uint32_t)lane >> 3) ^ (((uint32_t)row >> 1) & 3u)) << 4) + ((uint32_t)lane & 7u) * 2u;
}
__device__ __forceinline__ void block_in16(uint32_t block, int lane, const uint16_t* src, const PlainBlock& g) {
#pragma unroll 8
  for (int r = 0; r < 32; ++r) {
    const uint16_t v = r < g.rows ? src[g.at + r * g.pitch] : (uint16_t)0;
    asm volatile("st.shared.u16 [%0], %1;" ::"r"(place16(block, r, lane)), "h"(v) : "memory");
  }
}
__device__ __forceinline__ void block_out16(uint32_t block, int lane, uint16_t* dst, const PlainBlock& g) {
#pragma unroll 8
  for (int r = 0; r < 32; ++r) {
    uint16_t v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(place16(block, r, lane)) : "memory");
    if (r < g.rows) dst[g.at + r * g.pitch] = v;
  }
}
__device__ __forceinline__ void block_out32(uint32_t block, int lane, float* dst, const PlainBlock& g, bool accumulate) {
#pragma unroll 8
  for (int r = 0; r < 32; ++r) {
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v)
                 : "r"(block + (uint32_t)r * 128u + ((((uint32_t)lane >> 2) ^ ((uint32_t)r & 7u)) << 4) + ((uint32_t)lane & 3u) * 4u)
                 : "memory");
    if (r < g.rows) dst[g.at + r * g.pitch] = accumulate ? dst[g.at + r * g.pitch] + v : v;
  }
}
__device__ __forceinline__ void add_row16(uint32_t block, int lane, float (&v)[32]) {
  const uint32_t at = block + (uint32_t)lane * 64u, sw = (uint32_t)(lane >> 1) & 3u;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint4 w;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w)
                 : "r"(at + (((uint32_t)j ^ sw) << 4)) : "memory");
    add_octet(w, v + 8 * j);
  }
}

}  // namespace morello
