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
template <int kInFlight = 8>
__device__ __forceinline__ void block_in16(uint32_t block, int lane, const uint16_t* src, const PlainBlock& g) {
#pragma unroll kInFlight
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

// put_row16 and add_row16 of 16 pairs; 16 f32 make a row as long (the lower or the upper eight pairs).
__device__ __forceinline__ uint32_t bf16_pack_pair(sm100::f32x2 v) {
  const float2 f = sm100::pair_values(v);
  return bf16_pack(f.x, f.y);
}
__device__ __forceinline__ void put_pairs16(uint32_t block, int lane, const sm100::f32x2 (&v)[16]) {
  const uint32_t at = block + (uint32_t)lane * 64u, sw = (uint32_t)(lane >> 1) & 3u;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    st_shared_v4(at + (((uint32_t)j ^ sw) << 4), bf16_pack_pair(v[4 * j]), bf16_pack_pair(v[4 * j + 1]), bf16_pack_pair(v[4 * j + 2]),
                 bf16_pack_pair(v[4 * j + 3]));
}
template <int kHalf>
__device__ __forceinline__ void put_pairs32(uint32_t block, int lane, const sm100::f32x2 (&v)[16]) {
  const uint32_t at = block + (uint32_t)lane * 64u, sw = (uint32_t)(lane >> 1) & 3u;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 a = sm100::pair_values(v[8 * kHalf + 2 * j]), b = sm100::pair_values(v[8 * kHalf + 2 * j + 1]);
    st_shared_v4(at + (((uint32_t)j ^ sw) << 4), __float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
  }
}
__device__ __forceinline__ void add_pairs16(uint32_t block, int lane, sm100::f32x2 (&v)[16]) {
  const uint32_t at = block + (uint32_t)lane * 64u, sw = (uint32_t)(lane >> 1) & 3u;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint32_t w[4];
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                 : "r"(at + (((uint32_t)j ^ sw) << 4)) : "memory");
#pragma unroll
    for (int q = 0; q < 4; ++q) v[4 * j + q] = sm100::add2(v[4 * j + q], sm100::pair_of(bf16_low(w[q]), bf16_high(w[q])));
  }
}
// A block of 32 rows of 16 f32 out to memory, two rows at a time: g.at is that of the block's first element here, cols its
// columns that exist.
__device__ __forceinline__ void half_block_out32(uint32_t block, int lane, float* dst, const PlainBlock& g, int cols) {
  const int col = lane & 15;
#pragma unroll 8
  for (int r0 = 0; r0 < 32; r0 += 2) {
    const int r = r0 + (lane >> 4);
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v)
                 : "r"(block + (uint32_t)r * 64u + ((((uint32_t)col >> 2) ^ (((uint32_t)r >> 1) & 3u)) << 4) + ((uint32_t)col & 3u) * 4u)
                 : "memory");
    if (r < g.rows && col < cols) dst[g.at + r * g.pitch + col] = v;
  }
}

}  // namespace morello
