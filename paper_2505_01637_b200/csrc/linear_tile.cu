// Tensor-core products with an epilogue: the forward pass, the input gradient and the weight
// gradient of linear layers, dense or with the weights of every row's expert.
//
// Persistent thread blocks walk output tiles, one CTA (cta_group::1, 128 x N) or a CTA pair
// (cta_group::2, 256 x N) per tile, warps specialised into a TMA producer, an MMA issuer and four
// epilogue warps; the two TMEM accumulators let the epilogue of one tile run under the main loop of
// the next.
//
// Either operand may be stored along or across the contraction (K-major or MN-major boxes of 64 x 64
// elements in the 128-byte swizzle), which makes the three products of a layer one kernel:
//   forward          Y = X W         A = X along, B = W across ([k][n]) or along ([n][k])
//   input gradient   dX = dZ W^T     A = dZ along, B = W the other way round
//   weight gradient  dW = X^T dZ     both across: the contraction runs over the rows
// Gated layers: a tile of N accumulator columns holds N / 2 columns of either half of W, so the gate and
// its partner meet in one thread's registers.
// Experts: their rows begin at multiples of 128, so a 128-row tile belongs to one expert and the weight
// gradient's contraction runs over its rows alone (rounded up to 16, where padding rows are zero).
//
// Epilogue, two warps per quarter of the rows, each with half of the tile's columns.  Where the TMA
// engine can address Y, Z and the residual: a thread holds one row of 32 columns, the residual's block
// arrives in shared memory by TMA while the accumulator is awaited, y replaces it there and leaves by TMA, Z
// beside it (blocks of 32 rows in the 64- or 128-byte swizzle).  Anything else (n % 8 != 0, odd
// addresses): a warp parks 32 rows x 64 accumulator columns (f32) in shared memory and reads them back
// with eight (gated: four) lanes to a row, so that any n and alignment is a matter of predicates.
#include <algorithm>

#include "activation.cuh"
#include "linear.h"
#include "sm100.cuh"
#include "tensormap.h"

namespace morello {
namespace {

using namespace sm100;

constexpr int kRowsPerCta = 128;
constexpr int kTileK = 64;
constexpr int kBytesA = kRowsPerCta * kTileK * 2;   // 16 KiB
constexpr int kBoxBytes = 64 * kTileK * 2;          // a 64 x 64 box: 8 KiB
constexpr int kAccStride = 256;
constexpr int kTmemColumns = 2 * kAccStride;
constexpr int kEpiWarps = 8;
constexpr int kThreads = 64 + 32 * kEpiWarps;
constexpr int kMaxStages = 8;
constexpr int kEpiBlockBytes = 8 * 1024;            // per warp: four blocks of 32 x 32 bf16, or 32 x 64 f32
constexpr int kEpiBytes = kEpiWarps * kEpiBlockBytes;
constexpr int kBlock16 = 32 * 32 * 2;               // 32 rows x 32 columns of bf16
constexpr int kSmemBudget = 227 * 1024;

template <bool kPair, int kTileN>
struct Shape {
  static constexpr int kCtas = kPair ? 2 : 1;
  static constexpr int kTileM = kRowsPerCta * kCtas;
  static constexpr int kColsB = kTileN / kCtas;
  static constexpr int kBoxesB = kColsB / 64;
  static constexpr int kStageBytes = kBytesA + kBoxesB * kBoxBytes;
  static constexpr int kFit = (kSmemBudget - kEpiBytes - 1024 - 512) / kStageBytes;
  static constexpr int kStages = kFit < kMaxStages ? kFit : kMaxStages;
  static constexpr size_t kSmemBytes = (size_t)kStages * kStageBytes + kEpiBytes + 1024 + 512;
  static_assert(kColsB % 64 == 0 && kTileN <= kAccStride, "tile shape");
};

struct TileParams {
  int64_t m;             // rows of one output
  int n;                 // columns of one output
  int k_blocks;          // contraction blocks (kContract: of the expert, from counts)
  int m_tiles, n_tiles, raster;
  int64_t tiles;         // kRows: decided on the device
  int b_up;
  uint8_t mode, a_mn, b_mn, zero_padding;
  // experts
  const int32_t* block_expert;
  const int32_t* offsets;
  const int32_t* counts;
  int experts;
  // epilogue
  uint8_t act, out_f32, accumulate, vec, tma;
  int z_pitch;           // columns of a row of Z and of the bias: n or 2 n
  const uint16_t* bias;
  const uint16_t* residual;
  void* Y;
  uint16_t* Z;
  uint32_t* status;
};

struct Barriers {
  uint64_t full[kMaxStages];
  uint64_t empty[kMaxStages];
  uint64_t acc_full[2];
  uint64_t acc_empty[2];
  uint64_t resid[kEpiWarps][2];
  uint32_t tmem_base;
  int abort_flag;
};

struct Item {
  int mt, nt;
  int group;        // expert (bias, weights, output of kContract)
  int k_blocks;
  int k_row0;       // kContract: first row of the contraction
  int k_steps;      // 16-deep steps of the last contraction block
  int live_end;     // rows of the output from here on hold no token (kRows), else m
};

// Tiles are walked in groups of `raster` rows of tiles, row-fastest inside a group, so that the tiles
// in flight share a few rows of A and a few columns of B in L2.
__device__ __forceinline__ void raster_decode(int raster, int m_tiles, int n_tiles, int within, int* mt, int* nt) {
  const int per_group = raster * n_tiles;
  const int grp = within / per_group, r = within - grp * per_group;
  const int rows = min(raster, m_tiles - grp * raster);
  *nt = r / rows;
  *mt = grp * raster + (r - *nt * rows);
}

template <bool kPair>
__device__ __forceinline__ Item decode_item(const TileParams& p, int m_tiles, int64_t t) {
  Item it;
  it.k_row0 = 0;
  it.k_blocks = p.k_blocks;
  it.k_steps = kTileK / 16;
  it.group = 0;
  it.live_end = (int)p.m;
  int within = (int)t;
  if (p.mode == (int)TileMode::kContract) {
    const int per = m_tiles * p.n_tiles;
    it.group = (int)(t / per);
    within = (int)(t - (int64_t)it.group * per);
    it.k_row0 = p.offsets[it.group];
    const int count = p.counts[it.group];
    it.k_blocks = (count + kTileK - 1) / kTileK;
    // Rows past the next multiple of 16 are never multiplied: they may hold anything.
    it.k_steps = (count - (it.k_blocks - 1) * kTileK + 15) / 16;
  }
  raster_decode(p.raster, m_tiles, p.n_tiles, within, &it.mt, &it.nt);
  if (p.mode == (int)TileMode::kRows) {
    it.group = p.block_expert[it.mt];
    it.live_end = p.offsets[it.group] + p.counts[it.group];
  }
  return it;
}

// Eight columns of one row, on their way out.
template <int kAct>
__device__ __forceinline__ void act8(float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = act_value<kAct>(v[e]);
}
__device__ __forceinline__ void act8_by(int act, float (&v)[8]) {
  if (act == kActNone) return;
  if (act == kActRelu) act8<kActRelu>(v);
  else if (act == kActGelu) act8<kActGelu>(v);
  else if (act == kActGeluTanh) act8<kActGeluTanh>(v);
  else act8<kActSilu>(v);
}
__device__ __forceinline__ void load8(const uint16_t* src, bool vec, int cols, float (&v)[8]) {
  if (vec) {
    const uint4 w = *reinterpret_cast<const uint4*>(src);
    v[0] = bf16_low(w.x); v[1] = bf16_high(w.x); v[2] = bf16_low(w.y); v[3] = bf16_high(w.y);
    v[4] = bf16_low(w.z); v[5] = bf16_high(w.z); v[6] = bf16_low(w.w); v[7] = bf16_high(w.w);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < cols ? bf16_value(src[e]) : 0.f;
  }
}
__device__ __forceinline__ void store8(uint16_t* dst, bool vec, int cols, const float (&v)[8]) {
  if (vec) {
    *reinterpret_cast<uint4*>(dst) = make_uint4(bf16_pack(v[0], v[1]), bf16_pack(v[2], v[3]),
                                                bf16_pack(v[4], v[5]), bf16_pack(v[6], v[7]));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < cols) dst[e] = bf16_round(v[e]);
  }
}
__device__ __forceinline__ void store8_f32(float* dst, bool vec, int cols, bool accumulate, float (&v)[8]) {
  if (vec) {
    float4* q = reinterpret_cast<float4*>(dst);
    if (accumulate) {
      const float4 a = q[0], b = q[1];
      v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w;
      v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
    }
    q[0] = make_float4(v[0], v[1], v[2], v[3]);
    q[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < cols) dst[e] = accumulate ? dst[e] + v[e] : v[e];
  }
}
// v += the eight staged columns at 16-byte chunks c0, c0 + 1 of the row; lanes of the upper half of a
// row read the second chunk first, which keeps the eight lanes of an access on different banks.
__device__ __forceinline__ void staged8(uint32_t row_addr, uint32_t c0, uint32_t sw, bool second_first, float (&v)[8]) {
  const uint32_t a0 = row_addr + (((c0 + (second_first ? 1u : 0u)) ^ sw) << 4);
  const uint32_t a1 = row_addr + (((c0 + (second_first ? 0u : 1u)) ^ sw) << 4);
  float x[8];
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]) : "r"(a0));
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]) : "r"(a1));
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] += second_first ? x[(e + 4) & 7] : x[e];
}

constexpr uint32_t kFullMask = 0xffffffffu;

struct EpilogueItem {
  int row0, col0;        // first row of the warp's quarter, first output column of the tile
  uint32_t taddr;
  const uint16_t* bias;
  int live_end;
  int group;             // third coordinate of Y
  bool empty_sum;
};

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
// A thread's 32 columns to or from its row of a 32 x 32 bf16 block in the 64-byte swizzle: the row's
// 16-byte chunk j sits at chunk j ^ ((row / 2) % 4).
__device__ __forceinline__ void put_row16(uint32_t block, int lane, const float (&v)[32]) {
  const uint32_t at = block + (uint32_t)lane * 64u, sw = (uint32_t)(lane >> 1) & 3u;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    st_shared_v4(at + (((uint32_t)j ^ sw) << 4), bf16_pack(v[8 * j], v[8 * j + 1]), bf16_pack(v[8 * j + 2], v[8 * j + 3]),
                 bf16_pack(v[8 * j + 4], v[8 * j + 5]), bf16_pack(v[8 * j + 6], v[8 * j + 7]));
}
__device__ __forceinline__ void add_row16(uint32_t block, int lane, float (&v)[32]) {
  const uint32_t at = block + (uint32_t)lane * 64u, sw = (uint32_t)(lane >> 1) & 3u;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint32_t w[4];
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at + (((uint32_t)j ^ sw) << 4)) : "memory");
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      v[8 * j + 2 * q] += bf16_low(w[q]);
      v[8 * j + 2 * q + 1] += bf16_high(w[q]);
    }
  }
}
__device__ __forceinline__ void sums32(uint32_t taddr, bool empty, float (&v)[32]) {
  uint32_t r[32];
  if (!empty) {
    tmem_ld_32x32(taddr, r);
    tmem_ld_wait();
  } else {
#pragma unroll
    for (int e = 0; e < 32; ++e) r[e] = 0u;
  }
#pragma unroll
  for (int e = 0; e < 32; ++e) v[e] = __uint_as_float(r[e]);
}
__device__ __forceinline__ void add_bias32(const uint16_t* bias, int cols, float (&v)[32]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (8 * j >= cols) break;          // cols is a multiple of 8 here
    float b[8];
    load8(bias + 8 * j, true, 8, b);
#pragma unroll
    for (int q = 0; q < 8; ++q) v[8 * j + q] += b[q];
  }
}

// Columns [0, kCols) of the tile's output belong to each half's warps, 32 at a time.
template <int kTileN, bool kGated>
struct EpilogueShape {
  static constexpr int kOutCols = kGated ? kTileN / 2 : kTileN;
  static constexpr int kCols = kOutCols / 2 < 32 ? 32 : kOutCols / 2;
  static constexpr int kSteps = kCols / 32;
};

template <int kTileN, bool kGated, typename Wait, typename Release>
__device__ __forceinline__ bool epilogue_tma(const TileParams& p, const EpilogueItem& e, const CUtensorMap& map_y,
                                             const CUtensorMap& map_z, const CUtensorMap& map_r, uint8_t* mine,
                                             uint64_t* r_bar, int half, int lane, uint32_t& step_no, uint32_t& r_phase,
                                             volatile int* abort_flag, Wait&& wait_sums, Release&& release_sums) {
  using E = EpilogueShape<kTileN, kGated>;
  const int first = half * E::kCols;                   // of this warp's output columns
  const bool rows_live = e.row0 < p.m;
  auto live_at = [&](int s) { return rows_live && s < E::kSteps && e.col0 + first + 32 * s < p.n; };
  // Y's block of a step (bf16: 2 KiB, alternating; f32: 4 KiB, alternating unless Z or the residual needs the rest).
  const bool one_y = p.out_f32 && (p.Z || p.residual);
  auto y_block = [&](uint32_t n) {
    return mine + (p.out_f32 ? (one_y ? 0u : (n & 1u) * 2u * kBlock16) : (n & 1u) * kBlock16);
  };
  auto load_residual = [&](int s, uint32_t n) {        // lane 0
    const uint32_t b = n & 1u;
    mbar_arrive_expect_tx(&r_bar[b], kBlock16);
    tma_load_3d(mine + (p.out_f32 ? 2u * kBlock16 + b * kBlock16 : b * kBlock16), &map_r, &r_bar[b],
                e.col0 + first + 32 * s, e.row0, 0);
  };
  // The residual's blocks are Y's own (bf16), or the two behind Y's single block (f32).
  if (p.residual && lane == 0 && live_at(0)) {
    bulk_wait_group_read<0>();
    load_residual(0, step_no);
    if (live_at(1)) load_residual(1, step_no + 1);
  }
  if (!wait_sums()) return false;
  const int row = e.row0 + lane;
  const bool padding = p.zero_padding && row >= e.live_end;
#pragma unroll 1
  for (int s = 0; s < E::kSteps; ++s) {
    const int c = first + 32 * s;
    const bool live = live_at(s);
    float v[32];
    [[maybe_unused]] float u[kGated ? 32 : 1];
    if (live) {
      sums32(e.taddr + (uint32_t)c, e.empty_sum, v);
      if constexpr (kGated) sums32(e.taddr + (uint32_t)(kTileN / 2 + c), e.empty_sum, u);
    }
    if (s + 1 == E::kSteps) release_sums();
    if (!live) continue;
    const int col = e.col0 + c;
    if (e.bias) {
      add_bias32(e.bias + col, p.n - col, v);
      if constexpr (kGated) add_bias32(e.bias + p.n + col, p.n - col, u);
    }
    if (padding) {
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] = 0.f;
      if constexpr (kGated) {
#pragma unroll
        for (int i = 0; i < 32; ++i) u[i] = 0.f;
      }
    }
    const uint32_t n = step_no;
    // The blocks written below must have left: those of the step before last, or of the last step where
    // every step uses the same.
    if (lane == 0) {
      if (one_y || (kGated && p.Z)) bulk_wait_group_read<0>();
      else bulk_wait_group_read<1>();
    }
    __syncwarp();
    uint8_t* z0 = mine + 2 * kBlock16 + (kGated ? 0u : (n & 1u) * kBlock16);
    uint8_t* z1 = mine + 3 * kBlock16;
    if (p.Z) {
      put_row16(smem_u32(z0), lane, v);
      if constexpr (kGated) put_row16(smem_u32(z1), lane, u);
    }
    act32_by(p.act, v);
    if constexpr (kGated) {
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] *= u[i];
    }
    uint8_t* yb = y_block(n);
    if (p.residual) {
      const uint32_t b = n & 1u;
      bool there = mbar_wait(&r_bar[b], (r_phase >> b) & 1u, abort_flag, p.status, 37);
      there = __all_sync(kFullMask, there);
      r_phase ^= 1u << b;
      if (!there) return false;
      add_row16(smem_u32(p.out_f32 ? mine + 2 * kBlock16 + b * kBlock16 : yb), lane, v);
    }
    if (p.out_f32) {
      // 128-byte rows: chunk j at j ^ (row % 8).
      const uint32_t at = smem_u32(yb) + (uint32_t)lane * 128u, sw = (uint32_t)(lane & 7);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        st_shared_v4(at + (((uint32_t)j ^ sw) << 4), __float_as_uint(v[4 * j]), __float_as_uint(v[4 * j + 1]),
                     __float_as_uint(v[4 * j + 2]), __float_as_uint(v[4 * j + 3]));
    } else {
      put_row16(smem_u32(yb), lane, v);
    }
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
      if (p.accumulate) tma_reduce_add_3d(&map_y, yb, col, e.row0, e.group);
      else tma_store_3d(&map_y, yb, col, e.row0, e.group);
      if (p.Z) {
        tma_store_3d(&map_z, z0, col, 0, e.row0);
        if constexpr (kGated) tma_store_3d(&map_z, z1, col, 1, e.row0);
      }
      bulk_commit_group();
      // The residual two steps ahead goes where this step's was read (f32) or where the step before
      // left its y (bf16): that store has been read once this step's alone is pending.
      if (p.residual) {
        if (p.out_f32) {
          if (live_at(s + 2)) load_residual(s + 2, n + 2);
        } else if (s >= 1 && live_at(s + 1)) {
          bulk_wait_group_read<1>();
          load_residual(s + 1, n + 1);
        }
      }
    }
    ++step_no;
  }
  return true;
}

template <int kTileN, bool kGated, typename Wait, typename Release>
__device__ __forceinline__ bool epilogue_plain(const TileParams& p, const EpilogueItem& e, uint32_t block, int half, int lane,
                                               Wait&& wait_sums, Release&& release_sums) {
  constexpr int kOutCols = kGated ? kTileN / 2 : kTileN;
  // Reading back: kLanes lanes to a row, kRowsAt rows at a time.
  constexpr int kLanes = kGated ? 4 : 8, kRowsAt = 32 / kLanes;
  constexpr int kStep = kGated ? 32 : 64;          // output columns per block
  constexpr int kCols = kOutCols / 2 < kStep ? kStep : kOutCols / 2;
  const int sub = lane % kLanes, row_in = lane / kLanes;
  const bool swap = !kGated && sub >= 4;
  if (!wait_sums()) return false;
  const int64_t out_row0 = (int64_t)e.group * p.m;
  const int row_end = (int)min(p.m, (int64_t)e.row0 + 32);
#pragma unroll 1
  for (int c = half * kCols; c < half * kCols + kCols; c += kStep) {
    const bool live = c < kOutCols && e.row0 < p.m && e.col0 + c < p.n;
    if (live) {
      // 64 accumulator columns: the step's own, or its gate's and its partner's 32 each.
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float v[32];
        sums32(e.taddr + (kGated ? (uint32_t)(c + h * (kTileN / 2)) : (uint32_t)(c + 32 * h)), e.empty_sum, v);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          st_shared_v4(block + (uint32_t)lane * 256u + ((((uint32_t)(h * 8 + j)) ^ (uint32_t)(lane & 7)) << 4),
                       __float_as_uint(v[4 * j]), __float_as_uint(v[4 * j + 1]), __float_as_uint(v[4 * j + 2]),
                       __float_as_uint(v[4 * j + 3]));
      }
    }
    if (c + kStep >= half * kCols + kCols) release_sums();
    if (!live) continue;
    __syncwarp();
    const int col = e.col0 + c + sub * 8;
    const int cols = p.n - col;                  // columns left from here (may be <= 0 or >= 8)
    const bool vec = p.vec && cols >= 8;
    float b0[8], b1[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) b0[i] = b1[i] = 0.f;
    if (e.bias && cols > 0) {
      load8(e.bias + col, vec, cols, b0);
      if constexpr (kGated) load8(e.bias + p.n + col, vec, cols, b1);
    }
    if (cols > 0) {
#pragma unroll 4
      for (int i = 0; i < 32 / kRowsAt; ++i) {
        const int r_in = i * kRowsAt + row_in;
        const int row = e.row0 + r_in;
        if (row >= row_end) continue;
        const uint32_t row_addr = block + (uint32_t)r_in * 256u, sw = (uint32_t)(r_in & 7);
        float v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = b0[q];
        staged8(row_addr, 2u * sub, sw, swap, v);
        const int64_t out_row = out_row0 + row;
        const bool padding = p.zero_padding && row >= e.live_end;
        if constexpr (kGated) {
          float u[8];
#pragma unroll
          for (int q = 0; q < 8; ++q) u[q] = b1[q];
          staged8(row_addr, 8u + 2u * sub, sw, false, u);
          if (padding) {
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] = u[q] = 0.f;
          }
          if (p.Z) {
            store8(p.Z + out_row * p.z_pitch + col, vec, cols, v);
            store8(p.Z + out_row * p.z_pitch + p.n + col, vec, cols, u);
          }
          act8_by(p.act, v);
#pragma unroll
          for (int q = 0; q < 8; ++q) v[q] *= u[q];
        } else {
          if (padding) {
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] = 0.f;
          }
          if (p.Z) store8(p.Z + out_row * p.z_pitch + col, vec, cols, v);
          act8_by(p.act, v);
        }
        if (p.residual) {
          float x[8];
          load8(p.residual + out_row * p.n + col, vec, cols, x);
#pragma unroll
          for (int q = 0; q < 8; ++q) v[q] += x[q];
        }
        if (p.out_f32) store8_f32(static_cast<float*>(p.Y) + out_row * p.n + col, vec, cols, p.accumulate, v);
        else store8(static_cast<uint16_t*>(p.Y) + out_row * p.n + col, vec, cols, v);
      }
    }
    __syncwarp();      // the block is rewritten by the next step
  }
  return true;
}

template <bool kPair, int kTileN, bool kGated>
__global__ void __launch_bounds__(kThreads, 1)
linear_tile_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                   const __grid_constant__ CUtensorMap map_y, const __grid_constant__ CUtensorMap map_z,
                   const __grid_constant__ CUtensorMap map_r, const TileParams p) {
  using S = Shape<kPair, kTileN>;
  constexpr int kOutCols = kGated ? kTileN / 2 : kTileN;   // output columns of a tile
  extern __shared__ uint8_t smem_raw[];
  uint8_t* stages = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* epi = stages + (size_t)S::kStages * S::kStageBytes;
  Barriers* bars = reinterpret_cast<Barriers*>(epi + kEpiBytes);
  volatile int* abort_flag = &bars->abort_flag;

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const uint32_t rank = kPair ? cluster_ctarank() : 0u;
  const int64_t unit = kPair ? (blockIdx.x >> 1) : blockIdx.x;
  const int64_t units = kPair ? (gridDim.x >> 1) : gridDim.x;

  if (threadIdx.x == 0) {
    for (int s = 0; s < S::kStages; ++s) {
      mbar_init(&bars->full[s], 1);
      mbar_init(&bars->empty[s], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars->acc_full[i], 1);
      mbar_init(&bars->acc_empty[i], kEpiWarps * S::kCtas);
    }
    for (int i = 0; i < 2 * kEpiWarps; ++i) mbar_init(&bars->resid[i >> 1][i & 1], 1);
    bars->abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_descriptor(&map_a);
    tma_prefetch_descriptor(&map_b);
  }
  if (warp == 1) {
    if constexpr (kPair) {
      tmem_alloc_pair(&bars->tmem_base, kTmemColumns);
      tmem_relinquish_pair();
    } else {
      tmem_alloc(&bars->tmem_base, kTmemColumns);
      tmem_relinquish();
    }
  }
  tc_fence_before_sync();
  if constexpr (kPair) cluster_sync(); else __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = bars->tmem_base;

  pdl_wait();
  pdl_release();

  // The experts' rows that are live: known on the device only.
  int m_tiles = p.m_tiles;
  int64_t tiles = p.tiles;
  if (p.mode == (int)TileMode::kRows) {
    m_tiles = p.offsets[p.experts] / kExpertBlock;
    tiles = (int64_t)m_tiles * p.n_tiles;
  }

  if (warp == 0) {
    // ------------------------------------------------------------------ producer
    if (elect_one()) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      const uint32_t leader_full = kPair ? map_to_cta(smem_u32(&bars->full[0]), 0) : 0u;
      (void)leader_full;
      for (int64_t t = unit; t < tiles && ok; t += units) {
        const Item it = decode_item<kPair>(p, m_tiles, t);
        const int row0 = it.mt * S::kTileM + (int)rank * kRowsPerCta;
        const int z_b = p.mode == (int)TileMode::kRows ? it.group : 0;
        int cols[S::kBoxesB];      // stored column of every 64-column box of B
#pragma unroll
        for (int j = 0; j < S::kBoxesB; ++j) {
          const int at = (int)rank * S::kColsB + j * 64;      // accumulator column
          if constexpr (kGated)
            cols[j] = at < kTileN / 2 ? it.nt * kOutCols + at : p.b_up + it.nt * kOutCols + at - kTileN / 2;
          else
            cols[j] = it.nt * kOutCols + at;
        }
        for (int kb = 0; kb < it.k_blocks; ++kb) {
          if (!(ok = mbar_wait(&bars->empty[stage], phase ^ 1, abort_flag, p.status, 33))) break;
          uint8_t* sa = stages + (size_t)stage * S::kStageBytes;
          uint8_t* sb = sa + kBytesA;
          const int kc = it.k_row0 + kb * kTileK;
          const uint32_t full = leader_full + (uint32_t)stage * 8u;
          (void)full;
          if constexpr (kPair) {
            if (rank == 0) mbar_arrive_expect_tx(&bars->full[stage], 2 * S::kStageBytes);
          } else {
            mbar_arrive_expect_tx(&bars->full[stage], S::kStageBytes);
          }
          auto load = [&](void* dst, const CUtensorMap* map, int c0, int c1, int c2) {
            if constexpr (kPair) tma_load_3d_pair(dst, map, full, c0, c1, c2);
            else tma_load_3d(dst, map, &bars->full[stage], c0, c1, c2);
          };
          if (p.a_mn) {
            load(sa, &map_a, row0, kc, 0);
            load(sa + kBoxBytes, &map_a, row0 + 64, kc, 0);
          } else {
            load(sa, &map_a, kc, row0, 0);
          }
#pragma unroll
          for (int j = 0; j < S::kBoxesB; ++j) {
            if (p.b_mn) load(sb + j * kBoxBytes, &map_b, cols[j], kc, z_b);
            else load(sb + j * kBoxBytes, &map_b, kc, cols[j], z_b);
          }
          if (++stage == S::kStages) { stage = 0; phase ^= 1; }
        }
      }
    }
  } else if (warp == 1) {
    // ---------------------------------------------------------------- MMA issuer
    if (rank == 0 && elect_one()) {
      const uint32_t idesc = instr_desc_bf16(S::kTileM, kTileN, p.a_mn != 0, p.b_mn != 0);
      // Across the contraction: 64-column groups one box apart, 16 contraction rows = 2048 bytes.
      // Along it: 8-row groups 1024 bytes apart, 16 elements = 32 bytes along the row.
      const uint32_t step_a = p.a_mn ? 2048u : 32u, step_b = p.b_mn ? 2048u : 32u;
      const uint32_t lbo_a = p.a_mn ? kBoxBytes : 16u, lbo_b = p.b_mn ? kBoxBytes : 16u;
      int stage = 0;
      uint32_t phase = 0;
      int buf = 0;
      uint32_t acc_phase = 0;
      bool ok = true;
      for (int64_t t = unit; t < tiles && ok; t += units) {
        const Item it = decode_item<kPair>(p, m_tiles, t);
        if (!(ok = mbar_wait(&bars->acc_empty[buf], acc_phase ^ 1, abort_flag, p.status, 34))) break;
        tc_fence_after_sync();
        const uint32_t d_tmem = tmem_base + (uint32_t)buf * kAccStride;
        for (int kb = 0; kb < it.k_blocks; ++kb) {
          if (!(ok = mbar_wait(&bars->full[stage], phase, abort_flag, p.status, 35))) break;
          tc_fence_after_sync();
          const uint32_t sa = smem_u32(stages + (size_t)stage * S::kStageBytes);
          const uint32_t sb = sa + kBytesA;
          const int steps = kb + 1 == it.k_blocks ? it.k_steps : kTileK / 16;
#pragma unroll
          for (int j = 0; j < kTileK / 16; ++j) {
            if (j >= steps) break;
            const uint64_t da = smem_desc_sw128(sa + j * step_a, lbo_a, 1024);
            const uint64_t db = smem_desc_sw128(sb + j * step_b, lbo_b, 1024);
            if constexpr (kPair) mma_bf16_ss_pair(d_tmem, da, db, idesc, (kb | j) != 0 ? 1u : 0u);
            else mma_bf16_ss(d_tmem, da, db, idesc, (kb | j) != 0 ? 1u : 0u);
          }
          if constexpr (kPair) mma_commit_pair(&bars->empty[stage], 3);
          else mma_commit(&bars->empty[stage]);
          if (++stage == S::kStages) { stage = 0; phase ^= 1; }
        }
        if (!ok) break;
        if constexpr (kPair) mma_commit_pair(&bars->acc_full[buf], 3);
        else mma_commit(&bars->acc_full[buf]);
        if (++buf == 2) { buf = 0; acc_phase ^= 1; }
      }
    }
  } else {
    // ------------------------------------------------------------------ epilogue
    const int ew = warp - 2;
    const int quarter = warp & 3, half = ew >> 2;      // TMEM lanes 32 quarter ..; half of the columns
    uint8_t* mine = epi + (size_t)ew * kEpiBlockBytes;
    int buf = 0;
    uint32_t acc_phase = 0;
    uint32_t step_no = 0;                              // steps taken: the block of a step is step_no % 2
    uint32_t r_phase = 0;                              // bit b: phase of the residual barrier of block b
    bool ok = true;
    for (int64_t t = unit; t < tiles && ok; t += units) {
      const Item it = decode_item<kPair>(p, m_tiles, t);
      EpilogueItem e;
      e.row0 = it.mt * S::kTileM + (int)rank * kRowsPerCta + quarter * 32;
      e.col0 = it.nt * kOutCols;
      e.taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)buf * kAccStride;
      e.bias = p.bias ? p.bias + (int64_t)it.group * p.z_pitch : nullptr;
      e.live_end = it.live_end;
      e.empty_sum = it.k_blocks == 0;
      e.group = p.mode == (int)TileMode::kContract ? it.group : 0;
      auto wait_sums = [&] {
        bool done = mbar_wait(&bars->acc_full[buf], acc_phase, abort_flag, p.status, 36);
        done = __all_sync(kFullMask, done);
        tc_fence_after_sync();
        return done;
      };
      auto release_sums = [&] {
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) {
          if constexpr (kPair) mbar_arrive_cluster(map_to_cta(smem_u32(&bars->acc_empty[buf]), 0));
          else mbar_arrive(&bars->acc_empty[buf]);
        }
      };
      if (p.tma)
        ok = epilogue_tma<kTileN, kGated>(p, e, map_y, map_z, map_r, mine, bars->resid[ew], half, lane, step_no,
                                          r_phase, abort_flag, wait_sums, release_sums);
      else
        ok = epilogue_plain<kTileN, kGated>(p, e, smem_u32(mine), half, lane, wait_sums, release_sums);
      if (++buf == 2) { buf = 0; acc_phase ^= 1; }
    }
    // Shared memory must outlive the engine's reads, and the stores must have been performed before the
    // kernel counts as complete.
    if (lane == 0) bulk_wait_group<0>();
  }

  __syncwarp();
  tc_fence_before_sync();
  if constexpr (kPair) cluster_sync(); else __syncthreads();
  tc_fence_after_sync();
  if (warp == 1) {
    __syncwarp();
    if constexpr (kPair) tmem_dealloc_pair(tmem_base, kTmemColumns);
    else tmem_dealloc(tmem_base, kTmemColumns);
  }
}

struct Maps {
  CUtensorMap a{}, b{}, y{}, z{}, r{};
};

template <bool kPair, int kTileN, bool kGated>
cudaError_t launch_tile(const DeviceInfo& dev, const Maps& maps, const TileParams& p, int64_t max_items,
                        cudaStream_t stream) {
  using S = Shape<kPair, kTileN>;
  static PerDeviceOnce once;
  const cudaError_t e = once.run_current([] {
    return cudaFuncSetAttribute(linear_tile_kernel<kPair, kTileN, kGated>,
                                cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kSmemBytes);
  });
  if (e != cudaSuccess) return e;
  const int64_t units = std::min<int64_t>(max_items, kPair ? gemm_pair_units(dev.sms) : dev.sms);
  return launch_pdl(linear_tile_kernel<kPair, kTileN, kGated>, dim3((unsigned)(units * S::kCtas)), dim3(kThreads),
                    S::kSmemBytes, stream, S::kCtas, maps.a, maps.b, maps.y, maps.z, maps.r, p);
}

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

}  // namespace

cudaError_t tile_launch(const DeviceInfo& dev, const TileCall& c, cudaStream_t stream, uint64_t* launches) {
  if (c.m <= 0 || c.n <= 0) return cudaSuccess;
  const LinearEpilogue& ep = c.epi;
  const int width = ep.gated ? 2 : 1;
  TileParams p{};
  p.m = c.m;
  p.n = (int)c.n;
  p.k_blocks = (int)((c.k + kTileK - 1) / kTileK);
  p.b_up = (int)c.b_up;
  p.mode = (uint8_t)c.mode;
  p.a_mn = c.a_mn;
  p.b_mn = c.b_mn;
  p.zero_padding = c.zero_padding;
  p.block_expert = c.experts.block_expert;
  p.offsets = c.experts.offsets;
  p.counts = c.experts.counts;
  p.experts = (int)c.experts.experts;
  p.act = (uint8_t)ep.act;
  p.out_f32 = ep.out_f32;
  p.accumulate = ep.accumulate;
  p.vec = c.n % 8 == 0 && aligned16(ep.Y) && aligned16(ep.Z) && aligned16(ep.bias) && aligned16(ep.residual);
  p.tma = p.vec && !(ep.out_f32 && ep.residual && ep.Z);    // that one has no room for its blocks
  p.z_pitch = (int)(c.n * width);
  p.bias = ep.bias;
  p.residual = ep.residual;
  p.Y = ep.Y;
  p.Z = ep.Z;
  p.status = dev.status;

  // The tile: the least waves x columns, weighted by what the narrower and the one-CTA tiles cost per
  // column.  Experts: a 128-row block belongs to one expert, a pair of them may not.
  const int64_t groups = c.mode == TileMode::kContract ? c.experts.experts : 1;
  double best = 0;
  int best_pair = -1, best_n = 0;
  for (int pair = 0; pair < 2; ++pair) {
    if (pair && (c.mode == TileMode::kRows || c.m <= kRowsPerCta)) continue;
    const int64_t units = std::max(1, pair ? gemm_pair_units(dev.sms) : dev.sms);
    for (int tn = 256; tn >= 64; tn >>= 1) {
      if (tn == 64 && (pair || ep.gated)) continue;
      const int64_t out_cols = ep.gated ? tn / 2 : tn;
      const int64_t tile_m = kRowsPerCta << pair;
      // Experts' blocks: the count is the device's; half of the padding's bound is the guess.
      const int64_t m_tiles = c.mode == TileMode::kRows
                                  ? std::max<int64_t>(1, (c.experts.tokens * c.experts.topk / kExpertBlock + c.m / kExpertBlock) / 2)
                                  : (c.m + tile_m - 1) / tile_m;
      const int64_t items = groups * m_tiles * ((c.n + out_cols - 1) / out_cols);
      const double waves = (double)((items + units - 1) / units);
      const double cost = waves * tn * (pair ? 1.0 : 1.15) * (tn == 256 ? 1.0 : tn == 128 ? 1.25 : 1.6);
      if (best_n == 0 || cost < best) { best = cost; best_pair = pair; best_n = tn; }
    }
  }
  const int64_t tile_m = kRowsPerCta << best_pair, out_cols = ep.gated ? best_n / 2 : best_n;
  p.m_tiles = (int)((c.m + tile_m - 1) / tile_m);
  p.n_tiles = (int)((c.n + out_cols - 1) / out_cols);
  p.raster = 8;
  p.tiles = groups * p.m_tiles * (int64_t)p.n_tiles;

  Maps maps;
  cudaError_t e = cudaSuccess;
  if (c.mode == TileMode::kContract || c.k > 0) {
    e = make_tensor_map_3d(&maps.a, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, c.a.p, (uint64_t)c.a.cols, (uint64_t)c.a.rows,
                           (uint64_t)c.a.groups, 64, c.a_mn ? 64u : (uint32_t)kRowsPerCta, CU_TENSOR_MAP_SWIZZLE_128B);
    if (e == cudaSuccess)
      e = make_tensor_map_3d(&maps.b, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, c.b.p, (uint64_t)c.b.cols, (uint64_t)c.b.rows,
                             (uint64_t)c.b.groups, 64, 64, CU_TENSOR_MAP_SWIZZLE_128B);
    if (e != cudaSuccess) return e;
  }
  if (p.tma) {
    const uint64_t out_groups = (uint64_t)groups;
    e = make_tensor_map_3d(&maps.y, ep.out_f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
                           ep.out_f32 ? 4 : 2, ep.Y, (uint64_t)c.n, (uint64_t)c.m, out_groups, 32, 32,
                           ep.out_f32 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B);
    // Z's halves are a dimension of their own: a block at the right edge of the first must not reach the second.
    if (e == cudaSuccess && ep.Z)
      e = make_tensor_map_3d_box(&maps.z, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, ep.Z, (uint64_t)c.n, (uint64_t)width,
                                 (uint64_t)c.m, 32, 1, 32, CU_TENSOR_MAP_SWIZZLE_64B);
    if (e == cudaSuccess && ep.residual)
      e = make_tensor_map_3d(&maps.r, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, ep.residual, (uint64_t)c.n, (uint64_t)c.m, 1, 32,
                             32, CU_TENSOR_MAP_SWIZZLE_64B);
    if (e != cudaSuccess) return e;
  }
  const int code = best_pair * 10000 + best_n * 10 + (ep.gated ? 1 : 0);
  switch (code) {
    case 640: e = launch_tile<false, 64, false>(dev, maps, p, p.tiles, stream); break;
    case 1280: e = launch_tile<false, 128, false>(dev, maps, p, p.tiles, stream); break;
    case 2560: e = launch_tile<false, 256, false>(dev, maps, p, p.tiles, stream); break;
    case 1281: e = launch_tile<false, 128, true>(dev, maps, p, p.tiles, stream); break;
    case 2561: e = launch_tile<false, 256, true>(dev, maps, p, p.tiles, stream); break;
    case 11280: e = launch_tile<true, 128, false>(dev, maps, p, p.tiles, stream); break;
    case 12560: e = launch_tile<true, 256, false>(dev, maps, p, p.tiles, stream); break;
    case 11281: e = launch_tile<true, 128, true>(dev, maps, p, p.tiles, stream); break;
    case 12561: e = launch_tile<true, 256, true>(dev, maps, p, p.tiles, stream); break;
    default: return cudaErrorInvalidValue;
  }
  if (e == cudaSuccess) ++*launches;
  return e;
}

}  // namespace morello
