// Tensor-core products with an epilogue: the forward pass, the input gradient and the weight
// gradient of linear layers, dense or with the weights of every row's expert.
//
// Persistent thread blocks walk output tiles, one CTA (cta_group::1, 128 x N) or a CTA pair
// (cta_group::2, 256 x N) per tile, warps specialised into a TMA producer, an MMA issuer and eight
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
// gradient's contraction runs over its rows alone, rounded up to 16.  The rows that round it up are zeros in one operand at
// least: where neither was written by this library, the last contraction block of A comes in gathers of four rows, and those
// without a pair are asked for past the tensor's end, which reads as zeros.
//
// Epilogue: eight warps, two per quarter of the rows, which take its 32-column steps in turn; a thread
// holds one row of 32 columns.  Where the TMA engine can address Y and Z they leave through shared memory
// in blocks of 32 rows x 32 columns (64- or 128-byte swizzle), two of which a warp uses in turn; the residual is
// read straight into registers while the accumulator is awaited.  Anything else (n % 8 != 0, odd addresses) goes
// through the same blocks, which the warp then copies out (and the residual's in) a row at a time.
// A step is a chain of tensor-memory load, conversion, shared store, proxy fence and TMA store, about 1,100
// cycles; eight warps keep it under a main loop of 8 contraction blocks or more.  Twelve and sixteen warps were
// measured slower (their share of the registers spills: 4096 x 4096 x 4096 with GELU, bias, residual and Z
// 116, 123 and 127 us).
#include <algorithm>
#include <cmath>

#include "activation.cuh"
#include "column_sums.cuh"
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
constexpr int kEpiWarps = 8;                        // two per quarter of the rows
constexpr int kParts = kEpiWarps / 4;
constexpr int kThreads = 64 + 32 * kEpiWarps;
constexpr int kMaxStages = 8;
constexpr int kEpiBlockBytes = 4 * 1024;            // per warp: two blocks of 32 x 32 bf16, or one of f32
constexpr int kEpiBytes = kEpiWarps * kEpiBlockBytes;
constexpr int kBlock16 = 32 * 32 * 2;               // 32 rows x 32 columns of bf16
constexpr int kSmemBudget = 227 * 1024;
constexpr int kPairTable = 257;                     // experts whose pairs of blocks a CTA pair can look up, + 1

template <bool kPair, int kTileN>
struct Shape {
  static constexpr int kCtas = kPair ? 2 : 1;
  static constexpr int kTileM = kRowsPerCta * kCtas;
  static constexpr int kColsB = kTileN / kCtas;
  static constexpr int kBoxesB = kColsB / 64;
  static constexpr int kStageBytes = kBytesA + kBoxesB * kBoxBytes;
  static constexpr int kFit = (kSmemBudget - kEpiBytes - 1024 - 1536) / kStageBytes;
  static constexpr int kStages = kFit < kMaxStages ? kFit : kMaxStages;
  static constexpr size_t kSmemBytes = (size_t)kStages * kStageBytes + kEpiBytes + 1024 + 1536;
  static_assert(kColsB % 64 == 0 && kTileN <= kAccStride, "tile shape");
};

struct TileParams {
  int64_t m;             // rows of one output
  int n;                 // columns of one output
  int k_blocks;          // contraction blocks (kContract: of the expert, from counts)
  int m_tiles, n_tiles;
  int64_t tiles;         // kRows: decided on the device
  int lead;              // second product: its items that a unit takes in place of one of the first's
  int b_up;
  int a_rows;            // masked_a: rows of A, the first that it does not have
  uint8_t mode, a_mn, b_mn, zero_padding, halves;
  uint8_t masked_a;      // kContract: see TileCall
  // experts
  const int32_t* block_expert;
  const int32_t* offsets;
  const int32_t* counts;
  int experts;
  // epilogue
  uint8_t act, out_f32, accumulate, tma, copy;   // copy: bf16 Y is the sums, nothing else, by epilogue_copy
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
  uint32_t tmem_base;
  int abort_flag;
  int pairs_before[kPairTable];   // kRows, pairs: pairs of blocks of the experts before each
};

struct Item {
  int row0, nt;     // first row of the tile
  int row_end;      // its rows end here (kRows: the expert's blocks do), for what is written
  int n_off, cols;  // first accumulator column inside the tile's, and how many: the tile or half of it
  int group;        // expert (bias, weights, output of kContract)
  int k_blocks;
  int k_row0;       // kContract: first row of the contraction,
  int k_row_end;    // and the first past it that holds no pair
  int k_steps;      // 16-deep steps of the last contraction block
  int live_end;     // rows of the output from here on hold no token (kRows)
};

// Tiles are walked in groups of kRaster rows of tiles, row-fastest inside a group, so that the tiles in
// flight share a few rows of A and a few columns of B in L2.
constexpr int kRasterLog = 3, kRaster = 1 << kRasterLog;

// What the tile loop walks: whole tiles, then the column halves of the last wave's.  The units take turns, but the first
// `lead` items go to the units from `idle` on, which the product before left without a share of its last wave.
struct Walk {
  int m_tiles, n_tiles;
  int whole, items;
  int lead, idle;
};

// A role's place in the walk.  It moves by additions: an item is decoded by every role of a block, and with
// divisions that took 1,000 cycles, as long as two contraction blocks.
template <bool kPair, int kTileN>
class Cursor {
 public:
  __device__ __forceinline__ Cursor(const TileParams& p, const Walk& w, const int* pairs_before, int unit, int units)
      : p_(p), w_(w), pairs_before_(pairs_before), unit_(unit), units_(units) {
    const bool leads = unit >= w.idle && w.lead > 0;
    t_ = leads ? unit - w.idle : w.lead + unit;
    step_ = leads ? units - w.idle : units;
    if (leads && t_ >= w.lead) join();
    place();
  }
  __device__ __forceinline__ bool valid() const { return t_ < w_.items; }
  __device__ __forceinline__ bool is_half() const { return t_ >= w_.whole; }
  __device__ __forceinline__ void next() {
    t_ += step_;
    if (step_ != units_ && t_ >= w_.lead) {
      join();
      place();
    } else if (t_ < w_.whole) {
      at_ += step_;
      settle();
    } else {                         // once or twice a launch
      place();
    }
  }
  __device__ __forceinline__ Item item() const {
    constexpr int kTileM = kPair ? 2 * kRowsPerCta : kRowsPerCta;
    Item it;
    it.k_row0 = it.k_row_end = 0;
    it.k_blocks = p_.k_blocks;
    it.k_steps = kTileK / 16;
    it.group = 0;
    it.live_end = it.row_end = (int)p_.m;
    it.n_off = is_half() ? ((t_ - w_.whole) & 1) * (kTileN / 2) : 0;
    it.cols = is_half() ? kTileN / 2 : kTileN;
    const int rows = min(kRaster, w_.m_tiles - (grp_ << kRasterLog));
    it.nt = rows == kRaster ? at_ >> kRasterLog : at_ / rows;
    const int mt = (grp_ << kRasterLog) + at_ - it.nt * rows;
    it.row0 = mt * kTileM;
    if (p_.mode == (int)TileMode::kContract) {
      it.group = expert_;
      it.k_row0 = p_.offsets[expert_];
      const int count = p_.counts[expert_];
      it.k_row_end = it.k_row0 + count;
      it.k_blocks = (count + kTileK - 1) / kTileK;
      // Rows past the next multiple of 16 are never multiplied: they may hold anything.
      it.k_steps = (count - (it.k_blocks - 1) * kTileK + 15) / 16;
    } else if (p_.mode == (int)TileMode::kRows) {
      if constexpr (kPair) {
        int lo = 0, hi = p_.experts;      // the expert whose pairs hold number mt
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (pairs_before_[mid] <= mt) lo = mid; else hi = mid;
        }
        it.group = lo;
        it.row0 = p_.offsets[lo] + (mt - pairs_before_[lo]) * kTileM;
      } else {
        it.group = p_.block_expert[mt];
      }
      it.row_end = p_.offsets[it.group + 1];
      it.live_end = p_.offsets[it.group] + p_.counts[it.group];
    }
    return it;
  }

 private:
  // From the leading items on to the turns of all units.
  __device__ __forceinline__ void join() {
    t_ = w_.lead + unit_;
    step_ = units_;
  }
  __device__ __forceinline__ void place() {
    if (t_ >= w_.items) return;
    at_ = t_ < w_.whole ? t_ : w_.whole + ((t_ - w_.whole) >> 1);
    expert_ = grp_ = 0;
    settle();
  }
  // Carries at_ into the expert (kContract) and the group of rows of tiles it lies in.
  __device__ __forceinline__ void settle() {
    if (p_.mode == (int)TileMode::kContract) {
      const int per = w_.m_tiles * w_.n_tiles;
      at_ += grp_ * (kRaster * w_.n_tiles);
      grp_ = 0;
      while (at_ >= per) { at_ -= per; ++expert_; }
    }
    while (at_ >= kRaster * w_.n_tiles) { at_ -= kRaster * w_.n_tiles; ++grp_; }
  }
  const TileParams& p_;
  const Walk& w_;
  const int* pairs_before_;
  const int unit_, units_;
  int t_, step_, at_ = 0, grp_ = 0, expert_ = 0;
};

constexpr uint32_t kFullMask = 0xffffffffu;

struct EpilogueItem {
  int row0, col0;        // first row of the warp's quarter, first output column of the item
  int row_end;           // rows from here on are not the item's
  int width;             // output columns of the item
  uint32_t taddr;
  const uint16_t* bias;
  int live_end;
  int group;             // third coordinate of Y
  bool empty_sum;
  int chunks;            // parts the contraction's sums come in
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

// bf16 Y by TMA with nothing to be done to the sums (the gradients): steps of 64 columns, one block of 32 rows x 128
// bytes a warp.  Half the fences and stores of the steps below; where the contraction is short (the weights of an
// expert with few rows) the epilogue is what the kernel waits for.
template <typename Wait, typename Release>
__device__ __forceinline__ bool epilogue_copy(const TileParams& p, const EpilogueItem& e, const CUtensorMap& map_y,
                                              uint8_t* mine, int part, int lane, Wait&& wait_sums,
                                              Release&& release_sums) {
  const int steps = e.row0 < e.row_end ? (min(e.width, p.n - e.col0) + 63) / 64 : 0;
  if (!wait_sums()) return false;
  const bool padding = p.zero_padding && e.row0 + lane >= e.live_end;
  if (part >= steps) release_sums();
#pragma unroll 1
  for (int s = part; s < steps; s += kParts) {
    uint32_t r[64];
    start_sums32(e.taddr + 64u * s, e.empty_sum, *reinterpret_cast<uint32_t(*)[32]>(r));
    start_sums32(e.taddr + 64u * s + 32u, e.empty_sum, *reinterpret_cast<uint32_t(*)[32]>(r + 32));
    if (lane == 0) bulk_wait_group_read<0>();        // meanwhile: the block's last store has been read
    tmem_ld_wait();
    if (s + kParts >= steps) release_sums();
    __syncwarp();
    const uint32_t at = smem_u32(mine) + (uint32_t)lane * 128u, sw = (uint32_t)(lane & 7);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t w[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        w[q] = bf16_pack(__uint_as_float(r[8 * j + 2 * q]), __uint_as_float(r[8 * j + 2 * q + 1]));
        if (padding) w[q] = 0u;
      }
      st_shared_v4(at + (((uint32_t)j ^ sw) << 4), w[0], w[1], w[2], w[3]);
    }
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
      tma_store_3d(&map_y, mine, e.col0 + 64 * s, e.row0, e.group);
      bulk_commit_group();
    }
  }
  return true;
}

// Everything else: steps part, part + kParts, ... of 32 columns; Y and Z by TMA, or row by row.
// kPrecise (tiles of at most 128 columns): the sums come in e.chunks parts of the contraction, which are added here.
template <bool kGated, bool kPrecise, typename Wait, typename Release, typename Next>
__device__ __forceinline__ bool epilogue_full(const TileParams& p, const EpilogueItem& e, const CUtensorMap& map_y,
                                              const CUtensorMap& map_z, uint8_t* mine, int part, int lane,
                                              Wait&& wait_sums, Release&& release_sums, Next&& next_sums) {
  const int row = e.row0 + lane;
  const int steps = e.row0 < e.row_end ? min(e.width, (p.n - e.col0 + 31) & ~31) / 32 : 0;
  uint4 res[4];
  auto load_residual = [&](int s) {
    const int col = e.col0 + 32 * s;
    const uint4* src = reinterpret_cast<const uint4*>(p.residual + (int64_t)row * p.n + col);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      res[j] = row < e.row_end && col + 8 * j < p.n ? src[j] : make_uint4(0u, 0u, 0u, 0u);
  };
  if (p.residual && p.tma && part < steps) load_residual(part);
  const bool padding = p.zero_padding && row >= e.live_end;
  // The two blocks take turns; a block may be rewritten once the store from it has been read.
  uint32_t slot = 0;
  auto next_block = [&](bool known_free) {
    if (!known_free && lane == 0) bulk_wait_group_read<1>();
    __syncwarp();
    uint8_t* b = mine + slot * kBlock16;
    slot ^= 1u;
    return b;
  };
  // One step from its sums (and its gate's partner's).
  auto finish = [&](int s, float (&v)[32], float (&u)[kGated ? 32 : 1]) {
    const int col = e.col0 + 32 * s;
    bool free_block = true;      // the block this step writes first has been read: waited for with the sums
    if (e.bias) {
      add_bias32(e.bias + col, p.n - col, p.tma, v);
      if constexpr (kGated) add_bias32(e.bias + p.n + col, p.n - col, p.tma, u);
    }
    if (padding) {
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] = 0.f;
      if constexpr (kGated) {
#pragma unroll
        for (int i = 0; i < 32; ++i) u[i] = 0.f;
      }
    }
    const int rows_here = col + lane < p.n ? min(32, e.row_end - e.row0) : 0;
    const int64_t out_row = (int64_t)e.group * p.m + e.row0;
    if (p.Z) {
      auto send = [&](const float (&x)[32], int half) {
        uint8_t* b = next_block(free_block);
        free_block = false;
        put_row16(smem_u32(b), lane, x);
        if (!p.tma) {
          __syncwarp();
          block_out16(smem_u32(b), lane, p.Z, PlainBlock{out_row * p.z_pitch + half * p.n + col + lane, p.z_pitch, rows_here});
          __syncwarp();
          return;
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          tma_store_3d(&map_z, b, col, half, e.row0);
          bulk_commit_group();
        }
      };
      send(v, 0);
      if constexpr (kGated) send(u, 1);
    }
    act32_by(p.act, v);
    if constexpr (kGated) {
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] *= u[i];
    }
    const PlainBlock plain{out_row * p.n + col + lane, p.n, rows_here};
    if (p.residual && p.tma) {
#pragma unroll
      for (int j = 0; j < 4; ++j) add_octet(res[j], v + 8 * j);
      if (s + kParts < steps) load_residual(s + kParts);
    } else if (p.residual) {
      __syncwarp();
      block_in16(smem_u32(mine), lane, p.residual, plain);
      __syncwarp();
      add_row16(smem_u32(mine), lane, v);
      __syncwarp();
    }
    if (!p.tma) {
      if (p.out_f32) put_row32(smem_u32(mine), lane, v);
      else put_row16(smem_u32(mine), lane, v);
      __syncwarp();
      if (p.out_f32) block_out32(smem_u32(mine), lane, static_cast<float*>(p.Y), plain, p.accumulate);
      else block_out16(smem_u32(mine), lane, static_cast<uint16_t*>(p.Y), plain);
      __syncwarp();
      return;
    }
    uint8_t* b = mine;
    if (p.out_f32) {
      if (!free_block && lane == 0) bulk_wait_group_read<0>();      // both blocks are one
      __syncwarp();
      put_row32(smem_u32(b), lane, v);
      slot = 0;
    } else {
      b = next_block(free_block);
      put_row16(smem_u32(b), lane, v);
    }
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
      if (p.accumulate) tma_reduce_add_3d(&map_y, b, col, e.row0, e.group);
      else tma_store_3d(&map_y, b, col, e.row0, e.group);
      bulk_commit_group();
      // With f32 the next block written may be the upper half of this one.
      if (p.out_f32 && p.Z) bulk_wait_group_read<0>();
    }
  };
  auto free_first_block = [&] {
    if (lane == 0) {
      if (p.out_f32) bulk_wait_group_read<0>(); else bulk_wait_group_read<1>();
    }
  };
  if constexpr (kPrecise) {
    float sums[2][32];         // steps part and part + kParts; gated: the step's gate and its partner
#pragma unroll
    for (int i = 0; i < 32; ++i) sums[0][i] = sums[1][i] = 0.f;
#pragma unroll 1
    for (int chunk = 0; chunk < e.chunks; ++chunk) {
      if (!wait_sums()) return false;
      const uint32_t taddr = next_sums(chunk + 1 == e.chunks, false);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uint32_t r[32];
        start_sums32(taddr + 32u * part + (uint32_t)i * (kGated ? (uint32_t)e.width : 32u * kParts), e.empty_sum, r);
        tmem_ld_wait();
#pragma unroll
        for (int q = 0; q < 32; ++q) sums[i][q] += __uint_as_float(r[q]);
      }
      release_sums();
      next_sums(chunk + 1 == e.chunks, true);
    }
#pragma unroll
    for (int i = 0; i < (kGated ? 1 : 2); ++i) {
      const int s = part + i * kParts;
      if (s >= steps) break;
      free_first_block();
      if constexpr (kGated) finish(s, sums[0], sums[1]);
      else { float none[1]; finish(s, sums[i], none); }
    }
  } else {
    if (!wait_sums()) return false;
    if (part >= steps) release_sums();
#pragma unroll 1
    for (int s = part; s < steps; s += kParts) {
      const uint32_t c = 32u * s;
      float v[32], u[kGated ? 32 : 1];
      uint32_t r[32];
      [[maybe_unused]] uint32_t q[32];
      start_sums32(e.taddr + c, e.empty_sum, r);
      if constexpr (kGated) start_sums32(e.taddr + (uint32_t)e.width + c, e.empty_sum, q);
      free_first_block();        // meanwhile
      tmem_ld_wait();
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
      if constexpr (kGated) {
#pragma unroll
        for (int i = 0; i < 32; ++i) u[i] = __uint_as_float(q[i]);
      }
      if (s + kParts >= steps) release_sums();
      finish(s, v, u);
    }
  }
  // The next item begins with the first block again: nothing but the last store may be pending from the second.
  if (slot == 1u && lane == 0) bulk_wait_group_read<0>();
  return true;
}

// The products of a launch: one, or the two of a backward pass, whose tiles share the units out between them.
constexpr int kMaxProducts = 2;
struct TileBatch {
  CUtensorMap a[kMaxProducts], b[kMaxProducts], y[kMaxProducts];
  CUtensorMap z;                // of the first product
  CUtensorMap a_rows;           // A of the product with masked_a, by single rows
  TileParams p[kMaxProducts];
  ColumnSums sums;              // of two products, or empty
};

// kTwo: the batch has two products.  One is a form of its own so that its parameters are constants at fixed
// addresses (through an index the epilogue of a 64-deep product took 92 instead of 79 us).
// kPrecise: the tensor cores add to their f32 accumulator by truncation, an error of about 1e-9 of the result per
// element of the contraction (4e-6 at 4096), one way.  Where the output is f32 and the contraction long, the sums are
// taken out every kChunk blocks and added up in registers (to nearest): a few 1e-7 whatever the length.  A warp's
// share of a 128-column tile's sums fits its registers; wider tiles' would not.
constexpr int kChunk = 8;
template <bool kPair, int kTileN, bool kGated, bool kTwo, bool kPrecise>
__global__ void __launch_bounds__(kThreads, 1) linear_tile_kernel(const __grid_constant__ TileBatch batch) {
  using S = Shape<kPair, kTileN>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* stages = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* epi = stages + (size_t)S::kStages * S::kStageBytes;
  Barriers* bars = reinterpret_cast<Barriers*>(epi + kEpiBytes);
  volatile int* abort_flag = &bars->abort_flag;

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const uint32_t rank = kPair ? cluster_ctarank() : 0u;
  const int unit = (int)(kPair ? (blockIdx.x >> 1) : blockIdx.x);
  const int units = (int)(kPair ? (gridDim.x >> 1) : gridDim.x);

  if (threadIdx.x == 0) {
    for (int s = 0; s < S::kStages; ++s) {
      mbar_init(&bars->full[s], 1);
      mbar_init(&bars->empty[s], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars->acc_full[i], 1);
      mbar_init(&bars->acc_empty[i], kEpiWarps * S::kCtas);
    }
    bars->abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_descriptor(&batch.a[0]);
    tma_prefetch_descriptor(&batch.b[0]);
    if (batch.p[0].tma) tma_prefetch_descriptor(&batch.y[0]);
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

  pdl_wait();
  pdl_release();

  // The experts' rows that are live are known on the device only (the first product's, if any).
  if (kPair && batch.p[0].mode == (int)TileMode::kRows && warp == 2) {
    const TileParams& p = batch.p[0];
    int before = 0;
    for (int e0 = 0; e0 < p.experts; e0 += 32) {
      const int e = e0 + lane;
      const int blocks = e < p.experts ? (p.offsets[e + 1] - p.offsets[e]) / kExpertBlock : 0;
      const int mine = (blocks + 1) / 2;
      int sum = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(kFullMask, sum, d);
        if (lane >= d) sum += o;
      }
      if (e < p.experts) bars->pairs_before[e] = before + sum - mine;
      before += __shfl_sync(kFullMask, sum, 31);
    }
    if (lane == 0) bars->pairs_before[p.experts] = before;
  }
  tc_fence_before_sync();
  if constexpr (kPair) cluster_sync(); else __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = bars->tmem_base;

  // A product's walk; before: the items of the product before it.
  auto walk_of = [&](int q, int before, Walk* w) {
    const TileParams& p = batch.p[q];
    w->m_tiles = p.m_tiles;
    w->n_tiles = p.n_tiles;
    int tiles = (int)p.tiles;
    if (p.mode == (int)TileMode::kRows) {
      w->m_tiles = kPair ? bars->pairs_before[p.experts] : p.offsets[p.experts] / kExpertBlock;
      tiles = w->m_tiles * p.n_tiles;
    }
    w->idle = before % units;
    w->lead = w->idle > 0 ? min(p.lead * (units - w->idle), tiles) : 0;
    // The tiles of a last wave that would occupy at most half the units are cut into column halves.
    const int tail = (tiles - w->lead) % units;
    w->whole = p.halves && tiles > units && tail > 0 && 2 * tail <= units ? tiles - tail : tiles;
    w->items = w->whole + 2 * (tiles - w->whole);
  };

  if (warp == 0) {
    // ------------------------------------------------------------------ producer
    if (elect_one()) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      const uint32_t leader_full = kPair ? map_to_cta(smem_u32(&bars->full[0]), 0) : 0u;
      (void)leader_full;
      int before = 0;
      for (int q = 0; q < (kTwo ? 2 : 1); ++q) {
        const TileParams& p = batch.p[q];
        const CUtensorMap* map_a = &batch.a[q];
        const CUtensorMap* map_b = &batch.b[q];
        Walk w;
        walk_of(q, before, &w);
        // The k loop is kept short: one thread issues it, and everything in it delays the next load.
        const bool a_mn = p.a_mn != 0, b_mn = p.b_mn != 0;
        for (Cursor<kPair, kTileN> at(p, w, bars->pairs_before, unit, units); at.valid() && ok; at.next()) {
          const Item it = at.item();
          int row0 = it.row0 + (int)rank * kRowsPerCta;
          // An expert's odd block leaves the pair's second CTA without rows: zeros cost less power than the next
          // expert's rows, and nothing is fetched for them.
          if (kPair && p.mode == (int)TileMode::kRows && row0 >= it.row_end) row0 = (int)p.m;
          const int z_b = p.mode == (int)TileMode::kRows ? it.group : 0;
          const int cols_b = it.cols / S::kCtas, boxes_b = cols_b / 64;
          const uint32_t tx = (uint32_t)(kBytesA + boxes_b * kBoxBytes);
          const int col0 = kGated ? (it.nt * kTileN + it.n_off) / 2 : it.nt * kTileN + it.n_off;
          int cols[S::kBoxesB];      // stored column of every 64-column box of B
#pragma unroll
          for (int j = 0; j < S::kBoxesB; ++j) {
            const int at = (int)rank * cols_b + j * 64;      // accumulator column
            if constexpr (kGated) cols[j] = at < it.cols / 2 ? col0 + at : p.b_up + col0 + at - it.cols / 2;
            else cols[j] = col0 + at;
          }
          auto load = [&](void* dst, const CUtensorMap* map, int c0, int c1, int c2) {
            if constexpr (kPair) tma_load_3d_pair(dst, map, leader_full + (uint32_t)stage * 8u, c0, c1, c2);
            else tma_load_3d(dst, map, &bars->full[stage], c0, c1, c2);
          };
          auto expect = [&](uint32_t bytes) {
            if constexpr (kPair) {
              if (rank == 0) mbar_arrive_expect_tx(&bars->full[stage], 2 * bytes);
            } else {
              mbar_arrive_expect_tx(&bars->full[stage], bytes);
            }
          };
          const bool masked = !kGated && p.masked_a && it.k_row_end % 16 != 0;
          const int whole_blocks = masked ? it.k_blocks - 1 : it.k_blocks;
          int kc = it.k_row0;
          for (int kb = 0; kb < whole_blocks; ++kb, kc += kTileK) {
            if (!(ok = mbar_wait(&bars->empty[stage], phase ^ 1, abort_flag, p.status, 33))) break;
            uint8_t* sa = stages + (size_t)stage * S::kStageBytes;
            uint8_t* sb = sa + kBytesA;
            expect(tx);
            if (a_mn) {
              load(sa, map_a, row0, kc, 0);
              load(sa + kBoxBytes, map_a, row0 + 64, kc, 0);
            } else {
              load(sa, map_a, kc, row0, 0);
            }
#pragma unroll
            for (int j = 0; j < S::kBoxesB; ++j)
              if (j < boxes_b) load(sb + j * kBoxBytes, map_b, b_mn ? cols[j] : kc, b_mn ? kc : cols[j], z_b);
            if (++stage == S::kStages) { stage = 0; phase ^= 1; }
          }
          // The last block with A's rows masked.  Only the steps that are multiplied come: two boxes of 16 rows x 128 bytes
          // each.  (The up to 32 gathers of a tile cost the backward pass of 16,384 rows, 1024 -> 2048 on 32 experts, 1 %:
          // 139.1 -> 140.6 us; 1554 rows on 16 experts 30.7 -> 31.2.  A copy of dY with zeros, which layers with an
          // activation make anyway, would read and write 150 MB there.)
          if (masked && ok && (ok = mbar_wait(&bars->empty[stage], phase ^ 1, abort_flag, p.status, 33))) {
            uint8_t* sa = stages + (size_t)stage * S::kStageBytes;
            expect(tx - (uint32_t)(kTileK / 16 - it.k_steps) * 4096u);
#pragma unroll 1
            for (int r = 0; r < 16 * it.k_steps; r += 4) {
              int from[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) from[i] = kc + r + i < it.k_row_end ? kc + r + i : p.a_rows;
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                uint8_t* dst = sa + h * kBoxBytes + r * 128;
                if constexpr (kPair) tma_gather4_pair(dst, &batch.a_rows, leader_full + (uint32_t)stage * 8u, row0 + 64 * h, from[0], from[1], from[2], from[3]);
                else tma_gather4(dst, &batch.a_rows, &bars->full[stage], row0 + 64 * h, from[0], from[1], from[2], from[3]);
              }
            }
#pragma unroll
            for (int j = 0; j < S::kBoxesB; ++j)
              if (j < boxes_b) load(sa + kBytesA + j * kBoxBytes, map_b, cols[j], kc, z_b);
            if (++stage == S::kStages) { stage = 0; phase ^= 1; }
          }
        }
        before = w.items;
      }
    }
  } else if (warp == 1) {
    // ---------------------------------------------------------------- MMA issuer
    if (rank == 0 && elect_one()) {
      int stage = 0;
      uint32_t phase = 0;
      int buf = 0;
      uint32_t acc_phase = 0;
      bool ok = true;
      int before = 0;
      for (int q = 0; q < (kTwo ? 2 : 1); ++q) {
        const TileParams& p = batch.p[q];
        Walk w;
        walk_of(q, before, &w);
        const uint32_t idesc_tile = instr_desc_bf16(S::kTileM, kTileN, p.a_mn != 0, p.b_mn != 0);
        const uint32_t idesc_half = instr_desc_bf16(S::kTileM, kTileN / 2, p.a_mn != 0, p.b_mn != 0);
        // Across the contraction: 64-column groups one box apart, 16 contraction rows = 2048 bytes.
        // Along it: 8-row groups 1024 bytes apart, 16 elements = 32 bytes along the row.
        const uint32_t step_a = p.a_mn ? 2048u : 32u, step_b = p.b_mn ? 2048u : 32u;
        const uint32_t lbo_a = p.a_mn ? kBoxBytes : 16u, lbo_b = p.b_mn ? kBoxBytes : 16u;
        for (Cursor<kPair, kTileN> at(p, w, bars->pairs_before, unit, units); at.valid() && ok; at.next()) {
          // The place of the tile does not matter here; its width and, by expert, its depth do.
          int k_blocks = p.k_blocks, k_steps = kTileK / 16;
          if (p.mode == (int)TileMode::kContract) {
            const Item it = at.item();
            k_blocks = it.k_blocks;
            k_steps = it.k_steps;
          }
          const uint32_t idesc = at.is_half() ? idesc_half : idesc_tile;
          if (!(ok = mbar_wait(&bars->acc_empty[buf], acc_phase ^ 1, abort_flag, p.status, 34))) break;
          tc_fence_after_sync();
          uint32_t d_tmem = tmem_base + (uint32_t)buf * kAccStride;
          for (int kb = 0; kb < k_blocks; ++kb) {
            if constexpr (kPrecise) {
              if (kb > 0 && kb % kChunk == 0) {      // this part of the sums is complete: on to the other accumulator
                if constexpr (kPair) mma_commit_pair(&bars->acc_full[buf], 3);
                else mma_commit(&bars->acc_full[buf]);
                if (++buf == 2) { buf = 0; acc_phase ^= 1; }
                if (!(ok = mbar_wait(&bars->acc_empty[buf], acc_phase ^ 1, abort_flag, p.status, 38))) break;
                tc_fence_after_sync();
                d_tmem = tmem_base + (uint32_t)buf * kAccStride;
              }
            }
            if (!(ok = mbar_wait(&bars->full[stage], phase, abort_flag, p.status, 35))) break;
            tc_fence_after_sync();
            const uint32_t sa = smem_u32(stages + (size_t)stage * S::kStageBytes);
            const uint32_t sb = sa + kBytesA;
            const int at_kb = kPrecise ? kb % kChunk : kb;
            auto mma = [&](int j) {
              const uint64_t da = smem_desc_sw128(sa + j * step_a, lbo_a, 1024);
              const uint64_t db = smem_desc_sw128(sb + j * step_b, lbo_b, 1024);
              if constexpr (kPair) mma_bf16_ss_pair(d_tmem, da, db, idesc, (at_kb | j) != 0 ? 1u : 0u);
              else mma_bf16_ss(d_tmem, da, db, idesc, (at_kb | j) != 0 ? 1u : 0u);
            };
            if (kb + 1 < k_blocks || k_steps == kTileK / 16) {
#pragma unroll
              for (int j = 0; j < kTileK / 16; ++j) mma(j);
            } else {
              for (int j = 0; j < k_steps; ++j) mma(j);
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
        before = w.items;
      }
    }
  } else {
    // ------------------------------------------------------------------ epilogue
    const int ew = warp - 2;
    const int quarter = warp & 3, part = ew >> 2;      // TMEM lanes 32 quarter ..; share of the columns
    // Under the first tile's main loop.  As a launch of their own between the slopes and the products the sums cost 1.3 us
    // (1000 x 2056) to 5 us (16 experts, 777 x 2 rows, 2000 columns).
    if constexpr (kTwo) {
      if (batch.sums.db) column_sums(batch.sums, (int64_t)blockIdx.x * kEpiWarps + ew, (int64_t)gridDim.x * kEpiWarps, lane);
    }
    uint8_t* mine = epi + (size_t)ew * kEpiBlockBytes;
    int buf = 0;
    uint32_t acc_phase = 0;
    bool ok = true;
    int before = 0;
    for (int q = 0; q < (kTwo ? 2 : 1); ++q) {
      const TileParams& p = batch.p[q];
      const CUtensorMap& map_y = batch.y[q];
      const CUtensorMap& map_z = batch.z;
      Walk w;
      walk_of(q, before, &w);
      Cursor<kPair, kTileN> at(p, w, bars->pairs_before, unit, units);
      Item ahead{};
      if (at.valid()) ahead = at.item();
      bool more = at.valid();
      while (more && ok) {
        // The next item is decoded before this one's steps: its loads (an expert's rows) return under them.
        const Item it = ahead;
        at.next();
        if (at.valid()) ahead = at.item();
        more = at.valid();
        EpilogueItem e;
        e.row0 = it.row0 + (int)rank * kRowsPerCta + quarter * 32;
        e.row_end = it.row_end;
        e.col0 = kGated ? (it.nt * kTileN + it.n_off) / 2 : it.nt * kTileN + it.n_off;
        e.width = kGated ? it.cols / 2 : it.cols;
        e.taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)buf * kAccStride;
        e.bias = p.bias ? p.bias + (int64_t)it.group * p.z_pitch : nullptr;
        e.live_end = it.live_end;
        e.empty_sum = it.k_blocks == 0;
        e.chunks = kPrecise ? max(1, (it.k_blocks + kChunk - 1) / kChunk) : 1;
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
            if constexpr (kPair) mbar_arrive_cluster_relaxed(map_to_cta(smem_u32(&bars->acc_empty[buf]), 0));
            else mbar_arrive(&bars->acc_empty[buf]);
          }
        };
        // Where the current part of the sums is; or, done with it, on to the next part's accumulator.
        auto next_sums = [&](bool last, bool done) {
          if (done && !last && ++buf == 2) { buf = 0; acc_phase ^= 1; }
          return tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)buf * kAccStride;
        };
        if (!kPrecise && p.copy) ok = epilogue_copy(p, e, map_y, mine, part, lane, wait_sums, release_sums);
        else ok = epilogue_full<kGated, kPrecise>(p, e, map_y, map_z, mine, part, lane, wait_sums, release_sums, next_sums);
        if (++buf == 2) { buf = 0; acc_phase ^= 1; }
      }
      // A product's blocks are laid out as its outputs need them: none is pending when the next begins.
      if (lane == 0) bulk_wait_group_read<0>();
      __syncwarp();
      before = w.items;
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

template <bool kPair, int kTileN, bool kGated, bool kTwo, bool kPrecise>
cudaError_t launch_form(const DeviceInfo& dev, const TileBatch& batch, int64_t max_items, cudaStream_t stream) {
  using S = Shape<kPair, kTileN>;
  static PerDeviceOnce once;
  const cudaError_t e = once.run_current([] {
    return cudaFuncSetAttribute(linear_tile_kernel<kPair, kTileN, kGated, kTwo, kPrecise>,
                                cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kSmemBytes);
  });
  if (e != cudaSuccess) return e;
  const int64_t units = std::min<int64_t>(max_items, kPair ? gemm_pair_units(dev.sms) : dev.sms);
  return launch_pdl(linear_tile_kernel<kPair, kTileN, kGated, kTwo, kPrecise>, dim3((unsigned)(units * S::kCtas)), dim3(kThreads),
                    S::kSmemBytes, stream, S::kCtas, batch);
}
template <bool kPair, int kTileN, bool kPrecise>
cudaError_t launch_tile(const DeviceInfo& dev, const TileBatch& batch, bool gated, bool two, int64_t max_items,
                        cudaStream_t stream) {
  if (two)
    return gated ? cudaErrorInvalidValue : launch_form<kPair, kTileN, false, true, kPrecise>(dev, batch, max_items, stream);
  if constexpr (kTileN > 64) {
    if (gated) return launch_form<kPair, kTileN, true, false, kPrecise>(dev, batch, max_items, stream);
  }
  return launch_form<kPair, kTileN, false, false, kPrecise>(dev, batch, max_items, stream);
}

// A tile's column halves are whole 64-column boxes in every CTA (gated: of both halves of W).
bool can_halve(int pair, int tile_n, bool gated) { return tile_n / (pair || gated ? 2 : 1) / 2 >= 64; }

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// Up to these lengths the truncation stays within 1e-6 of the result (a gated layer multiplies two sums).  Parts cost
// 140 instead of 92 us on a cube of 4096, and where one of two products is summed in parts the other is too (f32 weight
// gradients of a gated 4096 x 2048 x 16384: 704 instead of 422 us).
constexpr int kPreciseFrom = 1024, kPreciseGated = 512;

// What a tile costs, in microseconds at full clocks: a contraction block (the MMAs of a 256-column tile, or what the
// roles' loops take for a narrower one) and the epilogue (which the next tile's main loop hides, if it is longer).
struct TileForm {
  int pair, tile_n;
  double block, epilogue;
};
constexpr TileForm kForms[] = {{1, 256, 0.28, 2.2}, {0, 256, 0.33, 2.2}, {1, 128, 0.19, 1.1}, {0, 128, 0.18, 1.1}, {0, 64, 0.175, 0.7}};

// Tiles of a product in a form, and the blocks of the contraction (experts: their numbers are the device's; half a
// tile of padding per expert, and an even share of the rows, are the guess).
int64_t tiles_of(const TileCall& c, const TileForm& f, double* blocks) {
  const int64_t out_cols = c.epi.gated ? f.tile_n / 2 : f.tile_n, tile_m = kRowsPerCta << f.pair;
  const int64_t pairs = c.experts.tokens * c.experts.topk;
  const int64_t live = std::max<int64_t>(1, std::min(pairs, c.experts.experts));
  int64_t m_tiles = (c.m + tile_m - 1) / tile_m, groups = 1;
  *blocks = (double)((c.k + kTileK - 1) / kTileK);
  if (c.mode == TileMode::kRows) m_tiles = std::max<int64_t>(1, (pairs + live * tile_m / 2) / tile_m);
  if (c.mode == TileMode::kContract) {
    groups = c.experts.experts;
    *blocks = (double)pairs / live / kTileK + 0.5;
  }
  return groups * m_tiles * ((c.n + out_cols - 1) / out_cols);
}

bool form_allowed(const TileCall& c, const TileForm& f) {
  if (f.pair && c.m <= kRowsPerCta) return false;
  if (f.pair && c.mode == TileMode::kRows && c.experts.experts >= kPairTable) return false;
  return f.tile_n > 64 || !c.epi.gated;
}

// Estimated time of a call's tiles in a form; lead: see TileParams.
double form_time(const DeviceInfo& dev, const TileCall* calls, int count, const TileForm& f, int* lead) {
  const int64_t units = std::max(1, f.pair ? gemm_pair_units(dev.sms) : dev.sms);
  double each[kMaxProducts];
  int64_t items[kMaxProducts];
  for (int q = 0; q < count; ++q) {
    double blocks = 0;
    items[q] = tiles_of(calls[q], f, &blocks);
    each[q] = std::max(blocks * f.block, f.epilogue) + 0.2;
  }
  *lead = count > 1 ? (int)std::min(1000.0, std::max(1.0, std::floor(each[0] / each[1] + 0.5))) : 0;
  // The units that hold a tile of the first product's last wave, and those that do not.
  const int64_t first = count > 1 ? items[0] : 0, held = first % units;
  double busy = 0, idle = 0;
  int64_t leading = 0;
  if (count > 1) {
    idle = (double)(first / units) * each[0];
    busy = idle + (held > 0 ? each[0] : 0);
    if (held > 0) {
      leading = std::min<int64_t>(*lead * (units - held), items[1]);
      idle += (double)((leading + units - held - 1) / (units - held)) * each[1];
    }
  }
  const int q = count - 1;
  const int64_t rest = items[q] - leading, tail = rest % units;
  const bool cut = can_halve(f.pair, f.tile_n, calls[q].epi.gated) && items[q] > units && 2 * tail <= units;
  const double last = tail == 0 ? 0 : cut ? 0.625 * each[q] : each[q];
  busy += (double)(rest / units) * each[q] + last;
  idle += (double)(rest / units) * each[q] + (tail > held ? last : 0);
  return std::max(busy, idle);
}

TileForm choose_form(const DeviceInfo& dev, const TileCall* calls, int count, bool precise, int* lead) {
  double best = 0;
  int at = -1;
  for (int i = 0; i < (int)(sizeof(kForms) / sizeof(kForms[0])); ++i) {
    bool allowed = !precise || kForms[i].tile_n == 128;
    for (int q = 0; q < count; ++q) allowed = allowed && form_allowed(calls[q], kForms[i]);
    int turn = 0;
    const double cost = form_time(dev, calls, count, kForms[i], &turn);
    if (allowed && (at < 0 || cost < best)) { best = cost; at = i; *lead = turn; }
  }
  return kForms[at < 0 ? 3 : at];
}

}  // namespace

cudaError_t tile_launch(const DeviceInfo& dev, const TileCall* calls, int count, const ColumnSums* sums,
                        cudaStream_t stream, uint64_t* launches) {
  if (count < 1 || count > kMaxProducts || (sums && count != 2)) return cudaErrorInvalidValue;
  for (int q = 0; q < count; ++q)
    if (calls[q].m <= 0 || calls[q].n <= 0 || (q > 0 && calls[q].mode == TileMode::kRows)) return cudaErrorInvalidValue;
  const bool gated = calls[0].epi.gated;
  // f32 results of a long contraction are summed in parts (see kPrecise).
  bool precise = false;
  for (int q = 0; q < count; ++q)
    precise = precise || (calls[q].precise && calls[q].k > (calls[q].epi.gated ? kPreciseGated : kPreciseFrom));
  int lead = 0;
  const TileForm form = choose_form(dev, calls, count, precise, &lead);
  TileBatch batch{};
  if (sums) batch.sums = *sums;
  int64_t items = 0;
  for (int q = 0; q < count; ++q) {
    const TileCall& c = calls[q];
    const LinearEpilogue& ep = c.epi;
    if (ep.gated != gated || (q > 0 && ep.Z)) return cudaErrorInvalidValue;
    const int width = ep.gated ? 2 : 1;
    const int64_t groups = c.mode == TileMode::kContract ? c.experts.experts : 1;
    TileParams& p = batch.p[q];
    p.m = c.m;
    p.n = (int)c.n;
    p.k_blocks = (int)((c.k + kTileK - 1) / kTileK);
    p.b_up = (int)c.b_up;
    p.mode = (uint8_t)c.mode;
    p.a_mn = c.a_mn;
    p.b_mn = c.b_mn;
    p.zero_padding = c.zero_padding;
    p.masked_a = c.masked_a;
    p.a_rows = (int)c.a.rows;
    p.block_expert = c.experts.block_expert;
    p.offsets = c.experts.offsets;
    p.counts = c.experts.counts;
    p.experts = (int)c.experts.experts;
    p.act = (uint8_t)ep.act;
    p.out_f32 = ep.out_f32;
    p.accumulate = ep.accumulate;
    p.tma = c.n % 8 == 0 && aligned16(ep.Y) && aligned16(ep.Z) && aligned16(ep.bias) && aligned16(ep.residual);
    // Y's map below goes by it, and so does the kernel's choice of epilogue: never in a launch that is summed in parts.
    p.copy = !precise && p.tma && !ep.gated && ep.act == kActNone && !ep.bias && !ep.residual && !ep.Z && !ep.out_f32;
    p.z_pitch = (int)(c.n * width);
    p.bias = ep.bias;
    p.residual = ep.residual;
    p.Y = ep.Y;
    p.Z = ep.Z;
    p.status = dev.status;
    p.halves = q + 1 == count && can_halve(form.pair, form.tile_n, ep.gated);
    p.lead = q > 0 ? lead : 0;
    const int64_t tile_m = kRowsPerCta << form.pair, out_cols = ep.gated ? form.tile_n / 2 : form.tile_n;
    const int64_t m_tiles = (c.m + tile_m - 1) / tile_m, n_tiles = (c.n + out_cols - 1) / out_cols;
    // Experts' pairs of blocks: up to one per block.
    const int64_t most = c.mode == TileMode::kRows ? (c.m / kExpertBlock) * n_tiles : groups * m_tiles * n_tiles;
    if (most >= (1ll << 30) || n_tiles >= (1 << 27)) return cudaErrorInvalidValue;   // items are ints
    p.m_tiles = (int)m_tiles;
    p.n_tiles = (int)n_tiles;
    p.tiles = groups * m_tiles * n_tiles;
    items += most;

    cudaError_t e = cudaSuccess;
    if (c.mode == TileMode::kContract || c.k > 0) {
      e = make_tensor_map_3d(&batch.a[q], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, c.a.p, (uint64_t)c.a.cols,
                             (uint64_t)c.a.rows, (uint64_t)c.a.groups, 64, c.a_mn ? 64u : (uint32_t)kRowsPerCta,
                             CU_TENSOR_MAP_SWIZZLE_128B);
      if (e == cudaSuccess)
        e = make_tensor_map_3d(&batch.b[q], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, c.b.p, (uint64_t)c.b.cols,
                               (uint64_t)c.b.rows, (uint64_t)c.b.groups, 64, 64, CU_TENSOR_MAP_SWIZZLE_128B);
      if (e == cudaSuccess && c.masked_a) e = make_gather_map(&batch.a_rows, c.a.p, (uint64_t)c.a.cols, (uint64_t)c.a.rows);
      if (e != cudaSuccess) return e;
    }
    if (p.tma) {
      e = make_tensor_map_3d(&batch.y[q], ep.out_f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
                             ep.out_f32 ? 4 : 2, ep.Y, (uint64_t)c.n, (uint64_t)c.m, (uint64_t)groups, p.copy ? 64 : 32, 32,
                             ep.out_f32 || p.copy ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B);
      // Z's halves are a dimension of their own: a block at the right edge of the first must not reach the second.
      if (e == cudaSuccess && ep.Z)
        e = make_tensor_map_3d_box(&batch.z, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, ep.Z, (uint64_t)c.n, (uint64_t)width,
                                   (uint64_t)c.m, 32, 1, 32, CU_TENSOR_MAP_SWIZZLE_64B);
      if (e != cudaSuccess) return e;
    }
  }
  cudaError_t e;
  const bool two = count == 2;
  switch (form.pair * 1000 + form.tile_n + (precise ? 1 : 0)) {
    case 64: e = launch_tile<false, 64, false>(dev, batch, gated, two, items, stream); break;
    case 128: e = launch_tile<false, 128, false>(dev, batch, gated, two, items, stream); break;
    case 256: e = launch_tile<false, 256, false>(dev, batch, gated, two, items, stream); break;
    case 1128: e = launch_tile<true, 128, false>(dev, batch, gated, two, items, stream); break;
    case 1256: e = launch_tile<true, 256, false>(dev, batch, gated, two, items, stream); break;
    case 129: e = launch_tile<false, 128, true>(dev, batch, gated, two, items, stream); break;
    case 1129: e = launch_tile<true, 128, true>(dev, batch, gated, two, items, stream); break;
    default: return cudaErrorInvalidValue;
  }
  if (e == cudaSuccess) ++*launches;
  return e;
}

}  // namespace morello
