// Products of microscaled 4-bit tensors on the tensor cores, with the linear layers' epilogue.
//
//   z[i,j] = alpha * sum_p (e s)_X[i,p] (e s)_W[j,p] + bias[j],  Y = act(z) + R or act(z_gate) * z_up + R
//
// The block-scaled MMA multiplies 64 elements of e2m1 a step and applies both operands' scales, which it reads from tensor
// memory.  Persistent blocks (or CTA pairs) walk output tiles, warps specialised into a TMA producer, an MMA issuer and
// sixteen epilogue warps.  A stage is 256 elements of the contraction: 128 bytes of every row in the 128-byte swizzle, and
// the scales of those rows, whole 512-byte atoms that the issuer copies to tensor memory ahead of the stage's four MMA
// steps, to one of two places in turn.
//
// A 256-column accumulator and two stages' scales (24 or 48 columns each) leave no room for a second one as wide in the 512
// columns of tensor memory (two of 192 columns would fit; not tried): the epilogue warps take all of a tile's sums into
// registers, hand the accumulator back, and finish the tile under the next one's main loop.  Gated tiles hold 128 columns
// of either half of W.
//
// 4096 x 4096 x 4096 takes 31 us (4.4 PFLOP/s), 8192 x 8192 x 8192 185 to 200 (5.5 to 5.9), gated 4096 x 4096 x (2 x 4096) with
// SiLU 53 (5.2), bound by the hand-over of the one accumulator, the copies of the scales and the board's power.
#include <algorithm>
#include <type_traits>

#include "activation_pairs.cuh"
#include "fp4.h"
#include "tensormap.h"
#include "tile_epilogue.cuh"

namespace morello {
namespace {

using namespace sm100;

constexpr uint32_t kFullMask = 0xffffffffu;
constexpr int kRowsPerCta = 128;
constexpr int kTileK = 256;                          // elements of a stage: 128 bytes of a row
constexpr int kSteps = kTileK / 64;
constexpr int kRowBytes = kTileK / 2;
constexpr int kBytesA = kRowsPerCta * kRowBytes;     // 16 KiB
constexpr int kAccColumns = 256;
constexpr int kScaleColumns = 64;                    // of tensor memory, per stage in turn
constexpr int kTmemColumns = 512;
constexpr int kEpiWarps = 16;                        // four per quarter of the rows
constexpr int kParts = kEpiWarps / 4;
constexpr int kThreads = 128 + 32 * kEpiWarps;       // a warpgroup for the producer and the issuer, four for the epilogue
// 640 threads are launched with 96 registers each; the epilogue's hold up to 64 sums besides.  (Eight epilogue warps with twice
// the sums each leave the schedulers short of warps: 4096 x 4096 x 4096 with GELU, bias and residual 46 us.)
constexpr int kFewRegisters = 32, kManyRegisters = 112;
static_assert(128 * kFewRegisters + 32 * kEpiWarps * kManyRegisters <= kThreads * 96, "registers of the launch");
constexpr int kMaxStages = 8;
constexpr int kBlockBytes = 32 * 64;                 // per warp: a block of 32 rows of 32 bf16 or 16 f32
constexpr int kEpiBytes = kEpiWarps * kBlockBytes;
constexpr int kSmemBudget = 227 * 1024;
constexpr int kRaster = 8;                           // rows of tiles per group of the tile order

template <bool kPair, int kTileN, bool kNv>
struct Shape {
  static constexpr int kCtas = kPair ? 2 : 1;
  static constexpr int kTileM = kRowsPerCta * kCtas;
  static constexpr int kColsB = kTileN / kCtas;                      // rows of W that a CTA loads
  static constexpr int kAtomsK = kNv ? 4 : 2;                        // atoms of a stage across
  static constexpr int kAtomsB = kTileN / kAtomRows;                 // and down, of W (every CTA needs them all)
  static constexpr int kScaleA = kAtomsK * kAtomBytes;
  static constexpr int kBytesB = kColsB * kRowBytes;
  static constexpr int kStageBytes = kBytesA + kBytesB + kScaleA * (1 + kAtomsB);
  static constexpr int kFit = (kSmemBudget - kEpiBytes - 1024 - 512) / kStageBytes;
  static constexpr int kStages = kFit < kMaxStages ? kFit : kMaxStages;
  static constexpr size_t kSmemBytes = (size_t)kStages * kStageBytes + kEpiBytes + 1024 + 512;
  static constexpr int kBuffers = kAccColumns / kTileN;
  static constexpr int kCols = kTileN / kParts;                      // accumulator columns of an epilogue thread
  static_assert(kColsB % kAtomRows == 0 && kAtomsK * 4 * (1 + kAtomsB) <= kScaleColumns, "tile shape");
};

struct Fp4Params {
  int64_t m;
  int n;
  int k_blocks, chunk;           // contraction blocks of a tile, and of a part of its sums
  int m_tiles, n_tiles, tiles;
  int up_rows, up_atoms;         // where the second half of W begins, in rows of W and of its scales' atoms
  uint8_t act, out_f32, tma;
  const float* alpha;
  const uint16_t* bias;
  const uint16_t* residual;
  void* Y;
  uint32_t* status;
};

struct Barriers {
  uint64_t full[kMaxStages];
  uint64_t empty[kMaxStages];
  uint64_t acc_full[2];
  uint64_t acc_empty[2];
  uint64_t res_full[kEpiWarps];      // the residual has come to a warp's block
  uint32_t tmem_base;
  int abort_flag;
};

// The tile's place: tiles are walked in groups of kRaster rows of tiles, row-fastest inside a group, so that the tiles in
// flight share a few rows of X and a few columns of W in L2.  (The last wave's tiles cut into column halves, where those fill
// at most half of the units, gained 1 % on a cube of 4096, and lost as much elsewhere: the board's power is the limit.)
__device__ __forceinline__ void tile_place(const Fp4Params& p, int t, int* mt, int* nt) {
  const int per = kRaster * p.n_tiles, group = t / per, at = t - group * per;
  const int rows = min(kRaster, p.m_tiles - group * kRaster);
  *nt = at / rows;
  *mt = group * kRaster + at - *nt * rows;
}

template <bool kPair, int kTileN, bool kGated, bool kNv>
__global__ void __launch_bounds__(kThreads, 1)
fp4_tile_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                const __grid_constant__ CUtensorMap map_sa, const __grid_constant__ CUtensorMap map_sb,
                const __grid_constant__ CUtensorMap map_y, const __grid_constant__ CUtensorMap map_r, const Fp4Params p) {
  using S = Shape<kPair, kTileN, kNv>;
  constexpr int kOutCols = kGated ? kTileN / 2 : kTileN;
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
    for (int i = 0; i < kEpiWarps; ++i) mbar_init(&bars->res_full[i], 1);
    bars->abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_descriptor(&map_a);
    tma_prefetch_descriptor(&map_b);
    tma_prefetch_descriptor(&map_sa);
    tma_prefetch_descriptor(&map_sb);
    if (p.tma) tma_prefetch_descriptor(&map_y);
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
  tc_fence_before_sync();
  if constexpr (kPair) cluster_sync(); else __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = bars->tmem_base;

  if (warp < 4) {
    registers_down<kFewRegisters>();
    if (warp == 0) {
    // ------------------------------------------------------------------ producer
    if (elect_one()) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      const uint32_t leader_full = kPair ? map_to_cta(smem_u32(&bars->full[0]), 0) : 0u;
      (void)leader_full;
      for (int t = unit; t < p.tiles && ok; t += units) {
        int mt, nt;
        tile_place(p, t, &mt, &nt);
        const int block_a = mt * S::kCtas + (int)rank;      // block of 128 rows of X
        // Rows of W and row of its scales' atoms that accumulator columns 128 a and up stand for.
        auto row_b = [&](int a) { return kGated ? nt * kAtomRows + (a ? p.up_rows : 0) : nt * kTileN + a * kAtomRows; };
        auto atom_b = [&](int a) { return kGated ? nt + (a ? p.up_atoms : 0) : nt * S::kAtomsB + a; };
        auto load = [&](void* dst, const CUtensorMap* map, int c0, int c1, int c2) {
          if constexpr (kPair) tma_load_3d_pair(dst, map, leader_full + (uint32_t)stage * 8u, c0, c1, c2);
          else tma_load_3d(dst, map, &bars->full[stage], c0, c1, c2);
        };
        for (int kb = 0; kb < p.k_blocks; ++kb) {
          if (!(ok = mbar_wait(&bars->empty[stage], phase ^ 1, abort_flag, p.status, 51))) break;
          uint8_t* sa = stages + (size_t)stage * S::kStageBytes;
          uint8_t* sb = sa + kBytesA;
          uint8_t* scales = sb + S::kBytesB;
          if constexpr (kPair) {
            if (rank == 0) mbar_arrive_expect_tx(&bars->full[stage], 2 * S::kStageBytes);
          } else {
            mbar_arrive_expect_tx(&bars->full[stage], S::kStageBytes);
          }
          load(sa, &map_a, kb * kRowBytes, block_a * kRowsPerCta, 0);
#pragma unroll
          for (int a = 0; a < S::kColsB / kAtomRows; ++a)
            load(sb + a * kAtomRows * kRowBytes, &map_b, kb * kRowBytes, row_b(kPair ? (int)rank : a), 0);
          load(scales, &map_sa, 0, kb * S::kAtomsK, block_a);
#pragma unroll
          for (int a = 0; a < S::kAtomsB; ++a)
            load(scales + (1 + a) * S::kScaleA, &map_sb, 0, kb * S::kAtomsK, atom_b(a));
          if (++stage == S::kStages) { stage = 0; phase ^= 1; }
        }
      }
    }
    } else if (warp == 1) {
    // ---------------------------------------------------------------- MMA issuer
    if (rank == 0 && elect_one()) {
      int stage = 0, buf = 0;
      uint32_t phase = 0, acc_phase = 0, turn = 0;
      bool ok = true;
      // Of an empty sum the epilogue awaits no accumulator, and an arrival must not come when the block has gone.
      const int tiles = p.k_blocks > 0 ? p.tiles : 0;
      for (int t = unit; t < tiles && ok; t += units) {
        uint32_t d_tmem = 0;
        int in_chunk = 0;
        for (int kb = 0; kb < p.k_blocks; ++kb) {
          if (in_chunk == p.chunk) {          // this part of the sums is complete
            if constexpr (kPair) mma_commit_pair(&bars->acc_full[buf], 3);
            else mma_commit(&bars->acc_full[buf]);
            if (++buf == S::kBuffers) { buf = 0; acc_phase ^= 1; }
            in_chunk = 0;
          }
          if (in_chunk == 0) {
            if (!(ok = mbar_wait(&bars->acc_empty[buf], acc_phase ^ 1, abort_flag, p.status, 52))) break;
            tc_fence_after_sync();
            d_tmem = tmem_base + (uint32_t)(buf * kTileN);
          }
          if (!(ok = mbar_wait(&bars->full[stage], phase, abort_flag, p.status, 53))) break;
          tc_fence_after_sync();
          const uint32_t sa = smem_u32(stages + (size_t)stage * S::kStageBytes);
          const uint32_t sb = sa + kBytesA, scales = sb + S::kBytesB;
          const uint32_t ta = tmem_base + kAccColumns + turn * kScaleColumns, tb = ta + S::kAtomsK * 4;
          turn ^= 1u;
#pragma unroll
          for (int j = 0; j < S::kAtomsK; ++j) {
            tmem_copy_32x16b<kPair>(ta + 4 * j, smem_desc_rows16(scales + j * kAtomBytes));
#pragma unroll
            for (int a = 0; a < S::kAtomsB; ++a)
              tmem_copy_32x16b<kPair>(tb + 4 * (j * S::kAtomsB + a),
                                      smem_desc_rows16(scales + (1 + a) * S::kScaleA + j * kAtomBytes));
          }
#pragma unroll
          for (int j = 0; j < kSteps; ++j) {
            // 64 elements are 32 bytes along the swizzled row; their scales are an atom's (e4m3) or half of one's.
            const int atom = kNv ? j : j / 2;
            mma_fp4_ss<kPair, kNv>(d_tmem, smem_desc_sw128(sa + j * 32, 16, 1024), smem_desc_sw128(sb + j * 32, 16, 1024),
                                   instr_desc_fp4(S::kTileM, kTileN, kNv, kNv ? 0 : j % 2 * 2), ta + 4 * atom,
                                   tb + 4 * S::kAtomsB * atom, (in_chunk | j) != 0 ? 1u : 0u);
          }
          ++in_chunk;
          if constexpr (kPair) mma_commit_pair(&bars->empty[stage], 3);
          else mma_commit(&bars->empty[stage]);
          if (++stage == S::kStages) { stage = 0; phase ^= 1; }
        }
        if (!ok) break;
        if constexpr (kPair) mma_commit_pair(&bars->acc_full[buf], 3);
        else mma_commit(&bars->acc_full[buf]);
        if (++buf == S::kBuffers) { buf = 0; acc_phase ^= 1; }
      }
      if (!ok) let_copies_land();
    }
    }
  } else {
    registers_up<kManyRegisters>();
    // ------------------------------------------------------------------ epilogue
    const int ew = warp - 4;
    const int quarter = warp & 3, part = ew >> 2;      // TMEM lanes 32 quarter ..; share of the columns
    uint8_t* mine = epi + (size_t)ew * kBlockBytes;
    const uint32_t block = smem_u32(mine);
    const float alpha = p.alpha ? *p.alpha : 1.f;
    // A thread's groups of 32 accumulator columns; gated: the gate's, then their partners'.
    constexpr int kGroups = S::kCols / 32, kOutGroups = kGated ? kGroups / 2 : kGroups;
    static_assert(kOutGroups == 1 || kOutGroups == 2, "steps of an item");
    auto group_column = [&](int g) {
      return kGated ? (g / kOutGroups) * (kTileN / 2) + part * (32 * kOutGroups) + g % kOutGroups * 32
                    : part * S::kCols + g * 32;
    };
    auto scale_and_bias = [&](f32x2(&v)[16], float bias) {
      const f32x2 factor = pair_of(alpha);
      if (p.bias) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          v[i] = fma2(v[i], factor, pair_of(__shfl_sync(kFullMask, bias, 2 * i), __shfl_sync(kFullMask, bias, 2 * i + 1)));
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = mul2(v[i], factor);
      }
    };
    int buf = 0;
    uint32_t acc_phase = 0, res_phase = 0;
    bool ok = true;
    for (int t = unit; t < p.tiles && ok; t += units) {
      int mt, nt;
      tile_place(p, t, &mt, &nt);
      const int64_t row0 = (int64_t)mt * S::kTileM + rank * kRowsPerCta + quarter * 32;
      const int col0 = nt * kOutCols + part * (32 * kOutGroups);      // first output column of this thread
      const int steps = row0 < p.m && col0 < p.n ? min(kOutGroups, (p.n - col0 + 31) / 32) : 0;
      // The residual's blocks come by TMA to where the output's leave from: the first while the sums are awaited, the next
      // while a step is worked on.  (Read straight into registers, 64 bytes of 32 rows, it cost 15 us of 49 on a cube of 4096.)
      const bool res_tma = p.residual && p.tma;
      auto load_residual = [&](int s) {
        if (lane != 0) return;
        bulk_wait_group_read<0>();
        mbar_arrive_expect_tx(&bars->res_full[ew], kBlockBytes);
        tma_load_3d(mine, &map_r, &bars->res_full[ew], col0 + 32 * s, (int)row0, 0);
      };
      if (res_tma && steps > 0) load_residual(0);
      const int rows_here = (int)max((int64_t)0, min((int64_t)32, p.m - row0));
      auto plain_block = [&](int s) {
        const int col = col0 + 32 * s;
        return PlainBlock{row0 * p.n + col + lane, p.n, lane < p.n - col ? rows_here : 0};
      };
      if (p.residual && !p.tma && steps > 0) {      // the same with loads: the next step's rows as far as L2
        if (steps > 1 && lane < rows_here) prefetch_l2(p.residual + (row0 + lane) * p.n + col0 + 32);
        block_in16<32>(block, lane, p.residual, plain_block(0));
      }
      // The bias of a step's columns, one to a lane.
      float bias[kOutGroups], bias_up[kGated ? kOutGroups : 1];
#pragma unroll
      for (int g = 0; g < kOutGroups; ++g) {
        const int col = col0 + 32 * g + lane;
        bias[g] = p.bias && col < p.n ? bf16_value(p.bias[col]) : 0.f;
        if constexpr (kGated) bias_up[g] = p.bias && col < p.n ? bf16_value(p.bias[p.n + col]) : 0.f;
      }
      f32x2 sums[kGroups][16];
      for (int done = 0; done < p.k_blocks && ok; done += p.chunk) {
        ok = mbar_wait(&bars->acc_full[buf], acc_phase, abort_flag, p.status, 54);
        ok = __all_sync(kFullMask, ok);
        tc_fence_after_sync();
        if (!ok) break;
        const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * kTileN);
        if (done == 0) {
          uint32_t r[kGroups][32];
#pragma unroll
          for (int g = 0; g < kGroups; ++g) tmem_ld_32x32(taddr + group_column(g), r[g]);
          tmem_ld_wait();
#pragma unroll
          for (int g = 0; g < kGroups; ++g)
#pragma unroll
            for (int i = 0; i < 16; ++i) sums[g][i] = pair_of(__uint_as_float(r[g][2 * i]), __uint_as_float(r[g][2 * i + 1]));
        } else {
#pragma unroll
          for (int g = 0; g < kGroups; ++g) {
            uint32_t r[32];
            tmem_ld_32x32(taddr + group_column(g), r);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i)
              sums[g][i] = add2(sums[g][i], pair_of(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1])));
          }
        }
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) {
          if constexpr (kPair) mbar_arrive_cluster_relaxed(map_to_cta(smem_u32(&bars->acc_empty[buf]), 0));
          else mbar_arrive(&bars->acc_empty[buf]);
        }
        if (++buf == S::kBuffers) { buf = 0; acc_phase ^= 1; }
      }
      if (!ok) break;
      if (p.k_blocks == 0) {
#pragma unroll
        for (int g = 0; g < kGroups; ++g)
#pragma unroll
          for (int i = 0; i < 16; ++i) sums[g][i] = 0;
      }
      // 32 columns of the output, the s-th of this thread's, from group g of its sums.
      auto step = [&](int s, auto group) {
        constexpr int g = decltype(group)::value;
        const int col = col0 + 32 * s;
        f32x2(&v)[16] = sums[g];
        if (res_tma && s > 0) load_residual(s);
        scale_and_bias(v, bias[g]);
        act_pairs_by(p.act, v);
        if constexpr (kGated) {
          f32x2(&u)[16] = sums[kOutGroups + g];
          scale_and_bias(u, bias_up[g]);
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = mul2(v[i], u[i]);
        }
        const int left = p.n - col;
        const PlainBlock plain = plain_block(s);
        if (res_tma) {
          ok = mbar_wait(&bars->res_full[ew], res_phase, abort_flag, p.status, 55);
          ok = __all_sync(kFullMask, ok);
          res_phase ^= 1u;
          if (!ok) return;
          add_pairs16(block, lane, v);
        } else if (p.residual) {
          if (s > 0) block_in16<16>(block, lane, p.residual, plain);
          __syncwarp();
          add_pairs16(block, lane, v);
        } else if (p.tma) {
          if (lane == 0) bulk_wait_group_read<0>();      // the block's last store has been read
        }
        __syncwarp();
        // The block out, or (f32) the first and the second half of the columns.
        auto send = [&](int at) {
          if (p.tma) {
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
              tma_store_3d(&map_y, mine, col + at, (int)row0, 0);
              bulk_commit_group();
            }
          } else {
            __syncwarp();
            if (p.out_f32) half_block_out32(block, lane, static_cast<float*>(p.Y), PlainBlock{row0 * p.n + col + at, p.n, rows_here}, left - at);
            else block_out16(block, lane, static_cast<uint16_t*>(p.Y), plain);
            __syncwarp();
          }
        };
        if (p.out_f32) {
          put_pairs32<0>(block, lane, v);
          send(0);
          if (left <= 16) return;
          if (p.tma && lane == 0) bulk_wait_group_read<0>();
          __syncwarp();
          put_pairs32<1>(block, lane, v);
          send(16);
        } else {
          put_pairs16(block, lane, v);
          send(0);
        }
      };
      if (steps > 0) step(0, std::integral_constant<int, 0>{});
      if constexpr (kOutGroups > 1) {
        if (steps > 1 && ok) step(1, std::integral_constant<int, 1>{});
      }
    }
    // Shared memory must outlive the engine's reads, and the stores must have been performed before the
    // kernel counts as complete.
    if (lane == 0) bulk_wait_group<0>();
    if (!ok) let_copies_land();      // the residual's
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

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// f32 sums are taken out of the accumulator every so many blocks and added up in registers: the tensor cores add by
// truncation.
constexpr int kPreciseChunk = 4;

template <bool kPair, int kTileN, bool kGated, bool kNv>
cudaError_t launch_form(const DeviceInfo& dev, const Fp4Call& c, Fp4Params p, cudaStream_t stream) {
  using S = Shape<kPair, kTileN, kNv>;
  static PerDeviceOnce once;
  cudaError_t e = once.run_current([] {
    // A launch with fewer registers than its warpgroups end up with would wait for them for good.
    cudaFuncAttributes attr{};
    const cudaError_t got = cudaFuncGetAttributes(&attr, fp4_tile_kernel<kPair, kTileN, kGated, kNv>);
    if (got != cudaSuccess) return got;
    if (attr.numRegs * kThreads < 128 * kFewRegisters + 32 * kEpiWarps * kManyRegisters) return cudaErrorInvalidConfiguration;
    return cudaFuncSetAttribute(fp4_tile_kernel<kPair, kTileN, kGated, kNv>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                (int)S::kSmemBytes);
  });
  if (e != cudaSuccess) return e;
  const int64_t out_cols = kGated ? kTileN / 2 : kTileN;
  const int64_t m_tiles = (c.m + S::kTileM - 1) / S::kTileM, n_tiles = (c.n + out_cols - 1) / out_cols;
  if (n_tiles >= (1 << 27) || m_tiles * n_tiles >= (1ll << 30)) return cudaErrorInvalidValue;      // counted in ints
  p.m_tiles = (int)m_tiles;
  p.n_tiles = (int)n_tiles;
  p.tiles = (int)(m_tiles * n_tiles);
  CUtensorMap a{}, b{}, sa{}, sb{}, y{}, r{};
  const int64_t pitch = fp4_pitch(c.k), across = fp4_atoms_across(kNv, c.k);
  auto rows_map = [&](CUtensorMap* m, const void* q, int64_t rows) {
    return make_tensor_map_3d(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, q, (uint64_t)pitch, (uint64_t)rows, 1, kRowBytes, kAtomRows,
                              CU_TENSOR_MAP_SWIZZLE_128B);
  };
  auto scales_map = [&](CUtensorMap* m, const void* s, int64_t down) {
    return make_tensor_map_3d(m, CU_TENSOR_MAP_DATA_TYPE_UINT32, 4, s, kAtomBytes / 4, (uint64_t)across, (uint64_t)down,
                              kAtomBytes / 4, S::kAtomsK, CU_TENSOR_MAP_SWIZZLE_NONE);
  };
  if (c.k > 0) {
    const int64_t parts = kGated ? 2 : 1;
    if ((e = rows_map(&a, c.X, c.m)) != cudaSuccess || (e = rows_map(&b, c.W, c.wide())) != cudaSuccess ||
        (e = scales_map(&sa, c.X_scales, fp4_atoms_down(c.m))) != cudaSuccess ||
        (e = scales_map(&sb, c.W_scales, parts * fp4_atoms_down(c.n))) != cudaSuccess)
      return e;
  }
  if (p.tma) {
    e = make_tensor_map_3d(&y, c.epi.out_f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
                           c.epi.out_f32 ? 4 : 2, c.epi.Y, (uint64_t)c.n, (uint64_t)c.m, 1, c.epi.out_f32 ? 16 : 32, 32,
                           CU_TENSOR_MAP_SWIZZLE_64B);
    if (e == cudaSuccess && c.epi.residual)
      e = make_tensor_map_3d(&r, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, c.epi.residual, (uint64_t)c.n, (uint64_t)c.m, 1, 32, 32,
                             CU_TENSOR_MAP_SWIZZLE_64B);
    if (e != cudaSuccess) return e;
  }
  const int units = std::min(p.tiles, kPair ? gemm_pair_units(dev.sms) : dev.sms);
  return launch_pdl(fp4_tile_kernel<kPair, kTileN, kGated, kNv>, dim3((unsigned)(units * S::kCtas)), dim3(kThreads),
                    S::kSmemBytes, stream, S::kCtas, a, b, sa, sb, y, r, p);
}

// What a tile costs, in microseconds: a block of 256 elements of the contraction, and the epilogue, which the next tile's
// main loop hides if it is longer.  Measured, of whole calls: pairs and single CTAs 31 and 38 us on a cube of 4096, 14.4 and
// 15.2 on 1024 x 4096 x 4096, 11.3 and 10.1 on 700 x 2048 x 4096, 20.0 and 18.7 on 4096 x 512 x 4096.
struct TileForm {
  bool pair;
  int tile_n;
  double block, epilogue;
};
constexpr TileForm kPair256{true, 256, 0.41, 4.0}, kOne256{false, 256, 0.56, 1.5}, kOne128{false, 128, 0.29, 2.0};
double form_time(const DeviceInfo& dev, const Fp4Call& c, const TileForm& f) {
  const int64_t tile_m = kRowsPerCta << (f.pair ? 1 : 0), cols = c.epi.gated ? f.tile_n / 2 : f.tile_n;
  const int64_t tiles = (c.m + tile_m - 1) / tile_m * ((c.n + cols - 1) / cols);
  const int64_t units = std::max(1, f.pair ? gemm_pair_units(dev.sms) : dev.sms);
  const double blocks = (double)((c.k + kTileK - 1) / kTileK);
  return (double)((tiles + units - 1) / units) * std::max(blocks * f.block, f.epilogue) + f.epilogue;
}

template <bool kNv>
cudaError_t launch_any(const DeviceInfo& dev, const Fp4Call& c, const Fp4Params& p, cudaStream_t stream) {
  const TileForm& one = c.epi.gated ? kOne256 : kOne128;
  const bool pair = c.m > kRowsPerCta && form_time(dev, c, kPair256) < form_time(dev, c, one);
  if (c.epi.gated)
    return pair ? launch_form<true, 256, true, kNv>(dev, c, p, stream) : launch_form<false, 256, true, kNv>(dev, c, p, stream);
  return pair ? launch_form<true, 256, false, kNv>(dev, c, p, stream) : launch_form<false, 128, false, kNv>(dev, c, p, stream);
}

}  // namespace

cudaError_t fp4_tile_launch(const DeviceInfo& dev, const Fp4Call& c, cudaStream_t stream, uint64_t* launches) {
  if (c.m <= 0 || c.n <= 0) return cudaSuccess;
  Fp4Params p{};
  p.m = c.m;
  p.n = (int)c.n;
  p.k_blocks = (int)((c.k + kTileK - 1) / kTileK);
  p.chunk = c.epi.out_f32 ? kPreciseChunk : std::max(1, p.k_blocks);
  p.up_rows = (int)c.n;
  p.up_atoms = (int)fp4_atoms_down(c.n);
  p.act = (uint8_t)c.epi.act;
  p.out_f32 = c.epi.out_f32;
  p.tma = c.n % 8 == 0 && aligned16(c.epi.Y) && aligned16(c.epi.bias) && aligned16(c.epi.residual);
  p.alpha = c.alpha;
  p.bias = c.epi.bias;
  p.residual = c.epi.residual;
  p.Y = c.epi.Y;
  p.status = dev.status;
  const cudaError_t e = c.nv ? launch_any<true>(dev, c, p, stream) : launch_any<false>(dev, c, p, stream);
  if (e == cudaSuccess) ++*launches;
  return e;
}

}  // namespace morello
