// Products of 4-bit tensors on few rows (at most 16): a decoding step.  The call streams the weights once and is bound by
// memory, and on small layers by the chain of a launch: 1 x 2048 x 16384 takes 6.4 us, gated 2 x 8192 7.2, 16 rows with bias,
// GELU and residual 8.3, of which the 17 MB are 2.6.
//
// Here and by the tile kernel, in us (contraction x columns): one row, 16384 x 2048 8.0 and 20.5, 4096 x 4096 5.7 and 8.2, 2048 x 16384 6.6 and 8.2; 16
// rows 9.6 and 20.5, 7.5 and 8.3, 7.8 and 8.2.  Where the contraction is a block or two and finishing the rows, one thread to
// a column of Y, is most of the work, the tile kernel is ahead at 16 rows (512 x 512 4.3 and 3.5, 256 x 65536 11.9 and 8.4) and
// even at 8 (256 x 65536 8.6 and 8.3).  With 32 and 64 rows that holds for wide layers too: 64 rows of 2048 x 16384 12.1 and
// 8.8, but 4096 x 4096 8.5 and 9.4; a form for so many rows is not kept.
//
// The operands trade places: a block owns 128 rows of W (columns of Y; gated: of either half), which become the M side of
// the MMA, and the rows of X, rounded up to 8 or 16, are its N side.  A contraction is cut over the blocks of
// a cluster, as many as keep two blocks on every SM; every block parks its sums in its shared memory and finishes its
// share of the rows, adding the slices in slice order through distributed shared memory, then the epilogue: one launch,
// no scratch, a fixed order.  The weights' first blocks are asked into L2 while the launch before drains.
//
// Gated: a block walks the contraction with its rows of either half in turn, into an accumulator each.
#include <algorithm>
#include <type_traits>

#include "activation.cuh"
#include "fp4.h"
#include "sm100.cuh"
#include "tensormap.h"

namespace morello {
namespace {

using namespace sm100;

constexpr uint32_t kFullMask = 0xffffffffu;
constexpr int kStrip = 128;                  // rows of W
constexpr int kTileK = 256;                  // elements of a stage: 128 bytes of a row
constexpr int kSteps = kTileK / 64;
constexpr int kRowBytes = kTileK / 2;
constexpr int kStripBytes = kStrip * kRowBytes;
constexpr int kThreads = 192;                // producer, issuer, four epilogue warps
constexpr int kMaxStages = 8;
constexpr int kRing = 108 * 1024;            // two blocks to an SM
constexpr int kPrefetch = 8;                 // stages asked into L2 before the wait
constexpr int kScaleColumns = 32;            // of tensor memory, per stage in turn
// Of tensor memory: accumulators of either half, the totals of their parts, and the scales of two stages.  Two blocks to an SM
// take half of it, so that blocks of different clusters never wait for one another's.
constexpr int kTmemColumns = 128;

template <int kRows, bool kNv>
struct Shape {
  static constexpr int kAtomsK = kNv ? 4 : 2;
  static constexpr int kScales = kAtomsK * kAtomBytes;
  static constexpr int kRowsBytes = kRows * kRowBytes;
  static constexpr int kStageBytes = kStripBytes + kRowsBytes + 2 * kScales;
  static constexpr int kFit = kRing / kStageBytes;
  static constexpr int kStages = kFit < kMaxStages ? kFit : kMaxStages;
  static constexpr size_t kSmemBytes = (size_t)kStages * kStageBytes + 1024 + 256;
  static constexpr int kBatch = kRows == 8 ? 4 : 8;      // rows a thread finishes at a time
  static_assert(2 * kRows * kStrip * 4 <= kStages * kStageBytes, "the parked sums reuse the stages");
  static_assert(4 * kRows + 2 * kScaleColumns <= kTmemColumns, "tensor memory");
};

struct Fp4RowsParams {
  int m, n;
  int k_blocks, per_slice, split, chunk;      // blocks of the contraction, of a slice, slices; blocks of a part of the sums
  int up_rows, up_atoms;
  uint8_t gated, act, out_f32;
  const float* alpha;
  const uint16_t* bias;
  const uint16_t* residual;
  void* Y;
  uint32_t* status;
};

struct Barriers {
  uint64_t full[kMaxStages];
  uint64_t empty[kMaxStages];
  uint64_t acc_full, acc_empty;
  uint32_t tmem_base;
  int abort_flag;
};

template <int kAct, int kBatch>
__device__ __forceinline__ void act_batch(float (&v)[kBatch]) {
#pragma unroll
  for (int q = 0; q < kBatch; ++q) v[q] = act_value<kAct>(v[q]);
}
template <int kBatch>
__device__ __forceinline__ void act_batch_by(int act, float (&v)[kBatch]) {
  if (act == kActNone) return;
  if (act == kActRelu) act_batch<kActRelu>(v);
  else if (act == kActGelu) act_batch<kActGelu>(v);
  else if (act == kActGeluTanh) act_batch<kActGeluTanh>(v);
  else act_batch<kActSilu>(v);
}

template <int kRows, bool kNv>
__global__ void __launch_bounds__(kThreads, 2)
fp4_rows_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
                const __grid_constant__ CUtensorMap map_sx, const __grid_constant__ CUtensorMap map_sw, const Fp4RowsParams p) {
  using S = Shape<kRows, kNv>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* stages = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  Barriers* bars = reinterpret_cast<Barriers*>(stages + (size_t)S::kStages * S::kStageBytes);
  volatile int* abort_flag = &bars->abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int slice = (int)blockIdx.x % p.split, strip = (int)blockIdx.x / p.split;
  const int kb0 = slice * p.per_slice, kb1 = min(p.k_blocks, kb0 + p.per_slice);
  const int halves = p.gated ? 2 : 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < S::kStages; ++s) {
      mbar_init(&bars->full[s], 1);
      mbar_init(&bars->empty[s], 1);
    }
    mbar_init(&bars->acc_full, 1);
    mbar_init(&bars->acc_empty, 4);
    bars->abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_descriptor(&map_x);
    tma_prefetch_descriptor(&map_w);
    tma_prefetch_descriptor(&map_sx);
    tma_prefetch_descriptor(&map_sw);
    for (int i = 0; i < min(kPrefetch, (kb1 - kb0) * halves); ++i) {
      const int half = p.gated ? i & 1 : 0, kb = kb0 + (p.gated ? i >> 1 : i);
      tma_prefetch_l2_3d(&map_w, kb * kRowBytes, strip * kStrip + half * p.up_rows, 0);
      tma_prefetch_l2_3d(&map_sw, 0, kb * S::kAtomsK, strip + half * p.up_atoms);
    }
  }
  if (warp == 1) {
    tmem_alloc(&bars->tmem_base, (uint32_t)kTmemColumns);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = bars->tmem_base;
  pdl_wait();
  pdl_release();

  // The epilogue's column; its bias and the residual of its first rows are read while the first blocks come.
  constexpr int kBatch = S::kBatch;
  const int t = (warp & 3) * 32 + lane, col = strip * kStrip + t;
  const bool mine = warp >= 2 && col < p.n;
  float alpha = 1.f, b0 = 0.f, b1 = 0.f;
  uint16_t res[kBatch];
  auto fetch = [&](int row) {
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      const int64_t r = row + q * p.split;
      res[q] = p.residual && mine && r < p.m ? p.residual[r * p.n + col] : (uint16_t)0;
    }
  };
  fetch(slice);
  if (mine) {
    if (p.alpha) alpha = *p.alpha;
    if (p.bias) b0 = bf16_value(p.bias[col]);
    if (p.bias && p.gated) b1 = bf16_value(p.bias[p.n + col]);
  }

  if (warp == 0) {
    // ------------------------------------------------------------------ producer
    if (elect_one()) {
      int stage = 0;
      uint32_t phase = 0;
      for (int i = 0; i < (kb1 - kb0) * halves; ++i) {
        if (!mbar_wait(&bars->empty[stage], phase ^ 1, abort_flag, p.status, 71)) break;
        const int half = p.gated ? i & 1 : 0, kb = kb0 + (p.gated ? i >> 1 : i);
        uint8_t* sw = stages + (size_t)stage * S::kStageBytes;
        uint8_t* sx = sw + kStripBytes;
        uint64_t* full = &bars->full[stage];
        mbar_arrive_expect_tx(full, S::kStageBytes);
        tma_load_3d(sw, &map_w, full, kb * kRowBytes, strip * kStrip + half * p.up_rows, 0);
        tma_load_3d(sx, &map_x, full, kb * kRowBytes, 0, 0);
        tma_load_3d(sx + S::kRowsBytes, &map_sw, full, 0, kb * S::kAtomsK, strip + half * p.up_atoms);
        tma_load_3d(sx + S::kRowsBytes + S::kScales, &map_sx, full, 0, kb * S::kAtomsK, 0);
        if (++stage == S::kStages) { stage = 0; phase ^= 1; }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ---------------------------------------------------------------- MMA issuer
    if (elect_one()) {
      int stage = 0, in_chunk = 0;
      uint32_t phase = 0, acc_phase = 0, turn = 0;
      bool ok = true;
      for (int i = 0; i < (kb1 - kb0) * halves && ok; ++i) {
        const int half = p.gated ? i & 1 : 0;
        if (half == 0 && in_chunk == p.chunk) {      // this part of the sums is complete: on when it has been taken out
          mma_commit(&bars->acc_full);
          if (!(ok = mbar_wait(&bars->acc_empty, acc_phase, abort_flag, p.status, 72))) break;
          tc_fence_after_sync();
          acc_phase ^= 1;
          in_chunk = 0;
        }
        if (!(ok = mbar_wait(&bars->full[stage], phase, abort_flag, p.status, 73))) break;
        tc_fence_after_sync();
        const uint32_t sw = smem_u32(stages + (size_t)stage * S::kStageBytes);
        const uint32_t sx = sw + kStripBytes, scales = sx + S::kRowsBytes;
        const uint32_t d_tmem = tmem_base + (uint32_t)(half * kRows);
        const uint32_t ta = tmem_base + (uint32_t)(kTmemColumns - 2 * kScaleColumns) + turn * kScaleColumns, tb = ta + S::kAtomsK * 4;
        turn ^= 1u;
#pragma unroll
        for (int j = 0; j < S::kAtomsK; ++j) {
          tmem_copy_32x16b<false>(ta + 4 * j, smem_desc_rows16(scales + j * kAtomBytes));
          tmem_copy_32x16b<false>(tb + 4 * j, smem_desc_rows16(scales + S::kScales + j * kAtomBytes));
        }
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
          const int atom = kNv ? j : j / 2;
          mma_fp4_ss<false, kNv>(d_tmem, smem_desc_sw128(sw + j * 32, 16, 1024), smem_desc_sw128(sx + j * 32, 16, 1024),
                                 instr_desc_fp4(kStrip, kRows, kNv, kNv ? 0 : j % 2 * 2), ta + 4 * atom, tb + 4 * atom,
                                 (in_chunk | j) != 0 ? 1u : 0u);
        }
        if (half + 1 == halves) ++in_chunk;
        mma_commit(&bars->empty[stage]);
        if (++stage == S::kStages) { stage = 0; phase ^= 1; }
      }
      // Of an empty sum nobody waits for a part, and an arrival must not come when the block has gone.
      if (ok && kb1 > kb0) mma_commit(&bars->acc_full);
      if (!ok) let_copies_land();
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------------ epilogue: sums out, part by part, and parked
    const uint32_t taddr = tmem_base + ((uint32_t)((warp & 3) * 32) << 16);
    float* part = reinterpret_cast<float*>(stages);      // [half][row][kStrip]; every MMA has completed by then
    uint32_t acc_phase = 0;
    bool ok = true;
    for (int kb = kb0; kb < kb1 && ok; kb += p.chunk) {
      ok = mbar_wait(&bars->acc_full, acc_phase, abort_flag, p.status, 74);
      ok = __all_sync(kFullMask, ok);
      tc_fence_after_sync();
      acc_phase ^= 1;
      if (!ok) break;
      const bool last = kb + p.chunk >= kb1, first = kb == kb0;
      // Parts before the last stay in tensor memory, beside the accumulators: the stages are still in use.
#pragma unroll 1
      for (int h = 0; h < halves; ++h) {
#pragma unroll 1
        for (int g = 0; g < p.m; g += 8) {
          uint32_t r[8], q[8];
          tmem_ld_32x8(taddr + (uint32_t)(h * kRows + g), r);
          if (!first) tmem_ld_32x8(taddr + (uint32_t)((2 + h) * kRows + g), q);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (!first) r[i] = __float_as_uint(__uint_as_float(r[i]) + __uint_as_float(q[i]));
          if (last) {
#pragma unroll
            for (int i = 0; i < 8; ++i) part[(h * kRows + g + i) * kStrip + t] = __uint_as_float(r[i]);
          } else {
            tmem_st_32x8(taddr + (uint32_t)((2 + h) * kRows + g), r);
          }
        }
      }
      if (!last) {
        tmem_st_wait();
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->acc_empty);
      }
    }
    if (kb1 <= kb0) {      // an empty sum
      for (int i = 0; i < halves * kRows; ++i) part[i * kStrip + t] = 0.f;
    }
    tc_fence_before_sync();
    __syncwarp();
  }
  // Every block's sums are parked, in all the cluster.
  __syncwarp();
  if (p.split > 1) cluster_sync(); else __syncthreads();

  if (mine && !*abort_flag) {
    const uint32_t part = smem_u32(stages) + (uint32_t)t * 4u;
    // Rows slice, slice + split, ... of this block's, kBatch of them at a time.
#pragma unroll 1
    for (int row = slice; row < p.m; row += kBatch * p.split) {
      float v[kBatch], u[kBatch], held[kBatch];
#pragma unroll
      for (int q = 0; q < kBatch; ++q) held[q] = bf16_value(res[q]);
      fetch(row + kBatch * p.split);
      auto sum = [&](uint32_t at, float(&x)[kBatch]) {
        float all[8][kBatch];        // every slice's in flight, then added in slice order
#pragma unroll
        for (int s = 0; s < 8; ++s)
          if (s < p.split) {
            const uint32_t peer = map_to_cta(at, (uint32_t)s);
#pragma unroll
            for (int q = 0; q < kBatch; ++q)
              all[s][q] = row + q * p.split < p.m ? ld_cluster_f32(peer + (uint32_t)(row + q * p.split) * (kStrip * 4u)) : 0.f;
          }
#pragma unroll
        for (int q = 0; q < kBatch; ++q) x[q] = all[0][q];
#pragma unroll
        for (int s = 1; s < 8; ++s)
          if (s < p.split) {
#pragma unroll
            for (int q = 0; q < kBatch; ++q) x[q] += all[s][q];
          }
      };
      sum(part, v);
#pragma unroll
      for (int q = 0; q < kBatch; ++q) v[q] = fmaf(v[q], alpha, b0);
      act_batch_by(p.act, v);
      if (p.gated) {
        sum(part + kRows * kStrip * 4u, u);
#pragma unroll
        for (int q = 0; q < kBatch; ++q) v[q] *= fmaf(u[q], alpha, b1);
      }
#pragma unroll
      for (int q = 0; q < kBatch; ++q) {
        const int64_t r = row + q * p.split;
        if (r >= p.m) continue;
        v[q] += held[q];
        if (p.out_f32) static_cast<float*>(p.Y)[r * p.n + col] = v[q];
        else static_cast<uint16_t*>(p.Y)[r * p.n + col] = bf16_round(v[q]);
      }
    }
  }
  // The parked sums have been read by every block of the cluster, the accumulator by every warp.
  __syncwarp();
  if (p.split > 1) cluster_sync();
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  if (warp == 1) {
    __syncwarp();
    tmem_dealloc(tmem_base, (uint32_t)kTmemColumns);
  }
}

constexpr int kPreciseChunk = 4;      // blocks of a part of f32 sums: see the tile kernel

template <int kRows, bool kNv>
cudaError_t launch(const DeviceInfo& dev, const Fp4Call& c, cudaStream_t stream) {
  using S = Shape<kRows, kNv>;
  static PerDeviceOnce once;
  cudaError_t e = once.run_current([] {
    return cudaFuncSetAttribute(fp4_rows_kernel<kRows, kNv>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kSmemBytes);
  });
  if (e != cudaSuccess) return e;
  Fp4RowsParams p{};
  p.m = (int)c.m;
  p.n = (int)c.n;
  p.k_blocks = (int)((c.k + kTileK - 1) / kTileK);
  p.up_rows = (int)c.n;
  p.up_atoms = (int)fp4_atoms_down(c.n);
  p.gated = c.epi.gated;
  p.act = (uint8_t)c.epi.act;
  p.out_f32 = c.epi.out_f32;
  p.alpha = c.alpha;
  p.bias = c.epi.bias;
  p.residual = c.epi.residual;
  p.Y = c.epi.Y;
  p.status = dev.status;
  // Slices: as many as keep two blocks on every SM.
  const int64_t strips = (c.n + kStrip - 1) / kStrip;
  int split = 1;
  while (split < 8 && strips * split * 2 <= 2 * (int64_t)dev.sms && p.k_blocks >= split * 2) split *= 2;
  while (split > 1 && (p.k_blocks + split - 1) / split * (split - 1) >= p.k_blocks) split /= 2;      // no empty slice
  p.split = split;
  p.per_slice = std::max(1, (p.k_blocks + split - 1) / split);
  p.chunk = c.epi.out_f32 ? std::min(p.per_slice, kPreciseChunk) : p.per_slice;
  CUtensorMap x{}, w{}, sx{}, sw{};
  if (c.k > 0) {
    const int64_t pitch = fp4_pitch(c.k), across = fp4_atoms_across(kNv, c.k), parts = p.gated ? 2 : 1;
    auto rows_map = [&](CUtensorMap* m, const void* q, int64_t rows, int box) {
      return make_tensor_map_3d(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, q, (uint64_t)pitch, (uint64_t)rows, 1, kRowBytes, (uint32_t)box,
                                CU_TENSOR_MAP_SWIZZLE_128B);
    };
    auto scales_map = [&](CUtensorMap* m, const void* s, int64_t down) {
      return make_tensor_map_3d(m, CU_TENSOR_MAP_DATA_TYPE_UINT32, 4, s, kAtomBytes / 4, (uint64_t)across, (uint64_t)down,
                                kAtomBytes / 4, S::kAtomsK, CU_TENSOR_MAP_SWIZZLE_NONE);
    };
    if ((e = rows_map(&x, c.X, c.m, kRows)) != cudaSuccess || (e = rows_map(&w, c.W, c.wide(), kStrip)) != cudaSuccess ||
        (e = scales_map(&sx, c.X_scales, 1)) != cudaSuccess ||
        (e = scales_map(&sw, c.W_scales, parts * fp4_atoms_down(c.n))) != cudaSuccess)
      return e;
  }
  return launch_pdl(fp4_rows_kernel<kRows, kNv>, dim3((unsigned)(strips * split)), dim3(kThreads), S::kSmemBytes, stream, split, x, w,
                    sx, sw, p);
}

template <bool kNv>
cudaError_t launch_any(const DeviceInfo& dev, const Fp4Call& c, cudaStream_t stream) {
  return c.m <= 8 ? launch<8, kNv>(dev, c, stream) : launch<16, kNv>(dev, c, stream);
}

}  // namespace

cudaError_t fp4_rows_launch(const DeviceInfo& dev, const Fp4Call& c, cudaStream_t stream, uint64_t* launches) {
  if (c.m <= 0 || c.n <= 0) return cudaSuccess;
  if (c.m > kFp4FewRows) return cudaErrorInvalidValue;
  const cudaError_t e = c.nv ? launch_any<true>(dev, c, stream) : launch_any<false>(dev, c, stream);
  if (e == cudaSuccess) ++*launches;
  return e;
}

}  // namespace morello
