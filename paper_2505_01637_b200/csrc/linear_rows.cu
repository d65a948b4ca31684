// Linear layers on few rows (at most 64, or at most 64 per expert): a decoding step.  The call
// streams the weights once and is bound by memory.
//
// The operands trade places: a block owns 128 columns of W (gated: 64 of either half), which become
// the M side of the MMA, and the rows of X, rounded up to 16, are its N side.  The MMA's cost
// follows the rows instead of a fixed 128, and a column of Y is one thread's.  Few strips and a long
// contraction: it is cut into 2, 4 or 8 slices, one block of a cluster each; every block parks its
// sums in its shared memory and finishes its share of the rows, adding the slices in slice order
// through distributed shared memory, then the epilogue: one launch, no scratch, a fixed order.
// Experts: grid.y is the block of the row layout; a block past the live ones leaves at once.
#include <algorithm>
#include <type_traits>

#include "activation.cuh"
#include "linear.h"
#include "sm100.cuh"
#include "tensormap.h"

namespace morello {
namespace {

using namespace sm100;

constexpr int kStrip = 128;
constexpr int kPart = 512;             // contraction elements of a part of precise sums
constexpr int kSpan = 64;              // contraction elements of one 128-byte swizzle span
constexpr int kThreads = 192;
constexpr int kMaxStages = 8;
constexpr int kPrefetch = 384;         // contraction elements asked into L2 before the wait

template <int kRows>
struct Shape {
  // Contraction elements of a stage.  The loops that issue loads and MMAs are one thread's each and take about 0.2 us
  // a stage, so stages are deep where two blocks' rings still hold three of them.
  static constexpr int kTileK = kRows <= 16 ? 128 : 64;
  static constexpr int kSpans = kTileK / kSpan;
  static constexpr int kStripBytes = kStrip * kTileK * 2;        // of W
  static constexpr int kRowsSpan = kRows * kSpan * 2;            // the rows of X, one span of them
  static constexpr int kStageBytes = kStripBytes + kSpans * kRowsSpan;
  // Two blocks fit an SM: another strip, or the next launch's, streams beside this one, and clusters of half-SM
  // blocks pack well (200 KiB rings: 8192 x 2048 on 32 rows in clusters of eight took two waves, 26 us).
  static constexpr int kRing = 109 * 1024;
  static constexpr int kFit = kRing / kStageBytes;
  static constexpr int kStages = kFit < kMaxStages ? kFit : kMaxStages;
  static constexpr int kPartBlocks = kPart / kTileK;
  static constexpr size_t kSmemBytes = (size_t)kStages * kStageBytes + 1024 + 256;
  static_assert(kRows * kStrip * 4 <= kStages * kStageBytes, "the parked sums reuse the stages");
};

// The strip's columns in one stage, as boxes: W across the contraction ([k][n]) two of 64 columns x kTileK; along it
// ([n][k]) one of 128 columns (gated: two of 64) per span.
template <int kRows, typename Box>
__device__ __forceinline__ void strip_boxes(bool b_mn, bool gated, int col0, int col1, int kc, Box&& box) {
  using S = Shape<kRows>;
  if (b_mn) {
    box(0, col0, kc);
    box(S::kStripBytes / 2, col1, kc);
  } else {
#pragma unroll
    for (int h = 0; h < S::kSpans; ++h) {
      box(h * kStrip * kSpan * 2, kc + h * kSpan, col0);
      if (gated) box(h * kStrip * kSpan * 2 + kStrip * kSpan, kc + h * kSpan, col1);
    }
  }
}

struct RowsParams {
  int m, n;              // rows (dense) and output columns
  int k_blocks, split, per_slice;
  int tmem_cols;
  int b_up;
  uint8_t b_mn, gated, grouped, zero_padding, gather;
  int topk, tokens;
  const int32_t* row_src;
  const int32_t* block_expert;
  const int32_t* offsets;
  const int32_t* counts;
  uint8_t act, out_f32, accumulate;
  int z_pitch;
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
  uint64_t acc_empty[2];     // precise sums
  uint32_t tmem_base;
  int abort_flag;
};

// Rows a thread finishes at a time.  The loops over them are rolled and their addresses advance by additions: a
// block runs this code once, from cold instruction caches and one warp to a scheduler, so every instruction
// counts (sixteen rows unrolled, with products for addresses and a switch per batch: 2.5 us of a 16 us launch).
constexpr int kBatch = 4;

template <int kAct>
__device__ __forceinline__ void act_batch(float (&v)[kBatch]) {
#pragma unroll
  for (int q = 0; q < kBatch; ++q) v[q] = act_value<kAct>(v[q]);
}
__device__ __forceinline__ void act_batch_by(int act, float (&v)[kBatch]) {
  if (act == kActNone) return;
  if (act == kActRelu) act_batch<kActRelu>(v);
  else if (act == kActGelu) act_batch<kActGelu>(v);
  else if (act == kActGeluTanh) act_batch<kActGeluTanh>(v);
  else act_batch<kActSilu>(v);
}

// A thread's column of the outputs and its rows: row i of them is row0 + lead + i * stride of the tensors.
struct Column {
  char* y;
  uint16_t* z;
  const uint16_t* r;
  int64_t y_step, z_step, r_step;     // bytes, elements, elements from one of its rows to the next
  int z_up;                           // from the gate's z to its partner's
  float b0, b1;
  bool f32, accumulate;
  uint16_t held[kBatch];              // residual of the next batch

  __device__ __forceinline__ void hold(int left) {
#pragma unroll
    for (int q = 0; q < kBatch; ++q) held[q] = r && q < left ? r[q * r_step] : (uint16_t)0;
  }
  // The next `left` (at most kBatch are taken) rows from their sums.
  template <bool kGated>
  __device__ __forceinline__ void finish(int act, int left, float (&v)[kBatch], float (&u)[kBatch]) {
    uint16_t res[kBatch];
#pragma unroll
    for (int q = 0; q < kBatch; ++q) res[q] = held[q];
    if (r) {
      r += kBatch * r_step;
      hold(left - kBatch);
    }
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      v[q] += b0;
      if constexpr (kGated) u[q] += b1;
    }
    if (z) {
#pragma unroll
      for (int q = 0; q < kBatch; ++q) {
        if (q < left) {
          z[q * z_step] = bf16_round(v[q]);
          if constexpr (kGated) z[q * z_step + z_up] = bf16_round(u[q]);
        }
      }
      z += kBatch * z_step;
    }
    act_batch_by(act, v);
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      if constexpr (kGated) v[q] *= u[q];
      v[q] += bf16_value(res[q]);
    }
    if (f32) {
#pragma unroll
      for (int q = 0; q < kBatch; ++q) {
        float* dst = reinterpret_cast<float*>(y + q * y_step);
        if (q < left) *dst = accumulate ? *dst + v[q] : v[q];
      }
    } else {
#pragma unroll
      for (int q = 0; q < kBatch; ++q)
        if (q < left) *reinterpret_cast<uint16_t*>(y + q * y_step) = bf16_round(v[q]);
    }
    y += kBatch * y_step;
  }
};

// One slice and no gate: the sums come straight from tensor memory, from one place or (more) two.
template <bool kPrecise>
__device__ __forceinline__ void finish_direct(Column& c, int act, uint32_t sums, uint32_t others, bool more, int rows, bool live) {
#pragma unroll 1
  for (int g = 0; g < rows; g += kBatch) {
    uint32_t r[kBatch];
    tmem_ld_32x4(sums + g, r);
    tmem_ld_wait();
    float v[kBatch], u[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) v[i] = __uint_as_float(r[i]);
    if (kPrecise && more) {
      tmem_ld_32x4(others + g, r);
      tmem_ld_wait();
#pragma unroll
      for (int i = 0; i < kBatch; ++i) v[i] += __uint_as_float(r[i]);
    }
    if (live) c.finish<false>(act, rows - g, v, u);
  }
}

// `rows` rows, `step` bytes of the parked sums apart, from those that the `split` blocks of the cluster have parked
// at shared address `part`.
template <bool kGated>
__device__ __forceinline__ void finish_parked(Column& c, int act, uint32_t part, uint32_t step, int rows, int split) {
#pragma unroll 1
  for (int j = 0; j < rows; j += kBatch) {
    float v[kBatch], u[kBatch];
    auto sum = [&](uint32_t at, float (&x)[kBatch]) {
      float t[8][kBatch];        // every slice's in flight, then added in slice order
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        if (s < split) {
          const uint32_t peer = map_to_cta(at, (uint32_t)s);
#pragma unroll
          for (int q = 0; q < kBatch; ++q) t[s][q] = j + q < rows ? ld_cluster_f32(peer + q * step) : 0.f;
        }
      }
#pragma unroll
      for (int q = 0; q < kBatch; ++q) x[q] = t[0][q];
#pragma unroll
      for (int s = 1; s < 8; ++s)
        if (s < split) {
#pragma unroll
          for (int q = 0; q < kBatch; ++q) x[q] += t[s][q];
        }
    };
    sum(part, v);
    if constexpr (kGated) sum(part + 64 * 4, u);
    c.finish<kGated>(act, rows - j, v, u);
    part += kBatch * step;
  }
}

// kPrecise: the sums come in parts of kPart elements (the tensor cores add by truncation: see the tile kernel), which two
// accumulators take in turn.  While one is filled the epilogue warps add the other to a total, which is in tensor memory
// too: held in registers, with all their code unrolled, 64 rows times 1024 x 32768 took 29 instead of 20.6 us.
template <int kRows, bool kPrecise>
__global__ void __launch_bounds__(kThreads, 2)       // two blocks to an SM, registers included
linear_rows_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                   const RowsParams p) {
  using S = Shape<kRows>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* stages = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  Barriers* bars = reinterpret_cast<Barriers*>(stages + (size_t)S::kStages * S::kStageBytes);
  volatile int* abort_flag = &bars->abort_flag;

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const int slice = (int)blockIdx.x % p.split;
  const int strip = (int)blockIdx.x / p.split;
  const int out_cols = p.gated ? kStrip / 2 : kStrip;       // output columns of a strip
  const int col0 = strip * out_cols;
  const int col1 = p.gated ? p.b_up + col0 : col0 + 64;     // stored column of the second box
  const int kb0 = slice * p.per_slice, kb1 = min(p.k_blocks, kb0 + p.per_slice);

  if (threadIdx.x == 0) {
    for (int s = 0; s < S::kStages; ++s) {
      mbar_init(&bars->full[s], 1);
      mbar_init(&bars->empty[s], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars->acc_full[i], 1);
      mbar_init(&bars->acc_empty[i], 4);
    }
    bars->abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_descriptor(&map_a);
    tma_prefetch_descriptor(&map_b);
    if (!p.grouped) {
      // The weights' first blocks into L2 while the predecessor drains.
      for (int kb = kb0; kb < min(kb1, kb0 + kPrefetch / S::kTileK); ++kb)
        strip_boxes<kRows>(p.b_mn, p.gated, col0, col1, kb * S::kTileK,
                           [&](int, int x, int y) { tma_prefetch_l2_3d(&map_b, x, y, 0); });
    }
  }
  // Which rows, and whose weights.  An expert's are known once the predecessor is done; a dense layer has set
  // everything up by then.
  int row0 = 0, rows = p.m, group = 0;
  if (p.grouped) {
    pdl_wait();
    row0 = (int)blockIdx.y * kExpertBlock;
    group = p.block_expert[blockIdx.y];
    if (group < 0) {            // past the live blocks: the whole cluster leaves
      pdl_release();
      return;
    }
    rows = min(kExpertBlock, p.offsets[group] + p.counts[group] - row0);
  }
  const int chunks = (rows + kRows - 1) / kRows;     // of rows; more than one only when an expert has many

  if (warp == 1) {
    tmem_alloc(&bars->tmem_base, (uint32_t)p.tmem_cols);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = bars->tmem_base;
  if (!p.grouped) pdl_wait();

  // The finishing of rows: this thread's column, and its rows lead + j * stride of a chunk (the cluster's
  // blocks share the rows out; gated: so do the two halves of the threads).
  const int t = (warp & 3) * 32 + lane;                 // the epilogue thread's accumulator lane
  const int j_col = p.gated ? t & 63 : t;
  const int col = col0 + j_col;
  const int stride = p.split * (p.gated ? 2 : 1);
  const int lead = p.gated ? slice * 2 + (t >> 6) : slice;
  const bool direct = p.split == 1 && !p.gated;
  const bool live = warp >= 2 && col < p.n;

  int stage = 0;
  uint32_t phase = 0, acc_phase = 0;
  int buf = 0;
  bool ok = true;
  for (int chunk = 0; chunk < chunks; ++chunk) {
    const int first = row0 + chunk * kRows;
    const int rows_here = min(kRows, rows - chunk * kRows);
    if (warp == 0) {
      // ---------------------------------------------------------------- producer
      // One lane, or, when the rows are gathered through the plan, the whole warp: a lane fetches four rows.
      if (p.gather || elect_one()) {
        const bool lead = !p.gather || lane == 0;
        int from[4] = {0, 0, 0, 0};
        if (p.gather && lane < kRows / 4) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int32_t src = p.row_src[first + lane * 4 + i];
            from[i] = src < 0 ? p.tokens : src / p.topk;      // past the last token: zeros
          }
        }
        for (int kb = kb0; kb < kb1; ++kb) {
          if (ok) ok = mbar_wait(&bars->empty[stage], phase ^ 1, abort_flag, p.status, 41);
          if (p.gather) ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          uint8_t* sb = stages + (size_t)stage * S::kStageBytes;
          uint64_t* full = &bars->full[stage];
          const int kc = kb * S::kTileK;
          if (lead) {
            mbar_arrive_expect_tx(full, S::kStageBytes);
            strip_boxes<kRows>(p.b_mn, p.gated, col0, col1, kc,
                               [&](int at, int x, int y) { tma_load_3d(sb + at, &map_b, full, x, y, group); });
          }
          if (p.gather) __syncwarp();
#pragma unroll
          for (int h = 0; h < S::kSpans; ++h) {
            uint8_t* sa = sb + S::kStripBytes + h * S::kRowsSpan;
            if (!p.gather) tma_load_3d(sa, &map_a, full, kc + h * kSpan, first, 0);
            else if (lane < kRows / 4)
              tma_gather4(sa + lane * 512, &map_a, full, kc + h * kSpan, from[0], from[1], from[2], from[3]);
          }
          if (++stage == S::kStages) { stage = 0; phase ^= 1; }
        }
        if (chunk + 1 == chunks) pdl_release();
      }
      __syncwarp();
    } else if (warp == 1) {
      // -------------------------------------------------------------- MMA issuer
      if (elect_one()) {
        const uint32_t idesc = instr_desc_bf16(kStrip, kRows, p.b_mn != 0, false);
        // W across the contraction: 64-column groups half a strip apart, 16 contraction rows = 2048 bytes.  Along it,
        // like the rows of X: 8-row groups 1024 bytes apart, 16 elements = 32 bytes, a span's rows after another's.
        const uint32_t step = p.b_mn ? 2048u : 32u, lbo = p.b_mn ? (uint32_t)(S::kStripBytes / 2) : 16u;
        const uint32_t span = p.b_mn ? 4u * 2048u : (uint32_t)(kStrip * kSpan * 2);
        uint32_t d_tmem = tmem_base;
        int in_part = 0;
        for (int kb = kb0; kb < kb1 && ok; ++kb) {
          if constexpr (kPrecise) {
            if (in_part == S::kPartBlocks) {
              mma_commit(&bars->acc_full[buf]);
              if (++buf == 2) { buf = 0; acc_phase ^= 1; }
              in_part = 0;
            }
            if (in_part == 0) {
              if (!(ok = mbar_wait(&bars->acc_empty[buf], acc_phase ^ 1, abort_flag, p.status, 44))) break;
              tc_fence_after_sync();
              d_tmem = tmem_base + (uint32_t)(buf * kRows);
            }
          }
          if (!(ok = mbar_wait(&bars->full[stage], phase, abort_flag, p.status, 42))) break;
          tc_fence_after_sync();
          const uint32_t sb = smem_u32(stages + (size_t)stage * S::kStageBytes);
          const uint32_t sa = sb + S::kStripBytes;
#pragma unroll
          for (int j = 0; j < S::kTileK / 16; ++j)
            mma_bf16_ss(d_tmem, smem_desc_sw128(sb + (j / 4) * span + (j % 4) * step, lbo, 1024),
                        smem_desc_sw128(sa + (j / 4) * S::kRowsSpan + (j % 4) * 32, 16, 1024), idesc,
                        (in_part | j) != 0 ? 1u : 0u);
          ++in_part;
          mma_commit(&bars->empty[stage]);
          if (++stage == S::kStages) { stage = 0; phase ^= 1; }
        }
        if (ok) mma_commit(&bars->acc_full[buf]);
        if (kPrecise && ++buf == 2) { buf = 0; acc_phase ^= 1; }
      }
      __syncwarp();
    } else {
      // ---------------------------------------------------------------- epilogue
      const int quarter = warp & 3;
      const int mine = lead < rows_here ? (rows_here - lead + stride - 1) / stride : 0;    // rows of this thread
      Column c;
      c.r = nullptr;
      c.z = nullptr;
      if (live) {
        const int64_t row = first + lead;
        const int size = p.out_f32 ? 4 : 2;
        c.f32 = p.out_f32;
        c.accumulate = p.accumulate;
        c.y = static_cast<char*>(p.Y) + (row * p.n + col) * size;
        c.y_step = (int64_t)stride * p.n * size;
        c.z_step = (int64_t)stride * p.z_pitch;
        c.z_up = p.n;
        c.r_step = (int64_t)stride * p.n;
        if (p.Z) c.z = p.Z + row * p.z_pitch + col;
        if (p.residual) c.r = p.residual + row * p.n + col;
        const uint16_t* bias = p.bias ? p.bias + (int64_t)group * p.z_pitch + col : nullptr;
        c.b0 = bias ? bf16_value(bias[0]) : 0.f;
        c.b1 = bias && p.gated ? bf16_value(bias[p.n]) : 0.f;
        c.hold(mine);
      }
      const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16), total = taddr + 2 * kRows;
      auto wait_sums = [&] {
        ok = mbar_wait(&bars->acc_full[buf], acc_phase, abort_flag, p.status, 43);
        ok = __all_sync(0xffffffffu, ok);
        tc_fence_after_sync();
      };
      auto hand_back = [&] {
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->acc_empty[buf]);
        if (++buf == 2) { buf = 0; acc_phase ^= 1; }
      };
      bool more = false;           // there is a total besides the last part
      if constexpr (kPrecise) {
        ok = true;
#pragma unroll 1
        for (int kb = kb0 + S::kPartBlocks; kb < kb1 && ok; kb += S::kPartBlocks) {
          wait_sums();
          if (!ok) break;
#pragma unroll 1
          for (int g = 0; g < rows_here; g += 16) {
            uint32_t r[16], q[16];
            tmem_ld_32x16(taddr + (uint32_t)(buf * kRows + g), r);
            if (more) {
              tmem_ld_32x16(total + g, q);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) + __uint_as_float(q[i]));
            } else {
              tmem_ld_wait();
            }
            tmem_st_32x16(total + g, r);
          }
          tmem_st_wait();
          hand_back();
          more = true;
        }
        if (ok) wait_sums();
      } else {
        wait_sums();
        acc_phase ^= 1;
      }
      const uint32_t last = taddr + (kPrecise ? (uint32_t)(buf * kRows) : 0u);
      if (ok) {
        // One slice and no gate: the sums are finished as they come.  Otherwise they are parked in the stages (every
        // MMA has completed, so those are free) as part[row][column of the strip].
        float* part = reinterpret_cast<float*>(stages);
        if (direct && kb1 > kb0) {
          finish_direct<kPrecise>(c, p.act, last, total, more, rows_here, live);
        } else {
#pragma unroll 1
          for (int g = 0; g < rows_here; g += 16) {
            uint32_t r[16];
            float sum[16];
            if (kb1 > kb0) {
              tmem_ld_32x16(last + g, r);
              tmem_ld_wait();
            } else {
#pragma unroll
              for (int i = 0; i < 16; ++i) r[i] = 0u;     // an empty sum
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[i] = __uint_as_float(r[i]);
            if (kPrecise && more) {
              tmem_ld_32x16(total + g, r);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 16; ++i) sum[i] += __uint_as_float(r[i]);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) part[(g + i) * kStrip + quarter * 32 + lane] = sum[i];
          }
        }
        if constexpr (kPrecise) hand_back();
        tc_fence_before_sync();
      }
      __syncwarp();
      if (!(direct && kb1 > kb0)) {
        if (p.split > 1) cluster_sync();
        else asm volatile("bar.sync 1, 128;" ::: "memory");     // the epilogue warps alone
        if (live && !*abort_flag) {
          const uint32_t part = smem_u32(stages) + (uint32_t)(lead * kStrip + j_col) * 4u;
          const uint32_t step = (uint32_t)(stride * kStrip) * 4u;
          if (p.gated) finish_parked<true>(c, p.act, part, step, mine, p.split);
          else finish_parked<false>(c, p.act, part, step, mine, p.split);
        }
        __syncwarp();
      }
    }
    if (warp < 2 && p.split > 1) cluster_sync();     // the epilogue warps' barrier above
    // The parked sums have been read by every block of the cluster, the accumulator by every warp.
    if (p.split > 1) {
      __syncwarp();
      cluster_sync();
    } else if (chunk + 1 < chunks) {
      __syncthreads();
    }
    if (chunk + 1 < chunks) {
      tc_fence_after_sync();
      fence_proxy_async_smem();   // ... before the next chunk's copies land on them
    }
  }
  // The rows that hold no token are zeros up to the next multiple of 16 (what the weight gradient's
  // contraction reads); a decoding step does not write 127 rows for one.
  if (live && p.zero_padding) {
    for (int i = rows + lead; i < (rows + 15) / 16 * 16; i += stride) {
      const int64_t row = row0 + i, out = row * p.n + col;
      if (p.Z) {
        p.Z[row * p.z_pitch + col] = 0;
        if (p.gated) p.Z[row * p.z_pitch + p.n + col] = 0;
      }
      if (p.out_f32) static_cast<float*>(p.Y)[out] = 0.f;
      else static_cast<uint16_t*>(p.Y)[out] = 0;
    }
  }

  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  if (warp == 1) {
    __syncwarp();
    tmem_dealloc(tmem_base, (uint32_t)p.tmem_cols);
  }
}

template <int kRows, bool kPrecise>
cudaError_t launch(const DeviceInfo& dev, const TileCall& c, RowsParams p, cudaStream_t stream) {
  using S = Shape<kRows>;
  static PerDeviceOnce once;
  cudaError_t e = once.run_current([] {
    return cudaFuncSetAttribute(linear_rows_kernel<kRows, kPrecise>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                (int)S::kSmemBytes);
  });
  if (e != cudaSuccess) return e;
  const int64_t out_cols = c.epi.gated ? kStrip / 2 : kStrip;
  const int64_t strips = (c.n + out_cols - 1) / out_cols;
  const int64_t blocks = p.grouped ? c.experts.rows / kExpertBlock : 1;
  // Slices: as many as keep every block slot of the device busy with at least 256 elements of the contraction.
  const int64_t live = p.grouped ? std::min(c.experts.experts, c.experts.tokens * c.experts.topk) : 1;
  const int64_t slots = (int64_t)dev.sms * 2;
  p.k_blocks = (int)((c.k + S::kTileK - 1) / S::kTileK);
  int split = 1;
  while (split < 8 && strips * live * split * 2 <= slots && p.k_blocks >= split * 2 * (256 / S::kTileK)) split *= 2;
  while (split > 1 && (p.k_blocks + split - 1) / split * (split - 1) >= p.k_blocks) split /= 2;   // no empty slice
  p.split = split;
  p.per_slice = (p.k_blocks + split - 1) / split;
  p.tmem_cols = 32;
  while (p.tmem_cols < (kPrecise ? 3 * kRows : kRows)) p.tmem_cols *= 2;      // at most half of the SM's: two blocks fit
  if (blocks > 65535 || strips * split >= (1ll << 31)) return cudaErrorInvalidValue;
  CUtensorMap ma{}, mb{};
  if (c.k > 0) {
    e = c.gather_a ? make_gather_map(&ma, c.a.p, (uint64_t)c.a.cols, (uint64_t)c.a.rows)
                   : make_tensor_map_3d(&ma, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, c.a.p, (uint64_t)c.a.cols,
                                        (uint64_t)c.a.rows, 1, kSpan, kRows, CU_TENSOR_MAP_SWIZZLE_128B);
    if (e == cudaSuccess)
      e = make_tensor_map_3d(&mb, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, c.b.p, (uint64_t)c.b.cols, (uint64_t)c.b.rows,
                             (uint64_t)c.b.groups, kSpan, c.b_mn ? S::kTileK : c.epi.gated ? kStrip / 2 : kStrip,
                             CU_TENSOR_MAP_SWIZZLE_128B);
    if (e != cudaSuccess) return e;
  }
  return launch_pdl(linear_rows_kernel<kRows, kPrecise>, dim3((unsigned)(strips * split), (unsigned)blocks), dim3(kThreads),
                    S::kSmemBytes, stream, split, ma, mb, p);
}

}  // namespace

cudaError_t rows_launch(const DeviceInfo& dev, const TileCall& c, cudaStream_t stream, uint64_t* launches) {
  if (c.m <= 0 || c.n <= 0) return cudaSuccess;
  const LinearEpilogue& ep = c.epi;
  RowsParams p{};
  p.grouped = c.mode == TileMode::kRows;
  const int64_t rows = p.grouped ? c.experts.tokens : c.m;
  if (rows > kLinearFewRows || c.a_mn || c.mode == TileMode::kContract) return cudaErrorInvalidValue;
  p.m = (int)c.m;
  p.n = (int)c.n;
  p.b_up = (int)c.b_up;
  p.b_mn = c.b_mn;
  p.gated = ep.gated;
  p.zero_padding = p.grouped && c.zero_padding;
  p.gather = c.gather_a;
  p.topk = (int)std::max<int64_t>(1, c.experts.topk);
  p.tokens = (int)c.experts.tokens;
  p.row_src = c.experts.row_src;
  p.block_expert = c.experts.block_expert;
  p.offsets = c.experts.offsets;
  p.counts = c.experts.counts;
  p.act = (uint8_t)ep.act;
  p.out_f32 = ep.out_f32;
  p.accumulate = ep.accumulate;
  p.z_pitch = (int)(c.n * (ep.gated ? 2 : 1));
  p.bias = ep.bias;
  p.residual = ep.residual;
  p.Y = ep.Y;
  p.Z = ep.Z;
  p.status = dev.status;
  cudaError_t e;
  auto go = [&](auto kernel_rows) {
    constexpr int kRows = decltype(kernel_rows)::value;
    return c.precise && c.k > kPart ? launch<kRows, true>(dev, c, p, stream) : launch<kRows, false>(dev, c, p, stream);
  };
  if (rows <= 16) e = go(std::integral_constant<int, 16>{});
  else if (rows <= 32) e = go(std::integral_constant<int, 32>{});
  else if (rows <= 48) e = go(std::integral_constant<int, 48>{});
  else e = go(std::integral_constant<int, 64>{});
  if (e == cudaSuccess) ++*launches;
  return e;
}

}  // namespace morello
