// Layer norm of rows (mean-centred or root-mean-square), its gradients, and the sums over rows that are the
// gradients of gamma and beta.
//
//   forward    y = (x - mu) r gamma + beta,  mu = mean(x) (rms: 0),  r = 1 / sqrt(mean((x - mu)^2) + eps)
//   backward   h = (x - mu) r, g = dy gamma:  dx = r (g - mean(g) - h mean(g h)) + R  (rms: without mean(g))
//              dgamma = sum over rows of dy h, dbeta = sum over rows of dy
//
// Both passes are bound by memory: a row is read once, held in registers by a team of 32 to 512 threads, reduced and
// written.  The variance is that of the differences from a mean (two sweeps over the registers), never a difference of
// sums.  A warp takes its own mean and the squares about it, and one barrier later every thread joins the warps' three
// numbers (Chan, Golub and LeVeque's formula for joining variances), so a row costs one barrier.
//
// The backward pass's threads keep the columns they own through all the rows of a block, so dgamma and dbeta add up in
// registers; the blocks' sums are joined by a second launch in the order of the blocks.  No atomics: the same sums in the
// same order every time.
#include <algorithm>

#include "../../include/morello.h"
#include "activation.cuh"
#include "linear.h"
#include "sm100.cuh"

namespace morello {
namespace {

using namespace sm100;

constexpr uint32_t kFull = 0xffffffffu;
constexpr int kBlockThreads = 256;

struct NormParams {
  int64_t m;
  int n;
  float eps, inv_n;
  const void* X;
  const uint16_t* gamma;
  const uint16_t* beta;
  uint16_t* Y;
  float* mean;
  float* rstd;
  uint32_t* status;
};

struct NormBackwardParams {
  int64_t m;
  int n;
  float inv_n;
  const void* X;
  const uint16_t* gamma;
  const float* mean;
  const float* rstd;
  const uint16_t* dY;
  const void* R;
  void* dX;
  float* partial;        // [blocks][2][n]: the blocks' sums for dgamma and dbeta
  bool beta;             // dbeta is wanted
  uint32_t* status;
};

// Sum over kLanes neighbouring lanes, in every one of them.
template <int kLanes = 32>
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = kLanes / 2; d > 0; d >>= 1) v += __shfl_xor_sync(kFull, v, d);
  return v;
}

// The barrier of one team of a block (all of it: barrier 0).
template <int kT>
__device__ __forceinline__ void team_barrier(int team) {
  if constexpr (kT >= kBlockThreads) __syncthreads();
  else asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "n"(kT) : "memory");
}

// A thread's columns of a row.  kVec 8: octets of columns, 8 (t + i T) ..., 16-byte accesses; needs n % 8 == 0 and
// aligned tensors.  kVec 1: single columns t + i T.  Element e of the thread: columns are known to exist by has(e).
template <int kT, int kVec, int kIter>
struct Columns {
  int t, n;
  __device__ __forceinline__ int of(int e) const {
    return kVec == 8 ? (t + e / 8 * kT) * 8 + e % 8 : t + e * kT;
  }
  __device__ __forceinline__ bool has(int e) const { return of(e - e % kVec) < n; }
};

// The raw elements of those columns, bf16 or f32, as they came from memory.
template <int kT, int kVec, int kIter, bool kF32>
struct Held {
  static constexpr int kWords = kVec == 1 ? kIter : kVec * kIter * (kF32 ? 4 : 2) / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const void* row, const Columns<kT, kVec, kIter>& c) {
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      const bool has = c.has(i * kVec);
      if constexpr (kVec == 8) {
        constexpr int kQuads = kF32 ? 2 : 1;
#pragma unroll
        for (int q = 0; q < kQuads; ++q) {
          uint4 v = make_uint4(0u, 0u, 0u, 0u);
          if (has) v = reinterpret_cast<const uint4*>(row)[(c.t + i * kT) * kQuads + q];
          uint32_t* o = w + (i * kQuads + q) * 4;
          o[0] = v.x; o[1] = v.y; o[2] = v.z; o[3] = v.w;
        }
      } else if constexpr (kF32) {
        w[i] = has ? __float_as_uint(static_cast<const float*>(row)[c.t + i * kT]) : 0u;
      } else {
        w[i] = has ? (uint32_t)static_cast<const uint16_t*>(row)[c.t + i * kT] << 16 : 0u;
      }
    }
  }
  // Octet i, as four pairs.
  __device__ __forceinline__ void pairs(int i, f32x2 (&v)[4]) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (kF32) v[j] = pair_of(__uint_as_float(w[i * 8 + 2 * j]), __uint_as_float(w[i * 8 + 2 * j + 1]));
      else v[j] = pair_of(bf16_low(w[i * 4 + j]), bf16_high(w[i * 4 + j]));
    }
  }
  __device__ __forceinline__ float get(int e) const {
    if constexpr (kVec == 1 || kF32) return __uint_as_float(w[e]);
    else return e % 2 ? bf16_high(w[e / 2]) : bf16_low(w[e / 2]);
  }
};

// Stores one octet (kVec 8) or one element of a row, column `col` on.
template <int kVec, bool kF32>
__device__ __forceinline__ void put_part(void* row, int col, const float* v) {
  if constexpr (kVec == 8 && kF32) {
    float4* o = reinterpret_cast<float4*>(static_cast<float*>(row) + col);
    o[0] = make_float4(v[0], v[1], v[2], v[3]);
    o[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else if constexpr (kVec == 8) {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(row) + col) =
        make_uint4(bf16_pack(v[0], v[1]), bf16_pack(v[2], v[3]), bf16_pack(v[4], v[5]), bf16_pack(v[6], v[7]));
  } else if constexpr (kF32) {
    static_cast<float*>(row)[col] = v[0];
  } else {
    static_cast<uint16_t*>(row)[col] = bf16_round(v[0]);
  }
}

// One octet or one element of a bf16 vector (gamma, beta); `missing` where there is none.
template <int kVec>
__device__ __forceinline__ void vector_part(const uint16_t* p, int col, float missing, float (&v)[kVec]) {
  if (!p) {
#pragma unroll
    for (int j = 0; j < kVec; ++j) v[j] = missing;
  } else if constexpr (kVec == 8) {
    const uint4 w = __ldg(reinterpret_cast<const uint4*>(p + col));
    v[0] = bf16_low(w.x); v[1] = bf16_high(w.x); v[2] = bf16_low(w.y); v[3] = bf16_high(w.y);
    v[4] = bf16_low(w.z); v[5] = bf16_high(w.z); v[6] = bf16_low(w.w); v[7] = bf16_high(w.w);
  } else {
    v[0] = bf16_value(__ldg(p + col));
  }
}

// Eight elements as four pairs.
__device__ __forceinline__ void octet_pairs(const uint4& w, f32x2 (&v)[4]) {
  v[0] = pair_of(bf16_low(w.x), bf16_high(w.x));
  v[1] = pair_of(bf16_low(w.y), bf16_high(w.y));
  v[2] = pair_of(bf16_low(w.z), bf16_high(w.z));
  v[3] = pair_of(bf16_low(w.w), bf16_high(w.w));
}
// Eight columns of gamma or beta; `missing` where there is no such vector.
__device__ __forceinline__ void vector_pairs(const uint16_t* p, int col, float missing, f32x2 (&v)[4]) {
  if (p) octet_pairs(*reinterpret_cast<const uint4*>(p + col), v);
  else v[0] = v[1] = v[2] = v[3] = pair_of(missing);
}
// An octet of a row in shared memory.
template <bool kF32>
__device__ __forceinline__ void shared_octet(const uint8_t* row, int col, f32x2 (&v)[4]) {
  if constexpr (kF32) {
    const float4* q = reinterpret_cast<const float4*>(row) + col / 4;
    const float4 a = q[0], b = q[1];
    v[0] = pair_of(a.x, a.y);
    v[1] = pair_of(a.z, a.w);
    v[2] = pair_of(b.x, b.y);
    v[3] = pair_of(b.z, b.w);
  } else {
    octet_pairs(*reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(row) + col), v);
  }
}
__device__ __forceinline__ uint32_t bf16_pack_pair(f32x2 v) {
  const float2 f = pair_values(v);
  return bf16_pack(f.x, f.y);
}
template <bool kF32>
__device__ __forceinline__ void put_octet(void* row, int col, const f32x2 (&v)[4]) {
  if constexpr (kF32) {
    float4* o = reinterpret_cast<float4*>(static_cast<float*>(row) + col);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const float2 a = pair_values(v[2 * q]), b = pair_values(v[2 * q + 1]);
      o[q] = make_float4(a.x, a.y, b.x, b.y);
    }
  } else {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(row) + col) =
        make_uint4(bf16_pack_pair(v[0]), bf16_pack_pair(v[1]), bf16_pack_pair(v[2]), bf16_pack_pair(v[3]));
  }
}

// What a warp knows of its part of a row: count values of mean `mean` + off / count, squares about `mean` with sum `squares`.
struct Part {
  float mean, off, squares, count;
};

// Joins the parts of a row: its mean is *base + *off, and the mean square about it is returned.  The mean is kept as two
// numbers, since what a single f32 rounds off a large mean is as large as the differences from it.
__device__ __forceinline__ float shift_of(const Part& a, float m0) { return fmaf(a.count, a.mean - m0, a.off); }
// About the row's mean, which is `away` from the part's: sum (d + away)^2 with sum d = off.
__device__ __forceinline__ float squares_of(const Part& a, float m0, float shift) {
  const float away = a.mean - m0 - shift;
  return a.squares + away * fmaf(a.count, away, 2.f * a.off);
}
template <int kWarps>
__device__ __forceinline__ float join_parts(const Part* parts, float inv_n, float* base, float* off) {
  const float m0 = parts[0].mean;
  float shift = 0.f, squares = 0.f;
  if constexpr (kWarps <= 4) {
#pragma unroll
    for (int w = 0; w < kWarps; ++w) shift += shift_of(parts[w], m0);
    shift *= inv_n;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) squares += squares_of(parts[w], m0, shift);
  } else {      // a lane to a part: so many would not fit the registers
    const int lane = (int)threadIdx.x % 32;
    Part a{m0, 0.f, 0.f, 0.f};
    if (lane < kWarps) a = parts[lane];
    shift = warp_sum(shift_of(a, m0)) * inv_n;
    squares = warp_sum(lane < kWarps ? squares_of(a, m0, shift) : 0.f);
  }
  *base = m0;
  *off = shift;
  return squares * inv_n;
}

// Teams of kT threads, a row each.
template <int kT, int kVec, int kIter, bool kF32, bool kRms>
__global__ void __launch_bounds__(kT > kBlockThreads ? kT : kBlockThreads) norm_kernel(const NormParams p) {
  constexpr int kTeams = kT < kBlockThreads ? kBlockThreads / kT : 1;
  constexpr int kWarps = kT / 32;
  constexpr int kCount = kVec * kIter;
  __shared__ Part parts[2][kTeams][kWarps];
  const int team = (int)threadIdx.x / kT, warp = (int)threadIdx.x % kT / 32, lane = (int)threadIdx.x % 32;
  const Columns<kT, kVec, kIter> c{(int)threadIdx.x % kT, p.n};
  float here = 0.f;
#pragma unroll
  for (int e = 0; e < kCount; ++e) here += c.has(e) ? 1.f : 0.f;
  const float count = warp_sum(here), inv_count = count > 0.f ? 1.f / count : 0.f;
  pdl_wait();
  pdl_release();
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * kTeams + team; row < p.m; row += (int64_t)gridDim.x * kTeams, turn ^= 1) {
    Held<kT, kVec, kIter, kF32> x;
    x.load(static_cast<const char*>(p.X) + row * p.n * (kF32 ? 4 : 2), c);
    Part mine{0.f, 0.f, 0.f, count};
    if constexpr (!kRms) {
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < kCount; ++e) s += x.get(e);
      mine.mean = warp_sum(s) * inv_count;
    }
    float off = 0.f, squares = 0.f;
#pragma unroll
    for (int e = 0; e < kCount; ++e) {
      const float d = c.has(e) ? x.get(e) - mine.mean : 0.f;
      if constexpr (!kRms) off += d;
      squares = fmaf(d, d, squares);
    }
    if constexpr (!kRms) mine.off = warp_sum(off);
    mine.squares = warp_sum(squares);
    float base, shift, square;
    if constexpr (kT == 32) {
      square = join_parts<1>(&mine, p.inv_n, &base, &shift);
    } else {
      if (lane == 0) parts[turn][team][warp] = mine;
      team_barrier<kT>(team);     // the other set of parts is written next: nobody is still reading it behind this barrier
      square = join_parts<kWarps>(parts[turn][team], p.inv_n, &base, &shift);
    }
    const float rstd = 1.f / sqrtf(square + p.eps);
    if (c.t == 0) {
      if (!kRms && p.mean) p.mean[row] = base + shift;
      if (p.rstd) p.rstd[row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      if (!c.has(i * kVec)) continue;
      float gamma[kVec], beta[kVec], y[kVec];
      vector_part<kVec>(p.gamma, c.of(i * kVec), 1.f, gamma);
      vector_part<kVec>(p.beta, c.of(i * kVec), 0.f, beta);
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        const float v = x.get(i * kVec + j);
        const float d = kRms ? v : (v - base) - shift;
        y[j] = fmaf(d * rstd, gamma[j], beta[j]);
      }
      put_part<kVec, false>(p.Y + row * p.n, c.of(i * kVec), y);
    }
  }
}

// The same by octets, two columns an instruction: n % 8 == 0 and 16-byte-aligned tensors.  Teams of 8 to 512 threads; up to
// kIter octets of a row to a thread, kept as they came.
template <int kT, int kIter, bool kF32, bool kRms>
__global__ void __launch_bounds__(kT > kBlockThreads ? kT : kBlockThreads) norm_octets_kernel(const NormParams p) {
  constexpr int kTeams = kT < kBlockThreads ? kBlockThreads / kT : 1;
  constexpr int kLanes = kT < 32 ? kT : 32, kWarps = kT / kLanes;
  __shared__ Part parts[2][kTeams][kWarps];
  const int team = (int)threadIdx.x / kT, warp = (int)threadIdx.x % kT / kLanes, lane = (int)threadIdx.x % kLanes;
  const Columns<kT, 8, kIter> c{(int)threadIdx.x % kT, p.n};
  float here = 0.f;
#pragma unroll
  for (int i = 0; i < kIter; ++i) here += c.has(i * 8) ? 8.f : 0.f;
  const float count = warp_sum<kLanes>(here), inv_count = count > 0.f ? 1.f / count : 0.f;
  pdl_wait();
  pdl_release();
  int turn = 0;
  // Teams of less than a warp leave the loop together: a row past the last is worked on like any other, but neither read nor written.
  for (int64_t row0 = (int64_t)blockIdx.x * kTeams; row0 < p.m; row0 += (int64_t)gridDim.x * kTeams, turn ^= 1) {
    const int64_t row = row0 + team;
    const bool live = row < p.m;
    if (kT >= 32 && !live) break;
    Held<kT, 8, kIter, kF32> x;
    const Columns<kT, 8, kIter> mine_of{c.t, live ? p.n : 0};
    x.load(static_cast<const char*>(p.X) + row * p.n * (kF32 ? 4 : 2), mine_of);
    Part mine{0.f, 0.f, 0.f, count};
    if constexpr (!kRms) {
      f32x2 sums = 0;
#pragma unroll
      for (int i = 0; i < kIter; ++i) {
        f32x2 v[4];
        x.pairs(i, v);
#pragma unroll
        for (int j = 0; j < 4; ++j) sums = add2(sums, v[j]);
      }
      mine.mean = warp_sum<kLanes>(pair_sum(sums)) * inv_count;
    }
    const f32x2 minus_mean = pair_of(-mine.mean);
    f32x2 off = 0, squares = 0;
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      if (!c.has(i * 8)) continue;
      f32x2 v[4];
      x.pairs(i, v);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x2 d = kRms ? v[j] : add2(v[j], minus_mean);
        if constexpr (!kRms) off = add2(off, d);
        squares = fma2(d, d, squares);
      }
    }
    if constexpr (!kRms) mine.off = warp_sum<kLanes>(pair_sum(off));
    mine.squares = warp_sum<kLanes>(pair_sum(squares));
    float base, shift, square;
    if constexpr (kWarps == 1) {
      square = join_parts<1>(&mine, p.inv_n, &base, &shift);
    } else {
      if (lane == 0) parts[turn][team][warp] = mine;
      team_barrier<kT>(team);     // the other set of parts is written next: nobody is still reading it behind this barrier
      square = join_parts<kWarps>(parts[turn][team], p.inv_n, &base, &shift);
    }
    const float rstd = 1.f / sqrtf(square + p.eps);
    if (c.t == 0 && live) {
      if (!kRms && p.mean) p.mean[row] = base + shift;
      if (p.rstd) p.rstd[row] = rstd;
    }
    const f32x2 factor = pair_of(rstd), minus_base = pair_of(-base), shifted = pair_of(-shift * rstd);
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      if (!mine_of.has(i * 8)) continue;
      f32x2 v[4], gamma[4], beta[4], y[4];
      x.pairs(i, v);
      vector_pairs(p.gamma, c.of(i * 8), 1.f, gamma);
      vector_pairs(p.beta, c.of(i * 8), 0.f, beta);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x2 h = kRms ? mul2(v[j], factor) : fma2(add2(v[j], minus_base), factor, shifted);
        y[j] = fma2(h, gamma[j], beta[j]);
      }
      put_octet<false>(p.Y + row * p.n, c.of(i * 8), y);
    }
  }
}

// --- rows through a ring in shared memory ------------------------------------------------------
//
// Whole batches: one or two persistent blocks of 16 warps to an SM.  A group is kTeams neighbouring rows, one to a team, and
// contiguous in memory: one bulk copy per tensor.  The first thread keeps the ring full: behind every group it has worked
// on it waits until the others are done with the one before, and has the next copied there.  The loads' latency, which a
// team that loads its own rows waits out at every row, is behind the ring.  (A warp of its own for the copies takes 3 of
// every 16 registers a thread, since registers are given to four warps at a time.)
constexpr int kRingThreads = 512;
constexpr int kMaxStages = 16;
struct RingBars {
  uint64_t full[kMaxStages];
  uint64_t empty[kMaxStages];
  int abort_flag;
};
struct RingShape {
  int stages;
  uint32_t stage_bytes;        // a group's rows of every tensor
};

struct RingTensor {
  const void* p;
  uint32_t row_bytes;
};
// Starts the copies of the group whose first row is `row` to a stage.
template <int kTeams, int kTensors>
__device__ __forceinline__ void ring_fill(RingBars* bars, uint8_t* smem, const RingShape& ring, int stage, int64_t row, int64_t m,
                                          const RingTensor (&tensors)[kTensors]) {
  const uint32_t rows = (uint32_t)min((int64_t)kTeams, m - row);
  uint32_t bytes = 0;
#pragma unroll
  for (int i = 0; i < kTensors; ++i) bytes += tensors[i].p ? rows * tensors[i].row_bytes : 0u;
  mbar_arrive_expect_tx(&bars->full[stage], bytes);
  uint8_t* dst = smem + (size_t)stage * ring.stage_bytes;
#pragma unroll
  for (int i = 0; i < kTensors; ++i) {
    if (!tensors[i].p) continue;
    bulk_load(dst, static_cast<const uint8_t*>(tensors[i].p) + row * tensors[i].row_bytes, rows * tensors[i].row_bytes,
              &bars->full[stage]);
    dst += kTeams * tensors[i].row_bytes;
  }
}
__device__ __forceinline__ void ring_init(RingBars* bars, int stages) {
  if (threadIdx.x == 0) {
    for (int i = 0; i < stages; ++i) {
      mbar_init(&bars->full[i], 1);
      mbar_init(&bars->empty[i], kRingThreads / 32);
    }
    bars->abort_flag = 0;
    mbar_fence_init();
  }
  __syncthreads();
}
// Where a block is in the ring.
struct RingPlace {
  int stage = 0, before = -1;        // the group's stage, and the one before it
  uint32_t phase = 0, phase_before = 0;
  int64_t fill;                      // first row of the next group to copy
  __device__ __forceinline__ void next(int stages) {
    before = stage;
    phase_before = phase;
    if (++stage == stages) { stage = 0; phase ^= 1; }
  }
};
template <int kTeams, int kTensors>
__device__ __forceinline__ void ring_start(RingBars* bars, uint8_t* smem, const RingShape& ring, RingPlace* at, int64_t m,
                                           const RingTensor (&tensors)[kTensors]) {
  at->fill = (int64_t)blockIdx.x * kTeams;
  if (threadIdx.x != 0) return;
  for (int i = 0; i < ring.stages && at->fill < m; ++i, at->fill += (int64_t)gridDim.x * kTeams)
    ring_fill<kTeams>(bars, smem, ring, i, at->fill, m, tensors);
}
// A warp is done with the group; the first thread has the stage before it filled again.
template <int kTeams, int kTensors>
__device__ __forceinline__ bool ring_next(RingBars* bars, uint8_t* smem, const RingShape& ring, RingPlace* at, int64_t m,
                                          const RingTensor (&tensors)[kTensors], uint32_t* status) {
  bool ok = true;
  __syncwarp();
  if (threadIdx.x % 32 == 0) mbar_arrive(&bars->empty[at->stage]);
  if (threadIdx.x == 0 && at->before >= 0 && at->fill < m) {
    ok = mbar_wait(&bars->empty[at->before], at->phase_before, &bars->abort_flag, status, 61);
    if (ok) ring_fill<kTeams>(bars, smem, ring, at->before, at->fill, m, tensors);
    at->fill += (int64_t)gridDim.x * kTeams;
  }
  at->next(ring.stages);
  return ok;
}
// A thread's octets of gamma or beta, kept through all its rows where registers allow (kIter 2), read again where not.
template <int kT, int kIter>
struct HeldVector {
  static constexpr bool kHold = kIter <= 2;
  const uint16_t* p;
  uint4 w[kHold ? kIter : 1];
  float missing;
  __device__ __forceinline__ HeldVector(const uint16_t* vector, float instead, const Columns<kT, 8, kIter>& c)
      : p(vector), missing(instead) {
    if constexpr (kHold) {
      const uint32_t pair = __float_as_uint(instead) | (__float_as_uint(instead) >> 16);      // exact in bf16
#pragma unroll
      for (int i = 0; i < kIter; ++i)
        w[i] = p && c.has(i * 8) ? *reinterpret_cast<const uint4*>(p + c.of(i * 8)) : make_uint4(pair, pair, pair, pair);
    }
  }
  __device__ __forceinline__ void get(int i, int col, f32x2 (&v)[4]) const {
    if constexpr (kHold) {
      octet_pairs(w[i], v);
    } else {
      vector_pairs(p, col, missing, v);
    }
  }
};
template <int kT>
__device__ __forceinline__ void ring_team_barrier(int team) {
  asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "n"(kT) : "memory");
}

template <int kT, int kIter, bool kF32, bool kRms>
__global__ void __launch_bounds__(kRingThreads, 1)
norm_backward_ring_kernel(const NormBackwardParams p, const RingShape ring) {
  constexpr int kTeams = kRingThreads / kT, kWarps = kT / 32;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ RingBars bars;
  __shared__ float2 parts[2][kTeams][kWarps];
  ring_init(&bars, ring.stages);
  pdl_wait();
  pdl_release();
  const uint32_t row16 = (uint32_t)p.n * 2, row_x = kF32 ? 2 * row16 : row16;
  const RingTensor tensors[3] = {{p.X, row_x}, {p.dY, row16}, {p.dX ? p.R : nullptr, row_x}};
  RingPlace at;
  ring_start<kTeams>(&bars, smem, ring, &at, p.m, tensors);
  const int team = (int)threadIdx.x / kT, warp = (int)threadIdx.x % kT / 32, lane = (int)threadIdx.x % 32;
  const Columns<kT, 8, kIter> c{(int)threadIdx.x % kT, p.n};
  const HeldVector<kT, kIter> gammas(p.gamma, 1.f, c);
  f32x2 sum_g[kIter][4], sum_b[kIter][4];
#pragma unroll
  for (int i = 0; i < kIter; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) sum_g[i][j] = sum_b[i][j] = 0;
  int turn = 0;
  bool ok = true;
  const int64_t step = (int64_t)gridDim.x * kTeams;
  int64_t row = (int64_t)blockIdx.x * kTeams + team;
  // The row's mean and rstd are fetched a row ahead.
  float mean = 0.f, rstd = 0.f, next_mean = 0.f, next_rstd = 0.f;
  auto fetch = [&](int64_t r) {
    if (r < p.m) {
      if constexpr (!kRms) next_mean = p.mean[r];
      next_rstd = p.rstd[r];
    }
  };
  fetch(row);
  for (int64_t row0 = (int64_t)blockIdx.x * kTeams; row0 < p.m; row0 += step, row += step, turn ^= 1) {
    mean = next_mean;
    rstd = next_rstd;
    fetch(row + step);
    if (ok) ok = mbar_wait(&bars.full[at.stage], at.phase, &bars.abort_flag, p.status, 63);
    ok = __all_sync(kFull, ok);
    const bool live = ok && row < p.m;
    const uint8_t* x_row = smem + (size_t)at.stage * ring.stage_bytes + team * row_x;
    const uint8_t* dy_row = smem + (size_t)at.stage * ring.stage_bytes + kTeams * row_x + team * row16;
    const uint8_t* r_row = smem + (size_t)at.stage * ring.stage_bytes + kTeams * (row_x + row16) + team * row_x;
    f32x2 p1 = 0, p2 = 0;      // sums of g and of g (x - mean)
    const f32x2 minus_mean = pair_of(-mean), factor = pair_of(rstd);
    if (live) {
#pragma unroll
      for (int i = 0; i < kIter; ++i) {
        if (!c.has(i * 8)) continue;
        f32x2 x[4], dy[4], gamma[4];
        shared_octet<kF32>(x_row, c.of(i * 8), x);
        shared_octet<false>(dy_row, c.of(i * 8), dy);
        gammas.get(i, c.of(i * 8), gamma);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f32x2 d = kRms ? x[j] : add2(x[j], minus_mean), g = mul2(dy[j], gamma[j]);
          if constexpr (!kRms) p1 = add2(p1, g);
          p2 = fma2(g, d, p2);
          sum_g[i][j] = fma2(dy[j], mul2(d, factor), sum_g[i][j]);
          sum_b[i][j] = add2(sum_b[i][j], dy[j]);
        }
      }
    }
    if (p.dX) {
      float s1 = 0.f, s2 = warp_sum(pair_sum(p2));
      if constexpr (!kRms) s1 = warp_sum(pair_sum(p1));
      if constexpr (kT > 32) {
        if (lane == 0) parts[turn][team][warp] = make_float2(s1, s2);
        ring_team_barrier<kT>(team);
        s1 = s2 = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          s1 += parts[turn][team][w].x;
          s2 += parts[turn][team][w].y;
        }
      }
      // dx = rstd g - rstd mean(g) - (mean(g h) rstd) rstd (x - mean) ...
      const f32x2 constant = pair_of(-rstd * s1 * p.inv_n), slope = pair_of(-(s2 * rstd * p.inv_n * rstd) * rstd);
      if (live) {
#pragma unroll
        for (int i = 0; i < kIter; ++i) {
          if (!c.has(i * 8)) continue;
          f32x2 x[4], dy[4], gamma[4], r[4], out[4];
          shared_octet<kF32>(x_row, c.of(i * 8), x);
          shared_octet<false>(dy_row, c.of(i * 8), dy);
          if (p.R) shared_octet<kF32>(r_row, c.of(i * 8), r);
          gammas.get(i, c.of(i * 8), gamma);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const f32x2 d = kRms ? x[j] : add2(x[j], minus_mean);
            out[j] = fma2(mul2(dy[j], gamma[j]), factor, kRms ? mul2(d, slope) : fma2(d, slope, constant));
            if (p.R) out[j] = add2(out[j], r[j]);
          }
          put_octet<kF32>(static_cast<char*>(p.dX) + row * row_x, c.of(i * 8), out);
        }
      }
    }
    ok = ring_next<kTeams>(&bars, smem, ring, &at, p.m, tensors, p.status) && ok;
  }
  if (!p.partial) return;
  // The teams' sums meet in the ring's memory, whose last copies every team has read.
  if constexpr (kTeams > 1) {
    float* joined = reinterpret_cast<float*>(smem);        // [team][2][kT * kIter * 8]
    constexpr int kWide = kT * kIter * 8;
    asm volatile("bar.sync 15, %0;" ::"n"(kRingThreads) : "memory");     // no team's own
    float* mine = joined + (size_t)team * 2 * kWide;
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      put_octet<true>(mine, c.of(i * 8), sum_g[i]);
      put_octet<true>(mine + kWide, c.of(i * 8), sum_b[i]);
    }
    asm volatile("bar.sync 15, %0;" ::"n"(kRingThreads) : "memory");     // no team's own
    if (!ok) return;
    float* out = p.partial + (int64_t)blockIdx.x * 2 * p.n;
    for (int col = (int)threadIdx.x; col < p.n; col += kRingThreads) {
      float g = 0.f, b = 0.f;
#pragma unroll
      for (int t = 0; t < kTeams; ++t) {
        g += joined[(size_t)t * 2 * kWide + col];
        b += joined[(size_t)t * 2 * kWide + kWide + col];
      }
      out[col] = g;
      if (p.beta) out[p.n + col] = b;
    }
  } else {
    if (!ok) return;
    float* out = p.partial + (int64_t)blockIdx.x * 2 * p.n;
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      if (!c.has(i * 8)) continue;
      put_octet<true>(out, c.of(i * 8), sum_g[i]);
      if (p.beta) put_octet<true>(out + p.n, c.of(i * 8), sum_b[i]);
    }
  }
}

// Rows longer than a team's registers: a block of 1024 threads sweeps the row three times (the second and third time from
// L2, where it fits).
constexpr int kLongThreads = 1024;
__device__ __forceinline__ float block_sum(float v, float* shared) {
  v = warp_sum(v);
  __syncthreads();          // the last sum has been read
  if (threadIdx.x % 32 == 0) shared[threadIdx.x / 32] = v;
  __syncthreads();
  return warp_sum(shared[threadIdx.x % 32]);
}
template <bool kF32>
__device__ __forceinline__ float element(const void* p, int64_t i) {
  if constexpr (kF32) return static_cast<const float*>(p)[i];
  else return bf16_value(static_cast<const uint16_t*>(p)[i]);
}

template <bool kF32, bool kRms>
__global__ void __launch_bounds__(kLongThreads) norm_long_kernel(const NormParams p) {
  __shared__ float shared[kLongThreads / 32];
  pdl_wait();
  pdl_release();
  for (int64_t row = blockIdx.x; row < p.m; row += gridDim.x) {
    const int64_t at = row * p.n;
    float base = 0.f, shift = 0.f;
    if constexpr (!kRms) {
      float s = 0.f;
      for (int64_t j = threadIdx.x; j < p.n; j += kLongThreads) s += element<kF32>(p.X, at + j);
      base = block_sum(s, shared) * p.inv_n;
    }
    float off = 0.f, squares = 0.f;
    for (int64_t j = threadIdx.x; j < p.n; j += kLongThreads) {
      const float d = element<kF32>(p.X, at + j) - base;
      off += d;
      squares = fmaf(d, d, squares);
    }
    if constexpr (!kRms) shift = block_sum(off, shared) * p.inv_n;
    const float square = block_sum(squares, shared) * p.inv_n - shift * shift;
    const float rstd = 1.f / sqrtf(square + p.eps);
    if (threadIdx.x == 0) {
      if (!kRms && p.mean) p.mean[row] = base + shift;
      if (p.rstd) p.rstd[row] = rstd;
    }
    for (int64_t j = threadIdx.x; j < p.n; j += kLongThreads) {
      const float d = (element<kF32>(p.X, at + j) - base) - shift;
      const float g = p.gamma ? bf16_value(p.gamma[j]) : 1.f, b = p.beta ? bf16_value(p.beta[j]) : 0.f;
      p.Y[at + j] = bf16_round(fmaf(d * rstd, g, b));
    }
  }
}

// The gradients, by the same teams.  kSums: dgamma (and dbeta) are wanted.
template <int kT, int kVec, int kIter, bool kF32, bool kRms, bool kSums>
__global__ void __launch_bounds__(kBlockThreads) norm_backward_kernel(const NormBackwardParams p) {
  constexpr int kTeams = kBlockThreads / kT;
  constexpr int kWarps = kT / 32;
  constexpr int kCount = kVec * kIter;
  __shared__ float2 parts[2][kTeams][kWarps];
  const int team = (int)threadIdx.x / kT, warp = (int)threadIdx.x % kT / 32, lane = (int)threadIdx.x % 32;
  const Columns<kT, kVec, kIter> c{(int)threadIdx.x % kT, p.n};
  float sum_g[kSums ? kCount : 1], sum_b[kSums ? kCount : 1];
  if constexpr (kSums) {
#pragma unroll
    for (int e = 0; e < kCount; ++e) sum_g[e] = sum_b[e] = 0.f;
  }
  pdl_wait();
  pdl_release();
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * kTeams + team; row < p.m; row += (int64_t)gridDim.x * kTeams, turn ^= 1) {
    const int64_t at = row * p.n;
    Held<kT, kVec, kIter, kF32> x;
    Held<kT, kVec, kIter, false> dy;
    Held<kT, kVec, kIter, kF32> r;
    x.load(static_cast<const char*>(p.X) + at * (kF32 ? 4 : 2), c);
    dy.load(p.dY + at, c);
    if (p.R) r.load(static_cast<const char*>(p.R) + at * (kF32 ? 4 : 2), c);
    const float mean = kRms ? 0.f : p.mean[row], rstd = p.rstd[row];
    float s1 = 0.f, s2 = 0.f;      // sums of g and of g (x - mean)
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      float gamma[kVec];
      vector_part<kVec>(c.has(i * kVec) ? p.gamma : nullptr, c.of(i * kVec), 1.f, gamma);
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        const int e = i * kVec + j;
        const float v = dy.get(e), d = x.get(e) - mean, g = v * gamma[j];
        if constexpr (!kRms) s1 += g;
        s2 = fmaf(g, c.has(e) ? d : 0.f, s2);
        if constexpr (kSums) {
          sum_g[e] = fmaf(v, c.has(e) ? d * rstd : 0.f, sum_g[e]);
          sum_b[e] += v;
        }
      }
    }
    if (!p.dX) continue;
    if constexpr (!kRms) s1 = warp_sum(s1);
    s2 = warp_sum(s2);
    if constexpr (kT > 32) {
      if (lane == 0) parts[turn][team][warp] = make_float2(s1, s2);
      team_barrier<kT>(team);
      s1 = s2 = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        s1 += parts[turn][team][w].x;
        s2 += parts[turn][team][w].y;
      }
    }
    const float mean_g = s1 * p.inv_n, slope = s2 * rstd * p.inv_n * rstd;     // slope: mean(g h) r, to go with x - mean
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      if (!c.has(i * kVec)) continue;
      float gamma[kVec], out[kVec];
      vector_part<kVec>(p.gamma, c.of(i * kVec), 1.f, gamma);
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        const int e = i * kVec + j;
        const float g = dy.get(e) * gamma[j], d = x.get(e) - mean;
        const float inner = fmaf(-slope, d, kRms ? g : g - mean_g);
        out[j] = p.R ? fmaf(rstd, inner, r.get(e)) : rstd * inner;
      }
      put_part<kVec, kF32>(static_cast<char*>(p.dX) + at * (kF32 ? 4 : 2), c.of(i * kVec), out);
    }
  }
  if constexpr (kSums) {
    // The teams of the block one after the other, then the block's row of partial sums.
    float* mine = p.partial + (int64_t)blockIdx.x * 2 * p.n;
    extern __shared__ float joined[];      // [2][kT * kCount] when there are several teams
    if constexpr (kTeams > 1) {
      for (int turn_of = kTeams - 1; turn_of > 0; --turn_of) {
        if (team == turn_of) {
#pragma unroll
          for (int e = 0; e < kCount; ++e) {
            const bool first = turn_of == kTeams - 1;
            float* s = joined + e * kT + c.t;
            s[0] = first ? sum_g[e] : s[0] + sum_g[e];
            s[kT * kCount] = first ? sum_b[e] : s[kT * kCount] + sum_b[e];
          }
        }
        __syncthreads();
      }
      if (team == 0) {
#pragma unroll
        for (int e = 0; e < kCount; ++e) {
          sum_g[e] += joined[e * kT + c.t];
          sum_b[e] += joined[e * kT + c.t + kT * kCount];
        }
      }
    }
    if (team == 0) {
#pragma unroll
      for (int i = 0; i < kIter; ++i) {
        if (!c.has(i * kVec)) continue;
        put_part<kVec, true>(mine, c.of(i * kVec), sum_g + i * kVec);
        if (p.beta) put_part<kVec, true>(mine + p.n, c.of(i * kVec), sum_b + i * kVec);
      }
    }
  }
}

// Rows longer than that: dx by a block of 1024 threads that sweeps the row twice, and the sums over rows by a launch of
// their own, 32 columns x 32 rows of threads to a block, that reads x and dy again.
template <bool kF32, bool kRms>
__global__ void __launch_bounds__(kLongThreads) norm_backward_long_kernel(const NormBackwardParams p) {
  __shared__ float shared[kLongThreads / 32];
  pdl_wait();
  pdl_release();
  for (int64_t row = blockIdx.x; row < p.m; row += gridDim.x) {
    const int64_t at = row * p.n;
    const float mean = kRms ? 0.f : p.mean[row], rstd = p.rstd[row];
    float s1 = 0.f, s2 = 0.f;
    for (int64_t j = threadIdx.x; j < p.n; j += kLongThreads) {
      const float g = bf16_value(p.dY[at + j]) * (p.gamma ? bf16_value(p.gamma[j]) : 1.f);
      s1 += g;
      s2 = fmaf(g, element<kF32>(p.X, at + j) - mean, s2);
    }
    s1 = kRms ? 0.f : block_sum(s1, shared);
    s2 = block_sum(s2, shared);
    const float mean_g = s1 * p.inv_n, slope = s2 * rstd * p.inv_n * rstd;
    for (int64_t j = threadIdx.x; j < p.n; j += kLongThreads) {
      const float g = bf16_value(p.dY[at + j]) * (p.gamma ? bf16_value(p.gamma[j]) : 1.f);
      float v = rstd * fmaf(-slope, element<kF32>(p.X, at + j) - mean, g - mean_g);
      if (p.R) v += element<kF32>(p.R, at + j);
      if constexpr (kF32) static_cast<float*>(p.dX)[at + j] = v;
      else static_cast<uint16_t*>(p.dX)[at + j] = bf16_round(v);
    }
  }
}

template <bool kF32>
__global__ void __launch_bounds__(1024) norm_columns_kernel(const NormBackwardParams p, int64_t rows_per_block) {
  __shared__ float2 shared[32][33];
  const int lane = threadIdx.x % 32, strip = threadIdx.x / 32;
  const int64_t col = (int64_t)blockIdx.x * 32 + lane;
  const int64_t first = (int64_t)blockIdx.y * rows_per_block, last = min(p.m, first + rows_per_block);
  pdl_wait();
  pdl_release();
  float2 s = make_float2(0.f, 0.f);
  if (col < p.n) {
    for (int64_t row = first + strip; row < last; row += 32) {
      const float v = bf16_value(p.dY[row * p.n + col]);
      const float h = (element<kF32>(p.X, row * p.n + col) - (p.mean ? p.mean[row] : 0.f)) * p.rstd[row];
      s.x = fmaf(v, h, s.x);
      s.y += v;
    }
  }
  shared[strip][lane] = s;
  __syncthreads();
  if (strip == 0 && col < p.n) {
    for (int i = 1; i < 32; ++i) {
      s.x += shared[i][lane].x;
      s.y += shared[i][lane].y;
    }
    float* mine = p.partial + (int64_t)blockIdx.y * 2 * p.n;
    mine[col] = s.x;
    mine[p.n + col] = s.y;
  }
}

// dgamma and dbeta from the blocks' sums: 32 columns to a block, eight warps that take every eighth part, then the eight
// in order.  grid.y: 0 dgamma, 1 dbeta.
struct NormSums {
  const float* partial;
  float* out[2];
  int n, parts;
  bool accumulate;
};
__global__ void __launch_bounds__(256) norm_sums_kernel(const NormSums p) {
  __shared__ float shared[8][32];
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int64_t col = (int64_t)blockIdx.x * 32 + lane;
  float* out = p.out[blockIdx.y];
  pdl_wait();
  pdl_release();
  if (!out) return;
  float s = 0.f;
  if (col < p.n) {
#pragma unroll 8
    for (int i = warp; i < p.parts; i += 8) s += p.partial[((int64_t)i * 2 + blockIdx.y) * p.n + col];
  }
  shared[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && col < p.n) {
#pragma unroll
    for (int w = 1; w < 8; ++w) s += shared[w][lane];
    out[col] = p.accumulate ? out[col] + s : s;
  }
}

// --- host -----------------------------------------------------------------------------------

constexpr int64_t kMaxExtent = (1ll << 31) - 1024;
constexpr int kMaxParts = 296;          // blocks whose sums the second launch joins: two to an SM of 148
constexpr int kTeamForward = 16384;     // columns a team of 512 threads holds
constexpr int kTeamBackward = 8192;     // columns a team of 256 threads holds beside its sums

bool aligned(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// The ring's teams: 16 columns to a thread, 32 in the longest rows.
int ring_team(int64_t n) {
  int t = 32;
  while (t < kRingThreads && n > t * 16) t *= 2;
  return t;
}
// Stages that fit `budget` bytes of shared memory beside the static part; below two the ring does not run.
RingShape ring_shape(int64_t n, int64_t column_bytes, int budget) {
  RingShape r;
  const int64_t bytes = kRingThreads / ring_team(n) * n * column_bytes;
  r.stage_bytes = (uint32_t)bytes;
  r.stages = (int)std::min<int64_t>(kMaxStages, budget / bytes);
  return r;
}

// Threads of a team: the fewest that hold the row in at most 32 columns each.
int team_of(int64_t n) { return n <= 1024 ? 32 : n <= 4096 ? 128 : n <= 8192 ? 256 : 512; }

// Blocks at most that leave sums of their own.
int64_t backward_parts(int64_t m, int64_t n) {
  if (n > kTeamBackward) return std::min<int64_t>(kMaxParts, m);
  const int64_t teams = kBlockThreads / team_of(n);
  return std::min<int64_t>(kMaxParts, (m + teams - 1) / teams);
}
size_t backward_bytes(int64_t m, int64_t n) { return (size_t)backward_parts(m, n) * 2 * n * 4; }

constexpr int kBackwardBudget = 224 * 1024;

template <auto kKernel, int kBudget, typename Params>
cudaError_t ring_launch(const Params& p, const RingShape& ring, int teams, int64_t most, size_t least_smem, cudaStream_t s) {
  static PerDeviceOnce once;
  const cudaError_t e = once.run_current(
      [] { return cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kBudget); });
  if (e != cudaSuccess) return e;
  const int64_t blocks = std::min(most, (p.m + teams - 1) / teams);
  return launch_pdl(kKernel, dim3((unsigned)blocks), dim3(kRingThreads),
                    std::max(least_smem, (size_t)ring.stages * ring.stage_bytes), s, 1, p, ring);
}
template <bool kF32, bool kRms>
cudaError_t backward_ring(const NormBackwardParams& p, const RingShape& ring, int64_t blocks, cudaStream_t s) {
#define MORELLO_RING(T, ITER)                                                                                          \
  return ring_launch<norm_backward_ring_kernel<T, ITER, kF32, kRms>, kBackwardBudget>(p, ring, kRingThreads / T, blocks, \
                                                                                      (size_t)kRingThreads * ITER * 64, s)
  if (p.n <= 256) MORELLO_RING(32, 1);
  if (p.n <= 512) MORELLO_RING(32, 2);
  if (p.n <= 1024) MORELLO_RING(64, 2);
  if (p.n <= 2048) MORELLO_RING(128, 2);
  if (p.n <= 4096) MORELLO_RING(256, 2);
  if (p.n <= 8192) MORELLO_RING(512, 2);
  MORELLO_RING(512, 4);
#undef MORELLO_RING
}

template <bool kF32, bool kRms>
cudaError_t forward_launch(const DeviceInfo& dev, const NormParams& p, bool vec, cudaStream_t s) {
  const int n = p.n;
  auto go = [&](auto kernel, int team) {
    const int threads = std::max(team, kBlockThreads), rows = threads / team;
    const int64_t blocks = std::min<int64_t>((p.m + rows - 1) / rows, (int64_t)dev.sms * 8);
    return launch_pdl(kernel, dim3((unsigned)blocks), dim3(threads), 0, s, 1, p);
  };
#define MORELLO_NORM(T, ITER) return go(norm_octets_kernel<T, ITER, kF32, kRms>, T)
#define MORELLO_NORM_ODD(T, ITER) return go(norm_kernel<T, 1, ITER, kF32, kRms>, T)
  if (n > kTeamForward) return launch_pdl(norm_long_kernel<kF32, kRms>, dim3((unsigned)std::min<int64_t>(p.m, (int64_t)dev.sms * 2)),
                                          dim3(kLongThreads), 0, s, 1, p);
  if (vec) {
    if (n <= 64) MORELLO_NORM(8, 1);
    if (n <= 128) MORELLO_NORM(16, 1);
    if (n <= 256) MORELLO_NORM(32, 1);
    if (n <= 512) MORELLO_NORM(32, 2);
    if (n <= 1024) MORELLO_NORM(32, 4);
    if (n <= 2048) MORELLO_NORM(128, 2);
    if (n <= 4096) MORELLO_NORM(128, 4);
    if (n <= 8192) MORELLO_NORM(256, 4);
    MORELLO_NORM(512, 4);
  }
  if (n <= 256) MORELLO_NORM_ODD(32, 8);
  if (n <= 1024) MORELLO_NORM_ODD(32, 32);
  if (n <= 2048) MORELLO_NORM_ODD(128, 16);
  if (n <= 4096) MORELLO_NORM_ODD(128, 32);
  if (n <= 8192) MORELLO_NORM_ODD(256, 32);
  MORELLO_NORM_ODD(512, 32);
#undef MORELLO_NORM
#undef MORELLO_NORM_ODD
}

template <bool kF32, bool kRms, bool kSums>
cudaError_t backward_rows_launch(const NormBackwardParams& p, int parts, bool vec, cudaStream_t s) {
  const int n = p.n, t = team_of(n);
  auto go = [&](auto kernel, int teams) {
    // The teams' sums meet in shared memory: kBlockThreads / teams threads of 32 columns at most.
    const size_t smem = kSums && teams > 1 ? (size_t)2 * (kBlockThreads / teams) * 32 * 4 : 0;
    return launch_pdl(kernel, dim3((unsigned)parts), dim3(kBlockThreads), smem, s, 1, p);
  };
#define MORELLO_NORM(T, VEC, ITER) return go(norm_backward_kernel<T, VEC, ITER, kF32, kRms, kSums>, kBlockThreads / T)
  if (vec) {
    if (t == 32) {
      if (n <= 256) MORELLO_NORM(32, 8, 1);
      if (n <= 512) MORELLO_NORM(32, 8, 2);
      MORELLO_NORM(32, 8, 4);
    }
    if (t == 128) {
      if (n <= 2048) MORELLO_NORM(128, 8, 2);
      MORELLO_NORM(128, 8, 4);
    }
    MORELLO_NORM(256, 8, 4);
  }
  if (t == 32) {
    if (n <= 256) MORELLO_NORM(32, 1, 8);
    MORELLO_NORM(32, 1, 32);
  }
  if (t == 128) {
    if (n <= 2048) MORELLO_NORM(128, 1, 16);
    MORELLO_NORM(128, 1, 32);
  }
  MORELLO_NORM(256, 1, 32);
#undef MORELLO_NORM
}

template <bool kF32, bool kRms>
cudaError_t backward_launch(const DeviceInfo& dev, const NormBackwardParams& p, float* dgamma, float* dbeta,
                            bool accumulate, bool vec, cudaStream_t s, uint64_t* launches) {
  cudaError_t e = cudaSuccess;
  const bool sums = dgamma || dbeta;
  int parts = (int)backward_parts(p.m, p.n);
  constexpr int kSize = kF32 ? 4 : 2;
  // With R or without: what a call asks for besides does not change the order of its sums.
  if (vec && p.n <= kRingThreads * 32 && ring_shape(p.n, 2 * kSize + 2, kBackwardBudget).stages >= 2) {
    const RingShape ring = ring_shape(p.n, kSize * (p.R && p.dX ? 2 : 1) + 2, kBackwardBudget);
    const int64_t teams = kRingThreads / ring_team(p.n);
    parts = (int)std::min<int64_t>(std::min(parts, dev.sms), (p.m + teams - 1) / teams);
    e = backward_ring<kF32, kRms>(p, ring, parts, s);
  } else if (p.n > kTeamBackward) {
    parts = (int)std::min<int64_t>(kMaxParts, (p.m + 127) / 128);
    if (p.dX) {
      const int64_t blocks = std::min<int64_t>(p.m, (int64_t)dev.sms * 2);
      e = launch_pdl(norm_backward_long_kernel<kF32, kRms>, dim3((unsigned)blocks), dim3(kLongThreads), 0, s, 1, p);
      if (e != cudaSuccess) return e;
      ++*launches;
    }
    if (!sums) return e;
    const int64_t per = (p.m + parts - 1) / parts;
    e = launch_pdl(norm_columns_kernel<kF32>, dim3((unsigned)((p.n + 31) / 32), (unsigned)parts), dim3(1024), 0, s, 1, p, per);
  } else {
    e = sums ? backward_rows_launch<kF32, kRms, true>(p, parts, vec, s)
             : backward_rows_launch<kF32, kRms, false>(p, parts, vec, s);
  }
  if (e != cudaSuccess) return e;
  ++*launches;
  if (!sums) return e;
  const NormSums ns{p.partial, {dgamma, dbeta}, p.n, parts, accumulate};
  e = launch_pdl(norm_sums_kernel, dim3((unsigned)((p.n + 31) / 32), dbeta ? 2u : 1u), dim3(256), 0, s, 1, ns);
  if (e == cudaSuccess) ++*launches;
  return e;
}

int check_norm(int rms, int x_type, int64_t m, int64_t n) {
  if (rms < 0 || rms > 1 || x_type < 0 || x_type > 1) return MORELLO_ERR_INVALID_ARGUMENT;
  if (m < 0 || n < 0 || m > kMaxExtent || n > kMaxExtent) return MORELLO_ERR_INVALID_SHAPE;
  return MORELLO_OK;      // m n elements of 4 bytes stay below 2^64
}

}  // namespace
}  // namespace morello

using namespace morello;

#pragma GCC visibility push(default)
extern "C" {

int morello_layer_norm(int rms, int x_type, int64_t m, int64_t n, float eps, const void* X, const void* gamma,
                       const void* beta, void* Y, float* mean, float* rstd, void* stream) {
  int rc;
  if ((rc = check_norm(rms, x_type, m, n)) != MORELLO_OK) return rc;
  if (!(eps >= 0.f)) return MORELLO_ERR_INVALID_ARGUMENT;
  const bool empty = m == 0 || n == 0, f32 = x_type == MORELLO_F32;
  if (!empty && (!X || !Y)) return MORELLO_ERR_NULL_POINTER;
  if (!aligned(X, f32 ? 4 : 2) || !aligned(gamma, 2) || !aligned(beta, 2) || !aligned(Y, 2) || !aligned(mean, 4) ||
      !aligned(rstd, 4))
    return MORELLO_ERR_MISALIGNED;
  DeviceInfo dev;
  void* none = nullptr;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if ((rc = operator_workspace(0, nullptr, 0, s, &none, &dev)) != MORELLO_OK || empty) return rc;
  const NormParams p{m, (int)n, eps, 1.f / (float)n, X, static_cast<const uint16_t*>(gamma),
                     static_cast<const uint16_t*>(beta), static_cast<uint16_t*>(Y), mean, rstd, dev.status};
  const bool vec = n % 8 == 0 && aligned(X, 16) && aligned(gamma, 16) && aligned(beta, 16) && aligned(Y, 16);
  cudaError_t e;
  if (f32) e = rms ? forward_launch<true, true>(dev, p, vec, s) : forward_launch<true, false>(dev, p, vec, s);
  else e = rms ? forward_launch<false, true>(dev, p, vec, s) : forward_launch<false, false>(dev, p, vec, s);
  if (e != cudaSuccess) return record_cuda_error(e);
  count_launches(1);
  return MORELLO_OK;
}

int morello_layer_norm_backward(int rms, int x_type, int accumulate, int64_t m, int64_t n, const void* X,
                                const void* gamma, const float* mean, const float* rstd, const void* dY, const void* R,
                                void* dX, float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes,
                                void* stream) {
  int rc;
  if ((rc = check_norm(rms, x_type, m, n)) != MORELLO_OK) return rc;
  if (accumulate < 0 || accumulate > 1) return MORELLO_ERR_INVALID_ARGUMENT;
  if (workspace && !aligned(workspace, 16)) return MORELLO_ERR_MISALIGNED;
  const bool empty = m == 0 || n == 0, f32 = x_type == MORELLO_F32, sums = dgamma || dbeta;
  if (!empty && (!X || !rstd || !dY || (!rms && !mean))) return MORELLO_ERR_NULL_POINTER;
  const uintptr_t to = f32 ? 4 : 2;
  if (!aligned(X, to) || !aligned(gamma, 2) || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(dY, 2) || !aligned(R, to) ||
      !aligned(dX, to) || !aligned(dgamma, 4) || !aligned(dbeta, 4))
    return MORELLO_ERR_MISALIGNED;
  DeviceInfo dev;
  void* ws = nullptr;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if ((rc = operator_workspace(sums ? backward_bytes(m, n) : 0, workspace, workspace_bytes, s, &ws, &dev)) != MORELLO_OK) return rc;
  cudaError_t e = cudaSuccess;
  if (empty) {
    // Empty sums: zero, or nothing added.
    if (dgamma && n > 0 && !accumulate) e = cudaMemsetAsync(dgamma, 0, (size_t)n * 4, s);
    if (e == cudaSuccess && dbeta && n > 0 && !accumulate) e = cudaMemsetAsync(dbeta, 0, (size_t)n * 4, s);
    return e == cudaSuccess ? MORELLO_OK : record_cuda_error(e);
  }
  if (!dX && !sums) return MORELLO_OK;
  const NormBackwardParams p{m, (int)n, 1.f / (float)n, X, static_cast<const uint16_t*>(gamma), rms ? nullptr : mean, rstd,
                             static_cast<const uint16_t*>(dY), R, dX, static_cast<float*>(ws), dbeta != nullptr, dev.status};
  const bool vec = n % 8 == 0 && aligned(X, 16) && aligned(gamma, 16) && aligned(dY, 16) && aligned(R, 16) && aligned(dX, 16) &&
                   aligned(ws, 16);
  uint64_t launches = 0;
  if (f32)
    e = rms ? backward_launch<true, true>(dev, p, dgamma, dbeta, accumulate != 0, vec, s, &launches)
            : backward_launch<true, false>(dev, p, dgamma, dbeta, accumulate != 0, vec, s, &launches);
  else
    e = rms ? backward_launch<false, true>(dev, p, dgamma, dbeta, accumulate != 0, vec, s, &launches)
            : backward_launch<false, false>(dev, p, dgamma, dbeta, accumulate != 0, vec, s, &launches);
  count_launches(launches);
  return e == cudaSuccess ? MORELLO_OK : record_cuda_error(e);
}

size_t morello_layer_norm_backward_workspace_bytes(int64_t m, int64_t n) {
  return check_norm(0, 0, m, n) == MORELLO_OK && n > 0 ? backward_bytes(m, n) : 0;
}

}  // extern "C"
#pragma GCC visibility pop
