// Layer norm of rows (mean-centred or root-mean-square), its gradients, and the sums over rows that are the
// gradients of gamma and beta.
//
//   forward    y = (x - mu) r gamma + beta,  mu = mean(x) (rms: 0),  r = 1 / sqrt(mean((x - mu)^2) + eps)
//   backward   h = (x - mu) r, g = dy gamma:  dx = r (g - mean(g) - h mean(g h)) + R  (rms: without mean(g))
//              dgamma = sum over rows of dy h, dbeta = sum over rows of dy
//
// A row is read once by a team of 8 to 512 threads, which hold it (backward: find it in shared memory again) until it has been
// reduced, and written.  In a row of calls 16384 x 4096 takes 49.5 us forward and 83.6 backward, 5.4 and 4.8 TB/s: bound by
// memory.  Short rows are not: 65536 x 128 takes 9.1 and 19.7 us with 65 and 53 % of the issue slots in use, and a warp's
// joins waited for in between.  Nor are rows off 16 bytes: 4096 x 2047 takes 16.5 and 30.6 us, at 17.8 and 28.0 M
// instructions for 8192 x 2047 (every element is an access of its own to shared memory, and a store), 57 and 58 % of the slots.
//
// The variance is that of the differences from a mean (two sweeps over the registers), never a difference of sums.  A warp
// takes its own mean and the squares about it, and one barrier later every thread joins the warps' three numbers (Chan,
// Golub and LeVeque's formula for joining variances), so a row costs one barrier.
//
// The backward pass's threads keep the columns they own through all the rows of a block, so dgamma and dbeta add up in
// registers; the blocks' sums are joined by a second launch in the order of the blocks.  No atomics: the same sums in the
// same order every time.
#include <algorithm>
#include <atomic>
#include <initializer_list>
#include <type_traits>

#include "../../include/morello.h"
#include "activation.cuh"
#include "linear.h"
#include "sm100.cuh"

namespace morello {
namespace {

using namespace sm100;

constexpr uint32_t kFull = 0xffffffffu;
constexpr int kBlockThreads = 256;
// Blocks that leave sums of their own, at most, but for very many rows: see ring_blocks().
constexpr int kMaxParts = 296;

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
  bool ring_r;           // longest rows: R comes through the ring; else, where that leaves no room for two stages, straight from memory
};

// Sum over kLanes neighbouring lanes, in every one of them.
template <int kLanes = 32>
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = kLanes / 2; d > 0; d >>= 1) v += __shfl_xor_sync(kFull, v, d);
  return v;
}

// The barrier of one team of a block of kThreads.
template <int kT, int kThreads>
__device__ __forceinline__ void team_barrier(int team) {
  if constexpr (kT == kThreads) __syncthreads();
  else asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "n"(kT) : "memory");
}

// A thread's columns of a row, by eights.  kVec 8: octets of columns, 8 (t + i T) ..., 16-byte accesses; needs n % 8 == 0
// and aligned tensors.  kVec 1: single columns t + (8 i + e) T, any n and alignment.
template <int kT, int kVec, int kIter>
struct Columns {
  int t, n;
  __device__ __forceinline__ int of(int i, int e) const { return first() + past(i, e); }
  // The same from the thread's first column on: a constant, so that addresses are one register's.
  static constexpr __device__ int past(int i, int e) { return kVec == 8 ? i * kT * 8 + e : (8 * i + e) * kT; }
  __device__ __forceinline__ int first() const { return kVec == 8 ? 8 * t : t; }
  __device__ __forceinline__ bool any(int i) const { return of(i, 0) < n; }       // of the eight
  __device__ __forceinline__ bool has(int i, int e) const { return kVec == 8 ? any(i) : of(i, e) < n; }
  // Whether the whole team has all of the i-th eight.
  __device__ __forceinline__ bool whole(int i) const { return kVec == 8 || 8 * (i + 1) * kT <= n; }
  __device__ __forceinline__ float count() const {
    float k = 0.f;
#pragma unroll
    for (int i = 0; i < kIter; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) k += has(i, e) ? 1.f : 0.f;
    return k;
  }
  // Zeros where there is no column.
  __device__ __forceinline__ void clear(int i, f32x2 (&v)[4]) const {
    if constexpr (kVec == 1) {
      if (whole(i)) return;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 f = pair_values(v[j]);
        v[j] = pair_of(has(i, 2 * j) ? f.x : 0.f, has(i, 2 * j + 1) ? f.y : 0.f);
      }
    }
  }
};

// Eight elements as four pairs.
__device__ __forceinline__ void octet_pairs(const uint4& w, f32x2 (&v)[4]) {
  v[0] = pair_of(bf16_low(w.x), bf16_high(w.x));
  v[1] = pair_of(bf16_low(w.y), bf16_high(w.y));
  v[2] = pair_of(bf16_low(w.z), bf16_high(w.z));
  v[3] = pair_of(bf16_low(w.w), bf16_high(w.w));
}
__device__ __forceinline__ uint32_t bf16_pack_pair(f32x2 v) {
  const float2 f = pair_values(v);
  return bf16_pack(f.x, f.y);
}

// The elements of a thread's octets, bf16 or f32, as they came from memory.
template <int kT, int kIter, bool kF32>
struct Held {
  uint32_t w[(kF32 ? 8 : 4) * kIter];
  __device__ __forceinline__ void load(const void* row, const Columns<kT, 8, kIter>& c) {
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      constexpr int kQuads = kF32 ? 2 : 1;
#pragma unroll
      for (int q = 0; q < kQuads; ++q) {
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (c.any(i)) v = static_cast<const uint4*>(row)[(c.t + i * kT) * kQuads + q];
        uint32_t* o = w + (i * kQuads + q) * 4;
        o[0] = v.x; o[1] = v.y; o[2] = v.z; o[3] = v.w;
      }
    }
  }
  __device__ __forceinline__ void pairs(int i, f32x2 (&v)[4]) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (kF32) v[j] = pair_of(__uint_as_float(w[i * 8 + 2 * j]), __uint_as_float(w[i * 8 + 2 * j + 1]));
      else v[j] = pair_of(bf16_low(w[i * 4 + j]), bf16_high(w[i * 4 + j]));
    }
  }
};

// Eight of a thread's columns of gamma or beta; `missing` where there is no such vector.
template <int kT, int kIter>
__device__ __forceinline__ void vector_pairs(const uint16_t* p, const Columns<kT, 8, kIter>& c, int i, float missing,
                                             f32x2 (&v)[4]) {
  if (p) octet_pairs(*reinterpret_cast<const uint4*>(p + c.of(i, 0)), v);
  else v[0] = v[1] = v[2] = v[3] = pair_of(missing);
}

// Stores eight columns of a row (kVec 8: they all exist).
template <bool kF32, int kT, int kVec, int kIter>
__device__ __forceinline__ void put_eight(void* row, const Columns<kT, kVec, kIter>& c, int i, const f32x2 (&v)[4]) {
  if constexpr (kVec == 8 && kF32) {
    float4* o = reinterpret_cast<float4*>(static_cast<float*>(row) + c.of(i, 0));
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const float2 a = pair_values(v[2 * q]), b = pair_values(v[2 * q + 1]);
      o[q] = make_float4(a.x, a.y, b.x, b.y);
    }
  } else if constexpr (kVec == 8) {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(row) + c.of(i, 0)) =
        make_uint4(bf16_pack_pair(v[0]), bf16_pack_pair(v[1]), bf16_pack_pair(v[2]), bf16_pack_pair(v[3]));
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 f = pair_values(v[j]);
      if constexpr (kF32) {
        float* dst = static_cast<float*>(row) + c.t;
        if (c.has(i, 2 * j)) dst[c.past(i, 2 * j)] = f.x;
        if (c.has(i, 2 * j + 1)) dst[c.past(i, 2 * j + 1)] = f.y;
      } else {
        const uint32_t both = bf16_pack(f.x, f.y);
        uint16_t* dst = static_cast<uint16_t*>(row) + c.t;
        if (c.has(i, 2 * j)) dst[c.past(i, 2 * j)] = (uint16_t)both;
        if (c.has(i, 2 * j + 1)) dst[c.past(i, 2 * j + 1)] = (uint16_t)(both >> 16);
      }
    }
  }
}

// Eight columns of a row in shared memory.  kVec 1: where the row ends its last column stands in for those that are missing.
template <bool kF32, int kT, int kVec, int kIter>
__device__ __forceinline__ void row_eight(const void* row, const Columns<kT, kVec, kIter>& c, int i, f32x2 (&v)[4]) {
  if constexpr (kVec == 8 && kF32) {
    const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(row) + c.of(i, 0));
    const float4 a = q[0], b = q[1];
    v[0] = pair_of(a.x, a.y);
    v[1] = pair_of(a.z, a.w);
    v[2] = pair_of(b.x, b.y);
    v[3] = pair_of(b.z, b.w);
  } else if constexpr (kVec == 8) {
    octet_pairs(*reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(row) + c.of(i, 0)), v);
  } else {
    auto one = [&](int e) {
      const int col = min(c.of(i, e), c.n - 1);
      if constexpr (kF32) return static_cast<const float*>(row)[col];
      else return bf16_value(static_cast<const uint16_t*>(row)[col]);
    };
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = pair_of(one(2 * j), one(2 * j + 1));
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
  return squares < 0.f ? 0.f : squares * inv_n;      // what rounding leaves of a row of one value
}

// d = x - mean of eight columns: their sum and their squares.
template <bool kRms>
__device__ __forceinline__ void spread(const f32x2 (&x)[4], f32x2 minus_mean, f32x2* off, f32x2* squares) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const f32x2 d = kRms ? x[j] : add2(x[j], minus_mean);
    if constexpr (!kRms) *off = add2(*off, d);
    *squares = fma2(d, d, *squares);
  }
}
// y = ((x - base) rstd - shift rstd) gamma + beta
struct ForwardFactors {
  f32x2 rstd, minus_base, shifted;
  template <bool kRms>
  __device__ __forceinline__ void y(const f32x2 (&x)[4], const f32x2 (&gamma)[4], const f32x2 (&beta)[4], f32x2 (&out)[4]) const {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      out[j] = fma2(kRms ? mul2(x[j], rstd) : fma2(add2(x[j], minus_base), rstd, shifted), gamma[j], beta[j]);
  }
};
// Joins the row's parts; one thread keeps its mean and rstd.
template <int kT, int kLanes, int kTeams, bool kRms, int kWarps>
__device__ __forceinline__ ForwardFactors forward_factors(const NormParams& p, Part (&parts)[kTeams][kWarps], const Part& mine, int team,
                                                          int warp, int lane, int64_t row, bool keeps) {
  float base, shift, square;
  if constexpr (kWarps == 1) {
    square = join_parts<1>(&mine, p.inv_n, &base, &shift);
  } else {
    if (lane == 0) parts[team][warp] = mine;
    team_barrier<kT, kT * kTeams>(team);     // the other set of parts is written next: nobody is still reading it behind this barrier
    square = join_parts<kWarps>(parts[team], p.inv_n, &base, &shift);
  }
  const float rstd = rsqrtf(square + p.eps);
  if (keeps) {
    if (!kRms && p.mean) p.mean[row] = base + shift;
    if (p.rstd) p.rstd[row] = rstd;
  }
  return ForwardFactors{pair_of(rstd), pair_of(-base), pair_of(-shift * rstd)};
}

// n % 8 == 0 and 16-byte-aligned tensors.  Teams of 8 to 512 threads, a row each and kIter of its octets to a thread, two
// columns an instruction.  A team's next row is on its way while it works on this one.
template <int kT, int kIter, bool kF32, bool kRms>
__global__ void __launch_bounds__(kT > kBlockThreads ? kT : kBlockThreads, kT > kBlockThreads || kIter < 4 ? 1 : kF32 ? 2 : 3)
norm_kernel(const NormParams p) {
  constexpr int kTeams = kT < kBlockThreads ? kBlockThreads / kT : 1;
  constexpr int kLanes = kT < 32 ? kT : 32, kWarps = kT / kLanes;
  __shared__ Part parts[2][kTeams][kWarps];
  const int team = (int)threadIdx.x / kT, warp = (int)threadIdx.x % kT / kLanes, lane = (int)threadIdx.x % kLanes;
  const Columns<kT, 8, kIter> c{(int)threadIdx.x % kT, p.n};
  const float count = warp_sum<kLanes>(c.count()), inv_count = count > 0.f ? 1.f / count : 0.f;
  pdl_wait();
  pdl_release();
  const int64_t step = (int64_t)gridDim.x * kTeams;
  int64_t row = (int64_t)blockIdx.x * kTeams + team;
  Held<kT, kIter, kF32> held;
  auto fetch = [&](int64_t r) {      // past the last row: the last one, to no use
    held.load(static_cast<const char*>(p.X) + min(r, p.m - 1) * p.n * (kF32 ? 4 : 2), c);
  };
  fetch(row);
  int turn = 0;
  // Rows past the last are worked on like any other, but neither read nor written: teams of less than a warp leave together.
  for (int64_t row0 = (int64_t)blockIdx.x * kTeams; row0 < p.m; row0 += step, row += step, turn ^= 1) {
    const bool live = row < p.m;
    if (kT >= 32 && !live) break;
    f32x2 x[kIter][4], sums = 0;
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      held.pairs(i, x[i]);
      if constexpr (!kRms) {
#pragma unroll
        for (int j = 0; j < 4; ++j) sums = add2(sums, x[i][j]);
      }
    }
    fetch(row + step);
    Part mine{0.f, 0.f, 0.f, count};
    if constexpr (!kRms) mine.mean = warp_sum<kLanes>(pair_sum(sums)) * inv_count;
    const f32x2 minus_mean = pair_of(-mine.mean);
    f32x2 off = 0, squares = 0;
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      if (!c.any(i)) continue;
      spread<kRms>(x[i], minus_mean, &off, &squares);
    }
    if constexpr (!kRms) mine.off = warp_sum<kLanes>(pair_sum(off));
    mine.squares = warp_sum<kLanes>(pair_sum(squares));
    const ForwardFactors f = forward_factors<kT, kLanes, kTeams, kRms>(p, parts[turn], mine, team, warp, lane, row, live && c.t == 0);
    if (!live) continue;
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      if (!c.any(i)) continue;
      f32x2 gamma[4], beta[4], y[4];
      vector_pairs(p.gamma, c, i, 1.f, gamma);
      vector_pairs(p.beta, c, i, 0.f, beta);
      f.y<kRms>(x[i], gamma, beta, y);
      put_eight<false>(p.Y + row * p.n, c, i, y);
    }
  }
}

// --- rows through a ring in shared memory ------------------------------------------------------
//
// The backward pass, and the forward pass of rows that are not whole octets: one persistent block of 16 warps to an SM.  A group is kTeams neighbouring rows, one to a team, and
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

// A tensor of rows, and the bytes of a stage that its part of a group takes: 32 more than its rows', so that their first byte
// can lie where it lies in its 16 bytes of memory, and a multiple of 16.
struct RingTensor {
  const void* p;
  uint32_t row_bytes, area;
};
__host__ __device__ constexpr uint32_t ring_area(uint32_t rows, uint32_t row_bytes) { return (rows * row_bytes + 47) / 16 * 16; }

// Starts the copies of the group whose first row is `row` to a stage.  A bulk copy moves whole 16 bytes: those that hold the
// group's rows, but where they reach past the tensor's ends, there its elements (2 bytes at a time) are copied one by one.
// kWhole: rows are whole 16 bytes.
template <int kTeams, bool kWhole, int kTensors>
__device__ __forceinline__ void ring_fill(RingBars* bars, uint8_t* smem, const RingShape& ring, int stage, int64_t row, int64_t m,
                                          const RingTensor (&tensors)[kTensors]) {
  const uint32_t rows = (uint32_t)min((int64_t)kTeams, m - row);
  if constexpr (kWhole) {
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
      dst += tensors[i].area;
    }
    return;
  }
  const uint8_t* from[kTensors];
  uint32_t head[kTensors], size[kTensors], bytes = 0;      // where the copy begins in its area, and how long it is
  uint8_t* dst = smem + (size_t)stage * ring.stage_bytes;
#pragma unroll
  for (int i = 0; i < kTensors; ++i) {
    if (!tensors[i].p) continue;
    const uint8_t* base = static_cast<const uint8_t*>(tensors[i].p);
    const uint8_t* first = base + row * tensors[i].row_bytes;
    const uint32_t skew = (uint32_t)reinterpret_cast<uintptr_t>(first) & 15u, end = skew + rows * tensors[i].row_bytes;
    uint32_t lo = 0u, hi = (end + 15u) & ~15u;
    auto singly = [&](uint32_t at, uint32_t stop) {
      for (; at < stop; at += 2) *reinterpret_cast<uint16_t*>(dst + at) = *reinterpret_cast<const uint16_t*>(first + (at - skew));
      fence_proxy_async_smem();      // a later copy to the same place comes behind it
    };
    if (first - skew < base) {
      lo = 16u;
      singly(skew, min(lo, end));
    }
    if (first - skew + hi > base + m * tensors[i].row_bytes) {
      hi = end & ~15u;
      singly(max(max(hi, lo), skew), end);
    }
    from[i] = first - skew + lo;
    head[i] = lo;
    size[i] = hi > lo ? hi - lo : 0u;
    bytes += size[i];
    dst += tensors[i].area;
  }
  mbar_arrive_expect_tx(&bars->full[stage], bytes);
  dst = smem + (size_t)stage * ring.stage_bytes;
#pragma unroll
  for (int i = 0; i < kTensors; ++i) {
    if (!tensors[i].p) continue;
    if (size[i] > 0) bulk_load(dst + head[i], from[i], size[i], &bars->full[stage]);
    dst += tensors[i].area;
  }
}
// Row `place` of the group whose first row is row0.
template <bool kWhole>
__device__ __forceinline__ const uint8_t* ring_row(const uint8_t* area, const RingTensor& t, int64_t row0, int place) {
  const uint32_t skew = kWhole ? 0u : (uint32_t)(reinterpret_cast<uintptr_t>(t.p) + (uintptr_t)row0 * t.row_bytes) & 15u;
  return area + skew + (uint32_t)place * t.row_bytes;
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
template <int kTeams, bool kWhole, int kTensors>
__device__ __forceinline__ void ring_start(RingBars* bars, uint8_t* smem, const RingShape& ring, RingPlace* at, int64_t m,
                                           const RingTensor (&tensors)[kTensors]) {
  at->fill = (int64_t)blockIdx.x * kTeams;
  if (threadIdx.x != 0) return;
  for (int i = 0; i < ring.stages && at->fill < m; ++i, at->fill += (int64_t)gridDim.x * kTeams)
    ring_fill<kTeams, kWhole>(bars, smem, ring, i, at->fill, m, tensors);
}
// A warp is done with the group's memory.
__device__ __forceinline__ void ring_release(RingBars* bars, const RingPlace& at) {
  __syncwarp();
  if (threadIdx.x % 32 == 0) mbar_arrive(&bars->empty[at.stage]);
}
// On to the next group; the first thread has the stage before this one's filled again.
template <int kTeams, bool kWhole, int kTensors>
__device__ __forceinline__ bool ring_next(RingBars* bars, uint8_t* smem, const RingShape& ring, RingPlace* at, int64_t m,
                                          const RingTensor (&tensors)[kTensors], uint32_t* status) {
  bool ok = true;
  // Of two stages it is the one just worked on: the one before it is the next (1024 x 16384 with R 44 instead of 51 us, f32
  // 2048 x 8192 44 instead of 61; of more stages the wait for this group's last warp costs as much as it gives).
  const bool now = ring.stages == 2;
  const int stage = now ? at->stage : at->before;
  if (threadIdx.x == 0 && stage >= 0 && at->fill < m) {
    ok = mbar_wait(&bars->empty[stage], now ? at->phase : at->phase_before, &bars->abort_flag, status, 61);
    if (ok) ring_fill<kTeams, kWhole>(bars, smem, ring, stage, at->fill, m, tensors);
    at->fill += (int64_t)gridDim.x * kTeams;
  }
  at->next(ring.stages);
  return ok;
}
// A thread's columns of gamma or beta.  Octets: kept through all its rows where registers allow (kIter 2), read again where not.
// Single columns: from a copy in shared memory.
template <int kT, int kVec, int kIter>
struct RingVector {
  static constexpr bool kHold = kVec == 8 && kIter <= 2;
  const uint16_t* p;
  float missing;
  Held<kT, kHold ? kIter : 1, false> held;
  __device__ __forceinline__ RingVector(const uint16_t* vector, float instead, uint16_t* copy, const Columns<kT, kVec, kIter>& c)
      : p(vector), missing(instead) {
    if constexpr (kVec == 1) {
      for (int col = (int)threadIdx.x; p && col < c.n; col += kRingThreads) copy[col] = p[col];
      if (p) p = copy;
    } else if constexpr (kHold) {
      if (p) held.load(p, c);
    }
  }
  __device__ __forceinline__ void get(const Columns<kT, kVec, kIter>& c, int i, f32x2 (&v)[4]) const {
    if (!p) {
      v[0] = v[1] = v[2] = v[3] = pair_of(missing);
    } else if constexpr (kHold) {
      held.pairs(i, v);
    } else if constexpr (kVec == 1) {
      row_eight<false>(p, c, i, v);
    } else {
      vector_pairs(p, c, i, missing, v);
    }
  }
};

// The threads of a block of the ring, in a barrier that is no team's own.
__device__ __forceinline__ void block_barrier() { asm volatile("bar.sync 15, %0;" ::"n"(kRingThreads) : "memory"); }

// The forward pass of rows that are not whole octets.
template <int kT, int kIter, bool kF32, bool kRms>
__global__ void __launch_bounds__(kRingThreads, 1) norm_ring_kernel(const NormParams p, const RingShape ring) {
  constexpr int kTeams = kRingThreads / kT, kLanes = kT < 32 ? kT : 32, kWarps = kT / kLanes;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ RingBars bars;
  __shared__ Part parts[2][kTeams][kWarps];
  ring_init(&bars, ring.stages);
  pdl_wait();
  pdl_release();
  const uint32_t row_bytes = (uint32_t)p.n * (kF32 ? 4 : 2);
  const RingTensor tensors[1] = {{p.X, row_bytes, ring_area(kTeams, row_bytes)}};
  RingPlace at;
  ring_start<kTeams, false>(&bars, smem, ring, &at, p.m, tensors);
  const int team = (int)threadIdx.x / kT, warp = (int)threadIdx.x % kT / 32, lane = (int)threadIdx.x % 32;
  const Columns<kT, 1, kIter> c{(int)threadIdx.x % kT, p.n};
  uint16_t* copies = reinterpret_cast<uint16_t*>(smem + (size_t)ring.stages * ring.stage_bytes);
  const RingVector<kT, 1, kIter> gammas(p.gamma, 1.f, copies, c), betas(p.beta, 0.f, copies + p.n, c);
  const float count = warp_sum<kLanes>(c.count()), inv_count = count > 0.f ? 1.f / count : 0.f;
  __syncthreads();
  int turn = 0;
  bool ok = true;          // once a wait gave up the rows go by unread and unwritten: the team's barriers still meet
  for (int64_t row0 = (int64_t)blockIdx.x * kTeams; row0 < p.m; row0 += (int64_t)gridDim.x * kTeams, turn ^= 1) {
    const int64_t row = row0 + team;
    if (ok) ok = mbar_wait(&bars.full[at.stage], at.phase, &bars.abort_flag, p.status, 63);
    ok = __all_sync(kFull, ok);
    const bool live = ok && row < p.m;
    f32x2 x[kIter][4], sums = 0;
    const uint8_t* src = ring_row<false>(smem + (size_t)at.stage * ring.stage_bytes, tensors[0], row0, team);
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      x[i][0] = x[i][1] = x[i][2] = x[i][3] = 0;
      if (!live) continue;
      row_eight<kF32>(src, c, i, x[i]);
      c.clear(i, x[i]);
#pragma unroll
      for (int j = 0; j < 4; ++j) sums = add2(sums, x[i][j]);
    }
    ring_release(&bars, at);
    Part mine{0.f, 0.f, 0.f, count};
    if constexpr (!kRms) mine.mean = warp_sum<kLanes>(pair_sum(sums)) * inv_count;
    f32x2 off = 0, squares = 0;
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      f32x2 d[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) d[j] = kRms ? x[i][j] : add2(x[i][j], pair_of(-mine.mean));
      c.clear(i, d);
      spread<kRms>(d, 0, &off, &squares);
    }
    if constexpr (!kRms) mine.off = warp_sum<kLanes>(pair_sum(off));
    mine.squares = warp_sum<kLanes>(pair_sum(squares));
    const ForwardFactors f = forward_factors<kT, kLanes, kTeams, kRms>(p, parts[turn], mine, team, warp, lane, row, live && c.t == 0);
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      if (!live || !c.any(i)) continue;
      f32x2 gamma[4], beta[4], y[4];
      gammas.get(c, i, gamma);
      betas.get(c, i, beta);
      f.y<kRms>(x[i], gamma, beta, y);
      put_eight<false>(p.Y + row * p.n, c, i, y);
    }
    ok = ring_next<kTeams, false>(&bars, smem, ring, &at, p.m, tensors, p.status) && ok;
  }
  if (!ok) let_copies_land();
}

// A row's x - mean, g = dy gamma and dy, eight columns of them.
template <bool kRms>
__device__ __forceinline__ void backward_terms(const f32x2 (&x)[4], const f32x2 (&dy)[4], const f32x2 (&gamma)[4], f32x2 minus_mean,
                                               f32x2 (&d)[4], f32x2 (&g)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    d[j] = kRms ? x[j] : add2(x[j], minus_mean);
    g[j] = mul2(dy[j], gamma[j]);
  }
}
// Their part of the row's two sums, and of dgamma and dbeta.
template <bool kRms>
__device__ __forceinline__ void backward_sums(const f32x2 (&d)[4], const f32x2 (&g)[4], const f32x2 (&dy)[4], f32x2 rstd, f32x2* p1,
                                              f32x2* p2, f32x2 (&sum_g)[4], f32x2 (&sum_b)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (!kRms) *p1 = add2(*p1, g[j]);
    *p2 = fma2(g[j], d[j], *p2);
    sum_g[j] = fma2(dy[j], mul2(d[j], rstd), sum_g[j]);
    sum_b[j] = add2(sum_b[j], dy[j]);
  }
}
// dx = rstd g - rstd mean(g) - (mean(g h) rstd) rstd (x - mean), from the row's sums of g (s1) and of g (x - mean) (s2).
struct BackwardFactors {
  f32x2 rstd, slope, constant;
  __device__ __forceinline__ BackwardFactors(float r, float s1, float s2, float inv_n)
      : rstd(pair_of(r)), slope(pair_of(-(s2 * r * inv_n * r) * r)), constant(pair_of(-r * s1 * inv_n)) {}
  template <bool kRms>
  __device__ __forceinline__ void dx(const f32x2 (&d)[4], const f32x2 (&g)[4], f32x2 (&out)[4]) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) out[j] = fma2(g[j], rstd, kRms ? mul2(d[j], slope) : fma2(d[j], slope, constant));
  }
};
__device__ __forceinline__ void add_four(f32x2 (&v)[4], const f32x2 (&r)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = add2(v[j], r[j]);
}

// The row is read from shared memory in both sweeps: kept in registers in between it took as long (and spilled with f32).
template <int kT, int kVec, int kIter, bool kF32, bool kRms>
__global__ void __launch_bounds__(kRingThreads, 1)
norm_backward_kernel(const NormBackwardParams p, const RingShape ring) {
  constexpr int kTeams = kRingThreads / kT, kLanes = kT < 32 ? kT : 32, kWarps = kT / kLanes;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ RingBars bars;
  __shared__ float2 parts[2][kTeams][kWarps];
  ring_init(&bars, ring.stages);
  pdl_wait();
  pdl_release();
  const uint32_t row16 = (uint32_t)p.n * 2, row_x = kF32 ? 2 * row16 : row16;
  const uint32_t area_x = ring_area(kTeams, row_x), area16 = ring_area(kTeams, row16);
  const RingTensor tensors[3] = {{p.X, row_x, area_x}, {p.dY, row16, area16}, {(kIter == 4 ? p.ring_r : p.dX != nullptr) ? p.R : nullptr, row_x, area_x}};
  RingPlace at;
  ring_start<kTeams, kVec == 8>(&bars, smem, ring, &at, p.m, tensors);
  const int team = (int)threadIdx.x / kT, warp = (int)threadIdx.x % kT / 32, lane = (int)threadIdx.x % 32;
  const Columns<kT, kVec, kIter> c{(int)threadIdx.x % kT, p.n};
  const RingVector<kT, kVec, kIter> gammas(p.gamma, 1.f, reinterpret_cast<uint16_t*>(smem + (size_t)ring.stages * ring.stage_bytes), c);
  if constexpr (kVec == 1) __syncthreads();
  f32x2 sum_g[kIter][4], sum_b[kIter][4];
#pragma unroll
  for (int i = 0; i < kIter; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) sum_g[i][j] = sum_b[i][j] = 0;
  int turn = 0;
  bool ok = true;          // once a wait gave up the rows go by unread and unwritten: the team's barriers still meet
  const int64_t step = (int64_t)gridDim.x * kTeams;
  int64_t row = (int64_t)blockIdx.x * kTeams + team;
  // The row's mean and rstd are fetched a row ahead.
  float next_mean = 0.f, next_rstd = 0.f;
  auto fetch = [&](int64_t r) {
    next_mean = !kRms && r < p.m ? p.mean[r] : 0.f;
    next_rstd = r < p.m ? p.rstd[r] : 0.f;
  };
  fetch(row);
  for (int64_t row0 = (int64_t)blockIdx.x * kTeams; row0 < p.m; row0 += step, row += step, turn ^= 1) {
    const float rstd = next_rstd;
    const f32x2 minus_mean = pair_of(-next_mean);
    fetch(row + step);
    if (ok) ok = mbar_wait(&bars.full[at.stage], at.phase, &bars.abort_flag, p.status, 62);
    ok = __all_sync(kFull, ok);
    const bool live = ok && row < p.m;
    const uint8_t* area = smem + (size_t)at.stage * ring.stage_bytes;
    const uint8_t* x_row = ring_row<kVec == 8>(area, tensors[0], row0, team);
    const uint8_t* dy_row = ring_row<kVec == 8>(area + area_x, tensors[1], row0, team);
    const uint8_t* r_row = ring_row<kVec == 8>(area + area_x + area16, tensors[2], row0, team);
    // Only the longest rows leave R no room (asked for at any length, this cost the others 5 %).
    if constexpr (kIter == 4) {
      if (!p.ring_r) r_row = static_cast<const uint8_t*>(p.R) + row * row_x;
    }
    auto terms = [&](int i, f32x2 (&d)[4], f32x2 (&g)[4], f32x2 (&dy)[4]) {
      f32x2 x[4], gamma[4];
      gammas.get(c, i, gamma);
      row_eight<kF32>(x_row, c, i, x);
      row_eight<false>(dy_row, c, i, dy);
      c.clear(i, dy);
      backward_terms<kRms>(x, dy, gamma, minus_mean, d, g);
    };
    f32x2 p1 = 0, p2 = 0;
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      if (!live || !c.any(i)) continue;
      f32x2 d[4], g[4], dy[4];
      terms(i, d, g, dy);
      backward_sums<kRms>(d, g, dy, pair_of(rstd), &p1, &p2, sum_g[i], sum_b[i]);
    }
    if (p.dX) {
      float s1 = kRms ? 0.f : warp_sum<kLanes>(pair_sum(p1)), s2 = warp_sum<kLanes>(pair_sum(p2));
      if constexpr (kT > 32) {
        if (lane == 0) parts[turn][team][warp] = make_float2(s1, s2);
        team_barrier<kT, kRingThreads>(team);
        s1 = s2 = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          s1 += parts[turn][team][w].x;
          s2 += parts[turn][team][w].y;
        }
      }
      const BackwardFactors f(rstd, s1, s2, p.inv_n);
#pragma unroll
      for (int i = 0; i < kIter; ++i) {
        if (!live || !c.any(i)) continue;
        f32x2 d[4], g[4], dy[4], out[4];
        terms(i, d, g, dy);
        f.dx<kRms>(d, g, out);
        if (p.R) {
          f32x2 r[4];
          row_eight<kF32>(r_row, c, i, r);
          add_four(out, r);
        }
        put_eight<kF32>(static_cast<char*>(p.dX) + row * row_x, c, i, out);
      }
    }
    ring_release(&bars, at);
    ok = ring_next<kTeams, kVec == 8>(&bars, smem, ring, &at, p.m, tensors, p.status) && ok;
  }
  if (!ok) let_copies_land();
  if (!p.partial) return;
  // The teams' sums meet in the ring's memory, whose last copies every team has read.
  constexpr int kWide = kT * kIter * 8;
  float* joined = reinterpret_cast<float*>(smem);        // [team][2][kWide]
  float* out = p.partial + (int64_t)blockIdx.x * 2 * p.n;
  if constexpr (kTeams > 1) {
    const Columns<kT, kVec, kIter> all{c.t, kWide};
    block_barrier();
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      put_eight<true>(joined + (size_t)team * 2 * kWide, all, i, sum_g[i]);
      put_eight<true>(joined + (size_t)team * 2 * kWide + kWide, all, i, sum_b[i]);
    }
    block_barrier();
    if (!ok) return;
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
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      if (!c.any(i)) continue;
      put_eight<true>(out, c, i, sum_g[i]);
      if (p.beta) put_eight<true>(out + p.n, c, i, sum_b[i]);
    }
  }
}

// Rows longer than a team's registers: a block of 1024 threads, two blocks to an SM, sweeps the row three times (the second and
// third time from L2, where it fits).  1024 x 32768 takes 75 us (f32 77), its backward pass 166.
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
// A thread's sums over its columns of a row, begun anew every kLongPart columns and joined in 64 bits: as one chain of f32
// additions a row of 2^24 equal values was off by more than 2^-16 of its sum.  add(j, part) adds column j's terms.
constexpr int kLongPart = 32;
template <int kSums, typename Add>
__device__ __forceinline__ void long_sums(int64_t n, float (&sums)[kSums], Add&& add) {
  double total[kSums];
#pragma unroll
  for (int i = 0; i < kSums; ++i) total[i] = 0.0;
  for (int64_t first = threadIdx.x; first < n; first += kLongPart * kLongThreads) {
    float part[kSums];
#pragma unroll
    for (int i = 0; i < kSums; ++i) part[i] = 0.f;
    if (first + (kLongPart - 1) * kLongThreads < n) {
#pragma unroll
      for (int e = 0; e < kLongPart; ++e) add(first + e * kLongThreads, part);
    } else {
#pragma unroll 4
      for (int64_t j = first; j < n; j += kLongThreads) add(j, part);
    }
#pragma unroll
    for (int i = 0; i < kSums; ++i) total[i] += part[i];
  }
#pragma unroll
  for (int i = 0; i < kSums; ++i) sums[i] = (float)total[i];
}

template <bool kF32, bool kRms>
__global__ void __launch_bounds__(kLongThreads, 2) norm_long_kernel(const NormParams p) {
  __shared__ float shared[kLongThreads / 32];
  pdl_wait();
  pdl_release();
  for (int64_t row = blockIdx.x; row < p.m; row += gridDim.x) {
    const int64_t at = row * p.n;
    const void* x = static_cast<const char*>(p.X) + at * (kF32 ? 4 : 2);
    float base = 0.f, shift = 0.f;
    if constexpr (!kRms) {
      float s[1];
      long_sums(p.n, s, [&](int64_t j, float (&part)[1]) { part[0] += element<kF32>(x, j); });
      base = block_sum(s[0], shared) * p.inv_n;
    }
    float s[2];      // differences and squares
    long_sums(p.n, s, [&](int64_t j, float (&part)[2]) {
      const float d = element<kF32>(x, j) - base;
      part[0] += d;
      part[1] = fmaf(d, d, part[1]);
    });
    if constexpr (!kRms) shift = block_sum(s[0], shared) * p.inv_n;
    float square = block_sum(s[1], shared) * p.inv_n - shift * shift;
    if (square < 0.f) square = 0.f;
    const float rstd = rsqrtf(square + p.eps);
    if (threadIdx.x == 0) {
      if (!kRms && p.mean) p.mean[row] = base + shift;
      if (p.rstd) p.rstd[row] = rstd;
    }
    for (int64_t j = threadIdx.x; j < p.n; j += kLongThreads) {
      const float d = (element<kF32>(x, j) - base) - shift;
      const float g = p.gamma ? bf16_value(p.gamma[j]) : 1.f, b = p.beta ? bf16_value(p.beta[j]) : 0.f;
      p.Y[at + j] = bf16_round(fmaf(d * rstd, g, b));
    }
  }
}

// Rows longer than that: dx by a block of 1024 threads that sweeps the row twice, and the sums over rows by a launch of
// their own, 32 columns x 32 rows of threads to a block, that reads x and dy again.
template <bool kF32, bool kRms>
__global__ void __launch_bounds__(kLongThreads, 2) norm_backward_long_kernel(const NormBackwardParams p) {
  __shared__ float shared[kLongThreads / 32];
  pdl_wait();
  pdl_release();
  for (int64_t row = blockIdx.x; row < p.m; row += gridDim.x) {
    const int64_t at = row * p.n;
    const float mean = kRms ? 0.f : p.mean[row], rstd = p.rstd[row];
    float s[2];      // g, and g (x - mean)
    const void* x = static_cast<const char*>(p.X) + at * (kF32 ? 4 : 2);
    const uint16_t* dy = p.dY + at;
    long_sums(p.n, s, [&](int64_t j, float (&part)[2]) {
      const float g = bf16_value(dy[j]) * (p.gamma ? bf16_value(p.gamma[j]) : 1.f);
      part[0] += g;
      part[1] = fmaf(g, element<kF32>(x, j) - mean, part[1]);
    });
    const float s1 = kRms ? 0.f : block_sum(s[0], shared), s2 = block_sum(s[1], shared);
    const float mean_g = s1 * p.inv_n, slope = s2 * rstd * p.inv_n * rstd;
    for (int64_t j = threadIdx.x; j < p.n; j += kLongThreads) {
      const float g = bf16_value(dy[j]) * (p.gamma ? bf16_value(p.gamma[j]) : 1.f);
      float v = rstd * fmaf(-slope, element<kF32>(x, j) - mean, g - mean_g);
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

// dgamma and dbeta from the blocks' sums: 32 columns to a block, eight warps that take every eighth part, then the eight in
// order (32 warps: 128 x 4096 7.5 instead of 6.3 us, both launches).  grid.y: 0 dgamma, 1 dbeta.
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
constexpr int64_t kRingColumns = 16384;     // a team of 512 threads with 32 columns each

bool aligned(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// Teams of 16 columns to a thread (32 in the longest rows, 8 in the shortest).
int team_of(int64_t n) {
  if (n <= 128) return n <= 64 ? 8 : 16;
  int t = 32;
  while (t < 512 && n > t * 16) t *= 2;
  return t;
}
// Stages of tensors of `sizes` bytes an element that fit shared memory beside `beside` bytes; below two the ring does not run.
constexpr int kRingBudget = 224 * 1024;
RingShape ring_shape(int64_t n, std::initializer_list<int> sizes, int64_t beside) {
  RingShape r{0, 0};
  if (n > kRingColumns) return r;
  const int teams = kRingThreads / team_of(n);
  for (const int size : sizes) r.stage_bytes += size ? ring_area((uint32_t)teams, (uint32_t)(n * size)) : 0u;
  r.stages = (int)std::min<int64_t>(kMaxStages, (kRingBudget - beside) / r.stage_bytes);
  return r;
}

// Blocks of the backward pass through the ring on so many SMs: one to each, but a block, whose threads add up a row of every
// group, takes kChain groups at most: of more rows there are two blocks to an SM, or three, one after the other (2^31 rows of one
// column were 226,719 additions in a row, and dgamma off by 1e-4).
constexpr int64_t kChain = 2048;
int64_t ring_blocks(int64_t groups, int64_t sms) {
  return std::min(groups, std::max<int64_t>(1, (groups + kChain * sms - 1) / (kChain * sms)) * sms);
}
// Blocks at most that leave sums of their own.  Rows too long for the ring: a block's share is this many at least.
constexpr int64_t kLongShare = 128;
int64_t backward_parts(int64_t m, int64_t n) {
  const int64_t rows = n > kRingColumns ? kLongShare : kRingThreads / team_of(n), shares = (m + rows - 1) / rows;
  const int64_t parts = std::min<int64_t>(kMaxParts, shares);
  return n > kRingColumns ? parts : std::max(parts, ring_blocks(shares, kMaxParts / 2));
}
size_t backward_bytes(int64_t m, int64_t n) { return (size_t)backward_parts(m, n) * 2 * n * 4; }

template <auto kKernel, typename Params>
cudaError_t ring_launch(const Params& p, const RingShape& ring, int teams, int64_t most, size_t beside, size_t least_smem, cudaStream_t s) {
  static PerDeviceOnce once;
  const cudaError_t e = once.run_current(
      [] { return cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingBudget); });
  if (e != cudaSuccess) return e;
  const int64_t blocks = std::min(most, (p.m + teams - 1) / teams);
  return launch_pdl(kKernel, dim3((unsigned)blocks), dim3(kRingThreads),
                    std::max(least_smem, (size_t)ring.stages * ring.stage_bytes + beside), s, 1, p, ring);
}
// Calls go with a team's threads and a thread's eights.
template <typename Go>
cudaError_t by_team(int64_t n, Go&& go) {
  using std::integral_constant;
  if (n <= 64) return go(integral_constant<int, 8>{}, integral_constant<int, 1>{});
  if (n <= 128) return go(integral_constant<int, 16>{}, integral_constant<int, 1>{});
  if (n <= 256) return go(integral_constant<int, 32>{}, integral_constant<int, 1>{});
  if (n <= 512) return go(integral_constant<int, 32>{}, integral_constant<int, 2>{});
  if (n <= 1024) return go(integral_constant<int, 64>{}, integral_constant<int, 2>{});
  if (n <= 2048) return go(integral_constant<int, 128>{}, integral_constant<int, 2>{});
  if (n <= 4096) return go(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  if (n <= 8192) return go(integral_constant<int, 512>{}, integral_constant<int, 2>{});
  return go(integral_constant<int, 512>{}, integral_constant<int, 4>{});
}

// Blocks: as many as are resident together, each with its share of the rows.
template <auto kKernel>
cudaError_t octets_launch(const DeviceInfo& dev, const NormParams& p, int team, cudaStream_t s) {
  const int threads = std::max(team, kBlockThreads), each = threads / team;
  // Of a kernel on devices of one kind, which all are: asked once.
  static std::atomic<int> resident{0};
  int r = resident.load(std::memory_order_relaxed);
  if (r == 0) {
    const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&r, kKernel, threads, 0);
    if (e != cudaSuccess) return e;
    resident.store(r = std::max(r, 1), std::memory_order_relaxed);
  }
  const int64_t blocks = std::min<int64_t>((p.m + each - 1) / each, (int64_t)dev.sms * r);
  return launch_pdl(kKernel, dim3((unsigned)blocks), dim3(threads), 0, s, 1, p);
}

template <bool kF32, bool kRms>
cudaError_t forward_launch(const DeviceInfo& dev, const NormParams& p, bool vec, cudaStream_t s) {
  const int n = p.n;
#define MORELLO_NORM(T, ITER) return octets_launch<norm_kernel<T, ITER, kF32, kRms>>(dev, p, T, s)
  const int64_t beside = n > kRingColumns ? 0 : 4 * n;       // gamma and beta
  const RingShape ring = ring_shape(n, {kF32 ? 4 : 2}, beside);
  if (vec ? n > kRingColumns : ring.stages < 2)
    return launch_pdl(norm_long_kernel<kF32, kRms>, dim3((unsigned)std::min<int64_t>(p.m, (int64_t)dev.sms * 2)),
                      dim3(kLongThreads), 0, s, 1, p);
  if (vec) {
    // 16 columns to a thread; 32 of long rows where there are many: half the teams' joins, and 16 bytes more of every thread
    // in flight (in a row of calls, 32 and 16 columns: 2048 x 8192 15.6 and 18.5 us, 16384 x 4096 49.5 and 53.0, 4096 x 4096 16.4
    // and 15.6, rms 13.8 and 14.6, f32 18.4 and 18.5; 128 x 4096 3.5 and 2.6; 4096 x 2048, where it is 16, 9.6 and 8.7).
    const bool many = p.m >= 4 * (int64_t)dev.sms;
    if (n <= 64) MORELLO_NORM(8, 1);
    if (n <= 128) MORELLO_NORM(16, 1);
    if (n <= 256) MORELLO_NORM(32, 1);
    if (n <= 512) MORELLO_NORM(32, 2);
    if (n <= 1024) MORELLO_NORM(64, 2);
    if (n <= 2048) MORELLO_NORM(128, 2);
    if (n <= 4096) {
      if (many) MORELLO_NORM(128, 4);
      MORELLO_NORM(256, 2);
    }
    if (n <= 8192) {
      if (many) MORELLO_NORM(256, 4);
      MORELLO_NORM(512, 2);
    }
    MORELLO_NORM(512, 4);
  }
  return by_team(n, [&](auto team, auto eights) {
    return ring_launch<norm_ring_kernel<team.value, eights.value, kF32, kRms>>(p, ring, kRingThreads / team.value, dev.sms,
                                                                               (size_t)beside, 0, s);
  });
#undef MORELLO_NORM
}

template <bool kF32, bool kRms>
cudaError_t backward_launch(const DeviceInfo& dev, NormBackwardParams p, float* dgamma, float* dbeta,
                            bool accumulate, bool vec, cudaStream_t s, uint64_t* launches) {
  cudaError_t e = cudaSuccess;
  const bool sums = dgamma || dbeta;
  int parts = (int)backward_parts(p.m, p.n);
  constexpr int kSize = kF32 ? 4 : 2;
  const int64_t beside = vec || p.n > kRingColumns ? 0 : 2 * p.n;       // gamma
  // With R or without: what a call asks for besides does not change the order of its sums.
  RingShape ring = ring_shape(p.n, {kSize, 2}, beside);
  if (ring.stages >= 2) {
    const RingShape with_r = ring_shape(p.n, {kSize, 2, kSize}, beside);
    p.ring_r = p.R && p.dX && with_r.stages >= 2;
    if (p.ring_r) ring = with_r;
    const int64_t teams = kRingThreads / team_of(p.n);
    parts = (int)std::min<int64_t>(parts, ring_blocks((p.m + teams - 1) / teams, dev.sms));
    e = by_team(p.n, [&](auto team, auto eights) {
      constexpr int kT = team.value, kIter = eights.value;
      constexpr size_t kJoined = (size_t)kRingThreads * kIter * 64;      // the teams' sums
      return vec ? ring_launch<norm_backward_kernel<kT, 8, kIter, kF32, kRms>>(p, ring, kRingThreads / kT, parts, 0, kJoined, s)
                 : ring_launch<norm_backward_kernel<kT, 1, kIter, kF32, kRms>>(p, ring, kRingThreads / kT, parts, (size_t)beside, kJoined, s);
    });
  } else {
    parts = (int)std::min<int64_t>(parts, (p.m + kLongShare - 1) / kLongShare);
    if (p.dX) {
      const int64_t blocks = std::min<int64_t>(p.m, (int64_t)dev.sms * 2);
      e = launch_pdl(norm_backward_long_kernel<kF32, kRms>, dim3((unsigned)blocks), dim3(kLongThreads), 0, s, 1, p);
      if (e != cudaSuccess) return e;
      ++*launches;
    }
    if (!sums) return e;
    const int64_t per = (p.m + parts - 1) / parts;
    e = launch_pdl(norm_columns_kernel<kF32>, dim3((unsigned)((p.n + 31) / 32), (unsigned)parts), dim3(1024), 0, s, 1, p, per);
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
                             static_cast<const uint16_t*>(dY), R, dX, static_cast<float*>(ws), dbeta != nullptr, dev.status, false};
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
