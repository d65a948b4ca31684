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
};

// Sum over the 32 lanes, in every lane.
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(kFull, v, d);
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
  static constexpr int kCount = kVec * kIter;
  int t, n;
  __device__ __forceinline__ int of(int e) const {
    return kVec == 8 ? (t + e / 8 * kT) * 8 + e % 8 : t + e * kT;
  }
  __device__ __forceinline__ bool has(int e) const { return of(e - e % kVec) < n; }
};

// The raw elements of those columns, bf16 or f32, as they came from memory.
template <int kT, int kVec, int kIter, bool kF32>
struct Held {
  using C = Columns<kT, kVec, kIter>;
  static constexpr int kWords = kVec == 1 ? C::kCount : C::kCount * (kF32 ? 4 : 2) / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const void* row, const C& c) {
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
  if constexpr (kWarps <= 8) {
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
  using C = Columns<kT, kVec, kIter>;
  constexpr int kCount = C::kCount;
  __shared__ Part parts[2][kTeams][kWarps];
  const int team = (int)threadIdx.x / kT, warp = (int)threadIdx.x % kT / 32, lane = (int)threadIdx.x % 32;
  const C c{(int)threadIdx.x % kT, p.n};
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
  using C = Columns<kT, kVec, kIter>;
  constexpr int kCount = C::kCount;
  __shared__ float2 parts[2][kTeams][kWarps];
  const int team = (int)threadIdx.x / kT, warp = (int)threadIdx.x % kT / 32, lane = (int)threadIdx.x % 32;
  const C c{(int)threadIdx.x % kT, p.n};
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

// Threads of a team: the fewest that hold the row in at most 32 columns each.
int team_of(int64_t n) { return n <= 1024 ? 32 : n <= 4096 ? 128 : n <= 8192 ? 256 : 512; }

int64_t backward_parts(int64_t m, int64_t n) {
  if (m == 0) return 0;
  if (n > kTeamBackward) return std::min<int64_t>(kMaxParts, (m + 127) / 128);
  const int64_t teams = kBlockThreads / team_of(n);
  return std::min<int64_t>(kMaxParts, (m + teams - 1) / teams);
}
size_t backward_bytes(int64_t m, int64_t n) { return (size_t)backward_parts(m, n) * 2 * n * 4; }

template <bool kF32, bool kRms>
cudaError_t forward_launch(const DeviceInfo& dev, const NormParams& p, bool vec, cudaStream_t s) {
  const int n = p.n, t = team_of(n);
  auto go = [&](auto kernel, int threads, int rows_per_block, int resident) {
    const int64_t blocks = std::min<int64_t>((p.m + rows_per_block - 1) / rows_per_block, (int64_t)dev.sms * resident);
    return launch_pdl(kernel, dim3((unsigned)blocks), dim3(threads), 0, s, 1, p);
  };
  if (n > kTeamForward) return go(norm_long_kernel<kF32, kRms>, kLongThreads, 1, 2);
#define MORELLO_NORM(T, VEC, ITER) \
  return go(norm_kernel<T, VEC, ITER, kF32, kRms>, T > kBlockThreads ? T : kBlockThreads, T < kBlockThreads ? kBlockThreads / T : 1, \
            T > kBlockThreads ? 2 : 8)
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
    if (t == 256) MORELLO_NORM(256, 8, 4);
    MORELLO_NORM(512, 8, 4);
  }
  if (t == 32) {
    if (n <= 256) MORELLO_NORM(32, 1, 8);
    MORELLO_NORM(32, 1, 32);
  }
  if (t == 128) {
    if (n <= 2048) MORELLO_NORM(128, 1, 16);
    MORELLO_NORM(128, 1, 32);
  }
  if (t == 256) MORELLO_NORM(256, 1, 32);
  MORELLO_NORM(512, 1, 32);
#undef MORELLO_NORM
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
  const int parts = (int)backward_parts(p.m, p.n);
  if (p.n > kTeamBackward) {
    if (p.dX) {
      const int64_t blocks = std::min<int64_t>(p.m, (int64_t)dev.sms * 2);
      e = launch_pdl(norm_backward_long_kernel<kF32, kRms>, dim3((unsigned)blocks), dim3(kLongThreads), 0, s, 1, p);
      if (e != cudaSuccess) return e;
      ++*launches;
    }
    if (sums) {
      const int64_t per = (p.m + parts - 1) / parts;
      e = launch_pdl(norm_columns_kernel<kF32>, dim3((unsigned)((p.n + 31) / 32), (unsigned)parts), dim3(1024), 0, s, 1, p, per);
    }
  } else {
    e = sums ? backward_rows_launch<kF32, kRms, true>(p, parts, vec, s)
             : backward_rows_launch<kF32, kRms, false>(p, parts, vec, s);
  }
  if (e != cudaSuccess || !sums) {
    if (e == cudaSuccess && p.n <= kTeamBackward) ++*launches;
    return e;
  }
  ++*launches;
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
                     static_cast<const uint16_t*>(beta), static_cast<uint16_t*>(Y), mean, rstd};
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
                             static_cast<const uint16_t*>(dY), R, dX, static_cast<float*>(ws), dbeta != nullptr};
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
