// The memory-bound companions of the linear layers' products: zero-padded copies of
// operands, the activation's slope with the bias gradient, and the weighted sum of a token's rows.
// Each is one pass over its data in 16-byte accesses where alignment allows.
#include <algorithm>

#include "activation.cuh"
#include "column_sums.cuh"
#include "linear.h"
#include "sm100.cuh"

namespace morello {
namespace {

using namespace sm100;

constexpr int kThreads = 256;
constexpr int kSlopeUnroll = 2;     // rows a thread has in flight: four blocks fit an SM's registers (with four rows, two
                                    // blocks, and 48 instead of 39 us on 18,400 x 2 x 1024)
constexpr int kSlopeLanes = 8;      // rows a block takes at a time

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// Elements per access that rows of `cols` elements from p on allow: 8, 4, 2 or 1.
int access_width(int64_t cols, const void* p) {
  for (int w = 8; w > 1; w /= 2)
    if (cols % w == 0 && reinterpret_cast<uintptr_t>(p) % (2 * w) == 0) return w;
  return 1;
}

// Eight elements from src on, of which `cols` exist, in accesses of `width` elements.
__device__ __forceinline__ uint4 load8_raw(const uint16_t* src, int width, int64_t cols) {
  if (cols >= 8) {
    if (width == 8) return *reinterpret_cast<const uint4*>(src);
    if (width == 4) {
      const uint2 a = reinterpret_cast<const uint2*>(src)[0], b = reinterpret_cast<const uint2*>(src)[1];
      return make_uint4(a.x, a.y, b.x, b.y);
    }
    // Rows of odd length start on 4-byte boundaries and off them in turn.
    if (width == 2 || (reinterpret_cast<uintptr_t>(src) & 2u) == 0) {
      const uint32_t* q = reinterpret_cast<const uint32_t*>(src);
      return make_uint4(q[0], q[1], q[2], q[3]);
    }
    const uint32_t first = src[0], last = src[7];
    const uint32_t* q = reinterpret_cast<const uint32_t*>(src + 1);
    const uint32_t a = q[0], b = q[1], c = q[2];
    return make_uint4(first | (a << 16), (a >> 16) | (b << 16), (b >> 16) | (c << 16), (c >> 16) | (last << 16));
  }
  uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t v = e < cols ? (uint32_t)src[e] : 0u;
    w[e >> 1] |= v << ((e & 1) * 16);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8_raw(uint16_t* dst, int width, int64_t cols, const uint4& w) {
  if (cols >= 8 && width == 8) {
    *reinterpret_cast<uint4*>(dst) = w;
  } else if (cols >= 8 && width == 4) {
    reinterpret_cast<uint2*>(dst)[0] = make_uint2(w.x, w.y);
    reinterpret_cast<uint2*>(dst)[1] = make_uint2(w.z, w.w);
  } else if (cols >= 8 && width == 2) {
    uint32_t* q = reinterpret_cast<uint32_t*>(dst);
    q[0] = w.x; q[1] = w.y; q[2] = w.z; q[3] = w.w;
  } else {
    const uint32_t q[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < cols) dst[e] = (uint16_t)(q[e >> 1] >> ((e & 1) * 16));
  }
}
__device__ __forceinline__ void unpack8(const uint4& w, float (&v)[8]) {
  v[0] = bf16_low(w.x); v[1] = bf16_high(w.x); v[2] = bf16_low(w.y); v[3] = bf16_high(w.y);
  v[4] = bf16_low(w.z); v[5] = bf16_high(w.z); v[6] = bf16_low(w.w); v[7] = bf16_high(w.w);
}
__device__ __forceinline__ uint4 pack8(const float (&v)[8]) {
  return make_uint4(bf16_pack(v[0], v[1]), bf16_pack(v[2], v[3]), bf16_pack(v[4], v[5]), bf16_pack(v[6], v[7]));
}

// A thread moves kCopyRows rows' worth of one 8-column group, their loads in flight together.
constexpr int kCopyRows = 4;
struct CopyParams {
  const uint16_t* src;
  uint4* dst;
  int64_t rows_in, cols_in, rows_out;
  int octets;                 // 8-column groups of a row of dst
  int spans;                  // > 0: blocks to a row group
  int width;                  // elements per access of src
  int row_groups;             // of kCopyRows rows in a group of dst
  int64_t threads;            // groups * row_groups * octets
  int topk;
  bool by_warp;               // gather in 16-byte accesses: a warp to a row
  const int32_t* row_src;     // gather
  const int32_t* live;        // number of live rows, or null
  const int32_t* counts;      // by group of dst: a group without rows is left alone, or null
};

struct CopyBatch {
  CopyParams job[kMaxCopies];
  int blocks0;                // blocks of the first job
  bool beside;                // made while the launch before runs: waits for it at the end
};

// Rows r0 .. of group g, columns 8 o .. of dst.
__device__ __forceinline__ void copy_rows(const CopyParams& p, int64_t g, int64_t r0, int o) {
  const int64_t left = p.cols_in - (int64_t)o * 8;
  const uint16_t* src[kCopyRows];
#pragma unroll
  for (int i = 0; i < kCopyRows; ++i) {
    const int64_t r = r0 + i;
    int64_t from = r;
    if (p.row_src && r < p.rows_out) {
      const int32_t s = p.row_src[r];
      from = s < 0 ? -1 : s / p.topk;
    }
    const bool there = r < p.rows_out && from >= 0 && from < p.rows_in && left > 0;
    src[i] = there ? p.src + (g * p.rows_in + from) * p.cols_in + (int64_t)o * 8 : nullptr;
  }
  uint4 w[kCopyRows];
  const bool octets = p.width == 8;        // one test for all rows, so that their loads go out together
#pragma unroll
  for (int i = 0; i < kCopyRows; ++i) w[i] = make_uint4(0u, 0u, 0u, 0u);
  if (octets) {
#pragma unroll
    for (int i = 0; i < kCopyRows; ++i)
      if (src[i]) w[i] = *reinterpret_cast<const uint4*>(src[i]);
  } else {
#pragma unroll
    for (int i = 0; i < kCopyRows; ++i)
      if (src[i]) w[i] = load8_raw(src[i], p.width, left);
  }
#pragma unroll
  for (int i = 0; i < kCopyRows; ++i)
    if (r0 + i < p.rows_out) p.dst[(g * p.rows_out + r0 + i) * p.octets + o] = w[i];
}

// Row r of dst in a gather: its token is looked up once for the whole row.  (As four rows of one column group to a thread,
// 16,384 rows of 2048 took 23 us instead of 16.6, most of it the addresses' arithmetic.)
constexpr int kGatherBatch = 4;
__device__ __forceinline__ void gather_row(const CopyParams& p, int64_t r, int lane) {
  const int32_t token = r < p.rows_out ? p.row_src[r] : -1;
  if (r >= p.rows_out || r >= *p.live) return;
  const uint4* src = token < 0 || token / p.topk >= p.rows_in ? nullptr : reinterpret_cast<const uint4*>(p.src) + (int64_t)(token / p.topk) * p.octets;
  uint4* dst = p.dst + r * p.octets;
  for (int o0 = lane; o0 < p.octets; o0 += 32 * kGatherBatch) {
    uint4 w[kGatherBatch];
#pragma unroll
    for (int i = 0; i < kGatherBatch; ++i) {
      w[i] = make_uint4(0u, 0u, 0u, 0u);
      if (src && o0 + 32 * i < p.octets) w[i] = src[o0 + 32 * i];
    }
#pragma unroll
    for (int i = 0; i < kGatherBatch; ++i)
      if (o0 + 32 * i < p.octets) dst[o0 + 32 * i] = w[i];
  }
}

__global__ void __launch_bounds__(kThreads) copy_kernel(const CopyBatch batch) {
  const bool second = (int)blockIdx.x >= batch.blocks0;
  const CopyParams p = second ? batch.job[1] : batch.job[0];     // by value: through an index every field is a load
  const int block = (int)blockIdx.x - (second ? batch.blocks0 : 0);
  if (p.by_warp) {
    if (!batch.beside) pdl_wait();
    pdl_release();
    gather_row(p, (int64_t)block * (kThreads / 32) + (threadIdx.x >> 5), threadIdx.x & 31);
    if (batch.beside) pdl_wait();
    return;
  }
  // Long rows: a block is a span of kThreads octets of a row group, one division for all its threads.  Short ones:
  // row groups and octets are numbered through (a 64-bit division is a hundred instructions, so 32 bits where they do).
  const bool small = p.threads < (1ll << 31);
  int64_t row_group;
  int o;
  bool mine = true;
  if (p.spans > 0) {
    row_group = (uint32_t)block / (uint32_t)p.spans;
    o = (block - (int)row_group * p.spans) * kThreads + threadIdx.x;
    mine = o < p.octets;
  } else {
    const int64_t idx = (int64_t)block * kThreads + threadIdx.x;
    row_group = small ? (int64_t)((uint32_t)idx / (uint32_t)p.octets) : idx / p.octets;
    o = (int)(idx - row_group * p.octets);
    mine = idx < p.threads;
  }
  const int64_t g = small ? (int64_t)((uint32_t)row_group / (uint32_t)p.row_groups) : row_group / p.row_groups;
  const int64_t r0 = (row_group - g * p.row_groups) * kCopyRows;
  // beside: what came before the launch that this one follows is complete, since this one starts when all blocks of that
  // one are past their own wait.  The wait at the end makes this one's end the end of both.
  if (!batch.beside) pdl_wait();
  pdl_release();
  if (mine && !(p.live && r0 >= *p.live) && !(p.counts && p.counts[g] == 0)) copy_rows(p, g, r0, o);
  if (batch.beside) pdl_wait();
}

struct SlopeParams {
  const uint16_t* dY;
  const uint16_t* Z;
  uint16_t* dZ;
  float* partial;
  int64_t rows, n, pitch;      // pitch: columns of a row of dZ, the width rounded up to 8
  int width_y, width_z, width_up;   // elements per access of dY, of Z, and of dZ's second half
  const int32_t* row_src;
  const int32_t* live;
};

// A block: 256 columns (32 groups of 8) x kSlopeRows rows, eight rows at a time.
// kOctets: every row is in 16-byte accesses (a test per access kept the loads from going out together), and the strips fit
// the grid's second dimension, 65,535 of them: the third, for layers of more than 16.7 million columns, costs registers (spills in
// five forms).
template <int kAct, bool kGated, bool kSums, bool kOctets>
__global__ void __launch_bounds__(kThreads, kSums ? 3 : 4) slope_kernel(const SlopeParams p) {
  __shared__ float sums[kSums ? kSlopeLanes : 1][kGated ? 2 : 1][256 + 8];
  const int group = threadIdx.x & 31, lane = threadIdx.x >> 5;
  const int64_t col = (int64_t)(kOctets ? blockIdx.y : blockIdx.z * gridDim.y + blockIdx.y) * 256 + group * 8;
  const int64_t row_begin = (int64_t)blockIdx.x * kSlopeRows;
  pdl_wait();
  pdl_release();
  if (p.live) {
    // An expert's tokens come first among its rows, which begin at a multiple of kSlopeRows: a first row without one means
    // none.  Nothing is read then, but zeros are left for the products, which run over such rows.
    const int32_t token = p.row_src[row_begin];
    if (row_begin >= *p.live) return;
    if (token < 0) {
      const int64_t octets = p.pitch / 8, end = min(p.rows, row_begin + kSlopeRows);
      uint4* dst = reinterpret_cast<uint4*>(p.dZ);
      for (int64_t r = row_begin + lane; p.dZ && r < end; r += kSlopeLanes)
        for (int64_t o = blockIdx.y * 32 + group; o < octets; o += gridDim.y * 32) dst[r * octets + o] = make_uint4(0u, 0u, 0u, 0u);
      return;
    }
  }
  const int64_t row_end = min(p.rows, row_begin + kSlopeRows);
  const int64_t left = p.n - col;
  float s0[8], s1[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) s0[e] = s1[e] = 0.f;
  if (left > 0) {
    const int64_t width = kGated ? 2 * p.n : p.n;
    const bool wants_z = kAct != kActNone || kGated;
#pragma unroll 1
    for (int64_t r0 = row_begin + lane; r0 < row_end; r0 += kSlopeUnroll * kSlopeLanes) {
      // The loads of the rows first.
      uint4 wd[kSlopeUnroll], w0[kSlopeUnroll], w1[kGated ? kSlopeUnroll : 1];
      bool holds[kSlopeUnroll];     // looked at after the loads: rows without a token may hold anything
#pragma unroll
      for (int i = 0; i < kSlopeUnroll; ++i) {
        const int64_t row = r0 + i * kSlopeLanes;
        holds[i] = row < row_end && (!p.row_src || p.row_src[row] >= 0);
        wd[i] = w0[i] = make_uint4(0u, 0u, 0u, 0u);
        if constexpr (kGated) w1[i] = make_uint4(0u, 0u, 0u, 0u);
        if (row >= row_end) continue;
        wd[i] = load8_raw(p.dY + row * p.n + col, kOctets ? 8 : p.width_y, kOctets ? 8 : left);
        if (wants_z) w0[i] = load8_raw(p.Z + row * width + col, kOctets ? 8 : p.width_z, kOctets ? 8 : left);
        if constexpr (kGated) w1[i] = load8_raw(p.Z + row * width + p.n + col, kOctets ? 8 : p.width_z, kOctets ? 8 : left);
      }
#pragma unroll
      for (int i = 0; i < kSlopeUnroll; ++i) {
        const int64_t row = r0 + i * kSlopeLanes;
        if (row >= row_end) break;
        float dy[8], z0[8], z1[8], d0[8], d1[8];
        unpack8(wd[i], dy);
        unpack8(w0[i], z0);
        if constexpr (kGated) unpack8(w1[i], z1);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float value;
          const float slope = act_slope<kAct>(z0[e], &value);
          if constexpr (kGated) {
            d0[e] = dy[e] * z1[e] * slope;
            d1[e] = dy[e] * value;
          } else {
            d0[e] = dy[e] * slope;
            d1[e] = 0.f;
          }
          if (!holds[i]) d0[e] = d1[e] = 0.f;
        }
        if (p.dZ) {
          uint16_t* dst = p.dZ + row * p.pitch + col;
          store8_raw(dst, 8, kOctets ? 8 : left, pack8(d0));        // rows of dZ are multiples of eight
          if constexpr (kGated) store8_raw(dst + p.n, kOctets ? 8 : p.width_up, kOctets ? 8 : left, pack8(d1));
          if (!kOctets && left <= 8)       // the columns that round the row up to eight
            for (int64_t c = width; c < p.pitch; ++c) p.dZ[row * p.pitch + c] = 0;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if constexpr (kSums) s0[e] += d0[e];
          if constexpr (kSums && kGated) s1[e] += d1[e];
        }
      }
    }
  }
  if constexpr (kSums) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      sums[lane][0][group * 8 + e] = s0[e];
      if constexpr (kGated) sums[lane][1][group * 8 + e] = s1[e];
    }
    __syncthreads();
    const int64_t c = (int64_t)(kOctets ? blockIdx.y : blockIdx.z * gridDim.y + blockIdx.y) * 256 + threadIdx.x;
    if (c < p.n) {
      const int64_t width = kGated ? 2 * p.n : p.n;
#pragma unroll
      for (int h = 0; h < (kGated ? 2 : 1); ++h) {
        float s = 0.f;
#pragma unroll
        for (int l = 0; l < kSlopeLanes; ++l) s += sums[l][h][threadIdx.x];
        p.partial[(int64_t)blockIdx.x * width + h * p.n + c] = s;
      }
    }
  }
}

__global__ void __launch_bounds__(kThreads) slope_sum_kernel(const ColumnSums c) {
  pdl_wait();
  pdl_release();
  column_sums(c, (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), (int64_t)gridDim.x * (kThreads / 32), threadIdx.x & 31);
}

struct CombineParams {
  const int32_t* slot;
  const float* weights;
  const void* Y;
  const uint16_t* residual;
  uint16_t* out;
  int64_t n, y_pitch;
  int topk;
  int64_t octets, threads;
  int width;                  // elements per access of residual and out
  bool vec_y;                 // f32 Y in 16-byte accesses
  int width_y;                // elements per access of bf16 Y
};

template <bool kF32>
__global__ void __launch_bounds__(kThreads) combine_kernel(const CombineParams p) {
  const int64_t idx = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  pdl_wait();
  pdl_release();
  if (idx >= p.threads) return;
  const int64_t t = p.threads < (1ll << 31) ? (int64_t)((uint32_t)idx / (uint32_t)p.octets) : idx / p.octets;
  const int64_t o = idx - t * p.octets;
  const int64_t col = o * 8, left = p.n - col;
  const bool vec_y = p.vec_y && left >= 8;
  float sum[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) sum[e] = 0.f;
  // Four places at a time, their rows' loads in flight together.
  for (int k0 = 0; k0 < p.topk; k0 += 4) {
    int32_t row[4];
    float w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool there = k0 + i < p.topk;
      row[i] = there ? p.slot[t * p.topk + k0 + i] : -1;
      w[i] = there && p.weights ? p.weights[t * p.topk + k0 + i] : 1.f;
    }
    float v[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
      if (row[i] < 0) continue;
      if constexpr (kF32) {
        const float* y = static_cast<const float*>(p.Y) + (int64_t)row[i] * p.y_pitch + col;
        if (vec_y) {
          const float4 a = reinterpret_cast<const float4*>(y)[0], b = reinterpret_cast<const float4*>(y)[1];
          v[i][0] = a.x; v[i][1] = a.y; v[i][2] = a.z; v[i][3] = a.w;
          v[i][4] = b.x; v[i][5] = b.y; v[i][6] = b.z; v[i][7] = b.w;
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (e < left) v[i][e] = y[e];
        }
      } else {
        unpack8(load8_raw(static_cast<const uint16_t*>(p.Y) + (int64_t)row[i] * p.y_pitch + col, p.width_y, left), v[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (row[i] < 0) continue;        // not routed: nothing is added, whatever the weight
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] = fmaf(w[i], v[i][e], sum[e]);
    }
  }
  if (p.residual) {
    float r[8];
    unpack8(load8_raw(p.residual + t * p.n + col, p.width, left), r);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] += r[e];
  }
  store8_raw(p.out + t * p.n + col, p.width, left, pack8(sum));
}

cudaError_t grid_for(int64_t threads, unsigned* blocks) {
  const int64_t n = (threads + kThreads - 1) / kThreads;
  if (n >= (1ll << 31)) return cudaErrorInvalidValue;
  *blocks = (unsigned)n;
  return cudaSuccess;
}

}  // namespace

cudaError_t copy_launch(const CopyJob* jobs, int count, bool beside, cudaStream_t stream, uint64_t* launches) {
  if (count > kMaxCopies) return cudaErrorInvalidValue;
  CopyBatch batch{};
  batch.beside = beside;
  int64_t blocks = 0;
  int at = 0;
  for (int i = 0; i < count; ++i) {
    const CopyJob& j = jobs[i];
    CopyParams p{};
    p.src = j.src;
    p.dst = reinterpret_cast<uint4*>(j.dst);
    p.rows_in = j.rows_in;
    p.cols_in = j.cols_in;
    p.rows_out = j.rows_out;
    p.octets = (int)(j.cols_out / 8);
    p.width = access_width(j.cols_in, j.src);
    p.row_groups = (int)((j.rows_out + kCopyRows - 1) / kCopyRows);
    p.threads = j.groups * p.row_groups * (int64_t)p.octets;
    if (j.by_expert) p.counts = j.by_expert->counts;
    if (j.experts) {
      p.live = j.experts->offsets + j.experts->experts;
      if (j.gather) {
        p.row_src = j.experts->row_src;
        p.topk = (int)j.experts->topk;
      }
    }
    // Spans where they leave few threads of a block without work.
    p.spans = p.octets % kThreads == 0 || p.octets > 4 * kThreads ? (p.octets + kThreads - 1) / kThreads : 0;
    p.by_warp = p.row_src && p.width == 8;
    const int64_t mine = p.by_warp ? (p.rows_out + kThreads / 32 - 1) / (kThreads / 32) : p.spans > 0 ? j.groups * (int64_t)p.row_groups * p.spans : (p.threads + kThreads - 1) / kThreads;
    if (mine <= 0) continue;
    if (at == 0) batch.blocks0 = (int)std::min<int64_t>(mine, (1ll << 31) - 1);
    batch.job[at++] = p;
    blocks += mine;
  }
  if (blocks == 0) return cudaSuccess;
  if (blocks >= (1ll << 31)) return cudaErrorInvalidValue;
  const cudaError_t e = launch_pdl(copy_kernel, dim3((unsigned)blocks), dim3(kThreads), 0, stream, 1, batch);
  if (e == cudaSuccess) ++*launches;
  return e;
}

size_t slope_partial_bytes(int64_t rows, int64_t n, bool gated) {
  return (size_t)((rows + kSlopeRows - 1) / kSlopeRows) * n * (gated ? 2 : 1) * 4;
}

cudaError_t slope_launch(const SlopeCall& c, cudaStream_t stream, uint64_t* launches) {
  if (c.n <= 0) return cudaSuccess;
  const int64_t parts = (c.rows + kSlopeRows - 1) / kSlopeRows;
  const int64_t width = c.gated ? 2 * c.n : c.n;
  cudaError_t e = cudaSuccess;
  if (parts > 0) {
    SlopeParams p{};
    p.dY = c.dY;
    p.Z = c.Z;
    p.dZ = c.dZ;
    p.partial = c.partial;
    p.rows = c.rows;
    p.n = c.n;
    p.pitch = (width + 7) / 8 * 8;
    p.width_y = access_width(c.n, c.dY);
    p.width_z = access_width(c.n, c.Z);
    p.width_up = access_width(c.n, nullptr);
    if (c.experts) {
      p.row_src = c.experts->row_src;
      p.live = c.experts->offsets + c.experts->experts;
    }
    const int64_t strips = (c.n + 255) / 256;
    if (parts >= (1ll << 31)) return cudaErrorInvalidValue;
    const unsigned deep = (unsigned)((strips + 65534) / 65535), wide = (unsigned)((strips + deep - 1) / deep);
    const dim3 grid((unsigned)parts, wide, deep);
    const bool with = p.partial != nullptr;
    const bool octets = p.width_y == 8 && p.width_z == 8 && deep == 1;
    auto go = [&](auto sums, auto none, auto sums_any, auto none_any) {
      return launch_pdl(octets ? (with ? sums : none) : (with ? sums_any : none_any), grid, dim3(kThreads), 0, stream, 1, p);
    };
    switch (c.act * 2 + (c.gated ? 1 : 0)) {
      case 0: e = go(slope_kernel<kActNone, false, true, true>, slope_kernel<kActNone, false, false, true>, slope_kernel<kActNone, false, true, false>,
                         slope_kernel<kActNone, false, false, false>); break;
      case 1: e = go(slope_kernel<kActNone, true, true, true>, slope_kernel<kActNone, true, false, true>, slope_kernel<kActNone, true, true, false>,
                         slope_kernel<kActNone, true, false, false>); break;
      case 2: e = go(slope_kernel<kActRelu, false, true, true>, slope_kernel<kActRelu, false, false, true>, slope_kernel<kActRelu, false, true, false>,
                         slope_kernel<kActRelu, false, false, false>); break;
      case 3: e = go(slope_kernel<kActRelu, true, true, true>, slope_kernel<kActRelu, true, false, true>, slope_kernel<kActRelu, true, true, false>,
                         slope_kernel<kActRelu, true, false, false>); break;
      case 4: e = go(slope_kernel<kActGelu, false, true, true>, slope_kernel<kActGelu, false, false, true>, slope_kernel<kActGelu, false, true, false>,
                         slope_kernel<kActGelu, false, false, false>); break;
      case 5: e = go(slope_kernel<kActGelu, true, true, true>, slope_kernel<kActGelu, true, false, true>, slope_kernel<kActGelu, true, true, false>,
                         slope_kernel<kActGelu, true, false, false>); break;
      case 6: e = go(slope_kernel<kActGeluTanh, false, true, true>, slope_kernel<kActGeluTanh, false, false, true>, slope_kernel<kActGeluTanh, false, true, false>,
                         slope_kernel<kActGeluTanh, false, false, false>); break;
      case 7: e = go(slope_kernel<kActGeluTanh, true, true, true>, slope_kernel<kActGeluTanh, true, false, true>, slope_kernel<kActGeluTanh, true, true, false>,
                         slope_kernel<kActGeluTanh, true, false, false>); break;
      case 8: e = go(slope_kernel<kActSilu, false, true, true>, slope_kernel<kActSilu, false, false, true>, slope_kernel<kActSilu, false, true, false>,
                         slope_kernel<kActSilu, false, false, false>); break;
      default: e = go(slope_kernel<kActSilu, true, true, true>, slope_kernel<kActSilu, true, false, true>, slope_kernel<kActSilu, true, true, false>,
                         slope_kernel<kActSilu, true, false, false>); break;
    }
    if (e != cudaSuccess) return e;
    ++*launches;
  }
  return e;
}

cudaError_t slope_sum_launch(const ColumnSums& c, cudaStream_t stream, uint64_t* launches) {
  const int64_t items = c.groups * ((c.width + kSumColumns - 1) / kSumColumns);
  if (items <= 0) return cudaSuccess;
  const int64_t blocks = std::min<int64_t>((items + kThreads / 32 - 1) / (kThreads / 32), 1 << 20);
  const cudaError_t e = launch_pdl(slope_sum_kernel, dim3((unsigned)blocks), dim3(kThreads), 0, stream, 1, c);
  if (e == cudaSuccess) ++*launches;
  return e;
}

cudaError_t combine_launch(const ExpertRows& x, bool y_f32, int64_t n, int64_t y_pitch, const float* weights,
                           const void* Y, const uint16_t* residual, uint16_t* out, cudaStream_t stream,
                           uint64_t* launches) {
  CombineParams p{};
  p.slot = x.slot;
  p.weights = weights;
  p.Y = Y;
  p.residual = residual;
  p.out = out;
  p.n = n;
  p.y_pitch = y_pitch;
  p.topk = (int)x.topk;
  p.octets = (n + 7) / 8;
  p.threads = x.tokens * p.octets;
  p.width = std::min(access_width(n, out), access_width(n, residual));
  p.vec_y = y_pitch % 8 == 0 && aligned16(Y);
  p.width_y = access_width(y_pitch, Y);
  if (p.threads <= 0) return cudaSuccess;
  unsigned blocks = 0;
  cudaError_t e = grid_for(p.threads, &blocks);
  if (e != cudaSuccess) return e;
  e = y_f32 ? launch_pdl(combine_kernel<true>, dim3(blocks), dim3(kThreads), 0, stream, 1, p)
            : launch_pdl(combine_kernel<false>, dim3(blocks), dim3(kThreads), 0, stream, 1, p);
  if (e == cudaSuccess) ++*launches;
  return e;
}

}  // namespace morello
