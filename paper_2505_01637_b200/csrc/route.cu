// Routing to experts: scores, the choice of the best, their weights, the gradient of the logits, and
// the plan that sorts the routed rows by expert.
//
// One warp per token.  Lane l holds experts l, l + 32, ...; a key is mapped to an unsigned integer of
// the same order.  With many experts per lane the choice is made among few: the topk-th largest of the lanes'
// maxima is a lower bound of the topk-th largest key, so only keys from there on, a dozen or so, are candidates;
// one to a lane, each counts the candidates before it, which is its place.  Few experts per lane, or more than 32
// candidates (rows of equal logits): the warp's maximum and the lowest index that has it, two integer reductions
// (redux) and a pass over the lane's keys per chosen expert.  All sums are in f32 in a fixed order.
#include <algorithm>
#include <type_traits>

#include "activation.cuh"
#include "route.h"
#include "sm100.cuh"

namespace morello {
namespace {

using namespace sm100;

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr uint32_t kFull = 0xffffffffu;
constexpr uint32_t kNone = 0xffffffffu;

// 0: out of the choice; 1: NaN, below every number; then the numbers in order (-0 equals +0).
__device__ __forceinline__ uint32_t order_of(float key) {
  if (key != key) return 1u;
  const uint32_t u = __float_as_uint(key + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(kFull, v, d);
  return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor_sync(kFull, v, d));
  return v;
}

template <bool kF32>
__device__ __forceinline__ float load_logit(const void* p, int64_t i) {
  if constexpr (kF32) return static_cast<const float*>(p)[i];
  else return bf16_value(static_cast<const uint16_t*>(p)[i]);
}

struct RouteParams {
  const void* logits;
  const float* bias;
  int32_t* idx;
  float* weights;
  int64_t tokens;
  int experts, topk, groups, topk_groups;
  bool sigmoid, renorm;
  float scale;
};

// From this many experts per lane on the choice is among candidates (at two per lane, 64 experts, that took 3.03 instead of
// 2.79 us on 16 tokens and 3.2 instead of 3.1 on 4096).
constexpr int kFewest = 4;

// kPer: experts per lane.  kWhole: every lane holds that many (a test per expert and phase: 10.7 instead of 9.2 us on
// 16384 x 256).
template <int kPer, bool kWhole, bool kF32, bool kSigmoid>
__global__ void __launch_bounds__(kThreads) route_kernel(const RouteParams p) {
  extern __shared__ uint32_t group_keys[];       // [kWarps][experts] when experts are grouped
  __shared__ uint64_t candidates[kWarps][32];    // key and ~expert: among equal keys the lower expert is the larger
  __shared__ int chosen[kWarps][32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t t = (int64_t)blockIdx.x * kWarps + warp;
  const int experts = kWhole ? 32 * kPer : p.experts;
  pdl_wait();
  pdl_release();
  if (t >= p.tokens) return;
  float x[kPer];
  uint32_t key[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int e = i * 32 + lane;
    x[i] = e < experts ? load_logit<kF32>(p.logits, t * experts + e) : 0.f;
  }
  float s[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) s[i] = kSigmoid ? 1.f / (1.f + expf(-x[i])) : x[i];
  if (p.bias) {
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (i * 32 + lane < experts) s[i] += p.bias[i * 32 + lane];
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) key[i] = i * 32 + lane < experts ? order_of(s[i]) : 0u;
  if (p.groups > 1) {
    // Lane g scores group g: the sum of its two largest keys (sigmoid) or its largest (softmax).
    uint32_t* mine = group_keys + (size_t)warp * experts;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (i * 32 + lane < experts) mine[i * 32 + lane] = key[i];
    __syncwarp();
    const int per = experts / p.groups;
    uint32_t score = 0u;
    if (lane < p.groups) {
      uint32_t first = 0u, second = 0u;
      for (int e = 0; e < per; ++e) {
        const uint32_t v = mine[lane * per + e];
        second = max(second, min(first, v));
        first = max(first, v);
      }
      score = first;
      if constexpr (kSigmoid) {
        auto value = [](uint32_t o) {
          return o <= 1u ? __uint_as_float(0x7fc00000u) : __uint_as_float((o & 0x80000000u) ? (o & 0x7fffffffu) : ~o);
        };
        score = per > 1 ? order_of(value(first) + value(second)) : first;
      }
    }
    int rank = 0;
    for (int g = 0; g < p.groups; ++g) {
      const uint32_t other = __shfl_sync(kFull, score, g);
      rank += (other > score || (other == score && g < lane)) ? 1 : 0;
    }
    const uint32_t keep = __ballot_sync(kFull, lane < p.groups && rank < p.topk_groups);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int e = i * 32 + lane;
      if (e < experts && !((keep >> (e / per)) & 1u)) key[i] = 0u;
    }
  }

  // Lane j ends up with the j-th choice.
  int my_idx = -1;
  bool done = false;
  if constexpr (kPer >= kFewest) {
    uint32_t left = 0u, bound = 0u;
#pragma unroll
    for (int i = 0; i < kPer; ++i) left = max(left, key[i]);
    // Equal maxima go together, which only lowers the bound.
    for (int j = 0; j < p.topk; ++j) {
      bound = __reduce_max_sync(kFull, left);
      if (left == bound) left = 0u;
    }
    // At least topk keys are >= bound (0 when lanes ran out: everything still in the choice is a candidate).
    bound = max(bound, 1u);
    int mine = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) mine += key[i] >= bound ? 1 : 0;
    int upto = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int o = __shfl_up_sync(kFull, upto, d);
      if (lane >= d) upto += o;
    }
    const int count = __shfl_sync(kFull, upto, 31);
    if (count <= 32) {
      uint64_t* at = &candidates[warp][upto - mine];
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (key[i] >= bound) *at++ = (uint64_t)key[i] << 32 | ~(uint32_t)(i * 32 + lane);
      __syncwarp();
      const uint64_t own = candidates[warp][lane];       // past count: what an earlier use left, not looked at
      int place = 0;
#pragma unroll 4
      for (int j = 0; j < count; ++j) place += candidates[warp][j] > own ? 1 : 0;
      if (lane < count && place < p.topk) chosen[warp][place] = (int)~(uint32_t)own;
      __syncwarp();
      if (lane < p.topk) my_idx = chosen[warp][lane];
      done = true;
    }
  }
  for (int j = 0; j < p.topk && !done; ++j) {
    uint32_t best = 0u;
#pragma unroll
    for (int i = 0; i < kPer; ++i) best = max(best, key[i]);
    best = __reduce_max_sync(kFull, best);
    uint32_t at = kNone;
#pragma unroll
    for (int i = kPer - 1; i >= 0; --i)
      if (key[i] == best) at = (uint32_t)(i * 32 + lane);
    at = __reduce_min_sync(kFull, at);
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (at == (uint32_t)(i * 32 + lane)) key[i] = 0u;
    if (lane == j) my_idx = (int)at;
  }
  const bool holds = lane < p.topk && my_idx >= 0 && my_idx < experts;
  const float my_x = holds ? load_logit<kF32>(p.logits, t * experts + my_idx) : -INFINITY;

  float w = 0.f;
  if constexpr (kSigmoid) {
    w = lane < p.topk ? 1.f / (1.f + expf(-my_x)) : 0.f;
  } else {
    float m = my_x;                        // among the chosen, whatever the others are, when only their shares count
    if (!p.renorm) {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (i * 32 + lane < experts) m = fmaxf(m, x[i]);
    }
    m = warp_max(m);
    if (m == -INFINITY) m = 0.f;           // nothing but masked logits: every weight is 0
    w = lane < p.topk ? expf(my_x - m) : 0.f;
    if (!p.renorm) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (i * 32 + lane < experts) sum += expf(x[i] - m);
      sum = warp_sum(sum);
      w = sum == 0.f ? 0.f : w / sum;
    }
  }
  if (p.renorm) {
    const float sum = warp_sum(w);
    w = sum == 0.f ? 0.f : w / sum;
  }
  if (lane < p.topk) {
    p.idx[t * p.topk + lane] = my_idx;
    p.weights[t * p.topk + lane] = w * p.scale;
  }
}

struct RouteBackParams {
  const void* logits;
  const int32_t* idx;
  const float* dweights;
  void* dlogits;
  int64_t tokens;
  int experts, topk;
  bool sigmoid, renorm;
  float scale;
  bool vec;          // rows of dlogits in four-element accesses
};

// With g = scale * dweights and w the weights before scaling:
//   softmax, all experts:   dx_e = w_e [chosen] g_e - p_e sum(g w)
//   softmax, renormalised:  dx_e = w_e (g_e - sum(g w)), chosen experts only
//   sigmoid:                dx_e = g_e s_e (1 - s_e)
//   sigmoid, renormalised:  dx_e = w_e (g_e - sum(g w)) (1 - s_e)
template <int kPer, bool kF32>
__global__ void __launch_bounds__(kThreads) route_backward_kernel(const RouteBackParams p) {
  __shared__ uint32_t named[kWarps][kPer];       // a bit per expert
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t t = (int64_t)blockIdx.x * kWarps + warp;
  pdl_wait();
  pdl_release();
  if (t >= p.tokens) return;
  const bool softmax_all = !p.sigmoid && !p.renorm;
  // Lane j: the j-th choice.
  int e_j = -1;
  float g = 0.f, x_j = 0.f;
  if (lane < p.topk) {
    e_j = p.idx[t * p.topk + lane];
    if (e_j < 0 || e_j >= p.experts) e_j = -1;
    if (e_j >= 0) {
      g = p.scale * p.dweights[t * p.topk + lane];
      x_j = load_logit<kF32>(p.logits, t * p.experts + e_j);
    }
  }
  float x[kPer];
  float m = -INFINITY, inv = 0.f;
  if (softmax_all) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int e = i * 32 + lane;
      x[i] = e < p.experts ? load_logit<kF32>(p.logits, t * p.experts + e) : -INFINITY;
      m = fmaxf(m, x[i]);
    }
    m = warp_max(m);
    if (m == -INFINITY) m = 0.f;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      x[i] = i * 32 + lane < p.experts ? expf(x[i] - m) : 0.f;
      sum += x[i];
    }
    sum = warp_sum(sum);
    inv = sum == 0.f ? 0.f : 1.f / sum;
  }
  float w = 0.f, d = 0.f;
  if (p.sigmoid) {
    const float s = e_j >= 0 ? 1.f / (1.f + expf(-x_j)) : 0.f;
    if (p.renorm) {
      const float sum = warp_sum(s);
      w = sum == 0.f ? 0.f : s / sum;
      const float dot = warp_sum(g * w);
      d = w * (g - dot) * (1.f - s);
    } else {
      d = g * s * (1.f - s);
    }
  } else if (p.renorm) {
    float mm = warp_max(e_j >= 0 ? x_j : -INFINITY);
    if (mm == -INFINITY) mm = 0.f;
    w = e_j >= 0 ? expf(x_j - mm) : 0.f;
    const float sum = warp_sum(w);
    w = sum == 0.f ? 0.f : w / sum;
    const float dot = warp_sum(g * w);
    d = w * (g - dot);
  } else {
    w = e_j >= 0 ? expf(x_j - m) * inv : 0.f;
    const float dot = warp_sum(g * w);
    d = g * w;
#pragma unroll
    for (int i = 0; i < kPer; ++i) x[i] *= -dot * inv;
  }
  if (!softmax_all) {
    // Everything but the chosen is zero: the row is cleared, then the chosen are set.
    const int64_t row = t * p.experts;
    if (lane < kPer) named[warp][lane] = 0u;
    // A caller's own choice may name an expert more than once: all its places get the sum of their terms, in order.  (Found
    // by a ballot per bit of the experts' numbers it took 0.9 us of 16384 x 256.)
    auto add_repeated = [&] {
      const bool again = e_j >= 0 && ((atomicOr(&named[warp][e_j >> 5], 1u << (e_j & 31)) >> (e_j & 31)) & 1u);
      if (!__any_sync(kFull, again)) return;
      float total = 0.f;
      for (int j = 0; j < p.topk; ++j) {
        const float v = __shfl_sync(kFull, d, j);
        if (__shfl_sync(kFull, e_j, j) == e_j) total += v;
      }
      d = total;
    };
    if constexpr (kF32) {
      float* dst = static_cast<float*>(p.dlogits) + row;
      if (p.vec) {
        for (int e = lane * 4; e < p.experts; e += 128) *reinterpret_cast<float4*>(dst + e) = make_float4(0.f, 0.f, 0.f, 0.f);
      } else {
        for (int e = lane; e < p.experts; e += 32) dst[e] = 0.f;
      }
      __syncwarp();
      add_repeated();
      if (e_j >= 0) dst[e_j] = d;
    } else {
      uint16_t* dst = static_cast<uint16_t*>(p.dlogits) + row;
      if (p.vec) {
        for (int e = lane * 4; e < p.experts; e += 128) *reinterpret_cast<uint2*>(dst + e) = make_uint2(0u, 0u);
      } else {
        for (int e = lane; e < p.experts; e += 32) dst[e] = 0;
      }
      __syncwarp();
      add_repeated();
      if (e_j >= 0) dst[e_j] = bf16_round(d);
    }
    return;
  }
  for (int j = 0; j < p.topk; ++j) {
    const int e = __shfl_sync(kFull, e_j, j);
    const float v = __shfl_sync(kFull, d, j);
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (e == i * 32 + lane) x[i] += v;
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int e = i * 32 + lane;
    if (e >= p.experts) continue;
    if constexpr (kF32) static_cast<float*>(p.dlogits)[t * p.experts + e] = x[i];
    else static_cast<uint16_t*>(p.dlogits)[t * p.experts + e] = bf16_round(x[i]);
  }
}

template <int kPer, bool kF32, bool kSigmoid>
cudaError_t launch_route_form(const RouteParams& p, unsigned blocks, cudaStream_t stream) {
  const size_t smem = p.groups > 1 ? (size_t)kWarps * p.experts * 4 : 0;
  return launch_pdl(p.experts == 32 * kPer ? route_kernel<kPer, true, kF32, kSigmoid> : route_kernel<kPer, false, kF32, kSigmoid>,
                    dim3(blocks), dim3(kThreads), smem, stream, 1, p);
}
template <bool kF32, bool kSigmoid>
cudaError_t launch_route(const RouteParams& p, unsigned blocks, cudaStream_t stream) {
  if (p.experts <= 32) return launch_route_form<1, kF32, kSigmoid>(p, blocks, stream);
  if (p.experts <= 64) return launch_route_form<2, kF32, kSigmoid>(p, blocks, stream);
  if (p.experts <= 128) return launch_route_form<4, kF32, kSigmoid>(p, blocks, stream);
  if (p.experts <= 256) return launch_route_form<8, kF32, kSigmoid>(p, blocks, stream);
  if (p.experts <= 512) return launch_route_form<16, kF32, kSigmoid>(p, blocks, stream);
  return launch_route_form<32, kF32, kSigmoid>(p, blocks, stream);
}
template <bool kF32>
cudaError_t launch_route_backward(const RouteBackParams& p, unsigned blocks, cudaStream_t stream) {
  const dim3 g(blocks), b(kThreads);
  if (p.experts <= 32) return launch_pdl(route_backward_kernel<1, kF32>, g, b, 0, stream, 1, p);
  if (p.experts <= 64) return launch_pdl(route_backward_kernel<2, kF32>, g, b, 0, stream, 1, p);
  if (p.experts <= 128) return launch_pdl(route_backward_kernel<4, kF32>, g, b, 0, stream, 1, p);
  if (p.experts <= 256) return launch_pdl(route_backward_kernel<8, kF32>, g, b, 0, stream, 1, p);
  if (p.experts <= 512) return launch_pdl(route_backward_kernel<16, kF32>, g, b, 0, stream, 1, p);
  return launch_pdl(route_backward_kernel<32, kF32>, g, b, 0, stream, 1, p);
}

// ---- the plan: a stable counting sort of the routed pairs by expert ---------------------------------
// Pairs (token, place) are numbered token * topk + place.  A chunk of kPlanChunk pairs is one block's; its
// warps take equal spans of it.  (1) every chunk counts its pairs per expert; (2) every block adds up the counts
// of the chunks before its own and of all, which gives the experts' first rows and its own pairs' among them; (3) it
// places its pairs: a warp's pairs of one expert find their order among the lanes.  A single
// chunk does all three in one launch; more than kPlanDirect chunks have (2) done by one block in between.

struct PlanParams {
  const int32_t* idx;
  int32_t* row_src;
  int32_t* block_expert;
  int32_t* offsets;
  int32_t* counts;
  int32_t* slot;
  int32_t* scratch;      // [chunks][experts]: counts, or (after the scan kernel) first rows
  int64_t pairs, rows;
  int experts, chunks;
};
constexpr int kPlanDirect = 128;

__device__ __forceinline__ int pair_expert(const PlanParams& p, int64_t i) {
  if (i >= p.pairs) return -1;
  const int e = p.idx[i];
  return e >= 0 && e < p.experts ? e : -1;
}

// A warp's span of the chunk, held in registers: round r of it is lane's pair at base + 32 r.
constexpr int kMaxRounds = kPlanChunk / 8 / 32;
struct Span {
  int64_t base;
  int rounds;
  int expert[kMaxRounds];
};
__device__ __forceinline__ Span load_span(const PlanParams& p, int64_t chunk) {
  Span s;
  const int span = kPlanChunk / (blockDim.x >> 5);
  s.base = chunk * kPlanChunk + (threadIdx.x >> 5) * span + (threadIdx.x & 31);
  s.rounds = span / 32;
#pragma unroll
  for (int r = 0; r < kMaxRounds; ++r) s.expert[r] = r < s.rounds ? pair_expert(p, s.base + 32 * r) : -1;
  return s;
}

// hist[expert * stride + warp] = pairs of the warp's span per expert; stride is odd, so that lanes that walk
// either way meet different banks.
__device__ __forceinline__ int hist_stride() { return (blockDim.x >> 5) + 1; }
__device__ void clear_histograms(const PlanParams& p, int32_t* hist) {
  for (int i = threadIdx.x; i < hist_stride() * p.experts; i += blockDim.x) hist[i] = 0;
  __syncthreads();
}
__device__ void fill_histograms(const Span& s, int32_t* hist) {
#pragma unroll
  for (int r = 0; r < kMaxRounds; ++r)
    if (s.expert[r] >= 0) atomicAdd(&hist[s.expert[r] * hist_stride() + (threadIdx.x >> 5)], 1);   // counts: any order
  __syncthreads();
}

// hist becomes the row of every warp's first pair of the expert.  One thread per expert, its counts in
// flight eight at a time.
__device__ void warp_starts(const PlanParams& p, int32_t* hist, const int32_t* first) {
  const int warps = blockDim.x >> 5;
  for (int e = threadIdx.x; e < p.experts; e += blockDim.x) {
    int32_t at = first[e];
    int32_t* row = hist + e * hist_stride();
    for (int w0 = 0; w0 < warps; w0 += 8) {
      int32_t n[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) n[i] = row[w0 + i];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        row[w0 + i] = at;
        at += n[i];
      }
    }
  }
  __syncthreads();
}

// The lanes whose expert is this lane's, from one ballot per bit of the numbers (match.any goes through the distinct
// values one by one, 2,000 cycles for a warp of them).  Lanes without a pair (-1) match each other.
__device__ __forceinline__ uint32_t same_expert(int e, int bits) {
  uint32_t same = __ballot_sync(kFull, e >= 0);
  if (e < 0) same = ~same;
  for (int b = 0; b < bits; ++b) {
    const uint32_t ones = __ballot_sync(kFull, (e >> b) & 1);
    same &= ((e >> b) & 1) ? ones : ~ones;
  }
  return same;
}

__device__ void place_pairs(const PlanParams& p, const Span& s, int32_t* hist) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int bits = 32 - __clz(p.experts);
#pragma unroll
  for (int r = 0; r < kMaxRounds; ++r) {
    if (r >= s.rounds) break;
    const int64_t i = s.base + 32 * r;
    const int e = s.expert[r];
    const uint32_t same = same_expert(e, bits);
    int32_t* next = hist + max(e, 0) * hist_stride() + warp;
    int row = -1;
    if (e >= 0) row = *next + __popc(same & ((1u << lane) - 1u));
    __syncwarp();
    if (e >= 0 && lane == __ffs(same) - 1) *next += __popc(same);
    __syncwarp();
    if (i < p.pairs) {
      p.slot[i] = row;
      if (row >= 0) p.row_src[row] = (int32_t)i;
    }
  }
}

// first[] = the first row of every expert, from total[] (its pairs; may be first[] itself); with `write` also offsets, counts and
// block_expert.  sums: one word per warp.
__device__ void scan_experts(const PlanParams& p, const int32_t* total, int32_t* first, int32_t* sums, bool write) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  int32_t carry = 0;
  for (int base = 0; base < p.experts; base += blockDim.x) {
    const int e = base + threadIdx.x;
    const int32_t pairs = e < p.experts ? total[e] : 0, blocks = (pairs + kExpertBlock - 1) / kExpertBlock;
    int32_t v = blocks;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int32_t o = __shfl_up_sync(kFull, v, d);
      if (lane >= d) v += o;
    }
    if (lane == 31) sums[warp] = v;
    __syncthreads();
    int32_t over = lane < warps ? sums[lane] : 0;      // the warps' sums, scanned by every warp for itself
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int32_t o = __shfl_up_sync(kFull, over, d);
      if (lane >= d) over += o;
    }
    const int32_t all = __shfl_sync(kFull, over, 31);
    const int32_t earlier = __shfl_sync(kFull, over, max(warp - 1, 0));
    const int32_t at = carry + (warp > 0 ? earlier : 0) + v - blocks;
    if (e < p.experts) {
      first[e] = at * kExpertBlock;
      if (write) {
        p.offsets[e] = at * kExpertBlock;
        p.counts[e] = pairs;
        for (int32_t b = 0; b < blocks; ++b) p.block_expert[at + b] = e;
      }
    }
    carry += all;
    __syncthreads();
  }
  if (!write) return;
  if (threadIdx.x == 0) p.offsets[p.experts] = carry * kExpertBlock;
  for (int64_t b = carry + threadIdx.x; b < p.rows / kExpertBlock; b += blockDim.x) p.block_expert[b] = -1;
}

// total[e] = pairs of expert e in all chunks, mine[e] = those in the chunks before `chunk`.
__device__ void add_chunks(const PlanParams& p, int chunk, int32_t* total, int32_t* mine) {
  for (int e = threadIdx.x; e < p.experts; e += blockDim.x) total[e] = mine[e] = 0;
  __syncthreads();
  // Several threads per expert, a few chunks each; sums of integers, in any order.
  const int groups = max(1, (int)blockDim.x / p.experts);
  const int g = threadIdx.x / p.experts;
  for (int e = threadIdx.x - g * p.experts; e < p.experts && g < groups; e += blockDim.x) {
    int32_t all = 0, before = 0;
    for (int c0 = g; c0 < p.chunks; c0 += 16 * groups) {
      int32_t n[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int c = c0 + i * groups;
        n[i] = c < p.chunks ? p.scratch[(int64_t)c * p.experts + e] : 0;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        all += n[i];
        if (c0 + i * groups < chunk) before += n[i];
      }
    }
    atomicAdd(&total[e], all);
    atomicAdd(&mine[e], before);
  }
  __syncthreads();
}

__global__ void __launch_bounds__(1024) plan_one_kernel(const PlanParams p) {
  extern __shared__ int32_t hist[];       // [experts][warps + 1], then total[experts], first[experts], sums
  const int warps = blockDim.x >> 5;
  int32_t* total = hist + hist_stride() * p.experts;
  int32_t* first = total + p.experts;
  int32_t* sums = first + p.experts;
  pdl_wait();
  pdl_release();
  const Span span = load_span(p, 0);
  for (int64_t i = threadIdx.x; i < p.rows; i += blockDim.x) p.row_src[i] = -1;
  clear_histograms(p, hist);
  fill_histograms(span, hist);
  for (int e = threadIdx.x; e < p.experts; e += blockDim.x) {
    int32_t n = 0;
#pragma unroll 8
    for (int w = 0; w < warps; ++w) n += hist[e * hist_stride() + w];
    total[e] = n;
  }
  __syncthreads();
  scan_experts(p, total, first, sums, true);
  warp_starts(p, hist, first);
  place_pairs(p, span, hist);
}

__global__ void __launch_bounds__(1024) plan_count_kernel(const PlanParams p) {
  extern __shared__ int32_t total[];
  pdl_wait();
  pdl_release();
  for (int e = threadIdx.x; e < p.experts; e += blockDim.x) total[e] = 0;
  __syncthreads();
  const int64_t base = (int64_t)blockIdx.x * kPlanChunk;
  for (int r = threadIdx.x; r < kPlanChunk; r += blockDim.x) {
    const int e = pair_expert(p, base + r);
    if (e >= 0) atomicAdd(&total[e], 1);
  }
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < p.rows; i += (int64_t)gridDim.x * blockDim.x)
    p.row_src[i] = -1;
  __syncthreads();
  for (int e = threadIdx.x; e < p.experts; e += blockDim.x) p.scratch[(int64_t)blockIdx.x * p.experts + e] = total[e];
}

__global__ void __launch_bounds__(1024) plan_scan_kernel(const PlanParams p) {
  extern __shared__ int32_t first[];      // [experts], then mine[experts], sums
  int32_t* mine = first + p.experts;
  int32_t* sums = mine + p.experts;
  pdl_wait();
  pdl_release();
  add_chunks(p, 0, first, mine);
  scan_experts(p, first, first, sums, true);
  __syncthreads();
  for (int e = threadIdx.x; e < p.experts; e += blockDim.x) {
    int32_t at = first[e];
    for (int c = 0; c < p.chunks; ++c) {
      int32_t* s = p.scratch + (int64_t)c * p.experts + e;
      const int32_t n = *s;
      *s = at;
      at += n;
    }
  }
}

__global__ void __launch_bounds__(1024) plan_place_kernel(const PlanParams p) {
  extern __shared__ int32_t hist[];       // [experts][warps + 1], then first and mine [experts], sums
  int32_t* first = hist + hist_stride() * p.experts;
  int32_t* mine = first + p.experts;
  int32_t* sums = mine + p.experts;
  // The pairs were there before the launch that this one follows, which has passed its own wait by now, and that one
  // writes neither them nor what is read here: the histograms are made beside it.
  pdl_release();
  const Span span = load_span(p, blockIdx.x);
  clear_histograms(p, hist);
  fill_histograms(span, hist);
  pdl_wait();
  if (p.chunks > kPlanDirect) {
    warp_starts(p, hist, p.scratch + (int64_t)blockIdx.x * p.experts);
  } else {
    add_chunks(p, blockIdx.x, first, mine);
    scan_experts(p, first, first, sums, blockIdx.x == 0);
    for (int e = threadIdx.x; e < p.experts; e += blockDim.x) first[e] += mine[e];
    __syncthreads();
    warp_starts(p, hist, first);
  }
  place_pairs(p, span, hist);
}

// ---- gradient of the weighted sum -----------------------------------------------------------------
struct CombineBackParams {
  const int32_t* row_src;
  const int32_t* live;
  const int32_t* slot;
  const float* weights;
  const void* Y;
  const uint16_t* dout;
  uint16_t* dY;
  float* dweights;
  int64_t n, pairs, rows, row_blocks;
  int topk;
};

// Eight elements of a row from column c on; `vec`: in 16-byte accesses (then all eight are there), else up to `left`.
__device__ __forceinline__ void load_octet(const uint16_t* p, bool vec, int64_t left, float (&v)[8]) {
  if (vec) {
    const uint4 q = *reinterpret_cast<const uint4*>(p);
    v[0] = bf16_low(q.x); v[1] = bf16_high(q.x); v[2] = bf16_low(q.y); v[3] = bf16_high(q.y);
    v[4] = bf16_low(q.z); v[5] = bf16_high(q.z); v[6] = bf16_low(q.w); v[7] = bf16_high(q.w);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < left ? bf16_value(p[e]) : 0.f;
  }
}
__device__ __forceinline__ void load_octet(const float* p, bool vec, int64_t left, float (&v)[8]) {
  if (vec) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < left ? p[e] : 0.f;
  }
}

// One warp per row of the layout; the blocks past row_blocks clear the weights' gradient of pairs that are
// not routed.  kVec: rows in 16-byte accesses, without a test per access, so that kBackBatch octets' loads of a lane go out
// together.  16,384 rows of 2048, bf16 and f32 Y: one 28.4 and 39.5 us, two 27.3 and 36.8, four 36.2 (registers) and 37.8.
constexpr int kBackBatch = 2;
template <bool kF32, bool kVec>
__global__ void __launch_bounds__(kThreads) combine_backward_kernel(const CombineBackParams p) {
  using Y = std::conditional_t<kF32, float, uint16_t>;
  constexpr int kBatch = kVec ? kBackBatch : 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_wait();
  pdl_release();
  if ((int64_t)blockIdx.x >= p.row_blocks) {
    const int64_t i = ((int64_t)blockIdx.x - p.row_blocks) * kThreads + threadIdx.x;
    if (p.dweights && i < p.pairs && p.slot[i] < 0) p.dweights[i] = 0.f;
    return;
  }
  const int64_t row = (int64_t)blockIdx.x * kWarps + warp;
  const int32_t src = row < p.rows ? p.row_src[row] : -1;
  if (row >= *p.live) return;
  const int64_t t = src < 0 ? 0 : src / p.topk;
  const float w = src < 0 ? 0.f : (p.weights ? p.weights[src] : 1.f);
  const bool dots = p.dweights && src >= 0;
  const uint16_t* g = p.dout + t * p.n;
  const Y* y = static_cast<const Y*>(p.Y) + row * p.n;
  float dot = 0.f;
  for (int64_t c0 = lane * 8; c0 < p.n; c0 += 256 * kBatch) {
    float d[kBatch][8], v[kBatch][8];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int64_t c = c0 + 256 * i, left = p.n - c;
#pragma unroll
      for (int e = 0; e < 8; ++e) d[i][e] = v[i][e] = 0.f;
      if (src >= 0 && left > 0) load_octet(g + c, kVec, left, d[i]);
      if (dots && left > 0) load_octet(y + c, kVec, left, v[i]);
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int64_t c = c0 + 256 * i, left = p.n - c;
      if (dots) {
#pragma unroll
        for (int e = 0; e < 8; ++e) dot = fmaf(d[i][e], v[i][e], dot);
      }
      if (!p.dY || left <= 0) continue;
      uint16_t* dst = p.dY + row * p.n + c;
      if constexpr (kVec) {
        *reinterpret_cast<uint4*>(dst) = make_uint4(bf16_pack(w * d[i][0], w * d[i][1]), bf16_pack(w * d[i][2], w * d[i][3]),
                                                    bf16_pack(w * d[i][4], w * d[i][5]), bf16_pack(w * d[i][6], w * d[i][7]));
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < left) dst[e] = bf16_round(w * d[i][e]);
      }
    }
  }
  if (dots) {
    dot = warp_sum(dot);
    if (lane == 0) p.dweights[src] = dot;
  }
}

}  // namespace

cudaError_t route_launch(const RouteCall& c, cudaStream_t stream, uint64_t* launches) {
  if (c.tokens <= 0) return cudaSuccess;
  const int64_t blocks = (c.tokens + kWarps - 1) / kWarps;
  if (blocks >= (1ll << 31)) return cudaErrorInvalidValue;
  RouteParams p{c.logits, c.bias, c.idx, c.weights, c.tokens, (int)c.experts, (int)c.topk, (int)c.groups,
                (int)c.topk_groups, c.sigmoid, c.renorm, c.scale};
  const cudaError_t e =
      c.logits_f32 ? (c.sigmoid ? launch_route<true, true> : launch_route<true, false>)(p, (unsigned)blocks, stream)
                   : (c.sigmoid ? launch_route<false, true> : launch_route<false, false>)(p, (unsigned)blocks, stream);
  if (e == cudaSuccess) ++*launches;
  return e;
}

cudaError_t route_backward_launch(const RouteCall& c, const int32_t* idx, const float* dweights, void* dlogits,
                                  cudaStream_t stream, uint64_t* launches) {
  if (c.tokens <= 0) return cudaSuccess;
  const int64_t blocks = (c.tokens + kWarps - 1) / kWarps;
  if (blocks >= (1ll << 31)) return cudaErrorInvalidValue;
  RouteBackParams p{c.logits, idx, dweights, dlogits, c.tokens, (int)c.experts, (int)c.topk, c.sigmoid, c.renorm,
                    c.scale, c.experts % 4 == 0 && reinterpret_cast<uintptr_t>(dlogits) % 16 == 0};
  const cudaError_t e = c.logits_f32 ? launch_route_backward<true>(p, (unsigned)blocks, stream)
                                     : launch_route_backward<false>(p, (unsigned)blocks, stream);
  if (e == cudaSuccess) ++*launches;
  return e;
}

cudaError_t plan_launch(const ExpertRows& x, const int32_t* idx, cudaStream_t stream, uint64_t* launches) {
  PlanParams p{};
  p.idx = idx;
  p.row_src = const_cast<int32_t*>(x.row_src);
  p.block_expert = const_cast<int32_t*>(x.block_expert);
  p.offsets = const_cast<int32_t*>(x.offsets);
  p.counts = const_cast<int32_t*>(x.counts);
  p.slot = const_cast<int32_t*>(x.slot);
  p.scratch = x.scratch;
  p.pairs = x.tokens * x.topk;
  p.rows = x.rows;
  p.experts = (int)x.experts;
  p.chunks = (int)((p.pairs + kPlanChunk - 1) / kPlanChunk);
  // A histogram per warp: 32 warps while that fits the 48 KiB every kernel may use, else eight.
  const int warps = p.experts <= 256 ? 32 : 8;
  const size_t hist = (size_t)(warps + 1) * p.experts * 4, lists = (size_t)p.experts * 8 + 32 * 4;
  const dim3 block(32 * warps);
  cudaError_t e;
  if (p.chunks <= 1) {
    e = launch_pdl(plan_one_kernel, dim3(1), block, hist + lists, stream, 1, p);
    if (e == cudaSuccess) ++*launches;
    return e;
  }
  e = launch_pdl(plan_count_kernel, dim3((unsigned)p.chunks), dim3(1024), (size_t)p.experts * 4, stream, 1, p);
  if (e == cudaSuccess) ++*launches;
  if (e == cudaSuccess && p.chunks > kPlanDirect) {
    e = launch_pdl(plan_scan_kernel, dim3(1), dim3(1024), lists, stream, 1, p);
    if (e == cudaSuccess) ++*launches;
  }
  if (e == cudaSuccess) e = launch_pdl(plan_place_kernel, dim3((unsigned)p.chunks), block, hist + lists, stream, 1, p);
  if (e == cudaSuccess) ++*launches;
  return e;
}

cudaError_t combine_backward_launch(const ExpertRows& x, bool y_f32, int64_t n, const float* weights, const void* Y,
                                    const uint16_t* dout, uint16_t* dY, float* dweights, cudaStream_t stream,
                                    uint64_t* launches) {
  CombineBackParams p{};
  p.row_src = x.row_src;
  p.live = x.offsets + x.experts;
  p.slot = x.slot;
  p.weights = weights;
  p.Y = Y;
  p.dout = dout;
  p.dY = dY;
  p.dweights = dweights;
  p.n = n;
  p.pairs = x.tokens * x.topk;
  p.topk = (int)x.topk;
  p.row_blocks = (x.rows + kWarps - 1) / kWarps;
  auto aligned = [](const void* q) { return reinterpret_cast<uintptr_t>(q) % 16 == 0; };
  p.rows = x.rows;
  const bool vec = n % 8 == 0 && aligned(dout) && aligned(dY) && aligned(Y);
  const int64_t blocks = p.row_blocks + (dweights ? (p.pairs + kThreads - 1) / kThreads : 0);
  if (blocks <= 0) return cudaSuccess;
  if (blocks >= (1ll << 31)) return cudaErrorInvalidValue;
  const dim3 grid((unsigned)blocks), block(kThreads);
  const cudaError_t e = launch_pdl(y_f32 ? (vec ? combine_backward_kernel<true, true> : combine_backward_kernel<true, false>)
                                         : (vec ? combine_backward_kernel<false, true> : combine_backward_kernel<false, false>),
                                   grid, block, 0, stream, 1, p);
  if (e == cudaSuccess) ++*launches;
  return e;
}

}  // namespace morello
