// Microscaled 4-bit tensors: quantisation and reading back.
//
// A block of 32 (or 16) elements along k shares a scale s, elements are e2m1: 0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives.
//   mx   s = 2^(floor(log2 amax) - 2): amax / s is in [4, 8), and what is beyond 6 becomes 6
//   nv   s = amax / 6 rounded to e4m3 (at most 448)
// and every element is x / s rounded to the nearest e2m1 value, ties to the even code.
//
// Rounding is exact: the result is that of the real quotient.  By a power of two a product is exact.  An e4m3 scale has at
// most 4 significant bits, a midpoint t of two e2m1 values 3, so t s is exact in f32.  q = x (1 / s) rounded to a multiple of 2^-13
// (by adding and taking away a large number) is t if x / s is t, and on the same side of every t as x / s where it is not t.
// Where it is t without x / s being t, the remainder x - q s, exact for q = t, tells: q + (x - q s) (1 / s) is x / s but
// for 2^-38, and rounds to f32 beside t, since x differs from t s by an ulp of x at least, more than half an ulp of t s.  A
// bf16 x (8 bits) differs from t s by 2^-8 of it at least: it needs no remainder.  Three instructions for two elements, and no
// division.  amax / 6 is the f32 quotient to nearest (Markstein's correction of a product with the rounded reciprocal),
// which never meets one of e4m3's midpoints (5 bits) from beside it, by the same argument.
//
// One read of X, one write: bound by memory once few enough instructions are spent on an element.  A lane takes 16 elements
// of a row of the [rows][k] layout, a warp 512 columns of four rows 32 apart, which share the 16 contiguous bytes of an
// atom's scales: a maximum and a scale a lane.  8192 x 4096 from bf16 16.8 us (nv) and 16.4 (mx), from f32 25.1; eight elements
// a lane, 16 instructions an element, took 21.3.  The [k][rows] layout is turned in registers: a lane takes 32 elements of
// four rows (f32: of one), a warp reads its lanes' rows side by side; 19 us, f32 24.5.  Reading back to bf16 takes 14.8 us.
#include <algorithm>
#include <type_traits>

#include "../../include/morello.h"
#include "fp4.h"
#include "octets.cuh"
#include "sm100.cuh"

namespace morello {
namespace {

using namespace sm100;

constexpr uint32_t kFull = 0xffffffffu;
constexpr int kThreads = 256;
constexpr int kWarpColumns = 512;   // of the quantisation

struct QuantizeParams {
  const void* X;
  const float* mult;
  uint8_t* q;
  uint8_t* scales;
  int64_t each, parts, k;      // rows of a part
  int64_t pitch;               // bytes of a row of q
  int down, across;            // atoms of a part
  int segments;                // turned: 256-element pieces of a row
  unsigned bands;              // groups of rows
  int width;                   // elements of X per access
};
// Blocks are numbered without long divisions (which took half of all instructions): grid.x along X's contiguous direction,
// the pieces of a row or (turned) the rows, grid.y across it (in turns, if more than 65,535).  The other way round the
// DRAM sees 512 bytes of every row, and 8192 x 4096 took 1.4 us more.

// Eight e2m1 codes, the first in the lowest four bits; beyond 6 is 6.
__device__ __forceinline__ uint32_t e2m1_codes(const f32x2 (&v)[4]) {
  const float2 a = pair_values(v[0]), b = pair_values(v[1]), c = pair_values(v[2]), d = pair_values(v[3]);
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y), "f"(d.x), "f"(d.y));
  return r;
}
__device__ __forceinline__ uint32_t e4m3_code(float v) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.f), "f"(v));
  return r & 0xffu;
}
__device__ __forceinline__ float f16_low(uint32_t h) {
  float f;
  asm("{\n\t.reg .b16 l, u;\n\tmov.b32 {l, u}, %1;\n\tcvt.f32.f16 %0, l;\n\t}" : "=f"(f) : "r"(h));
  return f;
}
__device__ __forceinline__ float f16_high(uint32_t h) {
  float f;
  asm("{\n\t.reg .b16 l, u;\n\tmov.b32 {l, u}, %1;\n\tcvt.f32.f16 %0, u;\n\t}" : "=f"(f) : "r"(h));
  return f;
}
__device__ __forceinline__ float e4m3_value(uint32_t code) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)code));
  return f16_low(h);
}
constexpr uint32_t kInfinity = 0x7f800000u;

// The scale's byte of a block whose largest magnitude has these bits; an infinity or a NaN in the block: NaN.
template <bool kNv>
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
  if constexpr (kNv) {
    constexpr float kSixth = 1.f / 6.f;
    const float a = __uint_as_float(amax), q = a * kSixth;
    return amax >= kInfinity ? 0x7fu : e4m3_code(fmaf(fmaf(-6.f, q, a), kSixth, q));
  }
  else return amax >= kInfinity ? 0xffu : (uint32_t)max((int)(amax >> 23) - 2, 0);
}
// Elements over the scale, before they are rounded to e2m1.  kWide: of more than 8 significant bits.
template <bool kNv, bool kWide>
struct Scaler {
  f32x2 inverse, minus_scale;
  // From the scale's byte.  A scale of 0 leaves codes of 0; behind a NaN scale the codes mean nothing.
  __device__ __forceinline__ explicit Scaler(uint32_t byte) {
    if constexpr (!kNv) {
      inverse = pair_of(byte == 0xffu ? 0.f : __uint_as_float((254u - byte) << 23));       // 2^(127 - byte)
    } else {
      const float s = e4m3_value(byte);
      inverse = pair_of(byte == 0u || byte == 0x7fu ? 0.f : fast_reciprocal(s));
      minus_scale = pair_of(-s);
    }
  }
  __device__ __forceinline__ f32x2 operator()(f32x2 x) const {
    if constexpr (!kNv) return mul2(x, inverse);
    constexpr float kSnap = 1536.f;      // sums with it are multiples of 2^-13
    const f32x2 q = add2(fma2(x, inverse, pair_of(kSnap)), pair_of(-kSnap));
    return kWide ? fma2(fma2(q, minus_scale, x), inverse, q) : q;
  }
};

// The larger of two pairs of 16-bit numbers.
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// Sixteen elements of X.
template <bool kF32>
struct Sixteen {
  uint32_t w[kF32 ? 16 : 8];
  __device__ __forceinline__ void load(const void* X, int64_t at, int64_t cols, int width) {
    auto put = [&](int i, const uint4& v) {
      w[4 * i] = v.x;
      w[4 * i + 1] = v.y;
      w[4 * i + 2] = v.z;
      w[4 * i + 3] = v.w;
    };
    if constexpr (kF32) {
      const float* src = static_cast<const float*>(X) + at;
      if (cols >= 16 && width >= 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) put(i, reinterpret_cast<const uint4*>(src)[i]);
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) w[e] = e < cols ? __float_as_uint(src[e]) : 0u;
      }
    } else {
      const uint16_t* src = static_cast<const uint16_t*>(X) + at;
#pragma unroll
      for (int i = 0; i < 2; ++i) put(i, cols > 8 * i ? load8_raw(src + 8 * i, width, cols - 8 * i) : make_uint4(0u, 0u, 0u, 0u));
    }
  }
  // The same for f32 rows off 16 bytes: the warp's piece of the row (from `at`, `cols` of its 512 elements exist) by
  // contiguous accesses, which spread() hands to the lanes that they are for.  (For bf16 rows, in words of two elements, that took
  // 40 us for 8192 x 4095; a lane's own accesses take 30.)
  __device__ __forceinline__ void load_piece(const void* X, int64_t at, int64_t cols, int lane) {
    static_assert(kF32, "single elements");
    const float* src = static_cast<const float*>(X) + at;
#pragma unroll
    for (int j = 0; j < 16; ++j) w[j] = 32 * j + lane < cols ? __float_as_uint(src[32 * j + lane]) : 0u;
  }
  static constexpr int kStride = 16 + 4;      // of lanes: eight lanes' accesses in different banks
  __device__ __forceinline__ void spread(uint32_t* shared, int lane) {
#pragma unroll
    for (int j = 0; j < 16; ++j) shared[(32 * j + lane) / 16 * kStride + lane % 16] = w[j];
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 v = *reinterpret_cast<const uint4*>(shared + lane * kStride + 4 * i);
      w[4 * i] = v.x;
      w[4 * i + 1] = v.y;
      w[4 * i + 2] = v.z;
      w[4 * i + 3] = v.w;
    }
    __syncwarp();
  }
  // Elements 8 i on.
  __device__ __forceinline__ void pairs(int i, f32x2 (&v)[4]) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (kF32) v[j] = pair_of(__uint_as_float(w[8 * i + 2 * j]), __uint_as_float(w[8 * i + 2 * j + 1]));
      else v[j] = pair_of(bf16_low(w[4 * i + j]), bf16_high(w[4 * i + j]));
    }
  }
  // Bits of the largest magnitude, as f32: NaN above infinity above the numbers.
  __device__ __forceinline__ uint32_t amax() const {
    uint32_t a = 0;
    if constexpr (kF32) {
#pragma unroll
      for (int i = 0; i < 16; ++i) a = max(a, w[i] & 0x7fffffffu);
      return a;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) a = max_u16x2(a, w[i] & 0x7fff7fffu);
      return max(a << 16, a & 0xffff0000u);
    }
  }
};
// The largest magnitude of a block's elements times the tensor's factor, from that of the elements: rounding keeps the order.
__device__ __forceinline__ uint32_t times(uint32_t amax, float mult) {
  return __float_as_uint(__uint_as_float(amax) * mult) & 0x7fffffffu;
}

// Where a warp of the [rows][k] layout works: band 4 (part * down + atom) + eighth, 16 columns a lane, rows 32 apart.
constexpr int kRowsAtOnce = 4;      // an atom's rows of the same 16 bytes
constexpr int kReadColumns = 256;   // of reading back
struct Band {
  unsigned atom_row;
  int r32;
  int64_t part_row, row0;      // the part's first row, and the warp's first inside it
  __device__ __forceinline__ Band(unsigned band, unsigned down, int64_t parts, int64_t each) {
    r32 = (int)(band & 3u) * 8 + (int)threadIdx.x / 32;
    atom_row = band >> 2;
    const unsigned part = parts > 1 ? atom_row / down : 0u;
    part_row = part * each;
    row0 = (int64_t)(atom_row - part * down) * kAtomRows + r32;
  }
};

// kShared: f32 rows off 16 bytes, through shared memory (8192 x 4095 32 us instead of 65).
template <bool kNv, bool kF32, bool kMult, bool kShared>
__global__ void __launch_bounds__(kThreads) quantize_kernel(const QuantizeParams p) {
  constexpr int kLanes = kNv ? 1 : 2, kBlock = 16 * kLanes;            // lanes of a block, its elements
  const int lane = threadIdx.x % 32;
  __shared__ __align__(16) uint32_t shared[kShared ? kThreads / 32 : 1][kShared ? 32 * Sixteen<kF32>::kStride : 4];
  pdl_wait();
  pdl_release();
  const int64_t col0 = (int64_t)blockIdx.x * kWarpColumns, col = col0 + lane * 16;
  const int64_t across = (int64_t)blockIdx.x * (kWarpColumns / (4 * kBlock)) + lane / (4 * kLanes);
  const float mult = kMult ? *p.mult : 1.f;
  for (unsigned band = blockIdx.y; band < p.bands; band += gridDim.y) {
    const Band at(band, (unsigned)p.down, p.parts, p.each);
    Sixteen<kF32> x[kRowsAtOnce];
    const int64_t first = at.part_row + at.row0;
#pragma unroll
    for (int i = 0; i < kRowsAtOnce; ++i) {
      const bool row = at.row0 + 32 * i < p.each;
      if constexpr (kShared) x[i].load_piece(p.X, (first + 32 * i) * p.k + col0, row ? p.k - col0 : 0, lane);
      else x[i].load(p.X, (first + 32 * i) * p.k + col, row ? p.k - col : 0, p.width);
    }
    uint32_t words[kRowsAtOnce];
    uint8_t* q = p.q + first * p.pitch + col / 2;
#pragma unroll
    for (int i = 0; i < kRowsAtOnce; ++i) {
      if constexpr (kShared) x[i].spread(shared[threadIdx.x / 32], lane);
      uint32_t amax = x[i].amax();
      if constexpr (kLanes > 1) amax = max(amax, __shfl_xor_sync(kFull, amax, 1));
      if constexpr (kMult) amax = times(amax, mult);
      const bool row = at.row0 + 32 * i < p.each, there = row && col / kBlock * kBlock < p.k;
      const uint32_t byte = there ? scale_byte<kNv>(amax) : 0u;
      const Scaler<kNv, kF32 || kMult> scaled(byte);
      uint32_t codes[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        f32x2 v[4];
        x[i].pairs(h, v);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = scaled(kMult ? mul2(v[j], pair_of(mult)) : v[j]);
        codes[h] = e2m1_codes(v);
      }
      if (row && col < 2 * p.pitch) *reinterpret_cast<uint2*>(q + 32 * i * p.pitch) = make_uint2(codes[0], codes[1]);
      uint32_t word = byte << (8 * (lane / kLanes % 4));
      word |= __shfl_xor_sync(kFull, word, kLanes);
      words[i] = word | __shfl_xor_sync(kFull, word, 2 * kLanes);
    }
    if (lane % (4 * kLanes) == 0 && across < p.across)
      *reinterpret_cast<uint4*>(p.scales + ((int64_t)at.atom_row * p.across + across) * kAtomBytes + at.r32 * 16) =
          make_uint4(words[0], words[1], words[2], words[3]);
  }
}

// 32 elements of four rows, `rows` apart, the first `here` of them in memory; kWhole: the four rows are neighbours (else off[]
// behind the first).
template <bool kWhole>
__device__ __forceinline__ void load_turned(const uint16_t* src, const int (&off)[4], int64_t rows, int here, uint2 (&w)[32]) {
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    uint32_t e[4];
#pragma unroll
    for (int h = 0; h < 4; ++h) e[h] = kWhole ? src[h] : src[off[h]];
    if (i + 1 < here) src += rows;
    asm("" : "+l"(src));
    w[i] = make_uint2(e[0] | e[1] << 16, e[2] | e[3] << 16);
  }
}

// X[k][rows]: a block turns 128 rows (f32: 32) x 256 elements, a warp 32 elements of each, a lane four neighbouring rows, which
// it reads together (one): 256 (128) bytes of memory a warp and element.
// kTogether: rows and parts are multiples of a lane's rows, and X aligned to them; f32 always.
template <bool kNv, bool kF32, bool kMult, bool kTogether>
__global__ void __launch_bounds__(kThreads, kF32 ? 4 : 2) quantize_turned_kernel(const QuantizeParams p) {
  constexpr int kBlocks = kNv ? 2 : 1;           // blocks of 32 elements
  constexpr int kBlock = 32 / kBlocks;
  constexpr int kLaneRows = kF32 ? 1 : 4, kTile = 32 * kLaneRows, kWords = kNv ? 4 : 2;
  using Word = std::conditional_t<kF32, uint32_t, uint16_t>;
  __shared__ __align__(16) uint8_t bytes[kTile][16 + 4];   // rows 20 bytes apart: words of different rows in different banks
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const unsigned tiles = (unsigned)p.down * (kAtomRows / kTile);      // of a part
  const unsigned part = p.parts > 1 ? blockIdx.x / tiles : 0u;
  const int64_t row0 = (int64_t)(blockIdx.x - part * tiles) * kTile;      // inside the part
  const int64_t left = p.each - row0 - kLaneRows * lane;                  // of this lane's rows that exist
  const int64_t at = part * p.each + row0 + kLaneRows * lane, rows = p.each * p.parts;
  pdl_wait();
  pdl_release();
  const float mult = kMult ? *p.mult : 1.f;
#pragma unroll 1
  for (int segment = (int)blockIdx.y; segment < p.segments; segment += (int)gridDim.y) {
    const int64_t col = (int64_t)segment * 256 + warp * 32;
    uint2 w[32];      // an element of the lane's rows
    const int here = (int)min((int64_t)32, p.k - col);      // elements that exist
    if constexpr (kTogether) {
      const Word* src = static_cast<const Word*>(p.X) + col * rows + at;
#pragma unroll
      for (int i = 0; i < 32; ++i, src += rows) {
        w[i] = make_uint2(0u, 0u);
        if (left > 0 && i < here) {
          if constexpr (kF32) w[i].x = *src;
          else w[i] = *reinterpret_cast<const uint2*>(src);
        }
        asm("" : "+l"(src));      // the next address from this one: all of them in registers at first took 25 us for 19
      }
    } else {
      static_assert(!kF32, "single rows");
      // Single elements, the last row's and the last element's in place of those that are missing: loads without a condition.
      // Where the tile's rows all exist, one address for a lane's four (8191 x 4096: 28.5 us, 41 with four).
      const Word* src = static_cast<const Word*>(p.X) + min(col, p.k - 1) * rows + part * p.each;
      int off[kLaneRows];
      const int64_t mine = min(row0 + kLaneRows * lane, p.each - 1);
#pragma unroll
      for (int h = 0; h < kLaneRows; ++h) off[h] = (int)(min(row0 + kLaneRows * lane + h, p.each - 1) - mine);
      if (row0 + kTile <= p.each) load_turned<true>(src + mine, off, rows, here, w);
      else load_turned<false>(src + mine, off, rows, here, w);
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (i >= here) w[i] = make_uint2(0u, 0u);
    }
    // Bits of the largest magnitude of every row's blocks (bf16: two rows a word).
    uint2 most[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
      most[b] = make_uint2(0u, 0u);
#pragma unroll
      for (int i = b * kBlock; i < (b + 1) * kBlock; ++i) {
        if constexpr (kF32) most[b].x = max(most[b].x, w[i].x & 0x7fffffffu);
        else most[b] = make_uint2(max_u16x2(most[b].x, w[i].x & 0x7fff7fffu), max_u16x2(most[b].y, w[i].y & 0x7fff7fffu));
      }
    }
#pragma unroll
    for (int h = 0; h < kLaneRows; ++h) {
      auto value = [&](const uint2& word) {
        if constexpr (kF32) return __uint_as_float(word.x);
        else return h % 2 ? bf16_high(h < 2 ? word.x : word.y) : bf16_low(h < 2 ? word.x : word.y);
      };
      uint32_t codes[4];
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        uint32_t amax = __float_as_uint(value(most[b]));
        if constexpr (kMult) amax = times(amax, mult);
        const bool there = left > h && col + b * kBlock < p.k;
        const uint32_t byte = there ? scale_byte<kNv>(amax) : 0u;
        bytes[kLaneRows * lane + h][warp * kBlocks + b] = (uint8_t)byte;
        const Scaler<kNv, kF32 || kMult> scaled(byte);
#pragma unroll
        for (int o = 0; o < kBlock / 8; ++o) {
          f32x2 v[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int i = b * kBlock + 8 * o + 2 * j;
            v[j] = pair_of(value(w[i]), value(w[i + 1]));
            if constexpr (kMult) v[j] = mul2(v[j], pair_of(mult));
            v[j] = scaled(v[j]);
          }
          codes[b * (kBlock / 8) + o] = e2m1_codes(v);
        }
      }
      if (left > h && col < p.k)
        *reinterpret_cast<uint4*>(p.q + (at + h) * p.pitch + col / 2) = make_uint4(codes[0], codes[1], codes[2], codes[3]);
    }
    __syncthreads();
    // The tile's scales, an atom's four bytes of a row at a time.
    for (int i = threadIdx.x; i < kTile * kWords; i += kThreads) {
      const int row = i % kTile, word = i / kTile;
      const int64_t r = row0 + row, atom = (int64_t)part * p.down + r / kAtomRows, across = (int64_t)segment * kWords + word;
      if (across < p.across)
        *reinterpret_cast<uint32_t*>(p.scales + (atom * p.across + across) * kAtomBytes + (r % 32) * 16 + r % kAtomRows / 32 * 4) =
            *reinterpret_cast<const uint32_t*>(&bytes[row][word * 4]);
    }
    __syncthreads();      // before the next piece's bytes
  }
}

struct DequantizeParams {
  const uint8_t* q;
  const uint8_t* scales;
  const float* alpha;
  void* Y;
  int64_t each, parts, k, pitch;
  int down, across;
  unsigned bands;
  int width;                   // elements of Y per access
};
// Eight codes times a scale.
__device__ __forceinline__ void codes_times(uint32_t codes, f32x2 scale, f32x2 (&v)[4]) {
  uint32_t h[4];
  asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(codes));
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = mul2(pair_of(f16_low(h[j]), f16_high(h[j])), scale);
}
// Where a warp's 256 elements of a row go through shared memory, so that its stores are contiguous.
constexpr int kReadWarps = kThreads / 32;
// bf16 rows off 16 bytes: words of two elements, 4 bytes aligned in memory.  `left` of the elements exist.
__device__ __forceinline__ void store_words(uint16_t* dst, int64_t left, int lane, const uint4& mine, uint32_t* shared) {
  *reinterpret_cast<uint4*>(shared + 4 * lane) = mine;
  __syncwarp();
  const int skew = (int)(reinterpret_cast<uintptr_t>(dst) >> 1) & 1;      // elements before the first whole word
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int word = 32 * j + lane, first = 2 * word + skew;
    uint32_t v = shared[word];
    if (skew) v = __funnelshift_r(v, shared[word + 1], 16);      // the word behind the last is not stored
    if (first + 1 < min(left, (int64_t)kReadColumns)) *reinterpret_cast<uint32_t*>(dst + first) = v;
    else if (first < min(left, (int64_t)kReadColumns)) dst[first] = (uint16_t)v;
  }
  if (skew && lane == 0) dst[0] = (uint16_t)shared[0];
  __syncwarp();
}
// f32, four elements an access where rows are on 16 bytes, single ones where not.
__device__ __forceinline__ void store_floats(float* dst, int64_t left, int lane, int width, const f32x2 (&v)[4], uint32_t* shared) {
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const float2 a = pair_values(v[2 * q]), b = pair_values(v[2 * q + 1]);
    reinterpret_cast<float4*>(shared)[2 * lane + q] = make_float4(a.x, a.y, b.x, b.y);
  }
  __syncwarp();
  if (width >= 4) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (4 * (32 * j + lane) < left) reinterpret_cast<uint4*>(dst)[32 * j + lane] = reinterpret_cast<const uint4*>(shared)[32 * j + lane];
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (32 * j + lane < left) dst[32 * j + lane] = __uint_as_float(shared[32 * j + lane]);
  }
  __syncwarp();
}
// A lane takes eight elements of each of its rows: a warp's stores are contiguous (sixteen a lane, as in the quantisation,
// leave half of every line to a second store: 22.1 us for 8192 x 4096 where this takes 14.8).
// kShared: through shared memory: f32, and bf16 rows off 8 bytes (8192 x 4095 22.5 us instead of 92; 4100 columns take 16.3 by
// two stores of a lane, 22.9 this way).
template <bool kNv, bool kF32, bool kShared>
__global__ void __launch_bounds__(kThreads) dequantize_kernel(const DequantizeParams p) {
  constexpr int kBlock = kNv ? 16 : 32;
  __shared__ __align__(16) uint32_t shared[kShared ? kReadWarps : 1][(kF32 ? kReadColumns : kReadColumns / 2) + 4];
  const int lane = threadIdx.x % 32;
  uint32_t* mine = shared[kShared ? threadIdx.x / 32 : 0];
  const int64_t col0 = (int64_t)blockIdx.x * kReadColumns, col = col0 + lane * 8;
  const bool any = col < p.k;
  pdl_wait();
  pdl_release();
  if (!kShared && !any) return;
  const float alpha = p.alpha ? *p.alpha : 1.f;
  const unsigned block = (unsigned)(col / kBlock);
  for (unsigned band = blockIdx.y; band < p.bands; band += gridDim.y) {
    const Band at(band, (unsigned)p.down, p.parts, p.each);
    const int64_t first = at.part_row + at.row0, here = p.each - at.row0;
    if (here <= 0) continue;
    uint4 scales = make_uint4(0u, 0u, 0u, 0u);
    if (any) scales = *reinterpret_cast<const uint4*>(p.scales + ((int64_t)at.atom_row * p.across + block / 4) * kAtomBytes + at.r32 * 16);
    const uint32_t words[kRowsAtOnce] = {scales.x, scales.y, scales.z, scales.w};
    const uint8_t* q = p.q + first * p.pitch + col / 2;
    uint32_t codes[kRowsAtOnce];
#pragma unroll
    for (int i = 0; i < kRowsAtOnce; ++i)
      codes[i] = any && 32 * i < here ? *reinterpret_cast<const uint32_t*>(q + 32 * i * p.pitch) : 0u;
#pragma unroll
    for (int i = 0; i < kRowsAtOnce; ++i) {
      if (32 * i >= here) break;      // of the whole warp
      const uint32_t byte = words[i] >> (8 * (block & 3)) & 0xffu;
      float s;
      if constexpr (kNv) s = byte == 0x7fu ? __uint_as_float(0x7fffffffu) : e4m3_value(byte);
      else s = byte == 0xffu ? __uint_as_float(0x7fffffffu) : __uint_as_float(byte == 0u ? 0x400000u : byte << 23);
      f32x2 v[4];
      codes_times(codes[i], pair_of(s), v);
      if (p.alpha) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = mul2(v[j], pair_of(alpha));
      }
      const int64_t to = (first + 32 * i) * p.k + col0;
      if constexpr (kF32) {
        store_floats(static_cast<float*>(p.Y) + to, p.k - col0, lane, p.width, v, mine);
      } else {
        const float2 a = pair_values(v[0]), b = pair_values(v[1]), c = pair_values(v[2]), d = pair_values(v[3]);
        const uint4 packed = make_uint4(bf16_pack(a.x, a.y), bf16_pack(b.x, b.y), bf16_pack(c.x, c.y), bf16_pack(d.x, d.y));
        uint16_t* dst = static_cast<uint16_t*>(p.Y) + to;
        if constexpr (kShared) store_words(dst, p.k - col0, lane, packed, mine);
        else store8_raw(dst + 8 * lane, p.width, p.k - col, packed);
      }
    }
  }
}

// --- host -----------------------------------------------------------------------------------

constexpr int64_t kMaxExtent = (1ll << 31) - 1024;
constexpr unsigned kMaxGridY = 65535;

bool aligned(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

int check_tensor(int format, int type, int64_t rows, int64_t parts, int64_t k) {
  if (format < 0 || format > 1 || type < 0 || type > 1) return MORELLO_ERR_INVALID_ARGUMENT;
  if (rows < 0 || k < 0 || parts < 1 || rows > kMaxExtent || k > kMaxExtent || rows % parts != 0) return MORELLO_ERR_INVALID_SHAPE;
  int64_t t;
  if (__builtin_mul_overflow(parts * fp4_atoms_down(rows / parts), fp4_atoms_across(format == MORELLO_NVFP4, k) * kAtomBytes, &t) ||
      __builtin_mul_overflow(rows, k * 4, &t))
    return MORELLO_ERR_INVALID_SHAPE;
  return MORELLO_OK;
}

// Elements per access that f32 rows of `cols` elements allow: 4, 2 or 1.
int access_width_f32(int64_t cols, const void* p) {
  for (int w = 4; w > 1; w /= 2)
    if (cols % w == 0 && aligned(p, 4 * w)) return w;
  return 1;
}

template <bool kNv, bool kF32, bool kMult>
cudaError_t quantize_launch(const QuantizeParams& p, bool turned, cudaStream_t s) {
  const dim3 grid = turned ? dim3(p.bands, std::min((unsigned)p.segments, kMaxGridY)) : dim3((unsigned)((p.k + kWarpColumns - 1) / kWarpColumns), std::min(p.bands, kMaxGridY));
  if constexpr (kF32) {
    if (!turned && p.width < 4) return launch_pdl(quantize_kernel<kNv, true, kMult, true>, grid, dim3(kThreads), 0, s, 1, p);
  }
  if (!turned) return launch_pdl(quantize_kernel<kNv, kF32, kMult, false>, grid, dim3(kThreads), 0, s, 1, p);
  if constexpr (!kF32) {
    if (p.width < 4) return launch_pdl(quantize_turned_kernel<kNv, false, kMult, false>, grid, dim3(kThreads), 0, s, 1, p);
  }
  return launch_pdl(quantize_turned_kernel<kNv, kF32, kMult, true>, grid, dim3(kThreads), 0, s, 1, p);
}

}  // namespace
}  // namespace morello

using namespace morello;

#pragma GCC visibility push(default)
extern "C" {

int64_t morello_fp4_bytes(int64_t rows, int64_t k) {
  return check_tensor(MORELLO_MXFP4, 0, rows, 1, k) == MORELLO_OK ? rows * fp4_pitch(k) : -1;
}

int64_t morello_fp4_scale_bytes(int format, int64_t rows, int64_t parts, int64_t k) {
  if (check_tensor(format, 0, rows, parts, k) != MORELLO_OK) return -1;
  return parts * fp4_atoms_down(rows / parts) * fp4_atoms_across(format == MORELLO_NVFP4, k) * kAtomBytes;
}

int morello_fp4_quantize(int format, int x_type, int x_layout, int64_t rows, int64_t parts, int64_t k, const void* X,
                         const float* mult, void* Q, void* scales, void* stream) {
  int rc;
  if (x_layout != MORELLO_W_ROWMAJOR && x_layout != MORELLO_W_COLMAJOR) return MORELLO_ERR_INVALID_ARGUMENT;
  if ((rc = check_tensor(format, x_type, rows, parts, k)) != MORELLO_OK) return rc;
  const bool empty = rows == 0 || k == 0, nv = format == MORELLO_NVFP4, f32 = x_type == MORELLO_F32;
  const bool turned = x_layout == MORELLO_W_ROWMAJOR;
  if (!empty && (!X || !Q || !scales)) return MORELLO_ERR_NULL_POINTER;
  if (!aligned(X, f32 ? 4 : 2) || !aligned(mult, 4) || !aligned(Q, 16) || !aligned(scales, 16)) return MORELLO_ERR_MISALIGNED;
  DeviceInfo dev;
  void* none = nullptr;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if ((rc = operator_workspace(0, nullptr, 0, s, &none, &dev)) != MORELLO_OK || empty) return rc;
  QuantizeParams p;
  p.X = X;
  p.mult = mult;
  p.q = static_cast<uint8_t*>(Q);
  p.scales = static_cast<uint8_t*>(scales);
  p.each = rows / parts;
  p.parts = parts;
  p.k = k;
  p.pitch = fp4_pitch(k);
  p.down = (int)fp4_atoms_down(p.each);
  p.across = (int)fp4_atoms_across(nv, k);
  const int64_t bands = parts * p.down * (turned ? (f32 ? 4 : 1) : 4);
  if (bands >= (1ll << 31)) return MORELLO_ERR_INVALID_SHAPE;
  p.segments = (int)((k + 255) / 256);
  p.bands = (unsigned)bands;
  // In the turned layout a lane's rows are read together where every part begins at a multiple of them.
  const int64_t contiguous = turned ? (p.each % 4 == 0 ? rows : 1) : k;
  p.width = f32 ? access_width_f32(contiguous, X) : access_width(contiguous, X);
  cudaError_t e;
  switch (nv * 4 + f32 * 2 + (mult ? 1 : 0)) {
    case 0: e = quantize_launch<false, false, false>(p, turned, s); break;
    case 1: e = quantize_launch<false, false, true>(p, turned, s); break;
    case 2: e = quantize_launch<false, true, false>(p, turned, s); break;
    case 3: e = quantize_launch<false, true, true>(p, turned, s); break;
    case 4: e = quantize_launch<true, false, false>(p, turned, s); break;
    case 5: e = quantize_launch<true, false, true>(p, turned, s); break;
    case 6: e = quantize_launch<true, true, false>(p, turned, s); break;
    default: e = quantize_launch<true, true, true>(p, turned, s); break;
  }
  if (e != cudaSuccess) return record_cuda_error(e);
  count_launches(1);
  return MORELLO_OK;
}

int morello_fp4_dequantize(int format, int y_type, int64_t rows, int64_t parts, int64_t k, const void* Q,
                           const void* scales, const float* alpha, void* Y, void* stream) {
  int rc;
  if ((rc = check_tensor(format, y_type, rows, parts, k)) != MORELLO_OK) return rc;
  const bool empty = rows == 0 || k == 0, nv = format == MORELLO_NVFP4, f32 = y_type == MORELLO_F32;
  if (!empty && (!Q || !scales || !Y)) return MORELLO_ERR_NULL_POINTER;
  if (!aligned(Q, 16) || !aligned(scales, 16) || !aligned(alpha, 4) || !aligned(Y, f32 ? 4 : 2)) return MORELLO_ERR_MISALIGNED;
  DeviceInfo dev;
  void* none = nullptr;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if ((rc = operator_workspace(0, nullptr, 0, s, &none, &dev)) != MORELLO_OK || empty) return rc;
  DequantizeParams p;
  p.q = static_cast<const uint8_t*>(Q);
  p.scales = static_cast<const uint8_t*>(scales);
  p.alpha = alpha;
  p.Y = Y;
  p.each = rows / parts;
  p.parts = parts;
  p.k = k;
  p.pitch = fp4_pitch(k);
  p.down = (int)fp4_atoms_down(p.each);
  p.across = (int)fp4_atoms_across(nv, k);
  const int64_t bands = parts * p.down * 4;
  if (bands >= (1ll << 31)) return MORELLO_ERR_INVALID_SHAPE;
  p.bands = (unsigned)bands;
  p.width = f32 ? access_width_f32(k, Y) : access_width(k, Y);
  const dim3 grid((unsigned)((k + kReadColumns - 1) / kReadColumns), std::min(p.bands, kMaxGridY)), block(kThreads);
  cudaError_t e;
  auto go = [&](auto kernel) { return launch_pdl(kernel, grid, block, 0, s, 1, p); };
  if (f32) e = nv ? go(dequantize_kernel<true, true, true>) : go(dequantize_kernel<false, true, true>);
  else if (p.width < 4) e = nv ? go(dequantize_kernel<true, false, true>) : go(dequantize_kernel<false, false, true>);
  else e = nv ? go(dequantize_kernel<true, false, false>) : go(dequantize_kernel<false, false, false>);
  if (e != cudaSuccess) return record_cuda_error(e);
  count_launches(1);
  return MORELLO_OK;
}

}  // extern "C"
#pragma GCC visibility pop
