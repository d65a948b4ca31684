// Internal declarations of the feed-forward operators: linear layers with an epilogue, their
// gradients, routing to experts and the experts' products.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "internal.h"

namespace morello {

// Rows of a block of the experts' row layout: every expert's rows begin at a multiple of it.
constexpr int kExpertBlock = 128;
// Entries of the routing table that one block of the plan's counting sort takes.
constexpr int kPlanChunk = 2048;

// The experts' row layout as the kernels read it (device pointers into the plan buffer).
struct ExpertRows {
  int64_t tokens = 0, topk = 0, experts = 0;
  int64_t rows = 0;                     // upper bound on the rows: a multiple of kExpertBlock
  const int32_t* row_src = nullptr;     // [rows]: token * topk + place, -1 for padding
  const int32_t* block_expert = nullptr;  // [rows / kExpertBlock]: expert of the block, -1 past the end
  const int32_t* offsets = nullptr;     // [experts + 1]: first row of every expert; the last: live rows
  const int32_t* counts = nullptr;      // [experts]: rows that hold a token
  const int32_t* slot = nullptr;        // [tokens][topk]: row of the token's place, -1 if not routed
  int32_t* scratch = nullptr;           // [chunks][experts]
};
// Upper bound on the rows of the layout, and the int32 words of the plan buffer.
int64_t expert_rows(int64_t tokens, int64_t topk, int64_t experts);
int64_t expert_plan_words(int64_t tokens, int64_t topk, int64_t experts);
ExpertRows expert_rows_of(int64_t tokens, int64_t topk, int64_t experts, const int32_t* plan);

// What happens to an accumulator on its way out: v = acc + bias; Z = v; y = act(v) (gated:
// act(v_gate) * v_up); Y = y + residual (accumulate: Y += y).
struct LinearEpilogue {
  int act = 0;
  bool gated = false;
  bool out_f32 = false;
  bool accumulate = false;              // f32 output only
  const uint16_t* bias = nullptr;       // bf16 [groups][width], width = n or 2 n (gated)
  const uint16_t* residual = nullptr;   // bf16 [m][n]
  void* Y = nullptr;                    // [groups or 1][m][n]
  uint16_t* Z = nullptr;                // bf16 [m][width]
};

// A dense bf16 matrix [groups][rows][cols] the TMA engine can address (16-byte-aligned base,
// cols % 8 == 0).
struct MatrixView {
  const uint16_t* p = nullptr;
  int64_t cols = 0, rows = 0, groups = 1;
};

// One product on the tile kernel.
//   kDense:    Y[m][n] = A x B
//   kRows:     the rows of A (and Y) are the experts' layout; B is the matrix of the row's expert
//   kContract: Y[e] = A x B over the rows of expert e (both operands have their rows along the
//              contraction: a_mn and b_mn)
enum class TileMode { kDense = 0, kRows = 1, kContract = 2 };
struct TileCall {
  TileMode mode = TileMode::kDense;
  MatrixView a, b;
  bool a_mn = false;       // A is stored with its output rows contiguous: [contraction][m]
  bool b_mn = false;       // B is stored [contraction][n] (true) or [n][contraction]
  int64_t m = 0, n = 0, k = 0;   // extents of one output (gated: n columns, B has 2 n); k unused by kContract
  int64_t b_up = 0;        // gated: where the second half of B's columns begins in its stored order
  bool zero_padding = false;     // kRows: rows that hold no token are written as zeros
  bool precise = false;          // f32 output whose sums are wanted as near as f32 allows
  bool masked_a = false;         // kContract: rows of A that hold no pair are taken as zeros (both operands are the caller's)
  bool gather_a = false;         // few-rows kernel: A is [tokens][cols], its rows fetched through the plan
  ExpertRows experts;
  LinearEpilogue epi;
};
// Column sums from partial sums of kSlopeRows rows each: db[g][c] = the partial sums of group g's rows, in a fixed order.
constexpr int kSlopeRows = 32;
struct ColumnSums {
  const float* partial = nullptr;    // [parts][width]
  float* db = nullptr;               // [groups][width]
  int64_t width = 0, parts = 0, groups = 1;
  const int32_t* offsets = nullptr;  // first row of every group (multiples of kSlopeRows) and
  const int32_t* counts = nullptr;   // rows of every group, or null: one group
  bool accumulate = false;
};
// One product, or two (of which only the first may be kRows), in one launch; two take the column sums with them.
cudaError_t tile_launch(const DeviceInfo& dev, const TileCall* calls, int count, const ColumnSums* sums,
                        cudaStream_t stream, uint64_t* launches);

// The few-rows kernel: at most kLinearFewRows rows (per expert), B streamed once.
constexpr int kLinearFewRows = 64;
cudaError_t rows_launch(const DeviceInfo& dev, const TileCall& call, cudaStream_t stream, uint64_t* launches);

// Copies with zero padding: dst[g][r][c] = src[g][row(r)][c] inside the source, else 0; dst's cols_out is a multiple of 8, its base 16-byte aligned.
struct CopyJob {
  const uint16_t* src = nullptr;
  uint16_t* dst = nullptr;
  int64_t groups = 1, rows_in = 0, cols_in = 0, rows_out = 0, cols_out = 0;
  const ExpertRows* experts = nullptr;  // rows past the live ones are left alone
  bool gather = false;                  // with experts: row r of dst is token row_src[r] / topk of src
  const ExpertRows* by_expert = nullptr;  // groups are experts: those without rows are left alone
};
constexpr int kMaxCopies = 2;
// One launch.  beside: the launch before it, of the same call, writes nothing that the copies read or overwrite, and
// they are made while it runs.
cudaError_t copy_launch(const CopyJob* jobs, int count, bool beside, cudaStream_t stream, uint64_t* launches);

// dZ = dY . act'(Z) into dZ [rows][width rounded up to 8] (bf16, the added columns zero; width = n or
// 2 n), and, when `partial` is given, the partial column sums of dZ in f32, of kSlopeRows
// rows each.  z may be null for act none without gating.
struct SlopeCall {
  int act = 0;
  bool gated = false;
  const uint16_t* dY = nullptr;
  const uint16_t* Z = nullptr;
  uint16_t* dZ = nullptr;     // null: only the column sums are wanted
  float* partial = nullptr;   // the column sums' parts, or null
  int64_t rows = 0, n = 0;    // rows of dY (with experts: the layout's rows)
  const ExpertRows* experts = nullptr;  // rows past the live ones are left alone, as are sums of kSlopeRows without a token
};
size_t slope_partial_bytes(int64_t rows, int64_t n, bool gated);
cudaError_t slope_launch(const SlopeCall& call, cudaStream_t stream, uint64_t* launches);
// The column sums alone.
cudaError_t slope_sum_launch(const ColumnSums& sums, cudaStream_t stream, uint64_t* launches);

// out[t] = residual[t] + sum_k weight[t][k] * Y[slot[t][k]]
cudaError_t combine_launch(const ExpertRows& x, bool y_f32, int64_t n, int64_t y_pitch, const float* weights,
                           const void* Y, const uint16_t* residual, uint16_t* out, cudaStream_t stream,
                           uint64_t* launches);

// Library-owned scratch of the current device, at least `need` bytes (as the products' own: one
// buffer, grown on demand, refused inside a stream capture), or the caller's; and the device.
int operator_workspace(size_t need, void* given, size_t given_bytes, cudaStream_t stream, void** out,
                       DeviceInfo* dev);

// A launch with programmatic stream serialisation: the kernel waits (griddepcontrol.wait) for its
// predecessor before it touches global memory.
template <typename... KArgs, typename... Args>
cudaError_t launch_pdl(void (*kern)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t stream,
                       int cluster, Args... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  int num = 1;
  if (cluster > 1) {
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    num = 2;
  }
  cfg.attrs = attr;
  cfg.numAttrs = num;
  return cudaLaunchKernelEx(&cfg, kern, static_cast<KArgs>(args)...);
}

}  // namespace morello
