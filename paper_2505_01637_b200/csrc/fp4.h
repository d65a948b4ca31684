// Microscaled 4-bit tensors: layout and internal declarations.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "linear.h"

namespace morello {

// A scale serves 32 elements (power of two) or 16 (e4m3).
constexpr int fp4_block(bool nv) { return nv ? 16 : 32; }
// Bytes of a row of packed elements: whole groups of 32, so that the TMA engine can address it.
constexpr int64_t fp4_pitch(int64_t k) { return (k + 31) / 32 * 16; }
// Scales lie in atoms of 128 rows x 4 blocks, 512 bytes, in the order the tensor cores read them: the four blocks' bytes of
// row r at 16 (r % 32) + 4 (r / 32).
constexpr int kAtomRows = 128;
constexpr int kAtomBytes = 512;
constexpr int64_t fp4_atoms_down(int64_t rows) { return (rows + kAtomRows - 1) / kAtomRows; }
constexpr int64_t fp4_atoms_across(bool nv, int64_t k) { return (k + 4 * fp4_block(nv) - 1) / (4 * fp4_block(nv)); }

// Y[m][n] = act(z) + R or act(z_gate) * z_up + R with z = alpha X W + bias: X[m][k] and W (a tensor of n or 2 n rows, in two
// parts) in 4 bits.
struct Fp4Call {
  bool nv = false;
  int64_t m = 0, n = 0, k = 0;
  const void *X = nullptr, *X_scales = nullptr, *W = nullptr, *W_scales = nullptr;
  const float* alpha = nullptr;
  LinearEpilogue epi;
  int64_t wide() const { return epi.gated ? 2 * n : n; }
};
// At most kFp4FewRows rows: W streamed once, the contraction cut over clusters (both sides' times at the head of fp4_rows.cu).
constexpr int kFp4FewRows = 16;
cudaError_t fp4_rows_launch(const DeviceInfo& dev, const Fp4Call& call, cudaStream_t stream, uint64_t* launches);
cudaError_t fp4_tile_launch(const DeviceInfo& dev, const Fp4Call& call, cudaStream_t stream, uint64_t* launches);

}  // namespace morello
