// C entry points of the feed-forward operators: argument checks, workspaces and the sequence of launches.
#include <algorithm>
#include <utility>

#include "../../include/morello.h"
#include "activation.cuh"
#include "linear.h"
#include "route.h"

namespace morello {

int64_t expert_rows(int64_t tokens, int64_t topk, int64_t experts) {
  const int64_t pairs = tokens * topk;
  return (pairs + (kExpertBlock - 1) * std::min(experts, pairs)) / kExpertBlock * kExpertBlock;
}

namespace {
int64_t plan_chunks(int64_t pairs) { return (pairs + kPlanChunk - 1) / kPlanChunk; }
}  // namespace

int64_t expert_plan_words(int64_t tokens, int64_t topk, int64_t experts) {
  const int64_t rows = expert_rows(tokens, topk, experts), pairs = tokens * topk;
  return rows + rows / kExpertBlock + (experts + 1) + experts + pairs + plan_chunks(pairs) * experts;
}

ExpertRows expert_rows_of(int64_t tokens, int64_t topk, int64_t experts, const int32_t* plan) {
  ExpertRows x;
  x.tokens = tokens;
  x.topk = topk;
  x.experts = experts;
  x.rows = expert_rows(tokens, topk, experts);
  x.row_src = plan;
  x.block_expert = x.row_src + x.rows;
  x.offsets = x.block_expert + x.rows / kExpertBlock;
  x.counts = x.offsets + experts + 1;
  x.slot = x.counts + experts;
  x.scratch = const_cast<int32_t*>(x.slot) + tokens * topk;
  return x;
}

namespace {

constexpr int64_t kMaxExtent = (1ll << 31) - 1024;   // tile coordinates are ints

bool aligned(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
int64_t round8(int64_t x) { return (x + 7) / 8 * 8; }
size_t round256(size_t x) { return (x + 255) / 256 * 256; }

// Carves a workspace; with a null base it only adds up.
struct Carver {
  char* base = nullptr;
  size_t at = 0;
  template <typename T>
  T* take(size_t bytes) {
    T* p = base ? reinterpret_cast<T*>(base + at) : nullptr;
    at += round256(bytes);
    return p;
  }
};

// One linear layer: dense (plan == nullptr) or with the experts' weights.
struct Layer {
  int act = 0;
  bool gated = false, w_cols = false, gather = false;
  int64_t m = 0, k = 0, n = 0;      // m: rows of Y (experts: the layout's)
  int64_t groups = 1;
  bool grouped = false;
  ExpertRows x;
  int64_t wide() const { return gated ? 2 * n : n; }
  int64_t x_rows() const { return gather ? x.tokens : m; }
};

// Few rows per weight matrix: the weights' stream is what counts.
bool few_rows(const Layer& l) { return (l.grouped ? l.x.tokens : l.m) <= kLinearFewRows; }

int check_extents(int64_t m, int64_t k, int64_t n, int64_t wide, int64_t groups) {
  if (m < 0 || k < 0 || n < 0) return MORELLO_ERR_INVALID_SHAPE;
  if (m > kMaxExtent || k > kMaxExtent || n > kMaxExtent || wide > kMaxExtent) return MORELLO_ERR_INVALID_SHAPE;
  int64_t t;
  if (__builtin_mul_overflow(m, round8(k), &t) || __builtin_mul_overflow(t, 4, &t) ||
      __builtin_mul_overflow(m, round8(wide), &t) || __builtin_mul_overflow(t, 4, &t) ||
      __builtin_mul_overflow(k, round8(n) * 2, &t) || __builtin_mul_overflow(t, groups, &t) ||
      __builtin_mul_overflow(t, 4, &t) || __builtin_mul_overflow(round8(k), wide, &t) ||
      __builtin_mul_overflow(t, groups, &t) || __builtin_mul_overflow(t, 4, &t))
    return MORELLO_ERR_INVALID_SHAPE;
  return MORELLO_OK;
}

int check_experts(int64_t tokens, int64_t topk, int64_t experts) {
  if (tokens < 0 || topk < 1 || experts < 1 || topk > kMaxTopk || experts > kMaxExperts) return MORELLO_ERR_INVALID_SHAPE;
  if (tokens > kMaxExtent / topk - (kExpertBlock + 1) * experts / topk - 1) return MORELLO_ERR_INVALID_SHAPE;
  return MORELLO_OK;
}

// Copies that a pass needs before its products, made by one launch.
struct Copies {
  CopyJob job[kMaxCopies];
  int count = 0;
  int launch(bool beside, cudaStream_t s, uint64_t* launches) {
    const cudaError_t e = copy_launch(job, count, beside, s, launches);
    return e == cudaSuccess ? MORELLO_OK : record_cuda_error(e);
  }
};

// X: [rows][k], padded when the TMA engine cannot address it; with `gather` its rows are copied in the
// experts' layout (the tile kernel's gathered loads, 32 of four rows per stage, were measured at twice the
// time of the whole product; the few-rows kernel gathers for itself).
void stage_x(const Layer& l, const void* X, bool gather, Carver& ws, bool dry, Copies* copies, MatrixView* out) {
  const uint16_t* src = static_cast<const uint16_t*>(X);
  const bool copy = gather || l.k % 8 != 0 || (!dry && !aligned(X, 16));
  out->rows = gather ? l.m : l.x_rows();
  out->groups = 1;
  out->cols = copy ? round8(l.k) : l.k;
  out->p = src;
  if (!copy) return;
  uint16_t* dst = ws.take<uint16_t>((size_t)out->rows * out->cols * 2);
  out->p = dst;
  if (!ws.base) return;
  CopyJob& j = copies->job[copies->count++];
  j.src = src;
  j.dst = dst;
  j.rows_in = l.x_rows();
  j.rows_out = out->rows;
  j.cols_in = l.k;
  j.cols_out = out->cols;
  j.gather = gather;
  if (gather || (l.grouped && !l.gather)) j.experts = &l.x;
}

// W for a product.  halves_apart: the forward pass of a gated layer reads its halves as two column
// ranges, each of which has to begin on a 16-byte boundary.
void stage_w(const Layer& l, const void* W, bool halves_apart, Carver& ws, bool dry, Copies* copies, MatrixView* out,
             int64_t* up) {
  const uint16_t* src = static_cast<const uint16_t*>(W);
  const int64_t parts = halves_apart && l.gated ? 2 : 1;       // column ranges of a row
  const int64_t cols_in = l.w_cols ? l.k : l.wide() / parts;
  const int64_t rows = l.w_cols ? l.wide() : l.k * parts;
  const bool copy = cols_in % 8 != 0 || (!dry && !aligned(W, 16));
  const int64_t cols = copy ? round8(cols_in) : cols_in;
  out->groups = l.groups;
  out->rows = l.w_cols ? l.wide() : l.k;
  out->cols = l.w_cols ? cols : cols * parts;
  out->p = src;
  if (up) *up = l.w_cols ? l.n : cols;
  if (!copy) return;
  uint16_t* dst = ws.take<uint16_t>((size_t)l.groups * rows * cols * 2);
  out->p = dst;
  if (!ws.base) return;
  CopyJob& j = copies->job[copies->count++];
  j.src = src;
  j.dst = dst;
  j.groups = l.groups;
  if (l.grouped) j.by_expert = &l.x;
  j.rows_in = rows;
  j.rows_out = rows;
  j.cols_in = cols_in;
  j.cols_out = cols;
}

struct ForwardArgs {
  const void *X, *W, *bias, *R;
  void *Y, *Z;
  bool y_f32;
};

int product(const DeviceInfo& dev, const Layer& l, const TileCall& c, cudaStream_t s, uint64_t* launches) {
  const cudaError_t e = few_rows(l) ? rows_launch(dev, c, s, launches) : tile_launch(dev, &c, 1, nullptr, s, launches);
  return e == cudaSuccess ? MORELLO_OK : record_cuda_error(e);
}

// `ws.base` null: only adds the workspace up (dev is not looked at).
int forward(const DeviceInfo& dev, const Layer& l, const ForwardArgs& a, Carver& ws, bool dry, cudaStream_t s,
            uint64_t* launches) {
  MatrixView x, w;
  int64_t up = 0;
  Copies copies;
  if (l.k > 0) {
    stage_x(l, a.X, l.gather && !few_rows(l), ws, dry, &copies, &x);
    stage_w(l, a.W, true, ws, dry, &copies, &w, &up);
  }
  if (!ws.base) return MORELLO_OK;
  if (const int rc = copies.launch(false, s, launches)) return rc;
  TileCall c;
  c.mode = l.grouped ? TileMode::kRows : TileMode::kDense;
  c.a = x;
  c.b = w;
  c.b_mn = !l.w_cols;
  c.m = l.m;
  c.n = l.n;
  c.k = l.k;
  c.b_up = up;
  c.gather_a = l.gather && few_rows(l);
  c.zero_padding = l.grouped;
  c.experts = l.x;
  c.epi.act = l.act;
  c.epi.gated = l.gated;
  c.epi.out_f32 = a.y_f32;
  c.precise = a.y_f32;
  c.epi.bias = static_cast<const uint16_t*>(a.bias);
  c.epi.residual = static_cast<const uint16_t*>(a.R);
  c.epi.Y = a.Y;
  c.epi.Z = static_cast<uint16_t*>(a.Z);
  return product(dev, l, c, s, launches);
}

struct BackwardArgs {
  const void *X, *W, *Z, *dY;
  void *dX, *dW;
  float* db;
  bool grad_f32, accumulate;
};

int backward(const DeviceInfo& dev, const Layer& l, const BackwardArgs& a, Carver& ws, bool dry, cudaStream_t s,
             uint64_t* launches) {
  const int64_t wide = l.wide(), wide8 = round8(wide);
  int rc;
  cudaError_t e;
  const bool want_dx = a.dX && l.k > 0, want_dw = a.dW && l.k > 0;
  // dZ: dY itself when the layer has no activation, else one pass that also adds up the bias gradient.
  const bool plain = l.act == kActNone && !l.gated;
  const bool direct = plain && l.n % 8 == 0 && (dry || aligned(a.dY, 16));
  const uint16_t* dz = static_cast<const uint16_t*>(a.dY);
  uint16_t* dz_own = nullptr;
  if (!direct && (want_dx || want_dw)) {
    dz_own = ws.take<uint16_t>((size_t)l.m * wide8 * 2);
    dz = dz_own;
  }
  float* partial = a.db || dry ? ws.take<float>(slope_partial_bytes(l.m, l.n, l.gated)) : nullptr;
  // The slopes' launch writes dZ and the partial sums; the copies of X and W run beside it.  The bias gradient's last sums
  // go with the products where those are one launch.
  const bool slopes = dz_own || a.db, one_launch = want_dx && want_dw && !few_rows(l);
  ColumnSums sums;
  if (ws.base && slopes) {
    SlopeCall c;
    c.act = l.act;
    c.gated = l.gated;
    c.dY = static_cast<const uint16_t*>(a.dY);
    c.Z = plain ? nullptr : static_cast<const uint16_t*>(a.Z);
    c.dZ = dz_own;
    c.partial = a.db ? partial : nullptr;
    c.rows = l.m;
    c.n = l.n;
    c.experts = l.grouped ? &l.x : nullptr;
    if ((e = slope_launch(c, s, launches)) != cudaSuccess) return record_cuda_error(e);
    sums.partial = partial;
    sums.db = a.db;
    sums.width = wide;
    sums.parts = (l.m + kSlopeRows - 1) / kSlopeRows;
    sums.accumulate = a.accumulate;
    if (l.grouped) {
      sums.groups = l.groups;
      sums.offsets = l.x.offsets;
      sums.counts = l.x.counts;
    }
  }
  const MatrixView z{dz, direct ? l.n : wide8, l.m, 1};
  MatrixView x, w;
  Copies copies;
  float* rows = nullptr;       // gather: dX of the layout's rows, summed by token at the end
  if (want_dx) {
    stage_w(l, a.W, false, ws, dry, &copies, &w, nullptr);
    if (l.gather) rows = ws.take<float>((size_t)l.m * l.k * 4);
  }
  if (want_dw) stage_x(l, a.X, l.gather, ws, dry, &copies, &x);
  if (!ws.base) return MORELLO_OK;
  if ((rc = copies.launch(slopes, s, launches)) != MORELLO_OK) return rc;
  if (a.db && !one_launch && (e = slope_sum_launch(sums, s, launches)) != cudaSuccess) return record_cuda_error(e);
  TileCall calls[2];
  int count = 0;
  if (want_dx) {
    TileCall& c = calls[count++];
    c.mode = l.grouped ? TileMode::kRows : TileMode::kDense;
    c.a = z;
    c.b = w;
    c.b_mn = l.w_cols;
    c.m = l.m;
    c.n = l.k;
    c.k = wide;
    c.zero_padding = l.grouped && !l.gather;
    c.experts = l.x;
    c.epi.out_f32 = l.gather;
    c.epi.Y = l.gather ? static_cast<void*>(rows) : a.dX;
    if (few_rows(l)) {
      if ((rc = product(dev, l, c, s, launches)) != MORELLO_OK) return rc;
      count = 0;
    }
  }
  if (want_dw) {
    TileCall& c = calls[count++];
    c = TileCall{};
    c.mode = l.grouped ? TileMode::kContract : TileMode::kDense;
    c.a = l.w_cols ? z : x;
    c.b = l.w_cols ? x : z;
    c.a_mn = c.b_mn = true;
    c.m = l.w_cols ? wide : l.k;
    c.n = l.w_cols ? l.k : wide;
    c.k = l.m;
    c.experts = l.x;
    // Gathered rows and slopes are written with zeros where there is no pair; X and dY as they came may hold any number there.
    c.masked_a = l.grouped && direct && !l.gather;
    c.epi.out_f32 = a.grad_f32;
    c.precise = a.grad_f32;
    c.epi.accumulate = a.accumulate;
    c.epi.Y = a.dW;
  }
  // The product with the longer tiles first: the other's fill up what its last wave leaves (experts: their rows first).
  if (count == 2 && !l.grouped && calls[1].k > calls[0].k) std::swap(calls[0], calls[1]);
  const ColumnSums* with = a.db && one_launch ? &sums : nullptr;
  if (count > 0 && (e = tile_launch(dev, calls, count, with, s, launches)) != cudaSuccess) return record_cuda_error(e);
  if (rows) {
    e = combine_launch(l.x, true, l.k, l.k, nullptr, rows, nullptr, static_cast<uint16_t*>(a.dX), s, launches);
    if (e != cudaSuccess) return record_cuda_error(e);
  }
  return MORELLO_OK;
}

int check_act(int act, int gated) {
  return act < 0 || act >= kActCount || gated < 0 || gated > 1 ? MORELLO_ERR_INVALID_ARGUMENT : MORELLO_OK;
}
int check_flag(int v) { return v == 0 || v == 1 ? MORELLO_OK : MORELLO_ERR_INVALID_ARGUMENT; }

// Workspace of a pass with 16-byte-aligned tensors.
template <typename Pass>
size_t dry_bytes(Pass&& pass) {
  Carver ws;
  uint64_t none = 0;
  pass(ws, none);
  return ws.at;
}

int run_forward(const Layer& l, const ForwardArgs& a, void* workspace, size_t workspace_bytes, void* stream) {
  if (workspace && !aligned(workspace, 16)) return MORELLO_ERR_MISALIGNED;
  if (l.m > 0 && l.n > 0) {
    if (!a.Y || (l.k > 0 && (!a.X || !a.W))) return MORELLO_ERR_NULL_POINTER;
    if (!aligned(a.X, 2) || !aligned(a.W, 2) || !aligned(a.bias, 2) || !aligned(a.R, 2) || !aligned(a.Z, 2) ||
        !aligned(a.Y, a.y_f32 ? 4 : 2))
      return MORELLO_ERR_MISALIGNED;
  }
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  Carver size;
  uint64_t launches = 0;
  DeviceInfo dev;
  int rc = MORELLO_OK;
  const bool empty = l.m == 0 || l.n == 0;
  if (!empty && (rc = forward(dev, l, a, size, false, s, &launches)) != MORELLO_OK) return rc;
  void* ws = nullptr;
  if ((rc = operator_workspace(size.at, workspace, workspace_bytes, s, &ws, &dev)) != MORELLO_OK || empty) return rc;
  Carver carve;
  carve.base = ws ? static_cast<char*>(ws) : reinterpret_cast<char*>(uintptr_t(256));   // nothing is taken
  rc = forward(dev, l, a, carve, false, s, &launches);
  count_launches(launches);
  return rc;
}

int run_backward(const Layer& l, const BackwardArgs& a, void* workspace, size_t workspace_bytes, void* stream) {
  const int64_t wide = l.wide();
  if (workspace && !aligned(workspace, 16)) return MORELLO_ERR_MISALIGNED;
  const bool plain = l.act == kActNone && !l.gated;
  if (l.m > 0 && wide > 0) {
    if (!a.dY || (!plain && !a.Z) || (a.dX && l.k > 0 && !a.W) || (a.dW && l.k > 0 && !a.X))
      return MORELLO_ERR_NULL_POINTER;
  }
  if (!aligned(a.X, 2) || !aligned(a.W, 2) || !aligned(a.Z, 2) || !aligned(a.dY, 2) || !aligned(a.dX, 2) ||
      !aligned(a.dW, a.grad_f32 ? 4 : 2) || !aligned(a.db, 4))
    return MORELLO_ERR_MISALIGNED;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  Carver size;
  uint64_t launches = 0;
  DeviceInfo dev;
  int rc = MORELLO_OK;
  const bool empty = l.m == 0 || wide == 0;
  if (!empty && (rc = backward(dev, l, a, size, false, s, &launches)) != MORELLO_OK) return rc;
  void* ws = nullptr;
  if ((rc = operator_workspace(size.at, workspace, workspace_bytes, s, &ws, &dev)) != MORELLO_OK) return rc;
  if (empty) {
    // Empty sums: zero, or nothing added.
    cudaError_t e = cudaSuccess;
    const size_t w_bytes = (size_t)l.groups * l.k * wide * (a.grad_f32 ? 4 : 2);
    if (a.dX && l.x_rows() > 0 && l.k > 0) e = cudaMemsetAsync(a.dX, 0, (size_t)l.x_rows() * l.k * 2, s);
    if (e == cudaSuccess && a.dW && w_bytes > 0 && !a.accumulate) e = cudaMemsetAsync(a.dW, 0, w_bytes, s);
    if (e == cudaSuccess && a.db && wide > 0 && !a.accumulate)
      e = cudaMemsetAsync(a.db, 0, (size_t)l.groups * wide * 4, s);
    return e == cudaSuccess ? MORELLO_OK : record_cuda_error(e);
  }
  Carver carve;
  carve.base = ws ? static_cast<char*>(ws) : reinterpret_cast<char*>(uintptr_t(256));   // nothing is taken
  rc = backward(dev, l, a, carve, false, s, &launches);
  count_launches(launches);
  return rc;
}

int dense_layer(int act, int gated, int w_layout, int64_t m, int64_t k, int64_t n, Layer* l) {
  int rc;
  if ((rc = check_act(act, gated)) != MORELLO_OK || (rc = check_flag(w_layout)) != MORELLO_OK) return rc;
  l->act = act;
  l->gated = gated != 0;
  l->w_cols = w_layout == MORELLO_W_COLMAJOR;
  l->m = m;
  l->k = k;
  l->n = n;
  return check_extents(m, k, n, gated ? (n > kMaxExtent ? n : 2 * n) : n, 1);
}

int expert_layer(int act, int gated, int w_layout, int gather, int64_t tokens, int64_t topk, int64_t experts, int64_t k,
                 int64_t n, const int32_t* plan, Layer* l) {
  int rc;
  if ((rc = check_flag(gather)) != MORELLO_OK || (rc = check_experts(tokens, topk, experts)) != MORELLO_OK) return rc;
  const int64_t rows = expert_rows(tokens, topk, experts);
  if ((rc = dense_layer(act, gated, w_layout, rows, k, n, l)) != MORELLO_OK) return rc;
  if ((rc = check_extents(rows, k, n, l->wide(), experts)) != MORELLO_OK) return rc;
  l->grouped = true;
  l->gather = gather != 0;
  l->groups = experts;
  if (rows > 0 && !plan) return MORELLO_ERR_NULL_POINTER;
  if (!aligned(plan, 4)) return MORELLO_ERR_MISALIGNED;
  l->x = expert_rows_of(tokens, topk, experts, plan);
  return MORELLO_OK;
}

const void* const kFake = reinterpret_cast<const void*>(uintptr_t(4096));   // 16-byte-aligned stand-in

}  // namespace
}  // namespace morello

using namespace morello;

#pragma GCC visibility push(default)
extern "C" {

int morello_linear(int act, int gated, int y_type, int w_layout, int64_t m, int64_t k, int64_t n, const void* X,
                   const void* W, const void* bias, const void* R, void* Y, void* Z, void* workspace,
                   size_t workspace_bytes, void* stream) {
  Layer l;
  int rc;
  if ((rc = check_flag(y_type)) != MORELLO_OK || (rc = dense_layer(act, gated, w_layout, m, k, n, &l)) != MORELLO_OK)
    return rc;
  return run_forward(l, ForwardArgs{X, W, bias, R, Y, Z, y_type == MORELLO_F32}, workspace, workspace_bytes, stream);
}

size_t morello_linear_workspace_bytes(int gated, int w_layout, int64_t m, int64_t k, int64_t n) {
  Layer l;
  if (dense_layer(kActNone, gated, w_layout, m, k, n, &l) != MORELLO_OK || m == 0 || n == 0) return 0;
  const ForwardArgs a{kFake, kFake, nullptr, nullptr, nullptr, nullptr, false};
  return dry_bytes([&](Carver& ws, uint64_t& none) { forward(DeviceInfo{}, l, a, ws, true, nullptr, &none); });
}

int morello_linear_backward(int act, int gated, int grad_type, int accumulate, int w_layout, int64_t m, int64_t k,
                            int64_t n, const void* X, const void* W, const void* Z, const void* dY, void* dX, void* dW,
                            float* dbias, void* workspace, size_t workspace_bytes, void* stream) {
  Layer l;
  int rc;
  if ((rc = check_flag(grad_type)) != MORELLO_OK || (rc = check_flag(accumulate)) != MORELLO_OK ||
      (rc = dense_layer(act, gated, w_layout, m, k, n, &l)) != MORELLO_OK)
    return rc;
  if (accumulate && grad_type != MORELLO_F32) return MORELLO_ERR_INVALID_ARGUMENT;
  return run_backward(l, BackwardArgs{X, W, Z, dY, dX, dW, dbias, grad_type == MORELLO_F32, accumulate != 0}, workspace,
                      workspace_bytes, stream);
}

size_t morello_linear_backward_workspace_bytes(int act, int gated, int w_layout, int64_t m, int64_t k, int64_t n) {
  Layer l;
  if (dense_layer(act, gated, w_layout, m, k, n, &l) != MORELLO_OK || m == 0 || n == 0) return 0;
  void* some = const_cast<void*>(kFake);
  const BackwardArgs a{kFake, kFake, kFake, kFake, some, some, static_cast<float*>(some), false, false};
  return dry_bytes([&](Carver& ws, uint64_t& none) { backward(DeviceInfo{}, l, a, ws, true, nullptr, &none); });
}

int64_t morello_expert_plan_rows(int64_t tokens, int64_t topk, int64_t experts) {
  return check_experts(tokens, topk, experts) == MORELLO_OK ? expert_rows(tokens, topk, experts) : -1;
}

int64_t morello_expert_plan_words(int64_t tokens, int64_t topk, int64_t experts) {
  return check_experts(tokens, topk, experts) == MORELLO_OK ? expert_plan_words(tokens, topk, experts) : -1;
}

int morello_expert_plan(int64_t tokens, int64_t topk, int64_t experts, const int32_t* idx, int32_t* plan, void* stream) {
  int rc;
  if ((rc = check_experts(tokens, topk, experts)) != MORELLO_OK) return rc;
  if (!plan || (!idx && tokens > 0)) return MORELLO_ERR_NULL_POINTER;
  if (!aligned(plan, 4) || !aligned(idx, 4)) return MORELLO_ERR_MISALIGNED;
  DeviceInfo dev;
  void* none = nullptr;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if ((rc = operator_workspace(0, nullptr, 0, s, &none, &dev)) != MORELLO_OK) return rc;
  uint64_t launches = 0;
  const cudaError_t e = plan_launch(expert_rows_of(tokens, topk, experts, plan), idx, s, &launches);
  count_launches(launches);
  return e == cudaSuccess ? MORELLO_OK : record_cuda_error(e);
}

int morello_expert_linear(int act, int gated, int y_type, int w_layout, int gather, int64_t tokens, int64_t topk,
                          int64_t experts, int64_t k, int64_t n, const int32_t* plan, const void* X, const void* W,
                          const void* bias, void* Y, void* Z, void* workspace, size_t workspace_bytes, void* stream) {
  Layer l;
  int rc;
  if ((rc = check_flag(y_type)) != MORELLO_OK ||
      (rc = expert_layer(act, gated, w_layout, gather, tokens, topk, experts, k, n, plan, &l)) != MORELLO_OK)
    return rc;
  return run_forward(l, ForwardArgs{X, W, bias, nullptr, Y, Z, y_type == MORELLO_F32}, workspace, workspace_bytes, stream);
}

size_t morello_expert_linear_workspace_bytes(int gated, int w_layout, int gather, int64_t tokens, int64_t topk,
                                             int64_t experts, int64_t k, int64_t n) {
  Layer l;
  if (expert_layer(kActNone, gated, w_layout, gather, tokens, topk, experts, k, n, static_cast<const int32_t*>(kFake),
                   &l) != MORELLO_OK || l.m == 0 || n == 0)
    return 0;
  const ForwardArgs a{kFake, kFake, nullptr, nullptr, nullptr, nullptr, false};
  return dry_bytes([&](Carver& ws, uint64_t& none) { forward(DeviceInfo{}, l, a, ws, true, nullptr, &none); });
}

int morello_expert_linear_backward(int act, int gated, int grad_type, int accumulate, int w_layout, int gather,
                                   int64_t tokens, int64_t topk, int64_t experts, int64_t k, int64_t n,
                                   const int32_t* plan, const void* X, const void* W, const void* Z, const void* dY,
                                   void* dX, void* dW, float* dbias, void* workspace, size_t workspace_bytes,
                                   void* stream) {
  Layer l;
  int rc;
  if ((rc = check_flag(grad_type)) != MORELLO_OK || (rc = check_flag(accumulate)) != MORELLO_OK ||
      (rc = expert_layer(act, gated, w_layout, gather, tokens, topk, experts, k, n, plan, &l)) != MORELLO_OK)
    return rc;
  if (accumulate && grad_type != MORELLO_F32) return MORELLO_ERR_INVALID_ARGUMENT;
  return run_backward(l, BackwardArgs{X, W, Z, dY, dX, dW, dbias, grad_type == MORELLO_F32, accumulate != 0}, workspace,
                      workspace_bytes, stream);
}

size_t morello_expert_linear_backward_workspace_bytes(int act, int gated, int w_layout, int gather, int64_t tokens,
                                                      int64_t topk, int64_t experts, int64_t k, int64_t n) {
  Layer l;
  if (expert_layer(act, gated, w_layout, gather, tokens, topk, experts, k, n, static_cast<const int32_t*>(kFake), &l) !=
          MORELLO_OK || l.m == 0 || n == 0)
    return 0;
  void* some = const_cast<void*>(kFake);
  const BackwardArgs a{kFake, kFake, kFake, kFake, some, some, static_cast<float*>(some), false, false};
  return dry_bytes([&](Carver& ws, uint64_t& none) { backward(DeviceInfo{}, l, a, ws, true, nullptr, &none); });
}

int morello_expert_combine(int y_type, int64_t tokens, int64_t topk, int64_t experts, int64_t n, const int32_t* plan,
                           const float* weights, const void* Y, const void* R, void* out, void* stream) {
  int rc;
  if ((rc = check_flag(y_type)) != MORELLO_OK || (rc = check_experts(tokens, topk, experts)) != MORELLO_OK) return rc;
  if ((rc = check_extents(expert_rows(tokens, topk, experts), 0, n, n, 1)) != MORELLO_OK) return rc;
  const bool empty = tokens == 0 || n == 0;
  if (!empty && (!plan || !Y || !out)) return MORELLO_ERR_NULL_POINTER;
  if (!aligned(plan, 4) || !aligned(weights, 4) || !aligned(Y, y_type == MORELLO_F32 ? 4 : 2) || !aligned(R, 2) ||
      !aligned(out, 2))
    return MORELLO_ERR_MISALIGNED;
  DeviceInfo dev;
  void* none = nullptr;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if ((rc = operator_workspace(0, nullptr, 0, s, &none, &dev)) != MORELLO_OK || empty) return rc;
  uint64_t launches = 0;
  const cudaError_t e =
      combine_launch(expert_rows_of(tokens, topk, experts, plan), y_type == MORELLO_F32, n, n, weights, Y,
                     static_cast<const uint16_t*>(R), static_cast<uint16_t*>(out), s, &launches);
  count_launches(launches);
  return e == cudaSuccess ? MORELLO_OK : record_cuda_error(e);
}

int morello_expert_combine_backward(int y_type, int64_t tokens, int64_t topk, int64_t experts, int64_t n,
                                    const int32_t* plan, const float* weights, const void* Y, const void* dout, void* dY,
                                    float* dweights, void* stream) {
  int rc;
  if ((rc = check_flag(y_type)) != MORELLO_OK || (rc = check_experts(tokens, topk, experts)) != MORELLO_OK) return rc;
  if ((rc = check_extents(expert_rows(tokens, topk, experts), 0, n, n, 1)) != MORELLO_OK) return rc;
  if (tokens > 0 && (!plan || (n > 0 && (!dout || (dweights && !Y))))) return MORELLO_ERR_NULL_POINTER;
  if (!aligned(plan, 4) || !aligned(weights, 4) || !aligned(Y, y_type == MORELLO_F32 ? 4 : 2) || !aligned(dout, 2) ||
      !aligned(dY, 2) || !aligned(dweights, 4))
    return MORELLO_ERR_MISALIGNED;
  DeviceInfo dev;
  void* none = nullptr;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if ((rc = operator_workspace(0, nullptr, 0, s, &none, &dev)) != MORELLO_OK || tokens == 0) return rc;
  uint64_t launches = 0;
  const cudaError_t e = combine_backward_launch(expert_rows_of(tokens, topk, experts, plan), y_type == MORELLO_F32, n,
                                                weights, Y, static_cast<const uint16_t*>(dout),
                                                static_cast<uint16_t*>(dY), dweights, s, &launches);
  count_launches(launches);
  return e == cudaSuccess ? MORELLO_OK : record_cuda_error(e);
}

int morello_route(int score, int renorm, float scale, int logits_type, int64_t tokens, int64_t experts, int64_t topk,
                  int64_t groups, int64_t topk_groups, const void* logits, const float* bias, int32_t* idx,
                  float* weights, void* stream) {
  int rc;
  if ((rc = check_flag(score)) != MORELLO_OK || (rc = check_flag(renorm)) != MORELLO_OK ||
      (rc = check_flag(logits_type)) != MORELLO_OK || (rc = check_experts(tokens, topk, experts)) != MORELLO_OK)
    return rc;
  if (groups < 1 || groups > kMaxGroups || experts % groups != 0 || topk_groups < 1 || topk_groups > groups ||
      topk > topk_groups * (experts / groups))
    return MORELLO_ERR_INVALID_SHAPE;
  if (tokens > 0 && (!logits || !idx || !weights)) return MORELLO_ERR_NULL_POINTER;
  if (!aligned(logits, logits_type == MORELLO_F32 ? 4 : 2) || !aligned(bias, 4) || !aligned(idx, 4) || !aligned(weights, 4))
    return MORELLO_ERR_MISALIGNED;
  DeviceInfo dev;
  void* none = nullptr;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if ((rc = operator_workspace(0, nullptr, 0, s, &none, &dev)) != MORELLO_OK) return rc;
  RouteCall c;
  c.sigmoid = score == MORELLO_SCORE_SIGMOID;
  c.renorm = renorm != 0;
  c.logits_f32 = logits_type == MORELLO_F32;
  c.scale = scale;
  c.tokens = tokens;
  c.experts = experts;
  c.topk = topk;
  c.groups = topk_groups == groups ? 1 : groups;     // every group stays: no choice of groups
  c.topk_groups = topk_groups;
  c.logits = logits;
  c.bias = bias;
  c.idx = idx;
  c.weights = weights;
  uint64_t launches = 0;
  const cudaError_t e = route_launch(c, s, &launches);
  count_launches(launches);
  return e == cudaSuccess ? MORELLO_OK : record_cuda_error(e);
}

int morello_route_backward(int score, int renorm, float scale, int logits_type, int64_t tokens, int64_t experts,
                           int64_t topk, const void* logits, const int32_t* idx, const float* dweights, void* dlogits,
                           void* stream) {
  int rc;
  if ((rc = check_flag(score)) != MORELLO_OK || (rc = check_flag(renorm)) != MORELLO_OK ||
      (rc = check_flag(logits_type)) != MORELLO_OK || (rc = check_experts(tokens, topk, experts)) != MORELLO_OK)
    return rc;
  if (topk > experts) return MORELLO_ERR_INVALID_SHAPE;
  if (tokens > 0 && (!logits || !idx || !dweights || !dlogits)) return MORELLO_ERR_NULL_POINTER;
  const uintptr_t to = logits_type == MORELLO_F32 ? 4 : 2;
  if (!aligned(logits, to) || !aligned(dlogits, to) || !aligned(idx, 4) || !aligned(dweights, 4))
    return MORELLO_ERR_MISALIGNED;
  DeviceInfo dev;
  void* none = nullptr;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if ((rc = operator_workspace(0, nullptr, 0, s, &none, &dev)) != MORELLO_OK) return rc;
  RouteCall c;
  c.sigmoid = score == MORELLO_SCORE_SIGMOID;
  c.renorm = renorm != 0;
  c.logits_f32 = logits_type == MORELLO_F32;
  c.scale = scale;
  c.tokens = tokens;
  c.experts = experts;
  c.topk = topk;
  c.logits = logits;
  uint64_t launches = 0;
  const cudaError_t e = route_backward_launch(c, idx, dweights, dlogits, s, &launches);
  count_launches(launches);
  return e == cudaSuccess ? MORELLO_OK : record_cuda_error(e);
}

}  // extern "C"
#pragma GCC visibility pop
