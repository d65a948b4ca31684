// Internal declarations of the routing to experts and its row plan.
#pragma once

#include "linear.h"

namespace morello {

constexpr int kMaxExperts = 1024;
constexpr int kMaxTopk = 32;
constexpr int kMaxGroups = 32;

struct RouteCall {
  bool sigmoid = false, renorm = false, logits_f32 = true;
  float scale = 1.f;
  int64_t tokens = 0, experts = 0, topk = 0, groups = 1, topk_groups = 1;
  const void* logits = nullptr;
  const float* bias = nullptr;
  int32_t* idx = nullptr;
  float* weights = nullptr;
};
cudaError_t route_launch(const RouteCall& c, cudaStream_t stream, uint64_t* launches);
cudaError_t route_backward_launch(const RouteCall& c, const int32_t* idx, const float* dweights, void* dlogits,
                                  cudaStream_t stream, uint64_t* launches);

// Fills the plan of idx [tokens][topk] (x's pointers are into the plan buffer).
cudaError_t plan_launch(const ExpertRows& x, const int32_t* idx, cudaStream_t stream, uint64_t* launches);

// dY[row] = weight * dout[token] (zero rows where the layout holds no token), dweights = <dout, Y>.
cudaError_t combine_backward_launch(const ExpertRows& x, bool y_f32, int64_t n, const float* weights, const void* Y,
                                    const uint16_t* dout, uint16_t* dY, float* dweights, cudaStream_t stream,
                                    uint64_t* launches);

}  // namespace morello
