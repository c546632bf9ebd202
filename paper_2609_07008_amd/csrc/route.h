// Arguments of the router (mla_moe_route).
#pragma once

#include "common.h"
#include "moe.h"

namespace mla {

constexpr int kRouteMaxGroups = 64;   // a lane ranks a group

struct RouteArgs {
  const void* logits;      // [N, E] f32 or bf16, rows `stride` apart
  const float* bias;       // [E] or null
  int32_t* expert_idx;     // [N, top_k]
  float* expert_w;         // [N, top_k]
  int32_t* fanout;         // [N] or null
  int32_t* expert_count;   // [E] or null
  int64_t n_rows;
  int64_t stride;
  int32_t n_experts;
  int32_t logits_bf16;
  int32_t sigmoid;         // 0: softmax over the row
  int32_t n_groups, top_groups, group_best;
  int32_t top_k, min_k;
  int32_t renormalize;
  float scale, tau;
};

hipError_t launch_moe_route(const RouteArgs& a, hipStream_t s);

}  // namespace mla
