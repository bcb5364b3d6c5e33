// Host-side launch interface of the routing kernels (aa_route.hip).
#pragma once

#include "aa_common.hpp"

namespace aa {

constexpr int kMaxExperts = AA_MAX_EXPERTS;
constexpr int kMaxChoices = AA_MAX_CHOICES;
constexpr int kPlanTile = 2048;  // pairs grouped by one block

struct RouteArgs {
  const void *logits;
  int32_t dtype, vec;  // vec (set at launch): a lane's logits can be moved at once
  int64_t ld;
  const int32_t *count;
  int32_t n_max, n_experts;
  const float *bias;
  aa_route_config cfg;
  int32_t *ids;
  float *weights;
};

struct RouteGradArgs {
  const void *logits;
  int32_t dtype, vec;
  int64_t ld;
  const int32_t *count;
  int32_t n_max, n_experts;
  aa_route_config cfg;
  const int32_t *ids;
  const float *dweights;
  void *dlogits;
  int64_t ld_out;
};

struct PlanArgs {
  const int32_t *ids;
  const int32_t *count;
  int32_t n_max, top_k, n_experts;
  int32_t *offsets, *order, *slot;
  int32_t *table;  // [tiles + 1][E]: counts of the tiles (scanned: of all before each, the last row the totals)
};

inline size_t plan_table_ints(int64_t n_max, int32_t top_k, int32_t n_experts) {
  const size_t tiles = ((size_t)n_max * top_k + kPlanTile - 1) / kPlanTile;
  return (tiles + 1) * (size_t)n_experts;
}

// plan: made in the same call (may be NULL)
hipError_t launch_route(const RouteArgs &a, const PlanArgs *plan, hipStream_t st);
hipError_t launch_route_grad(const RouteGradArgs &a, hipStream_t st);
hipError_t launch_expert_plan(const PlanArgs &a, hipStream_t st);

}  // namespace aa
