// Routing of tokens to experts (route.hip).  Internal to the library.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace rl {

struct RouteDesc {
  int dtype = 0;  // of the logits
  int64_t n = 0;
  int experts = 0, top = 1, sigmoid = 0, renorm = 0, groups = 1, kept = 1, group_top = 1;
  float scale = 1.f;
  const float* bias = nullptr;
  const void* logits = nullptr;
  int64_t ld = 0;
  float* weight = nullptr;
  int32_t *expert = nullptr, *place = nullptr, *source = nullptr, *ends = nullptr;  // backward: expert is read
  const float* dweight = nullptr;
  void* dlogits = nullptr;
  int64_t lddl = 0;
};
constexpr int kRouteMaxExperts = 1024, kRouteMaxTop = 64;
constexpr int64_t kRouteMaxTokens = 1 << 23;

constexpr int64_t kRouteGroups = 512;  // workgroups of a large call; counts of at most 65535 rows an expert in each of them
static_assert(kRouteMaxTokens / kRouteGroups + 1024 < 65536, "counts are 16 bits");

// How a call's choice is dealt out: lanes a token, as few as hold the choice and one more, from 16 on, with up to 16 experts each (`groups`: of experts,
// 1 without a limit).  route_lds: bytes of LDS a workgroup, wide: scores are added to.
struct RoutePlan {
  int lanes, per, waves, each, groups;  // per: experts a lane;  waves, each, groups: of a workgroup, its tokens, workgroups
  unsigned room;                        // bytes a wave has in LDS
};
RoutePlan route_plan(int64_t n, int64_t experts, int64_t top, int64_t groups);
unsigned route_lds(const RoutePlan& p, int64_t experts, bool wide);

size_t route_workspace(int64_t n, int64_t experts, int64_t top);
hipError_t route_forward(const RouteDesc& d, void* workspace, hipStream_t s);
hipError_t route_backward(const RouteDesc& d, hipStream_t s);

}  // namespace rl
