// The choice of a token's experts, shared by the router (tuna_route.cu) and the few-token layer (tuna_few.cu).
#ifndef TUNA_ROUTE_CUH
#define TUNA_ROUTE_CUH

#include "tuna_ops.cuh"

namespace tuna_ops {

constexpr int kMaxK = TUNA_MOE_MAX_K;

// What a router makes of a logit.  A NaN is a masked place, like -inf: never chosen.
__device__ __forceinline__ float logit_of(float v) { return v != v ? -INFINITY : v; }
// exp(z - m) where both may be infinite: the places that hold +inf share the weight.
__device__ __forceinline__ float exp_of(float z, float m) { return z == m ? 1.0f : expf(z - m); }
__device__ __forceinline__ float sigmoid_of(float z) { return 1.0f / (1.0f + expf(-z)); }

// A token's logits, VPL a lane in a group of LPT lanes: lane l holds experts l*VPL ...
template <int VPL, typename T>
__device__ __forceinline__ void load_logits(const T *row, int first, int experts, bool vec, float (&z)[VPL]) {
  if (vec && first + VPL <= experts) {
    load_row(row + first, z);
#pragma unroll
    for (int i = 0; i < VPL; ++i) z[i] = logit_of(z[i]);
  } else {
#pragma unroll
    for (int i = 0; i < VPL; ++i) z[i] = first + i < experts ? logit_of(to_f32(row[first + i])) : -INFINITY;
  }
}

// The choice for one token by its group of LPT lanes; lane s of the group leaves with slot s
// (k <= LPT).  k rounds of an argmax: within a lane over its VPL values, then the group's largest
// value, by shuffles or, where the group is the warp, in one instruction; the first lane that holds
// it tells its expert.  Ties go to the lower expert: within a lane a later one must be strictly
// larger, and lanes hold experts in order.
template <int LPT, int VPL>
__device__ __forceinline__ void choose(float (&z)[VPL], int lane, int k, int scoring, int renormalize, float scale, int &id, float &weight) {
  const int first = lane * VPL;
  uint32_t taken = 0;
  float mine = -INFINITY, top = -INFINITY;
  id = -1;
  for (int s = 0; s < k; ++s) {
    float best = -INFINITY;
    int at = 0;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      if (z[i] > best && !((taken >> i) & 1)) best = z[i], at = i;
    }
    int e = first + at;
    const float own = best;
    if constexpr (LPT == 32) {
      asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(best) : "f"(own));
    } else {
#pragma unroll
      for (int d = 1; d < LPT; d <<= 1) best = fmaxf(best, __shfl_xor_sync(~0u, best, d));
    }
    const uint32_t holders = __ballot_sync(~0u, own == best) >> (threadIdx.x & (32 - LPT));
    e = __shfl_sync(~0u, e, __ffs(holders) - 1, LPT);
    if (s == 0) top = best;
    if (best != -INFINITY) {  // (no early end: the other groups of the warp go on with the shuffles)
      if (e >= first && e < first + VPL) taken |= 1u << (e - first);
      if (s == lane) id = e, mine = best;
    }
  }
  float w = 0.0f;
  if (scoring == TUNA_MOE_SIGMOID) {
    if (id >= 0) w = sigmoid_of(mine);
  } else if (id >= 0) {
    w = exp_of(mine, top);
  }
  float sum = w;
  if (!renormalize && scoring == TUNA_MOE_SOFTMAX) {
    sum = 0.0f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) sum += z[i] == -INFINITY ? 0.0f : exp_of(z[i], top);
  }
#pragma unroll
  for (int d = 1; d < LPT; d <<= 1) sum += __shfl_xor_sync(~0u, sum, d);
  if (renormalize || scoring == TUNA_MOE_SOFTMAX) w = sum > 0.0f ? w / sum : 0.0f;
  weight = id >= 0 ? w * scale : 0.0f;
}

}  // namespace tuna_ops
#endif
