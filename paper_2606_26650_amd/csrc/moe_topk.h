// A token's experts: the k largest router logits and their softmax, shared by the routing call and the experts' layer.
#pragma once

#include "catq_internal.h"

namespace catq {

// Logits in order as integers: a larger logit has a larger key, -0 and +0 the
// same, a NaN the lowest of all (0).
__device__ __forceinline__ unsigned int logit_key(float x) {
  if (x != x) return 0u;
  const unsigned int u = x == 0.0f ? 0u : __float_as_uint(x);
  return (u >> 31) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_logit(unsigned int key) {
  if (key == 0u) return __builtin_nanf("");
  return __uint_as_float((key >> 31) ? key & 0x7fffffffu : ~key);
}

// The largest of a wave's values (not below 0), by data-parallel moves: within rows of 16 lanes, then across them.
__device__ __forceinline__ unsigned int wave_umax(unsigned int v) {
#define CATQ_MAX_MOVED(ctrl, rows) \
  v = max(v, (unsigned int)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, rows, 0xf, false))
  CATQ_MAX_MOVED(0x111, 0xf);
  CATQ_MAX_MOVED(0x112, 0xf);
  CATQ_MAX_MOVED(0x114, 0xf);
  CATQ_MAX_MOVED(0x118, 0xf);
  CATQ_MAX_MOVED(0x142, 0xa);
  CATQ_MAX_MOVED(0x143, 0xc);
#undef CATQ_MAX_MOVED
  return (unsigned int)__builtin_amdgcn_readlane((int)v, 63);
}

// One wavefront takes a token: top-k of the E >= k logits (largest first; equal
// values go to the lower expert id, NaN after every other) and the softmax over
// the k selected logits.  An expert is selected once whatever the logits hold:
// the ids index rows and experts, so they are valid and distinct also where
// logits are NaN or -inf (then it is the weights that turn NaN or 0).  PER logits
// per lane (E <= 64 PER).
// Lane j < k gets the j-th selected expert and its weight.  (With the maximum and its id passed through shuffles,
// a token of 128 experts and 8 slots took 7 us.)
template <int PER>
__device__ __forceinline__ void topk_token(const float* logits, int E, int k, int lane, int& id, float& weight) {
  unsigned int key[PER];   // 1 for a NaN (no other key is that small), 0 for none and for a selected one
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = lane + 64 * i;
    key[i] = e < E ? max(logit_key(logits[e]), 1u) : 0u;
  }
  float sel = -INFINITY;   // lane j: the j-th selected logit and its expert
  int sid = 0;
  for (int j = 0; j < k; ++j) {
    unsigned int best = key[0];
#pragma unroll
    for (int i = 1; i < PER; ++i) best = max(best, key[i]);
    best = wave_umax(best);
    int be = -1;           // the lowest id that has it
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const unsigned long long m = __ballot(key[i] == best);
      if (be < 0 && m) be = 64 * i + __builtin_ctzll(m);
    }
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (lane + 64 * i == be) key[i] = 0u;
    if (lane == j) {
      sel = key_logit(best == 1u ? 0u : best);
      sid = be;
    }
  }
  auto lane_of = [](float v, int j) {
    return __uint_as_float((unsigned int)__builtin_amdgcn_readlane((int)__float_as_uint(v), j));
  };
  const float ex = expf(sel - lane_of(sel, 0));
  float sum = 0.f;
  for (int j = 0; j < k; ++j) sum += lane_of(ex, j);
  id = sid;
  weight = ex * (1.0f / sum);
}

}  // namespace catq
