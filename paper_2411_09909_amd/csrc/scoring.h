// What the operators of include/amxfp4_scoring.h share: capped scores and biases that fall with distance. Not installed.
#pragma once
#include <math.h>

#include "../../include/amxfp4_scoring.h"
#include "device_formats.h"

namespace amx {

// What a kernel reads of amx_scores_t. All scores are in units of log2, so that the softmax takes exp2.
struct Scores {
  float in, cap;        // tanh(scale q.k / C) of a raw product s is 1 - 2 / (1 + exp2(s * in)); cap: C log2(e). 0: not capped
  float scale;          // softmax scale times log2(e), where not capped
  const float* slopes;  // of the query heads, or nullptr
};

constexpr float kLog2e = 1.4426950408889634f;

inline bool scores_valid(const amx_scores_t* s) {
  if (!s) return true;
  if (s->reserved != 0 || (reinterpret_cast<uintptr_t>(s->slopes) & 3)) return false;
  return s->cap == 0.f || (s->cap >= 0x1p-20f && s->cap <= 0x1p20f);
}

inline Scores scores_of(const amx_scores_t* s, float scale) {
  Scores r = {0.f, 0.f, scale * kLog2e, s ? s->slopes : nullptr};
  if (s && s->cap > 0.f) r.in = scale / s->cap * (2 * kLog2e), r.cap = s->cap * kLog2e;
  return r;
}

// cap * tanh from what the product is: the two hardware functions are right to about an ulp of 1, so the result to 2^-22 of the
// cap, absolutely. An infinite exponential gives the cap itself.
__device__ __forceinline__ float capped(float s, float in, float cap) {
  const float e = __builtin_amdgcn_exp2f(s * in);
  return __builtin_fmaf(-2.0f * cap, __builtin_amdgcn_rcpf(1.0f + e), cap);
}

}  // namespace amx
