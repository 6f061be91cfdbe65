// What the operators of include/amxfp4_scoring.h share: capped scores and biases that fall with distance. Not installed.
#pragma once
#include <math.h>

#include "../../include/amxfp4_scoring.h"
#include "device_formats.h"

namespace amx {

// What a kernel reads of amx_scores_t. All scores are in units of log2, so that the softmax takes exp2.
struct Scores {
  float in, cap;        // tanh(scale q.k / C) of a raw product s is 1 - 2 / (1 + exp2(s * in)); cap: C log2(e). 0: not capped
  float scale;          // softmax scale times log2(e)
  float small;          // raw products up to here may take the polynomial below (0: none)
  float k1, k2, k3, k4; // scale s (1 + k1' s^2 + ..): multiplied by the scale here
  const float* slopes;  // of the query heads, or nullptr
};

constexpr float kLog2e = 1.4426950408889634f;

inline bool scores_valid(const amx_scores_t* s) {
  if (!s) return true;
  if (s->reserved != 0 || (reinterpret_cast<uintptr_t>(s->slopes) & 3)) return false;
  return s->cap == 0.f || (s->cap >= 0x1p-20f && s->cap <= 0x1p20f);
}

// tanh z = z (1 + u (c1 + u (c2 + u (c3 + u c4)))), u = z^2, for |z| <= 0.45: coefficients fitted here for the least relative error, 2^-27.4, below FP32's own.
// Six instructions at the full rate where the formula with exp2 and a reciprocal takes five, two of them at a quarter of it. (Three coefficients are 2^-21.7
// off: times a cap of 50 enough for ten times as many weights of a prompt on the other side of a boundary of the cast as FP32 itself brings about. The fourth
// takes 1 to 4 % of capped calls; where times of their variants are compared in these files, both sides are still without it.)
constexpr float kSmall = 0.45f, kTanh[4] = {-0.333332479f, 0.13329199f, -0.0533394367f, 0.0180139281f};

inline Scores scores_of(const amx_scores_t* s, float scale) {
  Scores r = {};
  r.scale = scale * kLog2e, r.slopes = s ? s->slopes : nullptr;
  if (s && s->cap > 0.f) {
    const float c = scale / s->cap, u = c * c;
    r.in = c * (2 * kLog2e), r.cap = s->cap * kLog2e;
    // as far as the powers of c stay in range: with a wide cap fewer terms up to a smaller size, with a very narrow one none
    if (c < 0x1p12f && scale < 0x1p20f) {
      const int terms = c > 0x1p-12f && scale > 0x1p-20f ? 4 : c > 0x1p-30f ? 2 : 1;
      // (2^60: the polynomial squares the product)
      r.small = fminf((terms == 4 ? kSmall : terms == 2 ? 0.02f : 0x1p-12f) / c, 0x1p60f);
      r.k1 = r.scale * u * kTanh[0];
      if (terms >= 2) r.k2 = r.scale * u * u * kTanh[1];
      if (terms == 4) r.k3 = r.scale * u * u * u * kTanh[2], r.k4 = r.scale * u * u * u * u * kTanh[3];
    }
  }
  return r;
}

// The slope of a query head. Distances are below 2^31, and what a slope makes of them has to be finite: the nearest key has all the weight well before.
__device__ __forceinline__ float slope_of(const Scores& w, uint32_t head) {
  return fminf(fmaxf(w.slopes[head] * kLog2e, -0x1p90f), 0x1p90f);
}

// cap * tanh from what the product is: the two hardware functions are right to about an ulp of 1, so the result to 2^-22 of the
// cap, absolutely. An infinite exponential gives the cap itself.
__device__ __forceinline__ float capped(float s, float in, float cap) {
  const float e = __builtin_amdgcn_exp2f(s * in);
  return __builtin_fmaf(-2.0f * cap, __builtin_amdgcn_rcpf(1.0f + e), cap);
}

// The same of a product of at most Scores::small, plus a number.
__device__ __forceinline__ float capped_small(float s, const Scores& w, float plus) {
  const float u = s * s;
  const float p = __builtin_fmaf(u, __builtin_fmaf(u, __builtin_fmaf(u, __builtin_fmaf(u, w.k4, w.k3), w.k2), w.k1), w.scale);
  return __builtin_fmaf(s, p, plus);
}

// Of any product, each by what is its due.
__device__ __forceinline__ float capped_any(float s, const Scores& w) {
  return __builtin_fabsf(s) <= w.small ? capped_small(s, w, 0.f) : capped(s, w.in, w.cap);
}

}  // namespace amx
