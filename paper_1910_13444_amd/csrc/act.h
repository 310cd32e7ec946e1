// Activations of the linear layer: value and derivative with respect to the
// pre-activation, in fp32.
//   tanh   t,                   1 - t^2 (formed from exp, see tanh_ts)
//   relu   max(a, 0),           1 for a > 0, else 0
//   gelu   a Phi(a),            Phi(a) + a phi(a)      (normal distribution)
//   silu   a s, s = 1 / (1 + exp(-a)),   s + a s (1 - s)
#pragma once
#include "common.h"

namespace pigan {

// exp(x) by the hardware base-2 exponential; the rounding of the scaled
// argument leaves |x| 6e-8 relative, which the functions below meet only where
// the exponential is a small part of their result
__device__ __forceinline__ float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.4426950408889634f); }

// Normal distribution: Phi(a), and gauss = exp(-a^2 / 2).  With z = |a| / sqrt 2
// and t = 1 / (1 + 0.4 z) the tail is erfc(z) = t Q(t) exp(-z^2), Q the
// polynomial of degree 8 that is nearest to erfc(z) exp(z^2) / t on all of
// z >= 0 (1.3e-7 relative, 2.6e-7 with the roundings of the fp32 evaluation).
// The lower tail is therefore accurate in relative terms, where
// 0.5 (1 + erf) would cancel.
__device__ __forceinline__ float normal_cdf(float a, float& gauss) {
  const float z = fabsf(a) * 0.70710678118654752f;
  const float t = __builtin_amdgcn_rcpf(1.0f + 0.4f * z);
  float q = 0.05027513951063156f;
  q = q * t - 0.18294988572597504f;
  q = q * t + 0.16915729641914368f;
  q = q * t - 0.0056617371737957f;
  q = q * t + 0.14145344495773315f;
  q = q * t + 0.1685371994972229f;
  q = q * t + 0.20784327387809753f;
  q = q * t + 0.22566954791545868f;
  q = q * t + 0.22567586600780487f;
  gauss = fast_exp(-0.5f * a * a);
  const float tail = 0.5f * t * q * gauss;
  return a < 0.0f ? tail : 1.0f - tail;
}

// s = 1 / (1 + exp(-a)) and c = 1 - s, both without cancellation
__device__ __forceinline__ float logistic(float a, float& c) {
  const float e = fast_exp(-fabsf(a));
  const float r = __builtin_amdgcn_rcpf(1.0f + e);
  c = a < 0.0f ? r : e * r;
  return a < 0.0f ? e * r : r;
}

template <int ACT>
__device__ __forceinline__ float act_value(float a) {
  if constexpr (ACT == PIGAN_ACT_TANH) {
    float t, s;
    tanh_ts(a, t, s);
    return t;
  } else if constexpr (ACT == PIGAN_ACT_RELU) {
    return a < 0.0f ? 0.0f : a;      // a NaN stays one
  } else if constexpr (ACT == PIGAN_ACT_GELU) {
    float g;
    return a * normal_cdf(a, g);
  } else if constexpr (ACT == PIGAN_ACT_SILU) {
    float c;
    return a * logistic(a, c);
  } else {
    return a;
  }
}

template <int ACT>
__device__ __forceinline__ float act_slope(float a) {
  if constexpr (ACT == PIGAN_ACT_TANH) {
    float t, s;
    tanh_ts(a, t, s);
    return s;
  } else if constexpr (ACT == PIGAN_ACT_RELU) {
    return a > 0.0f ? 1.0f : 0.0f;
  } else if constexpr (ACT == PIGAN_ACT_GELU) {
    float g;
    const float p = normal_cdf(a, g);
    return p + a * g * 0.3989422804014327f;   // 1 / sqrt(2 pi)
  } else if constexpr (ACT == PIGAN_ACT_SILU) {
    float c;
    const float s = logistic(a, c);
    return s + a * s * c;
  } else {
    return 1.0f;
  }
}

// f<ACT>() with the activation of a launch: one branch for all lanes
#define PIGAN_ACT_SWITCH(act, ...)                                               \
  switch (act) {                                                                 \
    case PIGAN_ACT_TANH: { constexpr int ACT = PIGAN_ACT_TANH; __VA_ARGS__ } break; \
    case PIGAN_ACT_RELU: { constexpr int ACT = PIGAN_ACT_RELU; __VA_ARGS__ } break; \
    case PIGAN_ACT_GELU: { constexpr int ACT = PIGAN_ACT_GELU; __VA_ARGS__ } break; \
    case PIGAN_ACT_SILU: { constexpr int ACT = PIGAN_ACT_SILU; __VA_ARGS__ } break; \
    default: { constexpr int ACT = PIGAN_ACT_NONE; __VA_ARGS__ } break;          \
  }

}  // namespace pigan
