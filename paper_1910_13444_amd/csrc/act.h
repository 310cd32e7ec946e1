// Activations of the linear layer: value and derivative with respect to the
// pre-activation.
//   tanh   t,                   1 - t^2 (formed from exp)
//   relu   max(a, 0),           1 for a > 0, else 0
//   gelu   a Phi(a),            Phi(a) + a phi(a)      (normal distribution)
//   silu   a s, s = 1 / (1 + exp(-a)),   s + a s (1 - s)
//
// For 16-bit results in fp32 (errors of 1e-7 to 2e-6 relative, below), for fp32
// results in fp64, rounded once: there the fp32 forms' errors would be two to three
// times those of the rounding.
#pragma once
#include "common.h"

namespace pigan {

// ---------------------------------------------------------------------------
// in fp32
// ---------------------------------------------------------------------------
// exp(x) by the hardware base-2 exponential; the rounding of the scaled argument
// leaves 6e-8 |x| relative: 2e-6 at x = -a^2 / 2 of a = -6, less than 2^-8 of a unit
// of fp16 wherever the result is not below its range
__device__ __forceinline__ float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.4426950408889634f); }

// Normal distribution: Phi(a), and gauss = exp(-a^2 / 2).  With z = |a| / sqrt 2
// and t = 1 / (1 + 0.4 z) the tail is erfc(z) = t Q(t) exp(-z^2), Q the
// polynomial of degree 8 that is nearest to erfc(z) exp(z^2) / t on all of
// z >= 0 (1.3e-7 relative, 2.6e-7 with the roundings of the fp32 evaluation).
// The lower tail therefore has these errors and exp's in relative terms, where
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

// ---------------------------------------------------------------------------
// in fp64 (1e-9 relative, a hundredth of an fp32 rounding)
// ---------------------------------------------------------------------------
// 2^y for -2^20 < y <= 0; a NaN stays one.  2^f on |f| <= 1/2 by its nearest polynomial
// of degree 7 (4e-11 relative); the whole part of y is in the low bits of its sum with
// 1.5 * 2^52.
__device__ __forceinline__ double exp2_64(double y) {
  const double sum = y + 6755399441055744.0, f = y - (sum - 6755399441055744.0);
  double q = 1.5201918109007667e-05;
  q = q * f + 0.00015469291112801776;
  q = q * f + 0.001333392257928822;
  q = q * f + 0.009618027253755258;
  q = q * f + 0.0555041035342827;
  q = q * f + 0.24022651198157235;
  q = q * f + 0.6931471807284516;
  q = q * f + 0.999999999961682;
  return __builtin_ldexp(q, (int)(uint32_t)__builtin_bit_cast(uint64_t, sum));
}

// 1 / d for 1 <= d < 2^100: the fp32 reciprocal (2e-7) and a Newton step (4e-14)
__device__ __forceinline__ double rcp64(double d) {
  const double r = __builtin_amdgcn_rcpf((float)d);
  return r + r * (1.0 - d * r);
}

// |a|, but `most` beyond it (where the exponentials below are 0); a NaN stays one
__device__ __forceinline__ float size_to(float a, float most) { return fabsf(a) > most ? most : fabsf(a); }

// tanh and its slope, as tanh_ts
__device__ __forceinline__ void tanh64(float a, double& t, double& s) {
  const double x = a, a2 = x * x, e = exp2_64(size_to(a, 400.0f) * -2.8853900817779268), r = rcp64(1.0 + e);   // -2 / ln 2
  double q = 62.0 / 2835.0;
  q = q * a2 - 17.0 / 315.0;
  q = q * a2 + 2.0 / 15.0;
  q = q * a2 - 1.0 / 3.0;
  const double small = x + (x * a2) * q, big = copysign((1.0 - e) * r, x);
  t = fabsf(a) < 0.125f ? small : big;
  s = 4.0 * e * (r * r);
}

// as normal_cdf, by half the polynomial of degree 12 (4.4e-10 relative)
__device__ __forceinline__ double normal_cdf64(float a, double& gauss) {
  const double x = size_to(a, 57.0f), t = rcp64(1.0 + 0.28284271247461901 * x);   // 0.4 / sqrt 2
  double q = 0.009405752837212747;
  q = q * t - 0.05364639004433673;
  q = q * t + 0.1184391272407524;
  q = q * t - 0.11789789501917438;
  q = q * t + 0.04930509977688804;
  q = q * t - 0.027986399804715534;
  q = q * t + 0.013292126438845341;
  q = q * t + 0.033011687973272856;
  q = q * t + 0.06082717082829332;
  q = q * t + 0.0857635098091793;
  q = q * t + 0.10381036390080491;
  q = q * t + 0.11283792962537757;
  q = q * t + 0.11283791665947903;
  gauss = exp2_64(x * x * -0.72134752044448170);   // -1 / (2 ln 2)
  const double tail = t * q * gauss;
  return a < 0.0f ? tail : 1.0 - tail;
}

// as logistic
__device__ __forceinline__ double logistic64(float a, double& c) {
  const double e = exp2_64(size_to(a, 1000.0f) * -1.4426950408889634), r = rcp64(1.0 + e);
  c = a < 0.0f ? r : e * r;
  return a < 0.0f ? e * r : r;
}

// ---------------------------------------------------------------------------
// of results of type TO
// ---------------------------------------------------------------------------
template <int ACT, class TO>
__device__ __forceinline__ float act_value(float a) {
  constexpr bool X64 = sizeof(TO) == 4;
  if constexpr (ACT == PIGAN_ACT_TANH) {
    if constexpr (X64) {
      double t, s;
      tanh64(a, t, s);
      return (float)t;
    } else {
      float t, s;
      tanh_ts(a, t, s);
      return t;
    }
  } else if constexpr (ACT == PIGAN_ACT_RELU) {
    return a < 0.0f ? 0.0f : a;      // a NaN stays one
  } else if constexpr (ACT == PIGAN_ACT_GELU) {
    if constexpr (X64) {
      double g;
      return (float)(a * normal_cdf64(a, g));
    } else {
      float g;
      return a * normal_cdf(a, g);
    }
  } else if constexpr (ACT == PIGAN_ACT_SILU) {
    if constexpr (X64) {
      double c;
      return (float)(a * logistic64(a, c));
    } else {
      float c;
      return a * logistic(a, c);
    }
  } else {
    return a;
  }
}

// An infinite a (an fp16 pre-activation beyond 65504 is stored as one) has the
// slope's limit: a's size is bounded where the factors beside it have become 0.
template <int ACT, class TO>
__device__ __forceinline__ float act_slope(float a) {
  constexpr bool X64 = sizeof(TO) == 4;
  if constexpr (ACT == PIGAN_ACT_TANH) {
    if constexpr (X64) {
      double t, s;
      tanh64(a, t, s);
      return (float)s;
    } else {
      float t, s;
      tanh_ts(a, t, s);
      return s;
    }
  } else if constexpr (ACT == PIGAN_ACT_RELU) {
    return a > 0.0f ? 1.0f : 0.0f;
  } else if constexpr (ACT == PIGAN_ACT_GELU) {
    if constexpr (X64) {
      double g;
      const double p = normal_cdf64(a, g);
      return (float)(p + copysignf(size_to(a, 57.0f), a) * (g * 0.3989422804014327));   // 1 / sqrt(2 pi)
    } else {
      float g;
      const float p = normal_cdf(a, g);
      return p + __builtin_amdgcn_fmed3f(a, -64.0f, 64.0f) * g * 0.3989422804014327f;
    }
  } else if constexpr (ACT == PIGAN_ACT_SILU) {
    if constexpr (X64) {
      double c;
      const double s = logistic64(a, c);
      return (float)(s + copysignf(size_to(a, 1000.0f), a) * (s * c));
    } else {
      float c;
      const float s = logistic(a, c);
      return s + __builtin_amdgcn_fmed3f(a, -200.0f, 200.0f) * s * c;
    }
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
