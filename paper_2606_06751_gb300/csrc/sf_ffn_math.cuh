// sf_ffn_math.cuh - the activations of the gated feed-forward product and
// their derivatives, in 32 bits.
#pragma once

#include "sf_float.cuh"

namespace sf {

// Results that are rounded to 16 bits take the hardware's exponential and
// quotient.  The exponential's error grows with its argument x, 2 + 1.2 |x| units of
// 2^-23 of the value: 2^-16 where the result leaves the range of f32, and 2^-18 where a
// product leaves that of f16, against a rounding's 2^-8 and 2^-11.  A quotient by a
// number above 2^126, or by infinity, is 0 there.
template <bool kFast>
__device__ __forceinline__ float exp_of(float x) {
  return kFast ? __expf(x) : expf(x);
}
template <bool kFast>
__device__ __forceinline__ float quotient(float a, float b) {
  return kFast ? __fdividef(a, b) : a / b;
}

// act(g) and, in both(), its derivative.
template <int kAct, bool kFast>
struct Activation;

template <bool kFast>
struct Activation<SF_ACT_SILU, kFast> {
  static __device__ __forceinline__ float part(float g) { return quotient<kFast>(1.f, 1.f + exp_of<kFast>(-g)); }
  static __device__ __forceinline__ float value(float g) { return g * part(g); }
  static __device__ __forceinline__ void both(float g, float& a, float& slope) {
    const float s = part(g);
    a = g * s;
    slope = s * (1.f + g * (1.f - s));
  }
};

template <bool kFast>
struct Activation<SF_ACT_GELU, kFast> {
  // (1 + erf(g / sqrt 2)) / 2 = erfc(x) / 2 with x = -g / sqrt 2, and e = exp(-g^2 / 2).
  // For 16 bits erfc(x) = e t P(t), t = 1 / (1 + 0.375 x), x > 0: P is the polynomial of
  // degree 6 whose largest relative error of exp(x^2) erfc(x) over 0 <= x <= 10.3 is
  // least (linear programming on 1700 points; 6.2e-7).  With the roundings to f32, but
  // for e's own error, within 1.5e-6 of the value for g >= -6, 3e-6 for g >= -10 and
  // 5e-6 down to -13, where e is no longer a normal number.  A polynomial for erf, whose
  // bound is one on the absolute error, is off by a per cent of the value there.
  static __device__ __forceinline__ float part(float g, float& e) {
    e = exp_of<kFast>(-0.5f * g * g);
    if (!kFast) return 0.5f * erfcf(-0.70710678f * g);
    const float t = quotient<true>(1.f, fmaf(0.375f * 0.70710678f, fabsf(g), 1.f));
    float p = fmaf(t, -0.1351857889f, 0.3882570338f);
    p = fmaf(t, p, -0.1300511278f);
    p = fmaf(t, p, 0.2833913173f);
    p = fmaf(t, p, 0.1665358411f);
    p = fmaf(t, p, 0.2157146458f);
    p = fmaf(t, p, 0.2113373632f);
    const float tail = 0.5f * t * p * e;
    return g < 0.f ? tail : 1.f - tail;
  }
  static __device__ __forceinline__ float value(float g) {
    float e;
    return g * part(g, e);
  }
  static __device__ __forceinline__ void both(float g, float& a, float& slope) {
    float e;
    const float c = part(g, e);
    a = g * c;
    slope = c + 0.39894228f * g * e;
  }
};

template <bool kFast>
struct Activation<SF_ACT_GELU_TANH, kFast> {
  static constexpr float kTwo = 1.59576912f;  // 2 sqrt(2 / pi)
  // (1 + tanh y) / 2 = 1 / (1 + exp(-2 y))
  static __device__ __forceinline__ float part(float g) {
    return quotient<kFast>(1.f, 1.f + exp_of<kFast>(-kTwo * (g + 0.044715f * g * g * g)));
  }
  static __device__ __forceinline__ float value(float g) { return g * part(g); }
  static __device__ __forceinline__ void both(float g, float& a, float& slope) {
    const float s = part(g), bend = s * (1.f - s);
    a = g * s;
    slope = bend == 0.f ? s : s + g * bend * kTwo * (1.f + 0.134145f * g * g);  // g^2 may be infinite where bend is 0
  }
};

template <bool kFast>
struct Activation<SF_ACT_RELU, kFast> {
  static __device__ __forceinline__ float value(float g) { return g < 0.f ? 0.f : g; }  // NaN stays
  static __device__ __forceinline__ void both(float g, float& a, float& slope) {
    a = value(g);
    slope = g > 0.f ? 1.f : 0.f;
  }
};

}  // namespace sf
