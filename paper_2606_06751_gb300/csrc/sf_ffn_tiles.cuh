// sf_ffn_tiles.cuh - what the tensor-core kernels of the gated feed-forward
// operators share: the products' layouts and the stores of their tiles.
#pragma once

#include "sf_ffn_math.cuh"
#include "sf_launch.h"
#include "sf_tcgen05.cuh"

namespace sf {
namespace {

enum Product { kForward, kInner, kDx, kDw };

constexpr uint32_t kABytes = 128 * kDepthBytes;

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
// Pairs of SMs; one where there is no device to ask.
inline int64_t sm_pairs() { return sm_count() > 1 ? sm_count() / 2 : 1; }

template <int kProduct>
struct Layout {
  static constexpr bool kGated = kProduct == kForward || kProduct == kInner;
  static constexpr bool kAAlongK = kGated, kBAlongK = kProduct != kDw;
  static constexpr int kRows = kGated ? 64 : 128;  // of what is stored, in a CTA's 128 rows of D
};

// A tile's first m and n and, for dW, whether it is the second matrix's: n tiles
// in groups of 8 m tiles, whose operands stay in L2.
template <int kProduct>
__device__ __forceinline__ void tile_of(int64_t tile, int64_t m_tiles, int64_t n_tiles, int N, int64_t& m, int64_t& n,
                                        bool& second) {
  const int64_t all = n_tiles * (kProduct == kDw ? 2 : 1);
  const int64_t group = tile / (8 * all), first = group * 8;
  const int64_t in_group = m_tiles - first < 8 ? m_tiles - first : 8;
  const int64_t at = tile - group * 8 * all;
  m = (first + at % in_group) * (2 * Layout<kProduct>::kRows);
  n = at / in_group;
  second = kProduct == kDw && n >= n_tiles;
  if (second) n -= n_tiles;
  n *= N;
}

// K values to addresses `ld` apart: those of rows i * step < left.
template <typename T, int K>
__device__ __forceinline__ void store_down(T* p, int64_t ld, int step, int left, const T (&v)[K]) {
  if ((K - 1) * step < left) {
#pragma unroll
    for (int i = 0; i < K; ++i, p += ld) *p = v[i];
  } else {
#pragma unroll
    for (int i = 0; i < K; ++i, p += ld)
      if (i * step < left) *p = v[i];
  }
}

// An f32 as a sum of three bf16: the upper half cut off (no overflow), then the rest's
// nearest and its rest's.  Exact for 2^-109 and more, where all of its bits are bf16 numbers; what is
// below 2^-134 of a smaller one is lost.  An infinity or NaN is the first part alone.
__device__ __forceinline__ void parts_of(float v, __nv_bfloat16 (&p)[3]) {
  const bool real = finite(v);
  const float a = real ? __uint_as_float(__float_as_uint(v) & 0xffff0000u) : v;
  const float r = real ? v - a : 0.f;
  p[0] = __float2bfloat16_rn(a);
  p[1] = __float2bfloat16_rn(r);
  p[2] = __float2bfloat16_rn(r - __bfloat162float(p[1]));
}
// K values to the three parts' matrices [T] rows of ldg, one behind the other.
template <int K>
__device__ __forceinline__ void store_parts(const FfnJob& j, void* to, int64_t t, int step, int64_t f, int left,
                                            const float (&v)[K]) {
  __nv_bfloat16 p[3][K];
#pragma unroll
  for (int i = 0; i < K; ++i) {
    __nv_bfloat16 q[3];
    parts_of(v[i], q);
    p[0][i] = q[0], p[1][i] = q[1], p[2][i] = q[2];
  }
#pragma unroll
  for (int k = 0; k < 3; ++k)
    store_down(static_cast<__nv_bfloat16*>(to) + (k * j.T + t) * j.ldg + f, step * j.ldg, step, left, p[k]);
}

// K values of h, or of dg and du (and h), from their g and u: feature f of tokens
// t, t + step, ... before t + most and T.  One basic block, so that the K chains of exponential and quotient overlap.
template <typename T, int kProduct, int kAct, int K>
__device__ __forceinline__ void store_act(const FfnJob& j, int64_t t, int step, int64_t f, int most, const float (&g)[K],
                                          const float (&u)[K], const T (&dh)[K]) {
  using A = Activation<kAct, sizeof(T) == 2>;
  T v[K], w[K], x[K];
#pragma unroll
  for (int i = 0; i < K; ++i) {
    if constexpr (kProduct == kForward) {
      v[i] = from_f32<T>(A::value(g[i]) * u[i]);
    } else {
      float a, slope;
      A::both(g[i], a, slope);
      v[i] = from_f32<T>(a * u[i]);
      const float d = to_f32(dh[i]);
      w[i] = from_f32<T>(d * u[i] * slope);
      x[i] = from_f32<T>(d * a);
    }
  }
  const int left = static_cast<int>(min(int64_t(most), j.T - t));
  if (kProduct == kForward || j.h != nullptr) store_down(static_cast<T*>(j.h) + t * j.ldh + f, step * j.ldh, step, left, v);
  if constexpr (kProduct == kInner && sizeof(T) == 4) {
    store_parts(j, j.dg, t, step, f, left, w);
    store_parts(j, j.du, t, step, f, left, x);
  } else if constexpr (kProduct == kInner) {
    store_down(static_cast<T*>(j.dg) + t * j.ldg + f, step * j.ldg, step, left, w);
    store_down(static_cast<T*>(j.du) + t * j.ldg + f, step * j.ldg, step, left, x);
  }
}
template <typename T, int kProduct, int K>
__device__ __forceinline__ void store_gated(const FfnJob& j, int64_t t, int step, int64_t f, int most, const float (&g)[K],
                                            const float (&u)[K], const T (&dh)[K]) {
  if (f >= j.F || t >= j.T) return;
  switch (j.act) {
    case SF_ACT_GELU: return store_act<T, kProduct, SF_ACT_GELU>(j, t, step, f, most, g, u, dh);
    case SF_ACT_GELU_TANH: return store_act<T, kProduct, SF_ACT_GELU_TANH>(j, t, step, f, most, g, u, dh);
    case SF_ACT_RELU: return store_act<T, kProduct, SF_ACT_RELU>(j, t, step, f, most, g, u, dh);
    default: return store_act<T, kProduct, SF_ACT_SILU>(j, t, step, f, most, g, u, dh);
  }
}
__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

// Their upstream gradients, as they are: a conversion would wait for them.
template <typename T, int K>
__device__ __forceinline__ void load_dh(const FfnJob& j, int64_t t, int step, int64_t f, T (&dh)[K]) {
  const T* p = static_cast<const T*>(j.dh) + t * j.lddh + f;
  const int left = f < j.F && t < j.T ? static_cast<int>(min(int64_t(K) * step, j.T - t)) : 0;
#pragma unroll
  for (int i = 0; i < K; ++i, p += step * j.lddh) dh[i] = i * step < left ? *p : from_f32<T>(0.f);
}

// K values of dx or of a weight's gradient: column m of rows n, n + step, ... before n + most and the last.
template <typename T, int kProduct, int K>
__device__ __forceinline__ void store_plain(const FfnJob& j, bool second, int64_t m, int64_t n, int step, int most,
                                            const float (&v)[K]) {
  const int64_t rows = kProduct == kDx ? j.T : j.F;
  if (m >= j.H || n >= rows) return;
  const int left = static_cast<int>(min(int64_t(most), rows - n));
  void* w = kProduct == kDx ? j.dx : second ? j.dw_up : j.dw_gate;
  const int64_t ld = kProduct == kDx ? j.lddx : j.lddw;
  if (kProduct == kDw && sizeof(T) == 2 && j.dw_dtype == SF_F32) {
    float* p = static_cast<float*>(w) + n * ld + m;
    float x[K];
#pragma unroll
    for (int i = 0; i < K; ++i) x[i] = v[i];
    if (j.accumulate) {
#pragma unroll
      for (int i = 0; i < K; ++i)
        if (i * step < left) x[i] += p[i * step * ld];
    }
    store_down(p, step * ld, step, left, x);
  } else {
    T* p = static_cast<T*>(w) + n * ld + m;
    T x[K];
#pragma unroll
    for (int i = 0; i < K; ++i) x[i] = from_f32<T>(v[i]);
    if (kProduct == kDw && j.accumulate) {
#pragma unroll
      for (int i = 0; i < K; ++i)
        if (i * step < left) x[i] = from_f32<T>(to_f32(p[i * step * ld]) + v[i]);
    }
    store_down(p, step * ld, step, left, x);
  }
}

}  // namespace
}  // namespace sf
