// sf_route.cu - the router of a layer of experts and its gradient
// (sf_route_experts, sf_route_experts_grad).
//
// Forward: a warp a token, NV consecutive experts a lane in registers.  The
// choice values are made orderable as unsigned keys (0: not available), so a
// maximum is one 32-bit warp reduction; the k chosen are taken one by one, the
// lowest lane and expert first among equals.  Loads are counted in shared
// memory and added to the totals once a CTA.
#include <algorithm>

#include "sf_float.cuh"
#include "sf_launch.h"

namespace sf {
namespace {

constexpr int kWarps = 8, kThreads = kWarps * 32;

// Order-preserving key of a choice value; 0 for NaN and -inf (not available),
// one key for both zeros.
__device__ __forceinline__ uint32_t choice_key(float u) {
  const uint32_t b = __float_as_uint(u + 0.f);
  const uint32_t k = (b & 0x80000000u) ? ~b : b | 0x80000000u;
  return u > neg_inf() ? k : 0u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k);
}

// exp(z - m) of an expert that is available, m >= z; NaN stays NaN.
__device__ __forceinline__ float softmax_term(float z, float m) { return z == neg_inf() ? 0.f : expf(z - m); }

// Lane holds experts [lane * NV, lane * NV + NV); those past E are not available.
template <typename T, int NV, bool kSigmoid>
__global__ void __launch_bounds__(kThreads) route_kernel(const RouteJob j) {
  extern __shared__ int32_t shared[];  // loads [E]; with groups, keys [kWarps][E]
  int32_t* hist = shared;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int E = static_cast<int>(j.E), k = j.cfg.k, e0 = lane * NV;
  const bool grouped = j.cfg.top_groups < j.cfg.groups;
  uint32_t* keys = reinterpret_cast<uint32_t*>(shared + E) + warp * E;
  for (int e = threadIdx.x; e < E; e += kThreads) hist[e] = 0;
  __syncthreads();
  uint32_t bits = 0;
  for (int64_t t = blockIdx.x * int64_t(kWarps) + warp; t < j.T; t += int64_t(gridDim.x) * kWarps) {
    const T* row = static_cast<const T*>(j.logits) + t * j.ld;
    float z[NV];
    uint32_t key[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) z[i] = e0 + i < E ? to_f32(row[e0 + i]) : neg_inf();
    float zmax = neg_inf();
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const float b = j.bias != nullptr && e0 + i < E ? j.bias[e0 + i] : 0.f;
      float u = kSigmoid ? 1.f / (1.f + expf(-z[i])) : z[i];
      u = u + b;
      if (z[i] == neg_inf()) {
        u = neg_inf();
      } else if (u != u || (!kSigmoid && z[i] == -neg_inf())) {
        bits |= SF_ST_NONFINITE;
        u = z[i] = neg_inf();
      }
      key[i] = choice_key(u);
      zmax = fmaxf(zmax, z[i]);
    }
    if (grouped) {
      const int G = j.cfg.groups, per = E / G;
      __syncwarp();
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (e0 + i < E) keys[e0 + i] = key[i];
      __syncwarp();
      uint32_t gk = 0;  // this lane's group
      if (lane < G) {
        uint32_t a = 0, b = 0;
        for (int i = 0; i < per; ++i) {
          const uint32_t v = keys[lane * per + i];
          b = max(b, min(a, v));
          a = max(a, v);
        }
        if (a != 0) gk = choice_key(j.cfg.group_top > 1 && b != 0 ? key_value(a) + key_value(b) : key_value(a));
      }
      // a group is kept if fewer than top_groups others come before it
      int before = 0;
      for (int g = 0; g < G; ++g) {
        const uint32_t o = __shfl_sync(kFull, gk, g);
        before += o > gk || (o == gk && g < lane);
      }
      const uint32_t kept = __ballot_sync(kFull, lane < G && before < j.cfg.top_groups);
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (e0 + i < E && !((kept >> ((e0 + i) / per)) & 1u)) key[i] = 0;
    }
    // the chosen, one by one; lane c keeps the c-th
    int mine = -1;
    float mine_z = 0.f;
    for (int c = 0; c < k; ++c) {
      uint32_t best = 0;
      int at = 0;
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (key[i] > best) {
          best = key[i];
          at = i;
        }
      const uint32_t top = __reduce_max_sync(kFull, best);
      if (top == 0) break;
      const int owner = __ffs(__ballot_sync(kFull, best == top)) - 1;
      float zc = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (i == at) {
          zc = z[i];
          if (lane == owner) key[i] = 0;
        }
      const int e = __shfl_sync(kFull, e0 + at, owner);
      zc = __shfl_sync(kFull, zc, owner);
      if (lane == c) {
        mine = e;
        mine_z = zc;
      }
    }
    // weights
    float w = 0.f;
    if (kSigmoid) {
      w = mine >= 0 ? 1.f / (1.f + expf(-mine_z)) : 0.f;
    } else {
      float m = zmax;
      if (j.cfg.renorm) m = mine >= 0 ? mine_z : neg_inf();
      m = warp_max(m);
      w = mine >= 0 ? expf(mine_z - m) : 0.f;
      if (!j.cfg.renorm) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) s += softmax_term(z[i], m);
        w = w / warp_sum(s);
      }
    }
    if (j.cfg.renorm) {
      const float s = warp_sum(w);
      w = s > 0.f ? w / s : 0.f;
    }
    if (lane < k) {
      j.index[t * k + lane] = mine;
      j.weight[t * k + lane] = mine >= 0 ? w * j.cfg.scale : 0.f;
      if (mine >= 0) atomicAdd(hist + mine, 1);
    }
  }
  report(j.status, bits);
  if (j.load == nullptr) return;
  __syncthreads();
  if (j.only_cta) {  // the totals are this CTA's counts
    for (int e = threadIdx.x; e < E; e += kThreads) j.load[e] = hist[e];
    return;
  }
  griddep_wait();  // the totals have been cleared
  for (int e = threadIdx.x; e < E; e += kThreads)
    if (hist[e] != 0) atomicAdd(j.load + e, hist[e]);
}

template <typename T, int NV>
cudaError_t launch_route_nv(const RouteJob& j, bool after_clear, cudaStream_t stream) {
  const bool grouped = j.cfg.top_groups < j.cfg.groups;
  const size_t smem = size_t(j.E) * 4 * (grouped ? 1 + kWarps : 1);
  const int64_t ctas = (j.T + kWarps - 1) / kWarps;
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>(ctas, int64_t(sm_count()) * 8)));
  count_launch();
  const auto kern = j.cfg.score == SF_SCORE_SIGMOID ? route_kernel<T, NV, true> : route_kernel<T, NV, false>;
  return launch_after(kern, grid, dim3(kThreads), smem, stream, after_clear, j);
}

template <typename T>
cudaError_t launch_route_t(const RouteJob& j, bool after_clear, cudaStream_t stream) {
  const int64_t nv = (j.E + 31) / 32;
  if (nv <= 1) return launch_route_nv<T, 1>(j, after_clear, stream);
  if (nv <= 2) return launch_route_nv<T, 2>(j, after_clear, stream);
  if (nv <= 4) return launch_route_nv<T, 4>(j, after_clear, stream);
  if (nv <= 8) return launch_route_nv<T, 8>(j, after_clear, stream);
  if (nv <= 16) return launch_route_nv<T, 16>(j, after_clear, stream);
  return launch_route_nv<T, 32>(j, after_clear, stream);
}

// Gradient: a warp a token; the row is put together in shared memory.
template <typename T>
__global__ void __launch_bounds__(kThreads) route_grad_kernel(const RouteGradJob j) {
  extern __shared__ float rows[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int E = static_cast<int>(j.E), k = j.cfg.k;
  float* d = rows + warp * E;
  const bool sigmoid = j.cfg.score == SF_SCORE_SIGMOID, dense = !sigmoid && !j.cfg.renorm;
  uint32_t bits = 0;
  for (int64_t t = blockIdx.x * int64_t(kWarps) + warp; t < j.T; t += int64_t(gridDim.x) * kWarps) {
    const T* row = static_cast<const T*>(j.logits) + t * j.ld;
    int e = -1;
    float dw = 0.f, z = neg_inf();
    if (lane < k) {
      e = j.index[t * k + lane];
      if (e < -1 || e >= E) {
        bits |= SF_ST_INDEX;
        e = -1;
      }
      if (e >= 0) {
        dw = j.dweight[t * k + lane];
        z = to_f32(row[e]);
      }
    }
    float m = z, g = 0.f, s = 0.f, inner = 0.f;
    if (sigmoid) {
      const float p = e >= 0 ? 1.f / (1.f + expf(-z)) : 0.f;
      const float slope = e >= 0 ? p * (1.f / (1.f + expf(z))) : 0.f;
      if (j.cfg.renorm) {
        s = warp_sum(p);
        inner = warp_sum(p * dw);
        g = s > 0.f ? slope / s * (dw - inner / s) : 0.f;
      } else {
        g = slope * dw;
      }
    } else {
      if (dense)
        for (int i = lane; i < E; i += 32) m = fmaxf(m, to_f32(row[i]));
      m = warp_max(m);
      const float q = softmax_term(z, m);
      s = q;
      if (dense) {
        s = 0.f;
        for (int i = lane; i < E; i += 32) s += softmax_term(to_f32(row[i]), m);
      }
      s = warp_sum(s);
      inner = warp_sum(q * dw);
      if (!finite(s)) bits |= SF_ST_NONFINITE;
      s = finite(s) && s > 0.f ? 1.f / s : 0.f;  // no gradient without a distribution
      inner *= s;
      g = s > 0.f ? q * s * (dw - inner) : 0.f;
    }
    __syncwarp();
    for (int i = lane; i < E; i += 32)
      d[i] = dense && s > 0.f ? -softmax_term(to_f32(row[i]), m) * s * inner : 0.f;
    __syncwarp();
    if (e >= 0) d[e] = g;
    __syncwarp();
    T* out = static_cast<T*>(j.dlogits) + t * j.ldd;
    for (int i = lane; i < E; i += 32) out[i] = from_f32<T>(d[i] * j.cfg.scale);
  }
  report(j.status, bits);
}

template <typename T>
cudaError_t launch_grad_t(const RouteGradJob& j, cudaStream_t stream) {
  const int64_t ctas = (j.T + kWarps - 1) / kWarps;
  const int grid = static_cast<int>(std::min<int64_t>(ctas, int64_t(sm_count()) * 8));
  count_launch();
  route_grad_kernel<T><<<grid, kThreads, size_t(j.E) * 4 * kWarps, stream>>>(j);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_route(RouteJob j, bool accumulate, cudaStream_t stream) {
  bool after_clear = false;
  j.only_cta = !accumulate && j.T <= kWarps;
  if (j.load != nullptr && !accumulate && !j.only_cta) {
    ZeroList z;
    z.add(j.load, size_t(j.E) * sizeof(int32_t));
    const cudaError_t e = launch_zero_many(z, stream, &after_clear);
    if (e != cudaSuccess) return e;
  }
  return j.dtype == SF_F32    ? launch_route_t<float>(j, after_clear, stream)
         : j.dtype == SF_BF16 ? launch_route_t<__nv_bfloat16>(j, after_clear, stream)
                              : launch_route_t<__half>(j, after_clear, stream);
}

cudaError_t launch_route_grad(const RouteGradJob& j, cudaStream_t stream) {
  return j.dtype == SF_F32    ? launch_grad_t<float>(j, stream)
         : j.dtype == SF_BF16 ? launch_grad_t<__nv_bfloat16>(j, stream)
                              : launch_grad_t<__half>(j, stream);
}

}  // namespace sf
