// sf_route.cu - the router of a layer of experts and its gradient
// (sf_route_experts, sf_route_experts_grad).
//
// A warp a token, NV consecutive experts a lane.  What it costs is
// instructions, not memory: 256 values a token are scored, and the k largest
// found, in the time that memory takes for a kilobyte.
#include <algorithm>

#include "sf_float.cuh"
#include "sf_launch.h"

namespace sf {
namespace {

constexpr int kWarps = 8, kThreads = kWarps * 32;

__device__ __forceinline__ float redux_max(float v) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}

__device__ __forceinline__ float sigmoid(float z) { return 1.f / (1.f + expf(-z)); }
// exp(z - m) of an expert that is available, m >= z; NaN stays NaN.
__device__ __forceinline__ float softmax_term(float z, float m) { return z == neg_inf() ? 0.f : expf(z - m); }

// A lane's NV values of a row, from e0 = lane * NV; `fill` past the row's end.
// `packs`: whole 16-byte packs (NV values are some, they lie on their boundary
// and no lane's are cut off by the end).
template <typename T, int NV>
__device__ __forceinline__ void load_lane(const T* row, int e0, int E, bool packs, float fill, float (&z)[NV]) {
  constexpr int N = Pack<T>::kN;
  if constexpr (NV % N == 0) {
    if (packs) {
      if (e0 < E) {
#pragma unroll
        for (int p = 0; p < NV / N; ++p) {
          float f[N];
          unpack(load16(row + e0 + p * N), f, T());
#pragma unroll
          for (int q = 0; q < N; ++q) z[p * N + q] = f[q];
        }
      } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) z[i] = fill;
      }
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) z[i] = e0 + i < E ? to_f32(row[e0 + i]) : fill;
}

// Whether rows of E values, ld apart, can be taken in packs by lanes of NV values.
template <typename T, int NV>
bool in_packs(const void* p, int64_t E, int64_t ld) {
  return NV % Pack<T>::kN == 0 && E % NV == 0 && reinterpret_cast<uintptr_t>(p) % 16 == 0 &&
         ld % Pack<T>::kN == 0;
}

// The two largest of a group's choice values.
struct Top2 {
  float a = neg_inf(), b = neg_inf();
  __device__ __forceinline__ void add(float v) {
    b = fmaxf(b, fminf(a, v));
    a = fmaxf(a, v);
  }
  __device__ __forceinline__ void merge(float oa, float ob) {
    b = fmaxf(fminf(a, oa), fmaxf(b, ob));
    a = fmaxf(a, oa);
  }
};

// The k largest: a bound first, the k-th largest of the lanes' own maxima, which
// at least k values reach; the few that do (k to k + 3 of 256, as a rule) go one
// to a lane, which counts those before it.  That is 160 instructions where
// taking them one by one from all lanes' values, each time with a new maximum
// a lane, is 230; more than 32 (equal values) are taken that way.

template <typename T, int NV, bool kSigmoid>
__global__ void __launch_bounds__(kThreads) route_kernel(const RouteJob j, const bool packs) {
  extern __shared__ int32_t hist[];  // loads [E]; with groups, choice values [kWarps][E]
  __shared__ float2 all_keys[kWarps][32];
  __shared__ float all_logits[kWarps][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int E = static_cast<int>(j.E), k = j.cfg.k, e0 = lane * NV;
  const int G = j.cfg.groups, per = E / G;
  const bool grouped = j.cfg.top_groups < G;
  // groups of a power of two of lanes: by shuffles; others through shared memory
  const int group_lanes = per % NV == 0 ? per / NV : 0;
  const bool shuffles = group_lanes > 0 && (group_lanes & (group_lanes - 1)) == 0;
  float* values = reinterpret_cast<float*>(hist + E) + warp * E;
  float2* keys = all_keys[warp];
  float* logits = all_logits[warp];
  for (int e = threadIdx.x; e < E; e += kThreads) hist[e] = 0;
  float bias[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) bias[i] = j.bias != nullptr && e0 + i < E ? j.bias[e0 + i] : 0.f;
  __syncthreads();
  uint32_t bits = 0;
  for (int64_t t = blockIdx.x * int64_t(kWarps) + warp; t < j.T; t += int64_t(gridDim.x) * kWarps) {
    float z[NV], u[NV];
    load_lane<T, NV>(static_cast<const T*>(j.logits) + t * j.ld, e0, E, packs, neg_inf(), z);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const float v = (kSigmoid ? sigmoid(z[i]) : z[i]) + bias[i];
      const bool faulty = z[i] != neg_inf() && (v != v || (!kSigmoid && z[i] == -neg_inf()));
      if (faulty) {
        bits |= SF_ST_NONFINITE;
        z[i] = neg_inf();
      }
      u[i] = z[i] == neg_inf() ? neg_inf() : v;
    }
    if (grouped) {
      Top2 best;
      float value = neg_inf();  // of this lane's group
      if (shuffles) {
#pragma unroll
        for (int i = 0; i < NV; ++i) best.add(u[i]);
        for (int o = 1; o < group_lanes; o <<= 1)
          best.merge(__shfl_xor_sync(kFull, best.a, o), __shfl_xor_sync(kFull, best.b, o));
      } else {
        __syncwarp();
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if (e0 + i < E) values[e0 + i] = u[i];
        __syncwarp();
        if (lane < G)
          for (int i = 0; i < per; ++i) best.add(values[lane * per + i]);
      }
      value = j.cfg.group_top > 1 && best.b != neg_inf() ? best.a + best.b : best.a;
      // a group is kept if fewer than top_groups come before it
      const int mine = shuffles ? lane / group_lanes : lane, stride = shuffles ? group_lanes : 1;
      int before = 0;
      for (int g = 0; g < G; ++g) {
        const float o = __shfl_sync(kFull, value, g * stride);
        before += o > value || (o == value && g < mine);
      }
      const bool keep = before < j.cfg.top_groups;
      if (shuffles) {
#pragma unroll
        for (int i = 0; i < NV; ++i) u[i] = keep ? u[i] : neg_inf();
      } else {
        const uint32_t kept = __ballot_sync(kFull, lane < G && keep);
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if (e0 + i < E && !((kept >> ((e0 + i) / per)) & 1u)) u[i] = neg_inf();
      }
    }
    // the bound
    float top = u[0];
#pragma unroll
    for (int i = 1; i < NV; ++i) top = fmaxf(top, u[i]);
    float bound = neg_inf();
    for (int c = 0; c < k; ++c) {
      bound = redux_max(top);
      if (bound == neg_inf()) break;
      if (lane == __ffs(static_cast<int>(__ballot_sync(kFull, top == bound))) - 1) top = neg_inf();
    }
    // the values that reach it
    int n = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const bool in = u[i] >= bound && u[i] != neg_inf();
      const uint32_t b = __ballot_sync(kFull, in);
      const int at = n + __popc(b & ((1u << lane) - 1u));
      if (in && at < 32) {
        keys[at] = make_float2(u[i], __int_as_float(e0 + i));
        logits[at] = z[i];
      }
      n += __popc(b);
    }
    int e = -1, rank = 32;
    float zc = neg_inf();
    if (n <= 32) {
      __syncwarp();
      if (lane < n) {
        const float2 own = keys[lane];
        e = __float_as_int(own.y);
        zc = logits[lane];
        rank = 0;
        for (int i = 0; i < n; ++i) {
          const float2 o = keys[i];
          rank += o.x > own.x || (o.x == own.x && __float_as_int(o.y) < e);
        }
      }
      __syncwarp();
    } else {
      for (int c = 0; c < k; ++c) {
        float m = u[0];
#pragma unroll
        for (int i = 1; i < NV; ++i) m = fmaxf(m, u[i]);
        const float best = redux_max(m);
        if (best == neg_inf()) break;
        const int owner = __ffs(static_cast<int>(__ballot_sync(kFull, m == best))) - 1;
        int at = e0;
        float za = 0.f;
        bool found = lane != owner;
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if (!found && u[i] == best) {
            found = true;
            at = e0 + i;
            za = z[i];
            u[i] = neg_inf();
          }
        at = __shfl_sync(kFull, at, owner);
        za = __shfl_sync(kFull, za, owner);
        if (lane == c) {
          e = at;
          zc = za;
          rank = c;
        }
      }
    }
    const bool chosen = rank < k;
    // weights
    float w = 0.f;
    if (kSigmoid) {
      w = chosen ? sigmoid(zc) : 0.f;
    } else if (j.cfg.renorm) {
      const float m = redux_max(chosen ? zc : neg_inf());
      w = chosen ? expf(zc - m) : 0.f;
    } else {
      float m = z[0], s = 0.f;
#pragma unroll
      for (int i = 1; i < NV; ++i) m = fmaxf(m, z[i]);
      m = redux_max(m);
#pragma unroll
      for (int i = 0; i < NV; ++i) s += softmax_term(z[i], m);
      s = warp_sum(s);
      w = chosen ? expf(zc - m) / s : 0.f;
    }
    if (j.cfg.renorm) {
      const float s = warp_sum(w);
      w = s > 0.f ? w / s : 0.f;
    }
    if (chosen) {
      j.index[t * k + rank] = e;
      j.weight[t * k + rank] = w * j.cfg.scale;
      atomicAdd(hist + e, 1);
    }
    const int found = __popc(__ballot_sync(kFull, chosen));
    if (lane >= found && lane < k) {  // fewer experts than k
      j.index[t * k + lane] = -1;
      j.weight[t * k + lane] = 0.f;
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
  return launch_after(kern, grid, dim3(kThreads), smem, stream, after_clear, j, in_packs<T, NV>(j.logits, j.E, j.ld));
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

// Gradient: the chosen experts' lanes put their own values (or, where all
// experts have a gradient, their upstream gradients) into a row of zeros in
// shared memory, from which every lane takes its NV.
template <typename T, int NV>
__global__ void __launch_bounds__(kThreads) route_grad_kernel(const RouteGradJob j, const bool packs) {
  constexpr int N = Pack<T>::kN;
  extern __shared__ __align__(16) float rows[];  // [kWarps][32 * NV]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int E = static_cast<int>(j.E), k = j.cfg.k, e0 = lane * NV;
  float* d = rows + warp * (32 * NV);
  const bool sigmoids = j.cfg.score == SF_SCORE_SIGMOID, dense = !sigmoids && !j.cfg.renorm;
  uint32_t bits = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) d[i * 32 + lane] = 0.f;
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
    float g = 0.f, all[NV], s = 0.f, inner = 0.f;
    if (sigmoids) {
      const float p = e >= 0 ? sigmoid(z) : 0.f;
      const float slope = e >= 0 ? p * (1.f / (1.f + expf(z))) : 0.f;
      if (j.cfg.renorm) {
        s = warp_sum(p);
        inner = warp_sum(p * dw);
        g = s > 0.f ? slope / s * (dw - inner / s) : 0.f;
      } else {
        g = slope * dw;
      }
    } else {
      float m = z;
      if (dense) {
        load_lane<T, NV>(row, e0, E, packs, neg_inf(), all);
#pragma unroll
        for (int i = 0; i < NV; ++i) m = fmaxf(m, all[i]);
      }
      m = warp_max(m);
      const float q = softmax_term(z, m);
      s = q;
      if (dense) {
        s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          all[i] = softmax_term(all[i], m);
          s += all[i];
        }
      }
      s = warp_sum(s);
      inner = warp_sum(q * dw);
      if (!finite(s)) bits |= SF_ST_NONFINITE;
      s = finite(s) && s > 0.f ? 1.f / s : 0.f;  // no gradient without a distribution
      inner *= s;
      g = dense ? dw : s > 0.f ? q * s * (dw - inner) : 0.f;
    }
    __syncwarp();  // the row is zeros
    if (e >= 0) d[e] = g;
    __syncwarp();
    float v[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      v[i] = d[e0 + i];
      if (dense) v[i] = s > 0.f ? all[i] * s * (v[i] - inner) : 0.f;
      v[i] *= j.cfg.scale;
    }
    __syncwarp();
    if (e >= 0) d[e] = 0.f;
    T* out = static_cast<T*>(j.dlogits) + t * j.ldd;
    if constexpr (NV % N == 0) {
      if (packs) {
        if (e0 < E) {
#pragma unroll
          for (int p = 0; p < NV / N; ++p) {
            float f[N];
#pragma unroll
            for (int q = 0; q < N; ++q) f[q] = v[p * N + q];
            store16(out + e0 + p * N, pack(f, T()));
          }
        }
        continue;
      }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (e0 + i < E) out[e0 + i] = from_f32<T>(v[i]);
  }
  report(j.status, bits);
}

template <typename T, int NV>
cudaError_t launch_grad_nv(const RouteGradJob& j, cudaStream_t stream) {
  const int64_t ctas = (j.T + kWarps - 1) / kWarps;
  const int grid = static_cast<int>(std::min<int64_t>(ctas, int64_t(sm_count()) * 8));
  const bool packs = in_packs<T, NV>(j.logits, j.E, j.ld) && in_packs<T, NV>(j.dlogits, j.E, j.ldd);
  count_launch();
  route_grad_kernel<T, NV><<<grid, kThreads, size_t(kWarps) * 32 * NV * 4, stream>>>(j, packs);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_grad_t(const RouteGradJob& j, cudaStream_t stream) {
  const int64_t nv = (j.E + 31) / 32;
  if (nv <= 1) return launch_grad_nv<T, 1>(j, stream);
  if (nv <= 2) return launch_grad_nv<T, 2>(j, stream);
  if (nv <= 4) return launch_grad_nv<T, 4>(j, stream);
  if (nv <= 8) return launch_grad_nv<T, 8>(j, stream);
  if (nv <= 16) return launch_grad_nv<T, 16>(j, stream);
  return launch_grad_nv<T, 32>(j, stream);
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
