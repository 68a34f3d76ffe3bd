// sf_policy_loss.cu - the clipped policy loss with a KL term, from logits, with
// its gradient (sf_policy_loss).
//
// Per row the softmax statistics m = max x_j and S = sum exp(x_j - m), x = tau z,
// give lp = x_y - m - log S; loss and derivative c follow from a few scalars of
// the row, and the gradient is g w tau c ([j = y] - exp(x_j - m) / S).  One
// exponential an element for the statistics and one for the gradient, against
// an element's bytes in and out: a streaming kernel, bound by memory.
#include <algorithm>

#include "sf_float.cuh"
#include "sf_launch.h"

namespace sf {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// What a row's scalars say: the gradient's factor and the terms of the sums.
struct RowLoss {
  float logp = 0.f, loss = 0.f, factor = 0.f;
  float4 terms = {0.f, 0.f, 0.f, 0.f};  // weight times loss, pg, kl, clipped
  uint32_t bits = 0;
};

// zy: the chosen token's logit, m: the largest logit, S: sum exp(tau (z - m)).
__device__ __forceinline__ RowLoss row_loss(const PolicyJob& j, int64_t row, float w, float zy, float m, float S) {
  RowLoss r;
  const float A = j.advantage[row];
  const float lp = (zy - m) * j.cfg.inv_temperature - logf(S);
  const float ratio = expf(lp - j.old_logp[row]);
  const float held = fminf(fmaxf(ratio, 1.f - j.cfg.clip_low), 1.f + j.cfg.clip_high);
  const bool clipped = held * A < ratio * A;
  const float pg = -fminf(ratio * A, held * A);
  float kl = 0.f, loss = pg, c = clipped ? 0.f : -ratio * A;
  if (j.ref_logp != nullptr) {
    const float u = j.ref_logp[row] - lp;
    const float em = expm1f(u);
    kl = em - u;
    if (j.cfg.kl_coef != 0.f) {
      loss += j.cfg.kl_coef * kl;
      c -= j.cfg.kl_coef * em;
    }
  }
  const float g = j.grad_out != nullptr ? *j.grad_out : 1.f;
  const float f = c * w * g * j.cfg.inv_temperature;
  // S >= 1 where the logits are sound; a NaN logit makes S NaN, a +inf one m
  if (!finite(m) || !finite(S) || !finite(loss) || !finite(w * loss) || !finite(w * kl) || !finite(f) || ratio != ratio) {
    r.bits = SF_ST_NONFINITE;
    return r;
  }
  r.logp = lp;
  r.loss = loss;
  r.factor = f;
  r.terms = make_float4(w * loss, w * pg, w * kl, clipped ? w : 0.f);
  return r;
}

__device__ __forceinline__ void write_row(const PolicyJob& j, int64_t row, const RowLoss& r) {
  if (j.logp != nullptr) j.logp[row] = r.logp;
  if (j.token_loss != nullptr) j.token_loss[row] = r.loss;
  j.terms[row] = r.terms;
  report(j.status, r.bits);
}

__device__ __forceinline__ float row_weight(const PolicyJob& j, int64_t row) {
  return j.weight != nullptr ? j.weight[row] : j.mean;
}

template <typename T, int kThreads>
__device__ void zero_row(T* d, int64_t V) {
  const int head = head_of(d, V);
  const int64_t nv = (V - head) / Pack<T>::kN;
  for (int64_t i = threadIdx.x; i < head; i += kThreads) d[i] = from_f32<T>(0.f);
  for (int64_t i = threadIdx.x; i < nv; i += kThreads) store16(d + head + i * Pack<T>::kN, make_uint4(0, 0, 0, 0));
  for (int64_t i = head + nv * Pack<T>::kN + threadIdx.x; i < V; i += kThreads) d[i] = from_f32<T>(0.f);
}

// Running maximum and sum of one thread: s = sum exp(tau (z - m)).
struct MaxSum {
  float m = neg_inf(), s = 0.f;
  __device__ __forceinline__ void grow(float to, float scale) {
    if (to > m) {
      s *= exp2_fast((m - to) * scale);  // m = -inf: 0
      m = to;
    }
  }
  __device__ __forceinline__ void add(float z, float scale) {
    grow(z, scale);
    if (z != neg_inf()) s += exp2_fast((z - m) * scale);
  }
  __device__ __forceinline__ void merge(float om, float os, float scale) {
    grow(om, scale);
    s += om == neg_inf() ? os : os * exp2_fast((om - m) * scale);  // without a maximum os is 0, or NaN and stays
  }
};

// A CTA a row, two passes over it: statistics, then the gradient.  The second
// pass finds the row in L2 (152 SMs hold some 600 rows in flight).
constexpr int kStreamThreads = 512;

template <typename T, bool kGrad>
__global__ void __launch_bounds__(kStreamThreads) policy_stream_kernel(const PolicyJob j) {
  constexpr int N = Pack<T>::kN;
  __shared__ float2 buf[2][kStreamThreads / 32];
  const float scale = j.cfg.inv_temperature * kLog2e;
  const int tid = threadIdx.x;
  int par = 0;
  for (int64_t row = blockIdx.x; row < j.N; row += gridDim.x) {
    const float w = row_weight(j, row);
    const int64_t y = w != 0.f ? j.target[row] : 0;
    T* d = kGrad ? static_cast<T*>(j.dlogits) + row * j.ldd : nullptr;
    if (w == 0.f || y < 0 || y >= j.V) {
      RowLoss r;
      if (w != 0.f) r.bits = SF_ST_INDEX;
      if (tid == 0) write_row(j, row, r);
      if (kGrad) zero_row<T, kStreamThreads>(d, j.V);
      continue;
    }
    const T* z = static_cast<const T*>(j.logits) + row * j.ld;
    const float zy = to_f32(z[y]);
    const int head = head_of(z, j.V);
    const int64_t nv = (j.V - head) / N;
    const T* body = z + head;
    const int tail = static_cast<int>(j.V - head - nv * N);
    MaxSum a;
    if (tid < head) a.add(to_f32(z[tid]), scale);
    if (tid < tail) a.add(to_f32(body[nv * N + tid]), scale);
    for (int64_t i = tid; i < nv; i += kStreamThreads) {
      float f[N];
      unpack(load16(body + i * N), f, T());
      float m = f[0];
#pragma unroll
      for (int q = 1; q < N; ++q) m = fmaxf(m, f[q]);
      a.grow(m, scale);
      if (a.m != neg_inf()) {
#pragma unroll
        for (int q = 0; q < N; ++q) a.s += exp2_fast((f[q] - a.m) * scale);
      } else {
#pragma unroll
        for (int q = 0; q < N; ++q) a.s += f[q] == neg_inf() ? 0.f : f[q];  // NaN stays NaN
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
      a.merge(__shfl_xor_sync(kFull, a.m, o), __shfl_xor_sync(kFull, a.s, o), scale);
    if ((tid & 31) == 0) buf[par][tid >> 5] = make_float2(a.m, a.s);
    __syncthreads();
    MaxSum b;
#pragma unroll
    for (int q = 0; q < kStreamThreads / 32; ++q) b.merge(buf[par][q].x, buf[par][q].y, scale);
    par ^= 1;
    const RowLoss r = row_loss(j, row, w, zy, b.m, b.s);
    if (tid == 0) write_row(j, row, r);
    if (!kGrad) continue;
    if (r.bits != 0) {
      zero_row<T, kStreamThreads>(d, j.V);
      continue;
    }
    const float p = -r.factor / b.s;
    const auto grad = [&](float v, int64_t at) {
      return exp2_fast((v - b.m) * scale) * p + (at == y ? r.factor : 0.f);
    };
    if (tid < head) d[tid] = from_f32<T>(grad(to_f32(z[tid]), tid));
    if (tid < tail) d[head + nv * N + tid] = from_f32<T>(grad(to_f32(body[nv * N + tid]), head + nv * N + tid));
    const bool even = (reinterpret_cast<uintptr_t>(d + head) & 15u) == 0;  // both rows at the same offset
    for (int64_t i = tid; i < nv; i += kStreamThreads) {
      float f[N];
      unpack(load16(body + i * N), f, T());
      const int64_t at = head + i * N;
#pragma unroll
      for (int q = 0; q < N; ++q) f[q] = grad(f[q], at + q);
      if (even) {
        store16(d + at, pack(f, T()));
      } else {
#pragma unroll
        for (int q = 0; q < N; ++q) d[at + q] = from_f32<T>(f[q]);
      }
    }
  }
}

// The sums over the rows, added in 64 bits in a fixed order: rows of a block of
// kSumRows by one CTA each, then (where there are several) their sums by one.
constexpr int kSumThreads = 512, kSumRows = 8192;

__device__ void add_terms(double (&a)[4], const float4& t) {
  a[0] += t.x;
  a[1] += t.y;
  a[2] += t.z;
  a[3] += t.w;
}

__global__ void __launch_bounds__(kSumThreads) policy_sum_kernel(const float4* terms, int64_t N, double* part,
                                                                 float* stats) {
  __shared__ double buf[4][kSumThreads / 32];
  griddep_wait();
  double a[4] = {0., 0., 0., 0.};
  const int64_t from = int64_t(blockIdx.x) * kSumRows, to = from + kSumRows < N ? from + kSumRows : N;
  for (int64_t i = from + threadIdx.x; i < to; i += kSumThreads) add_terms(a, terms[i]);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const double s = block_sum<kSumThreads>(a[q], buf[q]);
    if (threadIdx.x == 0) {
      if (part != nullptr)
        part[int64_t(blockIdx.x) * 4 + q] = s;
      else
        stats[q] = static_cast<float>(s);
    }
  }
}

__global__ void __launch_bounds__(128) policy_sum_parts_kernel(const double* part, int64_t blocks, float* stats) {
  griddep_wait();
  const int q = threadIdx.x >> 5;
  double s = 0.;
  for (int64_t i = threadIdx.x & 31; i < blocks; i += 32) s += part[i * 4 + q];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(kFull, s, o);
  if ((threadIdx.x & 31) == 0) stats[q] = static_cast<float>(s);
}

template <typename T>
cudaError_t launch_rows(const PolicyJob& j, cudaStream_t stream) {
  const int grid = static_cast<int>(std::min<int64_t>(j.N, int64_t(sm_count()) * 4));
  count_launch();
  if (j.dlogits != nullptr)
    policy_stream_kernel<T, true><<<grid, kStreamThreads, 0, stream>>>(j);
  else
    policy_stream_kernel<T, false><<<grid, kStreamThreads, 0, stream>>>(j);
  return cudaGetLastError();
}

int64_t sum_blocks(int64_t N) { return (N + kSumRows - 1) / kSumRows; }

}  // namespace

size_t policy_loss_workspace(int64_t N) {
  return size_t(N) * sizeof(float4) + (sum_blocks(N) > 1 ? size_t(sum_blocks(N)) * 4 * sizeof(double) : 0);
}

cudaError_t launch_policy_loss(PolicyJob j, void* workspace, cudaStream_t stream) {
  j.terms = static_cast<float4*>(workspace);
  j.mean = 1.f / static_cast<float>(j.N);
  const cudaError_t e = j.dtype == SF_F32    ? launch_rows<float>(j, stream)
                        : j.dtype == SF_BF16 ? launch_rows<__nv_bfloat16>(j, stream)
                                             : launch_rows<__half>(j, stream);
  if (e != cudaSuccess) return e;
  const int64_t blocks = sum_blocks(j.N);
  double* part = blocks > 1 ? reinterpret_cast<double*>(j.terms + j.N) : nullptr;
  count_launch();
  const cudaError_t s = launch_after(policy_sum_kernel, dim3(static_cast<unsigned>(blocks)), dim3(kSumThreads), 0,
                                     stream, true, j.terms, j.N, part, j.stats);
  if (s != cudaSuccess || part == nullptr) return s;
  count_launch();
  return launch_after(policy_sum_parts_kernel, dim3(1), dim3(128), 0, stream, true, part, blocks, j.stats);
}

}  // namespace sf
