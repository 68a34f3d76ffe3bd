// sf_grad_norm.cu - the 2-norm over many gradient tensors, each tensor's own,
// and clipping (sf_grad_norm, sf_grad_clip).
//
// The tensors are cut into chunks of one size; a persistent grid takes the
// chunks in turn, writes each one's sum of squares and its CTA's total.  The
// tensors' pointers and sizes travel as a kernel parameter (up to 32 KB), so
// nothing has to be copied to the device or kept there.  A second kernel adds
// the totals (every CTA for itself: they are few) and, for clipping, scales
// the data; chunks are taken in reverse, as the last ones read are those that
// L2 still holds.  All sums go in a fixed order.  Bound by memory: one
// multiply-add and one conversion an element.
#include <algorithm>

#include "sf_float.cuh"
#include "sf_launch.h"

namespace sf {
namespace {

constexpr int kThreads = 256;
constexpr int kPerSm = 4;                          // CTAs of the grid per SM
constexpr int64_t kMinChunk = 4096;                // elements
constexpr int64_t kMaxChunk = int64_t(1) << 20;
constexpr int kUnroll = 8;                         // 16-byte loads in flight a thread
constexpr int kListMax = 1024;                     // tensors of one launch

// Part of the tensors, as a kernel parameter.
template <int M>
struct TensorList {
  const void* in[M];
  void* out[M];
  int64_t n[M];
  int32_t first[M + 1];  // chunks of the tensors before, within this list
  uint8_t type[M];
  int32_t count;
  int64_t chunk;    // elements
  double* partial;  // [first[count]] sums of squares of the chunks
  double* total;    // [gridDim.x] of the CTAs
};

__device__ __forceinline__ int tensor_of(const int32_t* first, int count, int chunk) {
  int lo = 0, hi = count;  // first[lo] <= chunk < first[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= chunk)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

template <typename T>
__device__ __forceinline__ uint32_t magnitude(T v);
template <>
__device__ __forceinline__ uint32_t magnitude<float>(float v) {
  return __float_as_uint(v) & 0x7fffffffu;
}
template <>
__device__ __forceinline__ uint32_t magnitude<__nv_bfloat16>(__nv_bfloat16 v) {
  return __bfloat16_as_ushort(v) & 0x7fffu;
}
template <>
__device__ __forceinline__ uint32_t magnitude<__half>(__half v) {
  return __half_as_ushort(v) & 0x7fffu;
}

// Sum of squares of n values at p, in every thread.  A thread sums what it has
// in flight in 32 bits (at most 16 squares to a sum) and adds that up in 64,
// so that equal values do not round the same way over and over.  Where the
// short sums overflow, or are so small that squares may have been lost below
// 2^-126 (a sum under 2^-80 of values that are not all 0), the chunk is summed
// again in 64 bits throughout.
template <typename T>
__device__ double sum_squares(const T* p, int64_t n, double* buf) {
  constexpr int N = Pack<T>::kN;
  const int head = head_of(p, n);
  const int64_t nv = (n - head) / N;
  const T* body = p + head;
  const int tail = static_cast<int>(n - head - nv * N);
  double sum = 0.;
  uint32_t any = 0;
  if (int(threadIdx.x) < head) {
    const float v = to_f32(p[threadIdx.x]);
    sum += v * v;
    any |= magnitude(p[threadIdx.x]);
  }
  if (int(threadIdx.x) < tail) {
    const float v = to_f32(body[nv * N + threadIdx.x]);
    sum += v * v;
    any |= magnitude(body[nv * N + threadIdx.x]);
  }
  for (int64_t i = threadIdx.x; i < nv; i += int64_t(kThreads) * kUnroll) {
    uint4 u[kUnroll];
#pragma unroll
    for (int q = 0; q < kUnroll; ++q)
      u[q] = i + q * kThreads < nv ? load16(body + (i + q * kThreads) * N) : make_uint4(0, 0, 0, 0);
    float a[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int q = 0; q < kUnroll; ++q) {
      float f[N];
      unpack(u[q], f, T());
#pragma unroll
      for (int e = 0; e < N; ++e) a[e & 3] = fmaf(f[e], f[e], a[e & 3]);
      const uint32_t mask = sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu;
      any |= (u[q].x | u[q].y | u[q].z | u[q].w) & mask;
    }
    sum += (a[0] + a[1]) + (a[2] + a[3]);
  }
  const double s = block_sum<kThreads>(sum, buf);
  const bool doubt = !(s <= 3.0e38) || (s < 8.0e-25 && __syncthreads_or(any != 0));
  __syncthreads();
  if (!doubt) return s;
  double d = 0.;
  for (int64_t i = threadIdx.x; i < n; i += kThreads) {
    const double v = to_f32(p[i]);
    d = fma(v, v, d);
  }
  d = block_sum<kThreads>(d, buf);
  __syncthreads();
  return d;
}

template <int M>
__global__ void __launch_bounds__(kThreads) grad_squares_kernel(const __grid_constant__ TensorList<M> list) {
  __shared__ double buf[kThreads / 32];
  griddep_wait();  // the workspace may still be read by the previous call's kernels
  const int chunks = list.first[list.count];
  double total = 0.;
  for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
    const int t = tensor_of(list.first, list.count, c);
    const int64_t from = int64_t(c - list.first[t]) * list.chunk;
    const int64_t n = list.n[t] - from < list.chunk ? list.n[t] - from : list.chunk;
    double s;
    if (list.type[t] == SF_F32)
      s = sum_squares(static_cast<const float*>(list.in[t]) + from, n, buf);
    else if (list.type[t] == SF_BF16)
      s = sum_squares(static_cast<const __nv_bfloat16*>(list.in[t]) + from, n, buf);
    else
      s = sum_squares(static_cast<const __half*>(list.in[t]) + from, n, buf);
    total += s;
    if (threadIdx.x == 0) list.partial[c] = s;
  }
  if (threadIdx.x == 0) list.total[blockIdx.x] = total;
}

struct NormOut {
  const double* total;
  int64_t totals;
  float *norm, *coef;
  float max_norm, eps;
  uint32_t* status;
};

// The norm over all tensors and the clipping coefficient, in every thread.
__device__ float finish_norm(const NormOut& o, double* buf, float& coef) {
  double s = 0.;
  for (int64_t i = threadIdx.x; i < o.totals; i += kThreads) s += o.total[i];
  s = block_sum<kThreads>(s, buf);
  const float norm = static_cast<float>(sqrt(s));
  coef = finite(norm) ? fminf(1.f, o.max_norm / (norm + o.eps)) : quiet_nan();
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    *o.norm = norm;
    if (o.coef != nullptr) *o.coef = coef;
    if (!finite(norm)) report(o.status, SF_ST_NONFINITE);
  }
  return norm;
}

// Norms of a list's tensors, a warp each, from the chunks' sums.
template <int M>
__device__ void tensor_norms(const TensorList<M>& list, float* out) {
  const int lane = threadIdx.x & 31;
  const int warp = (blockIdx.x * kThreads + threadIdx.x) >> 5, warps = (gridDim.x * kThreads) >> 5;
  for (int t = warp; t < list.count; t += warps) {
    double s = 0.;
    for (int c = list.first[t] + lane; c < list.first[t + 1]; c += 32) s += list.partial[c];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(kFull, s, o);
    if (lane == 0) out[t] = static_cast<float>(sqrt(s));
  }
}

template <int M>
__global__ void __launch_bounds__(kThreads)
    grad_norms_kernel(const __grid_constant__ TensorList<M> list, const NormOut o, float* tensor_norm) {
  __shared__ double buf[kThreads / 32];
  griddep_wait();
  float coef;
  if (blockIdx.x == 0 && o.norm != nullptr) finish_norm(o, buf, coef);
  if (tensor_norm != nullptr) tensor_norms(list, tensor_norm);
}

template <typename T>
__device__ void scale_chunk(const T* p, T* q, int64_t n, float coef) {
  constexpr int N = Pack<T>::kN;
  const int head = head_of(p, n);
  const int64_t nv = (n - head) / N;
  const int tail = static_cast<int>(n - head - nv * N);
  if (int(threadIdx.x) < head) q[threadIdx.x] = from_f32<T>(to_f32(p[threadIdx.x]) * coef);
  if (int(threadIdx.x) < tail) {
    const int64_t at = head + nv * N + threadIdx.x;
    q[at] = from_f32<T>(to_f32(p[at]) * coef);
  }
  const bool even = (reinterpret_cast<uintptr_t>(q + head) & 15u) == 0;  // both runs at the same offset
  for (int64_t i = threadIdx.x; i < nv; i += int64_t(kThreads) * kUnroll) {
    uint4 u[kUnroll];
#pragma unroll
    for (int e = 0; e < kUnroll; ++e)
      if (i + e * kThreads < nv) u[e] = load16(p + head + (i + e * kThreads) * N);
#pragma unroll
    for (int e = 0; e < kUnroll; ++e) {
      if (i + e * kThreads >= nv) break;
      float f[N];
      unpack(u[e], f, T());
#pragma unroll
      for (int k = 0; k < N; ++k) f[k] *= coef;
      const int64_t at = head + (i + e * kThreads) * N;
      if (even) {
        store16(q + at, pack(f, T()));
      } else {
#pragma unroll
        for (int k = 0; k < N; ++k) q[at + k] = from_f32<T>(f[k]);
      }
    }
  }
}

template <int M>
__global__ void __launch_bounds__(kThreads)
    grad_scale_kernel(const __grid_constant__ TensorList<M> list, const NormOut o, float* tensor_norm) {
  __shared__ double buf[kThreads / 32];
  griddep_wait();
  float coef;
  finish_norm(o, buf, coef);
  if (tensor_norm != nullptr) tensor_norms(list, tensor_norm);
  if (!finite(coef)) coef = 1.f;  // passed on unscaled
  for (int c = list.first[list.count] - 1 - int(blockIdx.x); c >= 0; c -= gridDim.x) {
    const int t = tensor_of(list.first, list.count, c);
    if (coef == 1.f && list.in[t] == list.out[t]) continue;
    const int64_t from = int64_t(c - list.first[t]) * list.chunk;
    const int64_t n = list.n[t] - from < list.chunk ? list.n[t] - from : list.chunk;
    if (list.type[t] == SF_F32)
      scale_chunk(static_cast<const float*>(list.in[t]) + from, static_cast<float*>(list.out[t]) + from, n, coef);
    else if (list.type[t] == SF_BF16)
      scale_chunk(static_cast<const __nv_bfloat16*>(list.in[t]) + from,
                  static_cast<__nv_bfloat16*>(list.out[t]) + from, n, coef);
    else
      scale_chunk(static_cast<const __half*>(list.in[t]) + from, static_cast<__half*>(list.out[t]) + from, n, coef);
  }
}

// How the tensors are cut: the chunk's size, and the chunks and launches that
// makes.  Eight chunks or more a CTA, so that none ends much later than the others.
struct Cut {
  int64_t chunk = kMinChunk, chunks = 0, launches = 0, grid = 0;
};

Cut cut_of(const int64_t* numel, int64_t n) {
  Cut c;
  int64_t total = 0;
  for (int64_t i = 0; i < n; ++i) total += numel[i];
  c.grid = int64_t(sm_count()) * kPerSm;
  c.chunk = std::min(kMaxChunk, std::max(kMinChunk, (total / (c.grid * 8) + kMinChunk - 1) / kMinChunk * kMinChunk));
  for (int64_t i = 0; i < n; ++i) c.chunks += (numel[i] + c.chunk - 1) / c.chunk;
  c.launches = std::max<int64_t>(1, (n + kListMax - 1) / kListMax);
  return c;
}

template <int M>
cudaError_t launch_lists(const GradJob& j, void* workspace, cudaStream_t stream) {
  const Cut cut = cut_of(j.numel, j.n);
  double* total = static_cast<double*>(workspace);
  double* partial = total + cut.launches * cut.grid;
  const bool clip = j.max_norm > 0.f;
  TensorList<M> list;
  list.chunk = cut.chunk;
  // pass 0: sums of squares of every list; pass 1: the norm, and the scaling
  for (int pass = 0; pass < 2; ++pass) {
    int64_t chunk0 = 0, total0 = 0;
    for (int64_t from = 0; from < std::max<int64_t>(1, j.n); from += M) {
      list.count = static_cast<int32_t>(std::min<int64_t>(M, j.n - from));
      int64_t chunks = 0;
      for (int i = 0; i < list.count; ++i) {
        list.in[i] = j.data[from + i];
        list.out[i] = j.out != nullptr ? j.out[from + i] : const_cast<void*>(j.data[from + i]);
        list.n[i] = j.numel[from + i];
        list.type[i] = static_cast<uint8_t>(j.dtype[from + i]);
        list.first[i] = static_cast<int32_t>(chunks);
        chunks += (list.n[i] + cut.chunk - 1) / cut.chunk;
        if (chunks > INT32_MAX) return cudaErrorInvalidValue;
      }
      list.first[list.count] = static_cast<int32_t>(chunks);
      list.partial = partial + chunk0;
      list.total = total + total0;
      const unsigned grid = static_cast<unsigned>(std::max<int64_t>(1, std::min(cut.grid, chunks)));
      chunk0 += chunks;
      total0 += grid;
      cudaError_t e;
      count_launch();
      if (pass == 0) {
        e = launch_after(grad_squares_kernel<M>, dim3(grid), dim3(kThreads), 0, stream, true, list);
      } else {
        NormOut o;
        o.total = total;
        o.totals = 0;
        for (int64_t f = 0, g; f < std::max<int64_t>(1, j.n); f += M) {  // the grids of pass 0
          int64_t k = 0;
          for (int64_t i = f; i < std::min(j.n, f + M); ++i) k += (j.numel[i] + cut.chunk - 1) / cut.chunk;
          g = std::max<int64_t>(1, std::min(cut.grid, k));
          o.totals += g;
        }
        o.norm = j.norm;
        o.coef = j.coef;
        o.max_norm = j.max_norm;
        o.eps = j.eps;
        o.status = j.status;
        float* norms = j.tensor_norm != nullptr ? j.tensor_norm + from : nullptr;
        if (clip) {
          e = launch_after(grad_scale_kernel<M>, dim3(grid), dim3(kThreads), 0, stream, true, list, o, norms);
        } else {
          const unsigned few = norms != nullptr ? (list.count * 32 + kThreads - 1) / kThreads : 1;
          e = launch_after(grad_norms_kernel<M>, dim3(std::max(1u, few)), dim3(kThreads), 0, stream, true, list, o, norms);
        }
      }
      if (e != cudaSuccess) return e;
    }
  }
  return cudaSuccess;
}

}  // namespace

size_t grad_workspace(const int64_t* numel, int64_t n) {
  const Cut c = cut_of(numel, n);
  return size_t(c.launches * c.grid + c.chunks) * sizeof(double);
}

cudaError_t launch_grad(const GradJob& j, void* workspace, cudaStream_t stream) {
  // a short list's parameters are launched faster
  return j.n <= 64 ? launch_lists<64>(j, workspace, stream) : launch_lists<kListMax>(j, workspace, stream);
}

}  // namespace sf
