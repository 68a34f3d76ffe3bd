// sf_grad_norm.cu - the 2-norm over many gradient tensors, each tensor's own,
// and clipping (sf_grad_norm, sf_grad_clip).
//
// The tensors, one after another, are one long run of 16-byte packs, each in a
// place of whole grains of 32 (so that no warp gets many small ones: 219 tensors
// of 8435 values in all took 42 us when they lay side by side).  It is cut into
// equal ranges, one a warp, or one a CTA whose warps take its blocks
// of 4 KB in turn: no warp waits for another, whatever the tensors' sizes.  A
// warp writes the sum of squares of each piece (range by tensor) it meets.
// Going on by one piece raises the range or the tensor, so range + tensor
// numbers the pieces.  The tensors' pointers and sizes travel as
// a kernel parameter (up to 32 KB): nothing is copied to the device or kept
// there.  A second kernel adds what the CTAs found (every CTA for itself: they
// are few) and, for clipping, scales the data, from the end of each range
// back, as L2 still holds what was read last.  All sums go in a fixed order.
// A few megabytes take one cluster of CTAs, one launch and no workspace.  Bound
// by memory: a conversion and a multiply-add an element.  1.5 G bf16 values
// of 400 tensors are normed in 418 us (7.2 TB/s), 1 G of 300 clipped into other
// buffers in 932 us (6.4 TB/s over two reads and a write).
#include <algorithm>

#include "sf_float.cuh"
#include "sf_launch.h"

namespace sf {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kPerSm = 4;       // CTAs of the grid per SM
constexpr int kUnroll = 8;      // packs in flight a thread
constexpr int64_t kGrain = 32;   // packs that a tensor's place is a multiple of, and the least of a range
constexpr int kListMax = 960;   // tensors of one launch: 33 bytes each of the 32764 there are for parameters

// Part of the tensors, as a kernel parameter.
template <int M>
struct TensorList {
  const void* in[M];
  void* out[M];
  int64_t n[M];
  int64_t off[M + 1];  // packs of the tensors before
  uint8_t type[M];
  int32_t count;
  int32_t group;    // warps of a range
  int64_t range;    // its packs
  double* partial;  // [range + tensor][group] sums of squares of the pieces
  double* total;    // of the CTAs
};

// The tensor that has pack `at` (at < off[count]): the last one that does not start after it, so never an empty one.
template <int M>
__device__ __forceinline__ int tensor_of(const TensorList<M>& list, int64_t at) {
  int lo = 0, hi = list.count;  // off[lo] <= at < off[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (list.off[mid] <= at)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// A warp's part of a range: warp `sub` of `group`.
struct Share {
  int lane, sub, group;
};

// Sum of squares of a warp's share of n values at p; lane 0's counts.  A lane sums what
// it has in flight in 32 bits (at most 16 squares to a sum) and adds that up
// as a pair, so that equal values do not round the same way over and over.
// Where the short sums overflow, or are so small that squares may have been
// lost below 2^-126 (a sum under 2^-80 of values that are not all 0), the
// piece is summed again in 64 bits.
template <typename T>
__device__ double sum_squares(const T* p, int64_t n, const Share& w) {
  const int lane = w.lane;
  constexpr int N = Pack<T>::kN;
  const int head = head_of(p, n);
  const int64_t nv = (n - head) / N;
  const T* body = p + head;
  const int tail = static_cast<int>(n - head - nv * N);
  Sum2 sum;
  uint32_t any = 0;
  if (w.sub == 0 && lane < head) {
    const float v = to_f32(p[lane]);
    sum.add(v * v);
    any |= v != 0.f;
  }
  if (w.sub == 0 && lane < tail) {
    const float v = to_f32(body[nv * N + lane]);
    sum.add(v * v);
    any |= v != 0.f;
  }
  const auto add = [&](const uint4(&u)[kUnroll]) {
    uint64_t a = 0, b = 0;  // two sums each
#pragma unroll
    for (int q = 0; q < kUnroll; ++q) {
      uint64_t z[N / 2];
      unpack2(u[q], z, T());
#pragma unroll
      for (int e = 0; e < N / 2; e += 2) {
        a = fma2(z[e], z[e], a);
        b = fma2(z[e + 1], z[e + 1], b);
      }
      any |= (u[q].x | u[q].y | u[q].z | u[q].w) & (sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu);
    }
    float x, y;
    split(add2(a, b), x, y);
    sum.add(x + y);
  };
  const int64_t step = 32 * kUnroll * w.group;
  int64_t i = 32 * kUnroll * w.sub + lane;
  for (; i + (kUnroll - 1) * 32 < nv; i += step) {
    uint4 u[kUnroll];
#pragma unroll
    for (int q = 0; q < kUnroll; ++q) u[q] = load16(body + (i + q * 32) * N);
    add(u);
  }
  if (i < nv) {
    uint4 u[kUnroll];
#pragma unroll
    for (int q = 0; q < kUnroll; ++q) u[q] = i + q * 32 < nv ? load16(body + (i + q * 32) * N) : make_uint4(0, 0, 0, 0);
    add(u);
  }
  __syncwarp();
  sum = warp_sum(sum);
  const bool small = sum.hi < 8.0e-25f && __any_sync(kFull, any != 0);
  if (sum.hi <= 3.0e38f && !small) return double(sum.hi) + double(sum.lo);
  double d = 0.;
  const auto again = [&](const T& x) {
    const double v = to_f32(x);
    d = fma(v, v, d);
  };
  if (w.sub == 0 && lane < head) again(p[lane]);
  if (w.sub == 0 && lane < tail) again(body[nv * N + lane]);
  for (i = 32 * kUnroll * w.sub + lane; i < nv; i += step)
    for (int64_t k = i; k < nv && k < i + 32 * kUnroll; k += 32)
      for (int q = 0; q < N; ++q) again(body[k * N + q]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) d += __shfl_xor_sync(kFull, d, o);
  return d;
}

// Calls f(type tag, tensor, first element, elements) for the pieces of a range,
// first to last or last to first.
template <bool kBack, int M, typename F>
__device__ __forceinline__ void for_pieces(const TensorList<M>& list, int64_t range, const F& f) {
  const int64_t total = list.off[list.count];
  int64_t from = range * list.range, to = from + list.range < total ? from + list.range : total;
  if (from >= to) return;
  int t = tensor_of(list, kBack ? to - 1 : from);
  while (from < to) {
    const int64_t a = from > list.off[t] ? from : list.off[t], b = to < list.off[t + 1] ? to : list.off[t + 1];
    if (a < b) {
      const int N = list.type[t] == SF_F32 ? 4 : 8;
      const int64_t first = (a - list.off[t]) * N, end = (b - list.off[t]) * N;
      const int64_t n = max(int64_t(0), (end < list.n[t] ? end : list.n[t]) - first);  // its place may end with nothing
      if (list.type[t] == SF_F32)
        f(float(), t, first, n);
      else if (list.type[t] == SF_BF16)
        f(__nv_bfloat16(), t, first, n);
      else
        f(__half(), t, first, n);
    }
    if (kBack) {
      to = a;
      --t;
    } else {
      from = b;
      ++t;
    }
  }
}

template <int M>
__device__ __forceinline__ Share share_of(const TensorList<M>& list) {
  const int warp = threadIdx.x >> 5;
  return {int(threadIdx.x & 31), warp % list.group, list.group};
}
template <int M>
__device__ __forceinline__ int64_t range_of(const TensorList<M>& list) {
  return (int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5)) / list.group;
}

template <int M>
__global__ void __launch_bounds__(kThreads, kPerSm) grad_squares_kernel(const __grid_constant__ TensorList<M> list) {
  __shared__ double totals[kWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const Share share = share_of(list);
  const int64_t range = range_of(list);
  griddep_wait();  // the gradients, and the workspace, which the previous call may still read
  double total = 0.;
  for_pieces<false>(list, range, [&](auto tag, int t, int64_t first, int64_t n) {
    const double s = sum_squares(static_cast<const decltype(tag)*>(list.in[t]) + first, n, share);
    total += s;
    if (lane == 0) list.partial[(range + t) * share.group + share.sub] = s;
  });
  if (lane == 0) totals[warp] = total;
  __syncthreads();
  if (threadIdx.x == 0) {
    double s = totals[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) s += totals[w];
    list.total[blockIdx.x] = s;
  }
}

struct NormOut {
  const double* total;
  int64_t totals;
  float *norm, *coef, *tensor_norm;
  float max_norm, eps;
  uint32_t* status;
};

// The root of a sum in 32 bits, where it has that range: 64-bit arithmetic is slow here.
__device__ __forceinline__ float root(double s) {
  return s > 1e-30 && s < 1e30 ? sqrtf(static_cast<float>(s)) : static_cast<float>(sqrt(s));
}

// The clipping coefficient, in every thread; CTA 0 writes the norm over all tensors.
__device__ float finish_norm(const NormOut& o) {
  __shared__ float shared_coef;
  if (threadIdx.x < 32) {
    double s = 0.;
    for (int64_t i = threadIdx.x; i < o.totals; i += 32) s += o.total[i];
#pragma unroll
    for (int k = 16; k > 0; k >>= 1) s += __shfl_xor_sync(kFull, s, k);
    if (threadIdx.x == 0) {
      const float norm = root(s);
      const float coef = finite(norm) ? fminf(1.f, o.max_norm / (norm + o.eps)) : quiet_nan();
      shared_coef = coef;
      if (blockIdx.x == 0) {
        *o.norm = norm;
        if (o.coef != nullptr) *o.coef = coef;
        if (!finite(norm)) report(o.status, SF_ST_NONFINITE);
      }
    }
  }
  __syncthreads();
  return shared_coef;
}

// Norms of a list's tensors from their pieces' sums, a CTA each.
template <int M>
__device__ void tensor_norms(const TensorList<M>& list, float* out) {
  __shared__ double buf[kWarps];
  for (int t = blockIdx.x; t < list.count; t += gridDim.x) {
    double s = 0.;
    if (list.n[t] > 0) {
      const int64_t first = (list.off[t] / list.range + t) * list.group;
      const int64_t end = ((list.off[t + 1] - 1) / list.range + t + 1) * list.group;
      for (int64_t i = first + threadIdx.x; i < end; i += kThreads) s += list.partial[i];
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(kFull, s, o);
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
      for (int w = 1; w < kWarps; ++w) s += buf[w];
      out[t] = root(s);
    }
    __syncthreads();
  }
}

template <int M>
__global__ void __launch_bounds__(kThreads)
    grad_norms_kernel(const __grid_constant__ TensorList<M> list, const NormOut o) {
  griddep_wait();
  if (o.tensor_norm != nullptr) tensor_norms(list, o.tensor_norm);
  if (blockIdx.x == 0) finish_norm(o);
}

// Fewer packs in flight than the sums have: each has its result beside it (with
// eight the registers do not do).
constexpr int kScaleUnroll = 4;

template <typename T>
__device__ void scale_piece(const T* p, T* q, int64_t n, float coef, const Share& w) {
  const int lane = w.lane;
  constexpr int N = Pack<T>::kN;
  const int head = head_of(p, n);
  const int64_t nv = (n - head) / N;
  const int tail = static_cast<int>(n - head - nv * N);
  if (w.sub == 0 && lane < tail) {
    const int64_t at = head + nv * N + lane;
    q[at] = from_f32<T>(to_f32(p[at]) * coef);
  }
  const bool even = (reinterpret_cast<uintptr_t>(q + head) & 15u) == 0;  // both runs at the same offset
  const auto scaled = [&](const uint4& u) {
    float f[N];
    unpack(u, f, T());
#pragma unroll
    for (int k = 0; k < N; ++k) f[k] *= coef;
    return pack(f, T());
  };
  const auto store = [&](int64_t at, const uint4& u) {
    if (even)
      store16(q + head + at * N, u);
    else
      store_elements(q + head + at * N, u);
  };
  const int64_t step = 32 * kScaleUnroll * w.group;
  int64_t i = nv - 1 - lane - 32 * kScaleUnroll * w.sub;
  for (; i - (kScaleUnroll - 1) * 32 >= 0; i -= step) {
    uint4 u[kScaleUnroll];
#pragma unroll
    for (int k = 0; k < kScaleUnroll; ++k) u[k] = load16(p + head + (i - k * 32) * N);
#pragma unroll
    for (int k = 0; k < kScaleUnroll; ++k) store(i - k * 32, scaled(u[k]));
  }
  if (i >= 0) {
    uint4 u[kScaleUnroll];
#pragma unroll
    for (int k = 0; k < kScaleUnroll; ++k)
      if (i - k * 32 >= 0) u[k] = load16(p + head + (i - k * 32) * N);
#pragma unroll
    for (int k = 0; k < kScaleUnroll; ++k)
      if (i - k * 32 >= 0) store(i - k * 32, scaled(u[k]));
  }
  __syncwarp();
  if (w.sub == 0 && lane < head) q[lane] = from_f32<T>(to_f32(p[lane]) * coef);
}

template <int M>
__global__ void __launch_bounds__(kThreads, kPerSm)
    grad_scale_kernel(const __grid_constant__ TensorList<M> list, const NormOut o) {
  const Share share = share_of(list);
  griddep_wait();
  float coef = finish_norm(o);
  if (!finite(coef)) coef = 1.f;  // passed on unscaled
  for_pieces<true>(list, range_of(list), [&](auto tag, int t, int64_t first, int64_t n) {
    if (coef == 1.f && list.in[t] == list.out[t]) return;
    using T = decltype(tag);
    scale_piece(static_cast<const T*>(list.in[t]) + first, static_cast<T*>(list.out[t]) + first, n, coef, share);
  });
  if (o.tensor_norm != nullptr) tensor_norms(list, o.tensor_norm);
}

// All of it by one cluster: each warp's sums of squares go to the first CTA's
// shared memory, which adds them up, in the same order whatever came first, and
// hands the coefficient back.  24 tensors of 4.8 MB: 12.2 us (two launches over
// all SMs 10.3, but 4 to 7 us more of the host's time); 219 of 8435 values 12.  The
// limit of 6 MB lies above that one comparison; many unaligned pieces are slow here
// (317 packed tensors of 5 MB clipped 43 us).
constexpr int kSmallCtas = 16, kSmallThreads = 512, kSmallWarps = kSmallCtas * kSmallThreads / 32;
constexpr int64_t kSmallPacks = 6 << 16;  // 6 MB

template <int M, bool kClip>
__global__ void __launch_bounds__(kSmallThreads, 1)
    grad_small_kernel(const __grid_constant__ TensorList<M> list, const NormOut o) {
  __shared__ double pieces[kSmallWarps + M];  // by range + tensor, of the first CTA
  __shared__ double part[kSmallThreads / 32];
  __shared__ float shared_coef;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t rank = cluster_rank();
  const int range = static_cast<int>(rank) * (kSmallThreads / 32) + warp;
  const Share share = {lane, 0, 1};
  if (rank == 0)
    for (int i = threadIdx.x; i < kSmallWarps + M; i += kSmallThreads) pieces[i] = 0.;
  cluster_sync();
  griddep_wait();  // the gradients
  for_pieces<false>(list, range, [&](auto tag, int t, int64_t first, int64_t n) {
    const double s = sum_squares(static_cast<const decltype(tag)*>(list.in[t]) + first, n, share);
    if (lane == 0)
      asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(at_rank(pieces + range + t, 0)), "d"(s) : "memory");
  });
  __syncwarp();
  cluster_sync();
  if (rank == 0) {
    double s = 0.;
    for (int i = threadIdx.x; i < kSmallWarps + list.count; i += kSmallThreads) s += pieces[i];
#pragma unroll
    for (int k = 16; k > 0; k >>= 1) s += __shfl_xor_sync(kFull, s, k);
    if (lane == 0) part[warp] = s;
    __syncthreads();
    if (warp == 0) {
      s = lane < kSmallThreads / 32 ? part[lane] : 0.;
#pragma unroll
      for (int k = 16; k > 0; k >>= 1) s += __shfl_xor_sync(kFull, s, k);
      const float norm = root(s);
      const float coef = finite(norm) ? fminf(1.f, o.max_norm / (norm + o.eps)) : quiet_nan();
      if (lane == 0) {
        *o.norm = norm;
        if (o.coef != nullptr) *o.coef = coef;
        if (!finite(norm)) report(o.status, SF_ST_NONFINITE);
      }
      if (kClip && lane < kSmallCtas)
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at_rank(&shared_coef, lane)), "f"(coef) : "memory");
    }
  }
  if (kClip) {
    __syncwarp();
    cluster_sync();
    float coef = shared_coef;
    if (!finite(coef)) coef = 1.f;  // passed on unscaled
    for_pieces<true>(list, range, [&](auto tag, int t, int64_t first, int64_t n) {
      if (coef == 1.f && list.in[t] == list.out[t]) return;
      using T = decltype(tag);
      scale_piece(static_cast<const T*>(list.in[t]) + first, static_cast<T*>(list.out[t]) + first, n, coef, share);
    });
  }
  if (rank != 0 || o.tensor_norm == nullptr) return;
  // each tensor's norm: by a thread where it has few pieces, else by a warp
  constexpr int kFew = 16;
  const auto pieces_of = [&](int t, int& first, int& end) {
    first = static_cast<int>(list.off[t] / list.range) + t;
    end = list.n[t] > 0 ? static_cast<int>((list.off[t + 1] - 1) / list.range) + t + 1 : first;
  };
  for (int t = threadIdx.x; t < list.count; t += kSmallThreads) {
    int first, end;
    pieces_of(t, first, end);
    if (end - first > kFew) continue;
    double q = 0.;
    for (int i = first; i < end; ++i) q += pieces[i];
    o.tensor_norm[t] = root(q);
  }
  for (int t = warp; t < list.count; t += kSmallThreads / 32) {
    int first, end;
    pieces_of(t, first, end);
    if (end - first <= kFew) continue;
    double q = 0.;
    for (int i = first + lane; i < end; i += 32) q += pieces[i];
#pragma unroll
    for (int k = 16; k > 0; k >>= 1) q += __shfl_xor_sync(kFull, q, k);
    if (lane == 0) o.tensor_norm[t] = root(q);
  }
}

// Packs of a tensor, and of its place.
int64_t packs_of(int64_t numel, int32_t dtype) {
  const int64_t N = dtype == SF_F32 ? 4 : 8;
  return (numel + N - 1) / N;
}
int64_t place_of(int64_t numel, int32_t dtype) { return (packs_of(numel, dtype) + kGrain - 1) / kGrain * kGrain; }

// The ranges of one list.  Long ranges are a CTA's: fewer places of memory are
// read at a time (2 GB of gradients clipped into other buffers: 932-944 us, with
// a warp's ranges 970), short ones a warp's (150 tensors of 60 MB in all: the
// warps of a CTA would take its tensors one after another).
struct Cut {
  int32_t group;
  int64_t range, grid;
};
Cut cut_of(int64_t packs) {
  const int64_t ctas = int64_t(sm_count()) * kPerSm, warps = ctas * kWarps;
  Cut c;
  c.group = packs >= warps * 2048 ? kWarps : 1;
  const int64_t most = warps / c.group;
  c.range = std::max(kGrain, ((packs + most - 1) / most + 31) / 32 * 32);
  const int64_t ranges = (packs + c.range - 1) / c.range;
  c.grid = std::max<int64_t>(1, (ranges * c.group + kWarps - 1) / kWarps);
  return c;
}

template <int M>
cudaError_t launch_small(TensorList<M>& list, const NormOut& o, bool clip, cudaStream_t stream) {
  const int64_t packs = list.off[list.count];
  list.group = 1;
  list.range = std::max(kGrain, ((packs + kSmallWarps - 1) / kSmallWarps + 31) / 32 * 32);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kSmallCtas);
  cfg.blockDim = dim3(kSmallThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = kSmallCtas;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  void* params[] = {&list, const_cast<NormOut*>(&o)};
  const void* kern = clip ? reinterpret_cast<const void*>(grad_small_kernel<M, true>)
                          : reinterpret_cast<const void*>(grad_small_kernel<M, false>);
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);  // 16 CTAs
  if (e != cudaSuccess) return e;
  count_launch();
  return cudaLaunchKernelExC(&cfg, kern, params);
}

template <int M>
cudaError_t launch_lists(const GradJob& j, void* workspace, cudaStream_t stream) {
  const int64_t lists = std::max<int64_t>(1, (j.n + M - 1) / M);
  const int64_t grid_max = int64_t(sm_count()) * kPerSm;
  double* total = static_cast<double*>(workspace);
  double* partial = total + lists * grid_max;
  TensorList<M> list;
  NormOut o;
  o.total = total;
  o.totals = 0;
  o.norm = j.norm;
  o.coef = j.coef;
  o.max_norm = j.max_norm;
  o.eps = j.eps;
  o.status = j.status;
  int64_t grid = 0;
  const auto fill = [&](int64_t l) {
    const int64_t from = l * M;
    list.count = static_cast<int32_t>(std::min<int64_t>(M, j.n - from));
    int64_t packs = 0;
    for (int i = 0; i < list.count; ++i) {
      list.in[i] = j.data[from + i];
      list.out[i] = j.out != nullptr ? j.out[from + i] : const_cast<void*>(j.data[from + i]);
      list.n[i] = j.numel[from + i];
      list.type[i] = static_cast<uint8_t>(j.dtype[from + i]);
      list.off[i] = packs;
      packs += place_of(list.n[i], j.dtype[from + i]);
    }
    list.off[list.count] = packs;
    const Cut c = cut_of(packs);
    list.group = c.group;
    list.range = c.range;
    list.partial = partial + l * (grid_max + M) * kWarps;
    grid = c.grid;
  };
  if (workspace == nullptr) {  // grad_small
    fill(0);
    o.tensor_norm = j.tensor_norm;
    return launch_small(list, o, j.max_norm > 0.f, stream);
  }
  for (int64_t l = 0; l < lists; ++l) {
    fill(l);
    list.total = total + o.totals;
    o.totals += grid;
    count_launch();
    const cudaError_t e = launch_after(grad_squares_kernel<M>, dim3(static_cast<unsigned>(grid)), dim3(kThreads), 0,
                                       stream, true, list);
    if (e != cudaSuccess) return e;
  }
  for (int64_t l = 0; l < lists; ++l) {
    if (lists > 1) fill(l);
    o.tensor_norm = j.tensor_norm != nullptr ? j.tensor_norm + l * M : nullptr;
    const bool clip = j.max_norm > 0.f;
    const int64_t ctas = clip ? grid : o.tensor_norm != nullptr ? std::max(1, list.count) : 1;
    count_launch();
    const cudaError_t e = launch_after(clip ? grad_scale_kernel<M> : grad_norms_kernel<M>,
                                       dim3(static_cast<unsigned>(ctas)), dim3(kThreads), 0, stream, true, list, o);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace

bool grad_small(const int64_t* numel, const int32_t* dtype, int64_t n) {
  if (n > kListMax) return false;
  int64_t packs = 0;
  for (int64_t i = 0; i < n && packs <= kSmallPacks; ++i) packs += packs_of(numel[i], dtype[i]);
  return packs <= kSmallPacks;
}

size_t grad_workspace(int64_t n) {
  const int64_t lists = std::max<int64_t>(1, (n + kListMax - 1) / kListMax), grid = int64_t(sm_count()) * kPerSm;
  return size_t(lists * (grid + (grid + kListMax) * kWarps)) * sizeof(double);
}

// The shorter the list, the faster its launch: 0.6 us a KB of parameters, 33 bytes a tensor.
cudaError_t launch_grad(const GradJob& j, void* workspace, cudaStream_t stream) {
  if (grad_small(j.numel, j.dtype, j.n)) workspace = nullptr;  // by size alone: the order of the sums is one
  if (j.n <= 32) return launch_lists<32>(j, workspace, stream);
  if (j.n <= 64) return launch_lists<64>(j, workspace, stream);
  if (j.n <= 160) return launch_lists<160>(j, workspace, stream);
  if (j.n <= 320) return launch_lists<320>(j, workspace, stream);
  if (j.n <= 480) return launch_lists<480>(j, workspace, stream);
  return launch_lists<kListMax>(j, workspace, stream);
}

}  // namespace sf
