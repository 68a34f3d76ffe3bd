// sf_ffn_few.cu - the gated feed-forward operators for a few tokens, on the f32
// units: the weights are read once, and what bounds a call is their bytes.
#include <algorithm>
#include <type_traits>

#include "sf_ffn_math.cuh"
#include "sf_ffn_tensor.h"

namespace sf {
namespace {

constexpr int kThreads = 256;

// Features of a warp, for their sake that the tokens are read for (us with 1 and 2, one GB300):
// even rows f32 4 x 2048 x 7452 28 and 25, 8 x 1024 x 4096 15 and 12, bf16 1 x 4096 x 12288 32.7 and 34.2;
// uneven rows f32 4 x 2009 x 7452 29 and 45, 8 x 2009 x 7452 95 and 67.
template <typename T, int kTokens, bool kEven>
constexpr int kFeaturesOf = kEven ? (sizeof(T) == 2 && kTokens == 1 ? 1 : 2) : kTokens <= 4 ? 1 : 2;

// One value of h, or of dg and du in f32 (and h), from its g and u.
template <typename T, int kAct, bool kInner>
__device__ __forceinline__ void store_value(const FfnJob& j, int64_t t, int64_t f, float g, float u) {
  using A = Activation<kAct, sizeof(T) == 2>;
  if constexpr (!kInner) {
    static_cast<T*>(j.h)[t * j.ldh + f] = from_f32<T>(A::value(g) * u);
  } else {
    float a, slope;
    A::both(g, a, slope);
    const float d = to_f32(static_cast<const T*>(j.dh)[t * j.lddh + f]);
    if (j.h != nullptr) static_cast<T*>(j.h)[t * j.ldh + f] = from_f32<T>(a * u);
    static_cast<float*>(j.dg)[t * j.ldg + f] = d * u * slope;
    static_cast<float*>(j.du)[t * j.ldg + f] = d * a;
  }
}

// A warp's rows of both weights times kTokens tokens.  Each lane sums every 32nd pack of
// 16 bytes (kEven: all rows start on 16 bytes) or value of a row, and the lanes' sums are
// added.  Bound by the weights' bytes (f32 1 x 4096 x 12288: 60 us, 99 % of the copy rate;
// 8 tokens 88 us); the tokens are read from L1, once for all of the warp's rows, which the
// weights do not pass through (that took 68 and 137 us).
template <typename T, int kTokens, bool kEven, bool kInner>
__global__ void __launch_bounds__(kThreads, kEven ? 2 : 4) ffn_rows_kernel(const FfnJob j) {
  constexpr int kFeatures = kFeaturesOf<T, kTokens, kEven>;
  constexpr int N = kEven ? Pack<T>::kN : 1, kAhead = kEven ? (kTokens <= 2 ? 4 : 2) : kFeatures == 1 ? 8 : 4;
  griddep_launch_dependents();
  const int lane = threadIdx.x & 31;
  const int64_t warp = (int64_t(blockIdx.y) * (kThreads / 32)) + (threadIdx.x >> 5);
  const int64_t f0 = warp * kFeatures, t0 = int64_t(blockIdx.x) * kTokens;
  if (f0 >= j.F) return;
  const T* x = static_cast<const T*>(j.x) + t0 * j.ldx;
  const T* w[2 * kFeatures];  // a feature's rows of both weights; a missing feature is the last one again
#pragma unroll
  for (int r = 0; r < kFeatures; ++r) {
    const int64_t f = min(f0 + r, j.F - 1);
    w[2 * r] = static_cast<const T*>(j.w_gate) + f * j.ldw;
    w[2 * r + 1] = static_cast<const T*>(j.w_up) + f * j.ldw;
  }
  int64_t x_at[kTokens];
#pragma unroll
  for (int t = 0; t < kTokens; ++t) x_at[t] = min(int64_t(t), j.T - 1 - t0) * j.ldx;
  float sum[2 * kFeatures][kTokens];
#pragma unroll
  for (int r = 0; r < 2 * kFeatures; ++r)
#pragma unroll
    for (int t = 0; t < kTokens; ++t) sum[r][t] = 0.f;
  using Raw = typename std::conditional<kEven, uint4, T>::type;  // as loaded: a conversion would wait
  const auto open = [](const Raw& raw, float (&v)[N]) {
    if constexpr (kEven)
      unpack(raw, v, T());
    else
      v[0] = to_f32(raw);
  };
  const int64_t whole = j.H / N;
  for (int64_t p0 = lane; p0 < whole; p0 += 32 * kAhead) {
    Raw raw[kAhead][2 * kFeatures];
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (p0 + 32 * k < whole) {
#pragma unroll
        for (int r = 0; r < 2 * kFeatures; ++r) {  // read once: the tokens stay in L1
          const T* p = w[r] + (p0 + 32 * k) * N;
          if constexpr (kEven)
            raw[k][r] = load16(p);
          else
            raw[k][r] = *p;
        }
      }
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (p0 + 32 * k < whole) {
        float v[2 * kFeatures][N];
#pragma unroll
        for (int r = 0; r < 2 * kFeatures; ++r) open(raw[k][r], v[r]);
#pragma unroll
        for (int t = 0; t < kTokens; ++t) {
          float y[N];
          open(*reinterpret_cast<const Raw*>(x + x_at[t] + (p0 + 32 * k) * N), y);
#pragma unroll
          for (int r = 0; r < 2 * kFeatures; ++r)
#pragma unroll
            for (int i = 0; i < N; ++i) sum[r][t] = fmaf(v[r][i], y[i], sum[r][t]);
        }
      }
  }
  for (int64_t c = whole * N + lane; c < j.H; c += 32) {
#pragma unroll
    for (int t = 0; t < kTokens; ++t)
#pragma unroll
      for (int r = 0; r < 2 * kFeatures; ++r) sum[r][t] = fmaf(to_f32(w[r][c]), to_f32(x[x_at[t] + c]), sum[r][t]);
  }
#pragma unroll
  for (int r = 0; r < 2 * kFeatures; ++r)
#pragma unroll
    for (int t = 0; t < kTokens; ++t) sum[r][t] = warp_sum(sum[r][t]);
  // lane t + kTokens r stores feature r of token t
  float g = 0.f, u = 0.f;
#pragma unroll
  for (int r = 0; r < kFeatures; ++r)
#pragma unroll
    for (int t = 0; t < kTokens; ++t)
      if (lane == t + kTokens * r) {
        g = sum[2 * r][t];
        u = sum[2 * r + 1][t];
      }
  const int64_t f = f0 + lane / kTokens, t = t0 + lane % kTokens;
  if (lane >= kTokens * kFeatures || f >= j.F || t >= j.T) return;
  switch (j.act) {
    case SF_ACT_GELU: return store_value<T, SF_ACT_GELU, kInner>(j, t, f, g, u);
    case SF_ACT_GELU_TANH: return store_value<T, SF_ACT_GELU_TANH, kInner>(j, t, f, g, u);
    case SF_ACT_RELU: return store_value<T, SF_ACT_RELU, kInner>(j, t, f, g, u);
    default: return store_value<T, SF_ACT_SILU, kInner>(j, t, f, g, u);
  }
}

template <typename T, int kTokens, bool kEven, bool kInner>
cudaError_t launch_warps(const FfnJob& j, cudaStream_t stream) {
  constexpr int kFeatures = kFeaturesOf<T, kTokens, kEven>;
  const int64_t warps = (j.F + kFeatures - 1) / kFeatures, blocks = (warps + kThreads / 32 - 1) / (kThreads / 32);
  // the tokens' groups of the same features side by side: they share the weights in L2
  const dim3 grid(static_cast<unsigned>((j.T + kTokens - 1) / kTokens), static_cast<unsigned>(blocks));
  count_launch();
  ffn_rows_kernel<T, kTokens, kEven, kInner><<<grid, kThreads, 0, stream>>>(j);
  return cudaGetLastError();
}
template <typename T, int kTokens, bool kInner>
cudaError_t launch_rows(const FfnJob& j, bool even, cudaStream_t stream) {
  if constexpr (sizeof(T) == 4 || kTokens <= 2) {  // uneven rows of 16 bits: up to two tokens
    if (!even) return launch_warps<T, kTokens, false, kInner>(j, stream);
  }
  return launch_warps<T, kTokens, true, kInner>(j, stream);
}
template <typename T, bool kInner>
cudaError_t launch_few(const FfnJob& j, bool even, cudaStream_t stream) {
  if (j.T == 1) return launch_rows<T, 1, kInner>(j, even, stream);
  if (j.T == 2) return launch_rows<T, 2, kInner>(j, even, stream);
  if constexpr (std::is_same<T, float>::value) {  // 16-bit types come here with up to four
    if (j.T > 4) return launch_rows<T, 8, kInner>(j, even, stream);
  }
  return launch_rows<T, 4, kInner>(j, even, stream);
}

// ---------------------------------------------------------------- the gradient, f32

constexpr int kColumns = 4, kBlock = kThreads * kColumns;  // of a thread, of a CTA
constexpr int kSlab = 128;                                   // features of a CTA, at most

// A thread's columns: four side by side (kEven), or every 256th.
template <bool kEven>
__device__ __forceinline__ int64_t column(int64_t c0, int i) {
  return kEven ? c0 + threadIdx.x * kColumns + i : c0 + threadIdx.x + i * kThreads;
}
template <bool kEven>
__device__ __forceinline__ void load_columns(const float* row, int64_t c0, int64_t H, float (&v)[kColumns]) {
  if (kEven && column<kEven>(c0, 0) + kColumns <= H) {
    unpack(load16(row + column<kEven>(c0, 0)), v, 0.f);
  } else {
#pragma unroll
    for (int i = 0; i < kColumns; ++i) v[i] = column<kEven>(c0, i) < H ? row[column<kEven>(c0, i)] : 0.f;
  }
}
template <bool kEven>
__device__ __forceinline__ void store_columns(float* row, int64_t c0, int64_t H, const float (&v)[kColumns]) {
  if (kEven && column<kEven>(c0, 0) + kColumns <= H) {
    store16(row + column<kEven>(c0, 0), pack(v, 0.f));
  } else {
#pragma unroll
    for (int i = 0; i < kColumns; ++i)
      if (column<kEven>(c0, i) < H) row[column<kEven>(c0, i)] = v[i];
  }
}

// The slab's dg and du, [feature][token].
template <int kTokens>
__device__ __forceinline__ void load_slab(const FfnJob& j, int64_t f0, int n, float (&dg)[kSlab][kTokens],
                                          float (&du)[kSlab][kTokens]) {
  for (int i = threadIdx.x; i < kSlab * kTokens; i += kThreads) {
    const int f = i % kSlab, t = i / kSlab;
    const bool in = f < n && t < j.T;
    dg[f][t] = in ? static_cast<const float*>(j.dg)[t * j.ldg + f0 + f] : 0.f;
    du[f][t] = in ? static_cast<const float*>(j.du)[t * j.ldg + f0 + f] : 0.f;
  }
  __syncthreads();
}

// The same columns to a row that may start anywhere.
template <bool kEven>
__device__ __forceinline__ void store_part(float* row, int64_t c0, int64_t H, const float (&v)[kColumns]) {
#pragma unroll
  for (int i = 0; i < kColumns; ++i)
    if (column<kEven>(c0, i) < H) row[column<kEven>(c0, i)] = v[i];
}

// A slab's part of dx, [slab][T][H]: the weights' rows go by once.
template <int kTokens, bool kEven>
__global__ void __launch_bounds__(kThreads) ffn_few_dx_kernel(const FfnJob j, float* parts, int slab) {
  __shared__ __align__(16) float dg[kSlab][kTokens], du[kSlab][kTokens];
  const int64_t f0 = int64_t(blockIdx.y) * slab, c0 = int64_t(blockIdx.x) * kBlock;
  const int n = static_cast<int>(min(int64_t(slab), j.F - f0));
  load_slab<kTokens>(j, f0, n, dg, du);
  const float *wg = static_cast<const float*>(j.w_gate) + f0 * j.ldw, *wu = static_cast<const float*>(j.w_up) + f0 * j.ldw;
  float sum[kTokens][kColumns] = {};
#pragma unroll 4
  for (int f = 0; f < n; ++f) {
    float a[kColumns], b[kColumns];
    load_columns<kEven>(wg + f * j.ldw, c0, j.H, a);
    load_columns<kEven>(wu + f * j.ldw, c0, j.H, b);
#pragma unroll
    for (int t = 0; t < kTokens; ++t)
#pragma unroll
      for (int i = 0; i < kColumns; ++i) sum[t][i] = fmaf(dg[f][t], a[i], fmaf(du[f][t], b[i], sum[t][i]));
  }
#pragma unroll
  for (int t = 0; t < kTokens; ++t)
    if (t < j.T) store_part<kEven>(parts + (blockIdx.y * j.T + t) * j.H, c0, j.H, sum[t]);
}

// A job's parts added up, every kQuarters-th by a thread, in a fixed order.
constexpr int kQuarters = 4, kSums = kThreads / kQuarters;
__global__ void __launch_bounds__(kThreads) ffn_sum_kernel(const FfnSum j) {
  __shared__ float sums[kQuarters][kSums];
  const int quarter = threadIdx.x / kSums, at = threadIdx.x % kSums;
  const int64_t all = j.rows * j.len;
  for (int64_t i0 = int64_t(blockIdx.x) * kSums; i0 < all; i0 += int64_t(gridDim.x) * kSums) {
    const int64_t i = i0 + at;
    float s = 0.f;
    if (i < all) {
#pragma unroll 16
      for (int k = quarter; k < j.parts; k += kQuarters) s += j.from[k * j.stride + i];
    }
    sums[quarter][at] = s;
    __syncthreads();
    if (quarter == 0 && i < all) {
#pragma unroll
      for (int q = 1; q < kQuarters; ++q) s += sums[q][at];
      const int64_t r = i / j.len;
      float* to = j.to + r * j.ld + i - r * j.len;
      *to = j.accumulate ? *to + s : s;
    }
    __syncthreads();
  }
}

// A slab's rows of both weights' gradients; the tokens stay in registers.
template <int kTokens, bool kEven>
__global__ void __launch_bounds__(kThreads) ffn_few_dw_kernel(const FfnJob j, int slab) {
  __shared__ __align__(16) float dg[kSlab][kTokens], du[kSlab][kTokens];
  const int64_t f0 = int64_t(blockIdx.y) * slab, c0 = int64_t(blockIdx.x) * kBlock;
  const int n = static_cast<int>(min(int64_t(slab), j.F - f0));
  load_slab<kTokens>(j, f0, n, dg, du);
  float x[kTokens][kColumns];
#pragma unroll
  for (int t = 0; t < kTokens; ++t)
    load_columns<kEven>(static_cast<const float*>(j.x) + min(int64_t(t), j.T - 1) * j.ldx, c0, j.H, x[t]);
  float *og = static_cast<float*>(j.dw_gate) + f0 * j.lddw, *ou = static_cast<float*>(j.dw_up) + f0 * j.lddw;
#pragma unroll 2
  for (int f = 0; f < n; ++f) {
    float a[kColumns] = {}, b[kColumns] = {};
#pragma unroll
    for (int t = 0; t < kTokens; ++t) {
      if (t >= j.T) break;  // 0 times a token again, which may be infinite
#pragma unroll
      for (int i = 0; i < kColumns; ++i) {
        a[i] = fmaf(dg[f][t], x[t][i], a[i]);
        b[i] = fmaf(du[f][t], x[t][i], b[i]);
      }
    }
    if (j.accumulate) {
      float p[kColumns], q[kColumns];
      load_columns<kEven>(og + f * j.lddw, c0, j.H, p);
      load_columns<kEven>(ou + f * j.lddw, c0, j.H, q);
#pragma unroll
      for (int i = 0; i < kColumns; ++i) {
        a[i] += p[i];
        b[i] += q[i];
      }
    }
    store_columns<kEven>(og + f * j.lddw, c0, j.H, a);
    store_columns<kEven>(ou + f * j.lddw, c0, j.H, b);
  }
}

// Features of a CTA: so many that two CTAs an SM have some, for a short sum over slabs.
int slab_of(int64_t H, int64_t F) {
  int slab = kSlab;
  while (slab > 16 && (F + slab - 1) / slab * ((H + kBlock - 1) / kBlock) < int64_t(2) * sm_count()) slab /= 2;
  return slab;
}
int64_t padded(int64_t F) { return (F + 3) / 4 * 4; }

template <int kTokens>
cudaError_t launch_grad(const FfnJob& j, float* parts, cudaStream_t stream) {
  const auto even = [](const void* p, int64_t rows, int64_t ld) { return ffn_rows_on16(p, rows > 1 ? ld : 0, SF_F32); };
  const bool weights = even(j.w_gate, j.F, j.ldw) && even(j.w_up, j.F, j.ldw), tokens = even(j.x, j.T, j.ldx);
  cudaError_t e = launch_rows<float, kTokens, true>(j, weights && tokens, stream);
  const int slab = slab_of(j.H, j.F);
  const int64_t slabs = (j.F + slab - 1) / slab;
  const dim3 grid(static_cast<unsigned>((j.H + kBlock - 1) / kBlock), static_cast<unsigned>(slabs));
  if (e == cudaSuccess && j.dx != nullptr) {
    count_launch();
    if (weights)
      ffn_few_dx_kernel<kTokens, true><<<grid, kThreads, 0, stream>>>(j, parts, slab);
    else
      ffn_few_dx_kernel<kTokens, false><<<grid, kThreads, 0, stream>>>(j, parts, slab);
    e = cudaGetLastError();
    if (e == cudaSuccess)
      e = launch_ffn_sum({parts, j.T * j.H, static_cast<int>(slabs), static_cast<float*>(j.dx), j.T, j.H, j.lddx, false},
                         stream);
  }
  if (e == cudaSuccess && j.dw_gate != nullptr) {
    count_launch();
    if (tokens && even(j.dw_gate, j.F, j.lddw) && even(j.dw_up, j.F, j.lddw))
      ffn_few_dw_kernel<kTokens, true><<<grid, kThreads, 0, stream>>>(j, slab);
    else
      ffn_few_dw_kernel<kTokens, false><<<grid, kThreads, 0, stream>>>(j, slab);
    e = cudaGetLastError();
  }
  return e;
}

}  // namespace

cudaError_t launch_ffn_sum(const FfnSum& j, cudaStream_t stream) {
  const int64_t blocks = (j.rows * j.len + kSums - 1) / kSums;
  count_launch();
  ffn_sum_kernel<<<static_cast<unsigned>(std::min<int64_t>(blocks, int64_t(sm_count()) * 8)), kThreads, 0, stream>>>(j);
  return cudaGetLastError();
}

cudaError_t launch_ffn_few(const FfnJob& j, bool even, cudaStream_t stream) {
  return j.dtype == SF_F32    ? launch_few<float, false>(j, even, stream)
         : j.dtype == SF_BF16 ? launch_few<__nv_bfloat16, false>(j, even, stream)
                              : launch_few<__half, false>(j, even, stream);
}

size_t ffn_few_workspace(int64_t T, int64_t H, int64_t F) {
  const int slab = slab_of(H, F);
  return 4 * (2 * size_t(T) * size_t(padded(F)) + size_t((F + slab - 1) / slab) * size_t(T) * size_t(H));
}

cudaError_t launch_ffn_few_grad(FfnJob j, void* workspace, cudaStream_t stream) {
  j.ldg = padded(j.F);
  j.dg = workspace;
  j.du = static_cast<float*>(workspace) + j.T * j.ldg;
  float* parts = static_cast<float*>(workspace) + 2 * j.T * j.ldg;
  if (j.T == 1) return launch_grad<1>(j, parts, stream);
  if (j.T <= 4) return launch_grad<4>(j, parts, stream);
  return launch_grad<8>(j, parts, stream);
}

}  // namespace sf
