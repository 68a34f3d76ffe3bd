// sf_ffn.cu - the gated feed-forward product h = act(x Wg^T) * (x Wu^T) and its
// gradient (sf_gated_ffn, sf_gated_ffn_grad): what the call launches, and f32 on
// the f32 units (bf16 and f16: sf_ffn_tensor.cu).
//
// Four products of one shape, rows x columns summed over k, by tiles of 128 x 128
// in registers:
//   forward   tokens x features over H; a tile's columns are 64 features of Wg
//             and the same 64 of Wu, so that a thread holds both factors of a
//             value of h
//   inner     the same, turned into dg = dh u act'(g) and du = dh act(g)
//   dx        tokens x H over the features of dg with Wg, then of du with Wu
//   dW        features of dg, then of du, x H over the tokens
// Bound by the multiply-adds: 128 an SM and clock.
#include <algorithm>

#include "sf_ffn_math.cuh"
#include "sf_ffn_tensor.h"

namespace sf {
namespace {

constexpr int kThreads = 256, kTile = 128, kDepth = 16, kHalf = kTile / 2, kRun = 128;
enum Product { kForward, kInner, kDx, kDw };

// Eight values along a row from p, `left` of which exist.
template <typename T>
__device__ __forceinline__ void load8(const T* p, int64_t left, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = i < left ? to_f32(p[i]) : 0.f;
}

template <typename T, int kProduct, int kAct>
__global__ void __launch_bounds__(kThreads) ffn_tile_kernel(const FfnJob j) {
  constexpr bool kGated = kProduct == kForward || kProduct == kInner;
  __shared__ float sa[2][kDepth][kTile + 4], sb[2][kDepth][kTile + 4];
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  const T *x = static_cast<const T*>(j.x), *wg = static_cast<const T*>(j.w_gate), *wu = static_cast<const T*>(j.w_up);
  T *dg = static_cast<T*>(j.dg), *du = static_cast<T*>(j.du);
  const int64_t feature_tiles = (j.F + kTile - 1) / kTile;
  // the tile's first row and column; dW: which of the two matrices
  const bool second = kProduct == kDw && blockIdx.x >= feature_tiles;
  const int64_t r0 = (int64_t(blockIdx.x) - (second ? feature_tiles : 0)) * kTile;
  const int64_t c0 = (int64_t(blockIdx.z) * 65535 + blockIdx.y) * (kGated ? kHalf : kTile);
  const int64_t rows = kProduct == kDw ? j.F : j.T, columns = kGated ? j.F : j.H;
  if (c0 >= columns) return;
  const int64_t per = kProduct == kDx ? j.F : kProduct == kDw ? j.T : j.H;  // the sum's length, for dx of each half
  const int64_t steps = (per + kDepth - 1) / kDepth, all = kProduct == kDx ? 2 * steps : steps;

  // the thread's eight values of each operand: along k of one row, or along the rows of one k
  const int lr = tid >> 1, lk = (tid & 1) * 8, tr = (tid & 15) * 8, tk = tid >> 4;
  float a[8], b[8];
  auto fetch = [&](int64_t step) {
    const bool up = kProduct == kDx && step >= steps;
    const int64_t k = (up ? step - steps : step) * kDepth;
    if constexpr (kProduct == kDw) {
      const int64_t t = k + tk;
      const T* g = second ? du : dg;
      load8(g + t * j.ldg + r0 + tr, t < per ? rows - r0 - tr : 0, a);
      load8(x + t * j.ldx + c0 + tr, t < per ? columns - c0 - tr : 0, b);
    } else {
      const int64_t r = r0 + lr;
      const T* p = kProduct == kDx ? (up ? du : dg) + r * j.ldg : x + r * j.ldx;
      load8(p + k + lk, r < rows ? per - k - lk : 0, a);
      if constexpr (kProduct == kDx) {
        const int64_t f = k + tk;
        load8((up ? wu : wg) + f * j.ldw + c0 + tr, f < per ? columns - c0 - tr : 0, b);
      } else {
        const int64_t f = c0 + (lr & (kHalf - 1));
        load8((lr < kHalf ? wg : wu) + f * j.ldw + k + lk, f < columns ? per - k - lk : 0, b);
      }
    }
  };
  auto stage = [&](int s) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (kProduct == kDw)
        sa[s][tk][tr + i] = a[i];
      else
        sa[s][lk + i][lr] = a[i];
      if (kGated)
        sb[s][lk + i][lr] = b[i];
      else
        sb[s][tk][tr + i] = b[i];
    }
  };

  // a run of kRun products is summed by itself and then added: the roundings of one long
  // chain are twice the error of a sum in pieces
  float sum[8][8], run[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int q = 0; q < 8; ++q) sum[i][q] = run[i][q] = 0.f;
  fetch(0);
  stage(0);
  __syncthreads();
  for (int64_t step = 0; step < all; ++step) {
    const int s = static_cast<int>(step & 1);
    if (step + 1 < all) fetch(step + 1);
#pragma unroll
    for (int k = 0; k < kDepth; ++k) {
      float u[8], v[8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        *reinterpret_cast<float4*>(u + 4 * h) = *reinterpret_cast<const float4*>(&sa[s][k][kHalf * h + 4 * ty]);
        *reinterpret_cast<float4*>(v + 4 * h) = *reinterpret_cast<const float4*>(&sb[s][k][kHalf * h + 4 * tx]);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int q = 0; q < 8; ++q) run[i][q] = fmaf(u[i], v[q], run[i][q]);
    }
    if ((step & (kRun / kDepth - 1)) == kRun / kDepth - 1 || step + 1 == all) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          sum[i][q] += run[i][q];
          run[i][q] = 0.f;
        }
    }
    if (step + 1 < all) stage(s ^ 1);
    __syncthreads();
  }

#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t r = r0 + kHalf * (i >> 2) + 4 * ty + (i & 3);
    if (r >= rows) continue;
    if constexpr (kGated) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {  // columns q of both halves are one feature's g and u
        const int64_t f = c0 + 4 * tx + q;
        if (f >= columns) continue;
        const float g = sum[i][q], u = sum[i][q + 4];
        using A = Activation<kAct, sizeof(T) == 2>;
        if constexpr (kProduct == kForward) {
          static_cast<T*>(j.h)[r * j.ldh + f] = from_f32<T>(A::value(g) * u);
        } else {
          float act, slope;
          A::both(g, act, slope);
          const float d = to_f32(static_cast<const T*>(j.dh)[r * j.lddh + f]);
          if (j.h != nullptr) static_cast<T*>(j.h)[r * j.ldh + f] = from_f32<T>(act * u);
          dg[r * j.ldg + f] = from_f32<T>(d * u * slope);
          du[r * j.ldg + f] = from_f32<T>(d * act);
        }
      }
    } else {
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const int64_t c = c0 + kHalf * (q >> 2) + 4 * tx + (q & 3);
        if (c >= columns) continue;
        float v = sum[i][q];
        if (kProduct == kDx) {
          static_cast<T*>(j.dx)[r * j.lddx + c] = from_f32<T>(v);
        } else if (j.dw_dtype == SF_F32) {
          float* p = static_cast<float*>(second ? j.dw_up : j.dw_gate) + r * j.lddw + c;
          *p = j.accumulate ? *p + v : v;
        } else {
          T* p = static_cast<T*>(second ? j.dw_up : j.dw_gate) + r * j.lddw + c;
          *p = from_f32<T>(j.accumulate ? to_f32(*p) + v : v);
        }
      }
    }
  }
}

// Rows of nothing, for weights without tokens.
__global__ void __launch_bounds__(kThreads) ffn_clear_kernel(char* gate, char* up, int64_t rows, int64_t bytes,
                                                             int64_t pitch) {
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
    for (int64_t i = threadIdx.x * int64_t(2); i < bytes; i += kThreads * 2) {
      *reinterpret_cast<unsigned short*>(gate + r * pitch + i) = 0;
      *reinterpret_cast<unsigned short*>(up + r * pitch + i) = 0;
    }
}

template <typename T, int kProduct>
cudaError_t launch_product(const FfnJob& j, cudaStream_t stream) {
  constexpr bool kGated = kProduct == kForward || kProduct == kInner;
  const int64_t row_tiles = kProduct == kDw ? 2 * ((j.F + kTile - 1) / kTile) : (j.T + kTile - 1) / kTile;
  const int64_t columns = kGated ? (j.F + kHalf - 1) / kHalf : (j.H + kTile - 1) / kTile;
  const dim3 grid(static_cast<unsigned>(row_tiles), static_cast<unsigned>(std::min<int64_t>(columns, 65535)),
                  static_cast<unsigned>((columns + 65534) / 65535));
  count_launch();
  if constexpr (kGated)
    with_activation(j.act, [&](auto act) { ffn_tile_kernel<T, kProduct, act.value><<<grid, kThreads, 0, stream>>>(j); });
  else
    ffn_tile_kernel<T, kProduct, 0><<<grid, kThreads, 0, stream>>>(j);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_type(const FfnJob& j, bool grad, cudaStream_t stream) {
  if (!grad) return launch_product<T, kForward>(j, stream);
  cudaError_t e = launch_product<T, kInner>(j, stream);
  if (e == cudaSuccess && j.dx != nullptr) e = launch_product<T, kDx>(j, stream);
  if (e == cudaSuccess && j.dw_gate != nullptr) e = launch_product<T, kDw>(j, stream);
  return e;
}

// Rows of 16-bit values that start anywhere, copied to rows that start on 16 bytes.
struct Spread {
  const unsigned short* from[3];
  uint4* to[3];
  int64_t rows[3], ld[3];
};
// A warp a run of 128 packs of a row.  A pack's 8 values lie in two of the source's
// 16-byte words; the second is the next lane's first, read once more.
__global__ void __launch_bounds__(kThreads) ffn_spread_kernel(const __grid_constant__ Spread s, int64_t len, int packs,
                                                              int runs) {
  griddep_launch_dependents();
  const int part = blockIdx.y, lane = threadIdx.x & 31;
  const int64_t all = s.rows[part] * runs, step = int64_t(gridDim.x) * (kThreads / 32);
  const int64_t last = s.rows[part] * int64_t(s.ld[part]) - (s.ld[part] - len);  // values from the first to the last
  for (int64_t i = int64_t(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5); i < all; i += step) {
    const int64_t r = i / runs;
    const int run = static_cast<int>(i - r * runs);
    const unsigned short* row = s.from[part] + r * s.ld[part];
    const int off = static_cast<int>(reinterpret_cast<uintptr_t>(row) >> 1 & 7u);
    uint4* to = s.to[part] + r * packs;
#pragma unroll 4
    for (int p = run * 128 + lane; p < min(packs, run * 128 + 128); p += 32) {
      const int64_t c = int64_t(p) * 8;
      const int64_t at = r * s.ld[part] + c - off;  // of the first word
      uint32_t w[9] = {0};
      if (at >= 0 && at + 16 <= last) {
        const uint4 a = load16(row + c - off), b = off != 0 ? load16(row + c - off + 8) : a;
        w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
        w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
        // by `off` values: whole words, then half a word
        const int words = off >> 1;
#pragma unroll
        for (int k = 0; k < 5; ++k) w[k] = words == 0 ? w[k] : words == 1 ? w[k + 1] : words == 2 ? w[k + 2] : w[min(k + 3, 8)];
        if (off & 1) {
#pragma unroll
          for (int k = 0; k < 4; ++k) w[k] = __funnelshift_r(w[k], w[k + 1], 16);
        }
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t lo = c + 2 * k < len ? row[c + 2 * k] : 0u, hi = c + 2 * k + 1 < len ? row[c + 2 * k + 1] : 0u;
          w[k] = lo | hi << 16;
        }
      }
      to[p] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}

size_t value_size(int32_t dtype) { return dtype == SF_F32 ? 4 : 2; }
size_t round16(size_t n) { return (n + 15) & ~size_t(15); }

}  // namespace

bool ffn_rows_on16(const void* p, int64_t ld, int32_t dtype) {
  return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (ld * int64_t(value_size(dtype))) % 16 == 0;
}

size_t ffn_workspace(int32_t dtype, int64_t T, int64_t H, int64_t F, bool aligned, bool grad) {
  const size_t inner = grad ? 2 * size_t(T) * round16(size_t(F) * value_size(dtype)) : 0;
  return inner + (dtype == SF_F32 || aligned ? 0 : size_t(T + 2 * F) * round16(size_t(H) * 2));
}

cudaError_t launch_ffn(FfnJob j, bool grad, void* workspace, cudaStream_t stream) {
  if (j.T == 0) {
    if (j.dw_gate == nullptr || j.accumulate) return cudaSuccess;
    const int64_t size = value_size(j.dw_dtype);
    count_launch();
    ffn_clear_kernel<<<static_cast<unsigned>(std::min<int64_t>(j.F, sm_count() * 8)), kThreads, 0, stream>>>(
        static_cast<char*>(j.dw_gate), static_cast<char*>(j.dw_up), j.F, j.H * size, j.lddw * size);
    return cudaGetLastError();
  }
  const size_t size = value_size(j.dtype), row = round16(size_t(j.F) * size);
  char* at = static_cast<char*>(workspace);
  if (grad) {
    j.dg = at;
    j.du = at + size_t(j.T) * row;
    j.ldg = int64_t(row / size);
    at += 2 * size_t(j.T) * row;
  }
  if (j.dtype == SF_F32) return launch_type<float>(j, grad, stream);
  if (!ffn_rows_on16(j.x, j.T > 1 ? j.ldx : 0, j.dtype) || !ffn_rows_on16(j.w_gate, j.F > 1 ? j.ldw : 0, j.dtype) ||
      !ffn_rows_on16(j.w_up, j.F > 1 ? j.ldw : 0, j.dtype)) {
    const int64_t packs = int64_t(round16(size_t(j.H) * 2) / 16);
    Spread s;
    const void** data[3] = {&j.x, &j.w_gate, &j.w_up};
    for (int i = 0; i < 3; ++i) {
      s.from[i] = static_cast<const unsigned short*>(*data[i]);
      s.to[i] = reinterpret_cast<uint4*>(at);
      s.rows[i] = i == 0 ? j.T : j.F;
      s.ld[i] = i == 0 ? j.ldx : j.ldw;
      *data[i] = at;
      at += size_t(s.rows[i]) * packs * 16;
    }
    const int64_t runs = (packs + 127) / 128, most = (std::max(j.T, j.F) * runs + kThreads / 32 - 1) / (kThreads / 32);
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>(most, int64_t(sm_count()) * 8)), 3);
    count_launch();
    ffn_spread_kernel<<<grid, kThreads, 0, stream>>>(s, j.H, static_cast<int>(packs), static_cast<int>(runs));
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    j.ldx = j.ldw = packs * 8;
  }
  return launch_ffn_tensor(j, grad, stream);
}

}  // namespace sf
