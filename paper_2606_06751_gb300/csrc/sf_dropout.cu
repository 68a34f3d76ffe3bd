// sf_dropout.cu - dropout with a mask from a counter-based generator
// (sf_dropout): out = residual + (kept ? x / (1 - p) : 0).
//
// The mask of 8 neighbouring columns is one call of Philox4x32-10 (Salmon,
// Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", SC11) on
// (pack, row, offset) under the seed: 16 bits a column, ten rounds of two 32-bit
// products.  Nothing of it is stored; a backward pass computes it again.  Each
// value is read and written once: bound by memory, with the generator's some 60
// integer instructions for 8 columns behind it.
#include <algorithm>

#include "sf_float.cuh"
#include "sf_launch.h"

namespace sf {
namespace {

constexpr int kThreads = 256, kCols = 8;

struct Key {
  uint32_t k0, k1, o0, o1;
};

__device__ __forceinline__ Key load_key(const uint64_t* key) {
  const uint64_t seed = key[0], offset = key[1];
  return {static_cast<uint32_t>(seed), static_cast<uint32_t>(seed >> 32), static_cast<uint32_t>(offset),
          static_cast<uint32_t>(offset >> 32)};
}

// Ten rounds; the multipliers and the key's increments are the paper's.
__device__ __forceinline__ uint4 philox(uint32_t pack, uint32_t row, const Key& key) {
  uint32_t c0 = pack, c1 = row, c2 = key.o0, c3 = key.o1, k0 = key.k0, k1 = key.k1;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = uint64_t(c0) * 0xD2511F53u, b = uint64_t(c2) * 0xCD9E8D57u;
    const uint32_t n0 = static_cast<uint32_t>(b >> 32) ^ c1 ^ k0, n2 = static_cast<uint32_t>(a >> 32) ^ c3 ^ k1;
    c0 = n0;
    c1 = static_cast<uint32_t>(b);
    c2 = n2;
    c3 = static_cast<uint32_t>(a);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return make_uint4(c0, c1, c2, c3);
}

// Bit j: column j of the pack is kept.
__device__ __forceinline__ uint32_t kept(const uint4& w, uint32_t t) {
  const uint32_t v[4] = {w.x, w.y, w.z, w.w};
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m |= ((v[i] & 0xffffu) >= t ? 1u : 0u) << (2 * i);
    m |= ((v[i] >> 16) >= t ? 1u : 0u) << (2 * i + 1);
  }
  return m;
}

// The rounded result: the product and the sum are rounded in f32 as written, then to T.
__device__ __forceinline__ float masked(float x, float r, bool keep, float scale) {
  return __fadd_rn(keep ? __fmul_rn(x, scale) : 0.f, r);
}

// Rows whose packs of 8 columns are all 16-byte aligned: a thread a pack, the
// packs of all rows one after another.
template <typename T, bool kResidual>
__global__ void __launch_bounds__(kThreads) dropout_pack_kernel(const DropoutJob j) {
  constexpr int N = Pack<T>::kN, P = kCols / N;  // 16-byte packs of a thread
  const Key key = load_key(j.key);
  const int64_t packs = (j.D + kCols - 1) / kCols, step = int64_t(gridDim.x) * kThreads;
  const int64_t first = int64_t(blockIdx.x) * kThreads + threadIdx.x;
  int64_t row = first / packs, at = first - row * packs;
  const int64_t rows_on = step / packs, at_on = step - rows_on * packs;
  const T *x = static_cast<const T*>(j.x), *res = static_cast<const T*>(j.residual);
  T* out = static_cast<T*>(j.out);
  while (row < j.N) {
    const int64_t c = at * kCols;
    const T *px = x + row * j.ldx + c, *pr = res + row * j.ldr + c;
    T* po = out + row * j.ldo + c;
    if (c + kCols <= j.D) {
      uint4 u[P], v[P];
#pragma unroll
      for (int p = 0; p < P; ++p) u[p] = load16(px + p * N);
      if (kResidual) {
#pragma unroll
        for (int p = 0; p < P; ++p) v[p] = load16(pr + p * N);
      }
      const uint32_t m = kept(philox(static_cast<uint32_t>(at), static_cast<uint32_t>(row), key), j.threshold);
#pragma unroll
      for (int p = 0; p < P; ++p) {
        float f[N], g[N];
        unpack(u[p], f, T());
        if (kResidual) unpack(v[p], g, T());
#pragma unroll
        for (int q = 0; q < N; ++q) f[q] = masked(f[q], kResidual ? g[q] : 0.f, m >> (p * N + q) & 1u, j.scale);
        store16(po + p * N, pack(f, T()));
      }
    } else {
      const uint32_t m = kept(philox(static_cast<uint32_t>(at), static_cast<uint32_t>(row), key), j.threshold);
      for (int q = 0; c + q < j.D; ++q)
        po[q] = from_f32<T>(masked(to_f32(px[q]), kResidual ? to_f32(pr[q]) : 0.f, m >> q & 1u, j.scale));
    }
    row += rows_on;
    at += at_on;
    if (at >= packs) {
      at -= packs;
      ++row;
    }
  }
}

// Any alignment: a warp takes 256 columns of a row.  Each lane computes the mask
// of one pack, and column 32 i + lane gets its bit from the lane of its pack, so
// that the lanes' elements lie side by side.
template <typename T, bool kResidual>
__global__ void __launch_bounds__(kThreads) dropout_lane_kernel(const DropoutJob j) {
  const Key key = load_key(j.key);
  const int lane = threadIdx.x & 31;
  const int64_t blocks = (j.D + 255) / 256, step = int64_t(gridDim.x) * (kThreads / 32);
  const int64_t first = int64_t(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5);
  int64_t row = first / blocks, at = first - row * blocks;
  const int64_t rows_on = step / blocks, at_on = step - rows_on * blocks;
  const T *x = static_cast<const T*>(j.x), *res = static_cast<const T*>(j.residual);
  T* out = static_cast<T*>(j.out);
  while (row < j.N) {
    const int64_t c = at * 256 + lane;
    const T *px = x + row * j.ldx + c, *pr = res + row * j.ldr + c;
    T* po = out + row * j.ldo + c;
    float f[kCols], g[kCols];
#pragma unroll
    for (int i = 0; i < kCols; ++i) {
      f[i] = c + 32 * i < j.D ? to_f32(px[32 * i]) : 0.f;
      g[i] = kResidual && c + 32 * i < j.D ? to_f32(pr[32 * i]) : 0.f;
    }
    const uint32_t m =
        kept(philox(static_cast<uint32_t>(at * 32 + lane), static_cast<uint32_t>(row), key), j.threshold);
#pragma unroll
    for (int i = 0; i < kCols; ++i) {
      const uint32_t bits = __shfl_sync(kFull, m, 4 * i + lane / 8);
      if (c + 32 * i < j.D) po[32 * i] = from_f32<T>(masked(f[i], g[i], bits >> (lane & 7) & 1u, j.scale));
    }
    row += rows_on;
    at += at_on;
    if (at >= blocks) {
      at -= blocks;
      ++row;
    }
  }
}

bool on16(const void* p, int64_t ld, size_t size) {
  return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld * static_cast<int64_t>(size) % 16 == 0;
}

template <typename T, bool kResidual>
cudaError_t launch_rows(const DropoutJob& j, cudaStream_t stream) {
  const bool even = on16(j.x, j.ldx, sizeof(T)) && on16(j.out, j.ldo, sizeof(T)) &&
                    (!kResidual || on16(j.residual, j.ldr, sizeof(T)));
  const int64_t work = even ? j.N * ((j.D + kCols - 1) / kCols) : j.N * ((j.D + 255) / 256) * 32;
  const int64_t grid = std::min<int64_t>((work + kThreads - 1) / kThreads, int64_t(sm_count()) * 8);
  count_launch();
  if (even)
    dropout_pack_kernel<T, kResidual><<<static_cast<unsigned>(grid), kThreads, 0, stream>>>(j);
  else
    dropout_lane_kernel<T, kResidual><<<static_cast<unsigned>(grid), kThreads, 0, stream>>>(j);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_type(const DropoutJob& j, cudaStream_t stream) {
  return j.residual != nullptr ? launch_rows<T, true>(j, stream) : launch_rows<T, false>(j, stream);
}

}  // namespace

cudaError_t launch_dropout(const DropoutJob& j, cudaStream_t stream) {
  return j.dtype == SF_F32    ? launch_type<float>(j, stream)
         : j.dtype == SF_BF16 ? launch_type<__nv_bfloat16>(j, stream)
                              : launch_type<__half>(j, stream);
}

}  // namespace sf
