// sf_dropout.cu - dropout with a mask from a counter-based generator
// (sf_dropout): out = residual + (kept ? x / (1 - p) : 0).
//
// The mask of 8 neighbouring columns is one call of Philox4x32-10 (Salmon,
// Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", SC11) on
// (pack, row, offset) under the seed: 16 bits a column, ten rounds of two 32-bit
// products.  Nothing of it is stored; a backward pass computes it again.  Each
// value is read and written once.  Bound by memory with a residual (16384 x 8192
// bf16: 118 to 123 us, 97 to 100 % of the copy rate) and by the integer units without
// (102 to 105 us, 75 to 78 %): some 160 instructions for 8 columns, of which the generator is 40 and the 8
// decisions with their selects 20.  CTAs of 128 threads: those of 256 take 138 and
// 107 us (whole CTAs fit the registers worse), 32 an SM in turn.
#include <algorithm>

#include "sf_float.cuh"
#include "sf_launch.h"

namespace sf {
namespace {

constexpr int kThreads = 128, kCols = 8, kTurns = 2, kRounds = 10, kPerSm = 32;

// The generator's keys of each round, in shared memory: they depend on the call
// alone, and a read for all lanes takes no slot of the integer units.
struct Keys {
  uint2 round[kRounds];
  uint2 offset;
};
__device__ __forceinline__ void load_keys(Keys& keys, const uint64_t* key) {
  if (threadIdx.x == 0) {
    const uint64_t seed = key[0], offset = key[1];
    uint32_t k0 = static_cast<uint32_t>(seed), k1 = static_cast<uint32_t>(seed >> 32);
    for (int r = 0; r < kRounds; ++r) {
      keys.round[r] = make_uint2(k0, k1);
      k0 += 0x9E3779B9u;
      k1 += 0xBB67AE85u;
    }
    keys.offset = make_uint2(static_cast<uint32_t>(offset), static_cast<uint32_t>(offset >> 32));
  }
  __syncthreads();
}

// Ten rounds for K counters; the multipliers and the keys' increments are the paper's.
template <int K>
__device__ __forceinline__ void philox(const uint32_t (&pack)[K], const uint32_t (&row)[K], const Keys& keys,
                                       uint4 (&c)[K]) {
  const uint2 o = keys.offset;
#pragma unroll
  for (int k = 0; k < K; ++k) c[k] = make_uint4(pack[k], row[k], o.x, o.y);
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const uint2 key = keys.round[r];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint64_t a = uint64_t(c[k].x) * 0xD2511F53u, b = uint64_t(c[k].z) * 0xCD9E8D57u;
      c[k] = make_uint4(static_cast<uint32_t>(b >> 32) ^ c[k].y ^ key.x, static_cast<uint32_t>(b),
                        static_cast<uint32_t>(a >> 32) ^ c[k].w ^ key.y, static_cast<uint32_t>(a));
    }
  }
}
__device__ __forceinline__ uint4 philox(uint32_t pack, uint32_t row, const Keys& keys) {
  const uint32_t p[1] = {pack}, r[1] = {row};
  uint4 w[1];
  philox(p, r, keys, w);
  return w[0];
}

// Whether column q of the pack is kept: its 16 bits are not below the threshold, which
// `high` holds in its upper half.  (All dropped, 65536 of 65536: the caller's to see.)
__device__ __forceinline__ bool keeps(const uint4& w, int q, uint32_t high) {
  const uint32_t v = q < 2 ? w.x : q < 4 ? w.y : q < 6 ? w.z : w.w;
  return (q & 1 ? v : v << 16) >= high;
}
// Bit j: column j of the pack is kept.
__device__ __forceinline__ uint32_t kept(const uint4& w, uint32_t high) {
  uint32_t m = 0;
#pragma unroll
  for (int q = 0; q < kCols; ++q) m |= keeps(w, q, high) ? 1u << q : 0u;
  return m;
}

// The rounded result: the product and the sum are rounded in f32 as written, then to T.
template <bool kResidual>
__device__ __forceinline__ float masked(float x, float r, bool keep, float scale) {
  const float v = __fmul_rn(x, scale);
  if (kResidual) return keep ? __fadd_rn(v, r) : r;
  return keep ? v : 0.f;
}

// A row's values that lie before its first 16-byte boundary's pack: `off` values
// behind a boundary, the same for all three rows.
template <typename T>
__device__ __forceinline__ int row_off(const DropoutJob& j, int64_t row) {
  return static_cast<int>(((reinterpret_cast<uintptr_t>(j.x) / sizeof(T)) + uint64_t(row) * uint64_t(j.ldx)) %
                          uint64_t(Pack<T>::kN));
}

// The columns from c of a row of D that exist.
template <typename T, int P>
__device__ __forceinline__ void load_some(const T* row, int64_t c, int64_t D, uint4 (&u)[P]) {
  constexpr int N = Pack<T>::kN;
#pragma unroll
  for (int q = 0; q < P * N; ++q)
    reinterpret_cast<T*>(&u[q / N])[q % N] = c + q >= 0 && c + q < D ? row[c + q] : from_f32<T>(0.f);
}

// How a warp's lanes lie on the packs: `lanes` (a power of two) side by side in a row, 32 / lanes
// rows below one another; the next of its kTurns turns is `packs_on` packs or `rows_on` rows further.
struct Tile {
  int shift;  // lanes = 1 << shift
  int packs_on, rows_on;
  int64_t rows, per_row, all;  // rows of a tile, tiles of a row, tiles
};

// Rows that start at the same distance from a 16-byte boundary in x, residual and
// out (kShift: not 0 in every row): a thread takes 8 columns between boundaries.
// Where a row starts `off` values behind a boundary its 8 columns lie in two packs of
// the mask: the lane before has the other.  The generator serves all turns of a warp at once.
template <typename T, bool kResidual, bool kShift>
__global__ void __launch_bounds__(kThreads) dropout_pack_kernel(const DropoutJob j, const Tile t) {
  constexpr int N = Pack<T>::kN, P = kCols / N;  // 16-byte packs of a thread
  __shared__ Keys keys;
  load_keys(keys, j.key);
  const int lane = threadIdx.x & 31, in_row = lane & ((1 << t.shift) - 1), below = lane >> t.shift;
  const int packs = static_cast<int>((j.D + (kShift ? N - 1 : 0) + kCols - 1) / kCols);
  const int64_t D = j.D;
  const T *x = static_cast<const T*>(j.x), *res = static_cast<const T*>(j.residual);
  T* out = static_cast<T*>(j.out);
  const int64_t step = int64_t(gridDim.x) * (kThreads / 32);
  const int64_t first = int64_t(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5);
  int64_t tile_row = first / t.per_row, seg = first - tile_row * t.per_row;
  const int64_t rows_step = step / t.per_row, seg_step = step - rows_step * t.per_row;
  for (int64_t tile = first; tile < t.all; tile += step) {
    const int64_t row0 = tile_row * t.rows + below;
    const int at0 = static_cast<int>(seg) * (kTurns * 32) + in_row;
    uint32_t rows[kTurns], ats[kTurns];
    int off[kTurns];
    int64_t c[kTurns];
    bool mine[kTurns], whole[kTurns];
    uint4 u[kTurns][P], v[kTurns][P], w[kTurns];
#pragma unroll
    for (int k = 0; k < kTurns; ++k) {
      const int64_t row = row0 + k * t.rows_on;
      const int at = at0 + k * t.packs_on;
      rows[k] = static_cast<uint32_t>(row);
      ats[k] = static_cast<uint32_t>(at);
      off[k] = kShift ? row_off<T>(j, row) : 0;
      c[k] = int64_t(at) * kCols - off[k];
      mine[k] = row < j.N && at < packs;
      whole[k] = mine[k] && c[k] >= 0 && c[k] + kCols <= D;
      if (whole[k]) {
#pragma unroll
        for (int p = 0; p < P; ++p) u[k][p] = load16(x + row * j.ldx + c[k] + p * N);
        if (kResidual) {
#pragma unroll
          for (int p = 0; p < P; ++p) v[k][p] = load16(res + row * j.ldr + c[k] + p * N);
        }
      } else if (mine[k]) {
        load_some(x + row * j.ldx, c[k], D, u[k]);
        if (kResidual) load_some(res + row * j.ldr, c[k], D, v[k]);
      }
    }
    philox(ats, rows, keys, w);
    uint32_t last = 0;  // the mask of the turn before
#pragma unroll
    for (int k = 0; k < kTurns; ++k) {
      uint32_t m = 0;
      if (kShift) {
        const uint32_t own = kept(w[k], j.high);
        uint32_t before = __shfl_up_sync(kFull, own, 1);
        const uint32_t end = __shfl_sync(kFull, last, 31);
        if (lane == 0) before = k > 0 ? end : kept(philox(ats[k] - 1, rows[k], keys), j.high);
        last = own;
        m = before >> (kCols - off[k]) | own << off[k];  // at a row's start columns before it, which are not stored
      }
      if (!mine[k]) continue;
      T* to = out + (row0 + k * t.rows_on) * j.ldo + c[k];
#pragma unroll
      for (int p = 0; p < P; ++p) {
        float f[N], g[N];
        unpack(u[k][p], f, T());
        if (kResidual) unpack(v[k][p], g, T());
#pragma unroll
        for (int q = 0; q < N; ++q)
          f[q] = masked<kResidual>(f[q], kResidual ? g[q] : 0.f,
                                   kShift ? m >> (p * N + q) & 1u : keeps(w[k], p * N + q, j.high), j.scale);
        u[k][p] = pack(f, T());
      }
      if (whole[k]) {
#pragma unroll
        for (int p = 0; p < P; ++p) store16(to + p * N, u[k][p]);
      } else {
#pragma unroll
        for (int q = 0; q < kCols; ++q)
          if (c[k] + q >= 0 && c[k] + q < D) to[q] = reinterpret_cast<const T*>(&u[k][q / N])[q % N];
      }
    }
    tile_row += rows_step;
    seg += seg_step;
    if (seg >= t.per_row) {
      seg -= t.per_row;
      ++tile_row;
    }
  }
}

// Any alignment: a warp takes 256 columns of a row.  Each lane computes the mask
// of one pack, and column 32 i + lane gets its bit from the lane of its pack, so
// that the lanes' elements lie side by side.  Bound by the instructions of single values:
// 16384 x 8192 bf16 with residual 183 us (119 at the copy rate), without 149 (79); f32 has
// half as many a byte, 4099 x 5001 40 us (36) and 31 (24).
template <typename T, bool kResidual>
__global__ void __launch_bounds__(kThreads) dropout_lane_kernel(const DropoutJob j) {
  __shared__ Keys keys;
  load_keys(keys, j.key);
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
        j.none ? 0u : kept(philox(static_cast<uint32_t>(at * 32 + lane), static_cast<uint32_t>(row), keys), j.high);
#pragma unroll
    for (int i = 0; i < kCols; ++i) {
      const uint32_t bits = __shfl_sync(kFull, m, 4 * i + lane / 8);
      if (c + 32 * i < j.D) po[32 * i] = from_f32<T>(masked<kResidual>(f[i], g[i], bits >> (lane & 7) & 1u, j.scale));
    }
    row += rows_on;
    at += at_on;
    if (at >= blocks) {
      at -= blocks;
      ++row;
    }
  }
}

template <typename T, bool kResidual>
cudaError_t launch_rows(const DropoutJob& j, cudaStream_t stream) {
  const auto off = [](const void* p) { return reinterpret_cast<uintptr_t>(p) & 15u; };
  const auto pitch = [](int64_t ld) { return uint64_t(ld) * sizeof(T) & 15u; };
  const bool alike = off(j.x) == off(j.out) && (!kResidual || off(j.x) == off(j.residual)) &&
                     (j.N == 1 || (pitch(j.ldx) == pitch(j.ldo) && (!kResidual || pitch(j.ldx) == pitch(j.ldr))));
  const bool even = alike && off(j.x) == 0 && (j.N == 1 || pitch(j.ldx) == 0);
  if (!alike || j.none) {
    const int64_t work = j.N * ((j.D + 255) / 256) * 32;
    const int64_t grid = std::min<int64_t>((work + kThreads - 1) / kThreads, int64_t(sm_count()) * kPerSm);
    count_launch();
    dropout_lane_kernel<T, kResidual><<<static_cast<unsigned>(grid), kThreads, 0, stream>>>(j);
    return cudaGetLastError();
  }
  const int64_t packs = (j.D + (even ? 0 : Pack<T>::kN - 1) + kCols - 1) / kCols;
  Tile t;
  t.shift = 0;
  while (t.shift < 5 && (1 << t.shift) < packs) ++t.shift;
  const bool wide = packs > 32;
  t.packs_on = wide ? 32 : 0;
  t.rows_on = wide ? 0 : 32 >> t.shift;
  t.rows = wide ? 1 : kTurns * t.rows_on;
  t.per_row = wide ? (packs + kTurns * 32 - 1) / (kTurns * 32) : 1;
  t.all = (j.N + t.rows - 1) / t.rows * t.per_row;
  const int64_t grid = std::min<int64_t>((t.all + kThreads / 32 - 1) / (kThreads / 32), int64_t(sm_count()) * kPerSm);
  count_launch();
  if (even)
    dropout_pack_kernel<T, kResidual, false><<<static_cast<unsigned>(grid), kThreads, 0, stream>>>(j, t);
  else
    dropout_pack_kernel<T, kResidual, true><<<static_cast<unsigned>(grid), kThreads, 0, stream>>>(j, t);
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
