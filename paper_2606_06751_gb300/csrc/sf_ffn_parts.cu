// sf_ffn_parts.cu - the gated feed-forward operators in f32 on the tensor cores.
//
// An f32 of 2^-109 or more is the sum of three bf16 (a1 its upper half, a2 and a3 what is left), so that
//   a b = a1 b1 + (a1 b2 + a2 b1) + (a2 b2 + a1 b3 + a3 b1)     to some 2^-24 of it,
// six products of bf16 at 16 times the f32 units' rate or more.  The tensor cores
// cut their f32 sums off instead of rounding them, by up to 2^-23 each time: a1 b1 and
// the rest are summed apart, so that the small terms lose nothing to the large ones, and
// runs of 256 k are summed there and the runs' sums in registers, rounded to nearest.
// The error is below that of one f32 chain over k.  An infinite input has parts
// (inf, 0, 0) and makes NaN where it meets a part that is 0.
//
// The parts are made first (4 bytes read, 6 written for a value), products as in
// sf_ffn_tensor.cu: 256 x 128 tiles of D by pairs of SMs.  A block of 64 k is 72 KB of
// parts an SM and 24 products of 16 k: bound by the tensor cores, six times the work
// of bf16 (2048 x 2048 x 4096 279 us, 246 TFLOP/s of f32 products; the parts 31 of them).
#include <algorithm>

#include "sf_ffn_tensor.h"
#include "sf_ffn_tiles.cuh"

namespace sf {
namespace {

constexpr int kThreads = 256;
constexpr int kGroups = 2, kStoreWarps = 4 * kGroups, kPairThreads = 128 + 32 * kStoreWarps;
constexpr int kMostN = 128, kRun = 4, kMaxStages = 6;  // kRun blocks of 64 k are summed at once
constexpr int kSwapBytes = kGroups * 4 * 8 * 32 * 4;    // groups, quadrants, columns, lanes

// ---------------------------------------------------------------- the parts

struct Sources {
  const float* from[3];
  __nv_bfloat16* to[3];
  int64_t rows[3], ld[3];
};

// A warp 256 columns of a row at a time.
__global__ void __launch_bounds__(kThreads) ffn_parts_of_kernel(const __grid_constant__ Sources s, int64_t len, int packs,
                                                               int runs) {
  griddep_launch_dependents();
  const int part = blockIdx.y, lane = threadIdx.x & 31;
  const int64_t all = s.rows[part] * runs, step = int64_t(gridDim.x) * (kThreads / 32);
  const int64_t pitch = int64_t(packs) * 8, next = s.rows[part] * pitch;
  const bool even = ((reinterpret_cast<uintptr_t>(s.from[part]) | uint64_t(s.ld[part]) * 4) & 15u) == 0;
  for (int64_t i = int64_t(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5); i < all; i += step) {
    const int64_t r = i / runs;
    const int p = static_cast<int>(i - r * runs) * 32 + lane;
    if (p >= packs) continue;
    const float* row = s.from[part] + r * s.ld[part];
    const int64_t c = int64_t(p) * 8;
    float v[8];
    if (even && c + 8 <= len) {
      unpack(load16(row + c), reinterpret_cast<float(&)[4]>(v[0]), 0.f);
      unpack(load16(row + c + 4), reinterpret_cast<float(&)[4]>(v[4]), 0.f);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = c + k < len ? row[c + k] : 0.f;
    }
    uint4 u[3];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      __nv_bfloat16 q[3];
      parts_of(v[k], q);
#pragma unroll
      for (int n = 0; n < 3; ++n) reinterpret_cast<__nv_bfloat16*>(&u[n])[k] = q[n];
    }
#pragma unroll
    for (int n = 0; n < 3; ++n) *reinterpret_cast<uint4*>(s.to[part] + n * next + r * pitch + c) = u[n];
  }
}

// ---------------------------------------------------------------- the products

struct Maps {
  CUtensorMap a0, a1, b0, b1;  // (column, row, part)
};

struct Shape {
  int64_t m_tiles, n_tiles;  // dW: n tiles of one of the two matrices
  int N, stages;
  int blocks, half;  // blocks of 64 k; dx: those of the first half
  int splits;        // dx, dW: ways in which the blocks of a tile are shared out; else 1
  float* sums;       // [splits][T][H] or [splits][2][F][H] where splits > 1
};

// A split's blocks.
__device__ __forceinline__ void blocks_of(const Shape& s, int split, int& first, int& last) {
  first = static_cast<int>(int64_t(s.blocks) * split / s.splits);
  last = static_cast<int>(int64_t(s.blocks) * (split + 1) / s.splits);
}

__device__ __forceinline__ void part_copy(uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y, int32_t part,
                                          uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2"
      " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(part), "r"(bar)
      : "memory");
}

template <int kProduct>
__device__ __forceinline__ void copy_parts(const Maps& maps, const Shape& s, int kb, int m, int n, bool second,
                                           uint32_t a, uint32_t b, uint32_t b_bytes, uint32_t bar) {
  const bool up = kProduct == kDx && kb >= s.half;
  const int k = (up ? kb - s.half : kb) * kBox;
  for (int p = 0; p < 3; ++p, a += kABytes, b += b_bytes) {
    if constexpr (Layout<kProduct>::kGated) {
      part_copy(a, &maps.a0, k, m, p, bar);
      part_copy(a + kBoxBytes, &maps.a1, k, m, p, bar);
      part_copy(b, &maps.b0, k, n, p, bar);
    } else {
      const CUtensorMap* w = up ? &maps.a1 : &maps.a0;
      part_copy(a, w, m, k, p, bar);
      part_copy(a + kBoxBytes, w, m + kBox, k, p, bar);
      if (kProduct == kDx)
        part_copy(b, up ? &maps.b1 : &maps.b0, k, n, p, bar);
      else
        part_copy(b, second ? &maps.b1 : &maps.b0, n, k, p, bar);
    }
  }
}

// A block's products: a1 b1 to `d`, the five smaller ones 128 columns further.
template <int kProduct>
__device__ __forceinline__ void multiply_parts(uint32_t d, uint32_t a, uint32_t b, uint32_t b_bytes, uint32_t desc,
                                               bool first) {
  using L = Layout<kProduct>;
#pragma unroll
  for (int k = 0; k < kBox / 16; ++k) {
    uint64_t x[3], y[3];
#pragma unroll
    for (int p = 0; p < 3; ++p) {
      x[p] = operand_of<L::kAAlongK>(a + p * kABytes + k * kStepBytes<L::kAAlongK>);
      y[p] = operand_of<L::kBAlongK>(b + p * b_bytes + k * kStepBytes<L::kBAlongK>);
    }
    const bool add = !(first && k == 0);
    tensor_product<2>(d, x[0], y[0], desc, add);
    tensor_product<2>(d + kMostN, x[0], y[2], desc, add);
    tensor_product<2>(d + kMostN, x[2], y[0], desc, true);
    tensor_product<2>(d + kMostN, x[1], y[1], desc, true);
    tensor_product<2>(d + kMostN, x[0], y[1], desc, true);
    tensor_product<2>(d + kMostN, x[1], y[0], desc, true);
  }
}

// Persistent pairs of CTAs.  Warp 0 copies, warp 1 of the pair's first CTA multiplies,
// warps from 4 add up the runs of a tile and store it, each 16 of every 32 columns.
template <int kProduct>
__global__ void __launch_bounds__(kPairThreads, 1) __cluster_dims__(2, 1, 1)
    ffn_parts_kernel(const __grid_constant__ Maps maps, const FfnJob j, const Shape s) {
  using L = Layout<kProduct>;
  extern __shared__ unsigned char raw[];
  __shared__ uint64_t full[kMaxStages], empty[kMaxStages], sums_full[2], sums_empty[2];
  __shared__ uint32_t tensor_at;
  __shared__ int abort;
  unsigned char* base = align_1024(raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t rank = cluster_rank();
  const int half_n = s.N / 2;
  const uint32_t b_bytes = uint32_t(half_n) * kDepthBytes, stage_bytes = 3 * (kABytes + b_bytes);
  // the splits of a tile one after another: they run at once
  const int64_t tiles = s.m_tiles * s.n_tiles * (kProduct == kDw ? 2 : 1) * s.splits;
  const int64_t pairs = gridDim.x / 2;

  if (tid == 0) {
    prefetch_tensormap(&maps.a0);
    prefetch_tensormap(&maps.a1);
    prefetch_tensormap(&maps.b0);
    prefetch_tensormap(&maps.b1);
    abort = 0;
    for (int i = 0; i < s.stages; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sums_full[i], 1);
      mbar_init(&sums_empty[i], 2 * kStoreWarps);
    }
    fence_barrier_init();
  }
  if (warp == 2) tensor_alloc<2>(&tensor_at, 512);
  griddep_launch_dependents();
  tensor_fence_before();
  cluster_sync();
  tensor_fence_after();
  griddep_wait();
  const uint32_t sums = tensor_at;

  if (warp == 0) {
    if (lane == 0) {
      int stage = 0;
      uint32_t parity = 1;
      bool ok = true;
      for (int64_t tile = blockIdx.x / 2; ok && tile < tiles; tile += pairs) {
        int64_t m, n;
        bool second;
        tile_of<kProduct>(tile / s.splits, s.m_tiles, s.n_tiles, s.N, m, n, second);
        int first, last;
        blocks_of(s, static_cast<int>(tile % s.splits), first, last);
        for (int kb = first; kb < last; ++kb) {
          ok = mbar_wait_bounded(&empty[stage], parity, &abort);
          if (!ok) break;
          const uint32_t a = smem_u32(base) + stage * stage_bytes;
          if (rank == 0) mbar_arrive_expect_tx(&full[stage], 2 * stage_bytes);
          copy_parts<kProduct>(maps, s, kb, static_cast<int>(m + rank * L::kRows), static_cast<int>(n + rank * half_n),
                               second, a, a + 3 * kABytes, b_bytes, at_rank(&full[stage], 0));
          if (++stage == s.stages) {
            stage = 0;
            parity ^= 1;
          }
        }
      }
      // the last products' arrivals have landed here before this CTA may end
      for (int i = 0; ok && i < s.stages; ++i) {
        ok = mbar_wait_bounded(&empty[stage], parity, &abort);
        if (++stage == s.stages) {
          stage = 0;
          parity ^= 1;
        }
      }
    }
  } else if (warp == 1) {
    if (rank == 0 && lane == 0) {
      const uint32_t desc = product_of(true, L::kAAlongK, L::kBAlongK, 256, s.N);
      int stage = 0;
      uint32_t parity = 0;
      int64_t run = 0;
      bool ok = true;
      for (int64_t tile = blockIdx.x / 2; ok && tile < tiles; tile += pairs) {
        int first, last;
        blocks_of(s, static_cast<int>(tile % s.splits), first, last);
        for (int kb0 = first; ok && kb0 < last; kb0 += kRun, ++run) {
          const int buf = static_cast<int>(run & 1);
          ok = mbar_wait_bounded(&sums_empty[buf], uint32_t(run >> 1 & 1) ^ 1u, &abort);
          if (!ok) break;
          tensor_fence_after();
          for (int kb = kb0; kb < min(kb0 + kRun, last); ++kb) {
            ok = mbar_wait_bounded(&full[stage], parity, &abort);
            if (!ok) break;
            tensor_fence_after();
            const uint32_t a = smem_u32(base) + stage * stage_bytes;
            multiply_parts<kProduct>(sums + buf * 256, a, a + 3 * kABytes, b_bytes, desc, kb == kb0);
            products_arrive<2>(&empty[stage]);
            if (++stage == s.stages) {
              stage = 0;
              parity ^= 1;
            }
          }
          if (ok) products_arrive<2>(&sums_full[buf]);
        }
      }
    }
  } else if (warp >= 4) {
    const int q = warp & 3, group = (warp - 4) >> 2;
    float* swap = reinterpret_cast<float*>(base + s.stages * stage_bytes) + group * (4 * 8 * 32);
    constexpr int kChunks = kMostN / 16 / kGroups;
    int64_t run = 0;
    for (int64_t tile = blockIdx.x / 2; tile < tiles; tile += pairs) {
      int64_t m, n;
      bool second;
      const int split = static_cast<int>(tile % s.splits);
      tile_of<kProduct>(tile / s.splits, s.m_tiles, s.n_tiles, s.N, m, n, second);
      m += rank * L::kRows;
      int first, last;
      blocks_of(s, split, first, last);
      float sum[kChunks][16];
#pragma unroll
      for (int c = 0; c < kChunks; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[c][i] = 0.f;
      for (int kb0 = first; kb0 < last; kb0 += kRun, ++run) {
        const int buf = static_cast<int>(run & 1);
        // after a timeout garbage, and a status
        if (!mbar_wait_bounded(&sums_full[buf], uint32_t(run >> 1 & 1), &abort) && lane == 0)
          report(j.status, SF_ST_TIMEOUT);
        tensor_fence_after();
        const uint32_t at = sums + buf * 256 + (uint32_t(q) << 21) + 16 * group;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
          if (32 * c + 16 * group >= s.N) break;
          uint32_t v[16], w[16];
          tensor_load16(at + 32 * c, v);
          tensor_load16(at + 32 * c + kMostN, w);
          tensor_loaded();
#pragma unroll
          for (int i = 0; i < 16; ++i) sum[c][i] += __uint_as_float(v[i]) + __uint_as_float(w[i]);
        }
        tensor_fence_before();
        __syncwarp();
        if (lane == 0) arrive_at(at_rank(&sums_empty[buf], 0));
      }
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        const int at = 32 * c + 16 * group;
        if (at >= s.N) break;
        if constexpr (L::kGated) {
          // quadrants 0 and 1 hold g, 2 and 3 u of the same features: each keeps half of the columns
          const int64_t f = m + 32 * (q & 1) + lane, t0 = n + at + (q < 2 ? 0 : 8);
          float dh[8], g[8], u[8];
          if constexpr (kProduct == kInner) load_dh<float>(j, t0, 1, f, dh);
          float* out = swap + q * 8 * 32 + lane;
          const float* in = swap + (q ^ 2) * 8 * 32 + lane;
#pragma unroll
          for (int i = 0; i < 8; ++i) out[32 * i] = q < 2 ? sum[c][8 + i] : sum[c][i];
          named_barrier(1 + group * 2 + (q & 1), 64);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float own = q < 2 ? sum[c][i] : sum[c][8 + i], other = in[32 * i];
            g[i] = q < 2 ? own : other;
            u[i] = q < 2 ? other : own;
          }
          named_barrier(1 + group * 2 + (q & 1), 64);
          store_gated<float, kProduct>(j, t0, 1, f, 8, g, u, dh);
        } else if (s.splits > 1) {
          const int64_t row = m + 32 * q + lane, column = n + at, columns = kProduct == kDx ? j.T : j.F;
          const int left = row < j.H && column < columns ? static_cast<int>(min(int64_t(16), columns - column)) : 0;
          const int64_t matrix = kProduct == kDx ? split : 2 * split + (second ? 1 : 0);
          store_down(s.sums + (matrix * columns + column) * j.H + row, j.H, 1, left, sum[c]);
        } else {
          store_plain<float, kProduct>(j, second, m + 32 * q + lane, n + at, 1, 16, sum[c]);
        }
      }
    }
  }
  __syncwarp();
  if (*static_cast<volatile int*>(&abort)) {  // let copies and products in flight end
    if (tid == 0) report(j.status, SF_ST_TIMEOUT);
    const uint64_t t0 = global_timer_ns();
    while (global_timer_ns() - t0 < 2000000u) {
    }
  }
  cluster_sync();
  if (warp == 2) tensor_free<2>(sums, 512);
}

// ---------------------------------------------------------------- host

// Three matrices of `rows` rows of `len` values, `ld` apart, one behind the other.
bool make_map(CUtensorMap* map, const void* p, int64_t rows, int64_t len, int64_t ld, int box_rows) {
  const EncodeFn encode = encode_fn();
  if (encode == nullptr) return false;
  const cuuint64_t dims[3] = {cuuint64_t(len), cuuint64_t(rows), 3};
  const cuuint64_t strides[2] = {cuuint64_t(ld) * 2, cuuint64_t(rows * ld) * 2};
  const cuuint32_t box[3] = {kBox, cuuint32_t(box_rows), 1}, ones[3] = {1, 1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(p), dims, strides, box, ones,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr size_t kSmem = 226 * 1024;  // of 227 KB, 1 KB for the barriers

struct Cut {
  int N, splits;
  int64_t m_tiles, n_tiles;
  double us;
};

// The width of the tiles, and for dx and dW, whose sums may be long and their tiles few, in how many
// ways k is split, by estimated time: a block of 64 k takes an SM the longer of its 24 products
// and its 3 x (16 KB + 64 N) bytes at 48 a clock; sums of splits are written and read once more.
// 175 x 193 x 5239: the gradient 190 us without splits, 58 with those of dx; 1247 x 72 x 993:
// 66 us without those of dW, 58 with them.
template <int kProduct>
Cut cut_of(int64_t M, int64_t Nall, int blocks) {
  const int two = kProduct == kDw ? 2 : 1;
  Cut best = {};
  best.us = 1e30;
  for (int N = kProduct == kDw ? 128 : 32; N <= kMostN; N += 32) {
    for (int splits = 1; splits == 1 || (!Layout<kProduct>::kGated && splits <= 16 && blocks >= 4 * splits);
         splits *= 2) {
      Cut c;
      c.N = N;
      c.splits = splits;
      c.m_tiles = ceil_div(M, 2 * Layout<kProduct>::kRows);
      c.n_tiles = ceil_div(Nall, N);
      const double rounds = double(ceil_div(c.m_tiles * c.n_tiles * two * splits, sm_pairs()));
      const double block = std::max(12.0 * N, 3.0 * (kABytes + 64.0 * N) / 48.0) / 1900.0;
      c.us = 6.0 + 0.02 * N + rounds * (1.0 + double(ceil_div(blocks, splits)) * block) +
             (splits > 1 ? two * (3.0 + 8.0 * splits * double(M) * double(Nall) / 6.5e6) : 0.0);
      if (c.us < best.us) best = c;
    }
  }
  return best;
}
// f32 values that the splits of dx, then of dW, need room for.
size_t split_values(int64_t T, int64_t H, int64_t F) {
  const int dx = cut_of<kDx>(H, T, static_cast<int>(2 * ceil_div(F, kBox))).splits;
  const int dw = cut_of<kDw>(H, F, static_cast<int>(ceil_div(T, kBox))).splits;
  return std::max(dx > 1 ? size_t(dx) * size_t(T) * size_t(H) : 0, dw > 1 ? 2 * size_t(dw) * size_t(F) * size_t(H) : 0);
}

template <int kProduct>
cudaError_t launch_product(const FfnJob& j, float* sums, cudaStream_t stream) {
  using L = Layout<kProduct>;
  Shape s = {};
  const int64_t k = kProduct == kDx ? j.F : kProduct == kDw ? j.T : j.H;
  s.half = static_cast<int>(ceil_div(k, kBox));
  s.blocks = kProduct == kDx ? 2 * s.half : s.half;
  const Cut c = cut_of<kProduct>(L::kGated ? j.F : j.H, kProduct == kDw ? j.F : j.T, s.blocks);
  s.N = c.N;
  s.splits = c.splits;
  s.sums = sums;
  const size_t stage = 3 * (kABytes + size_t(s.N / 2) * kDepthBytes);
  s.stages = static_cast<int>(std::min<size_t>(kMaxStages, (kSmem - 1024 - kSwapBytes) / stage));
  s.m_tiles = c.m_tiles;
  s.n_tiles = c.n_tiles;
  Maps maps;
  const int n_rows = kProduct == kDw ? kBox : s.N / 2;
  bool fine = L::kGated || (make_map(&maps.b0, j.dg, j.T, j.F, j.ldg, n_rows) && make_map(&maps.b1, j.du, j.T, j.F, j.ldg, n_rows));
  if (kProduct == kDw) {
    fine = fine && make_map(&maps.a0, j.x, j.T, j.H, j.ldx, kBox);
    maps.a1 = maps.a0;
  } else {
    fine = fine && make_map(&maps.a0, j.w_gate, j.F, j.H, j.ldw, kBox) && make_map(&maps.a1, j.w_up, j.F, j.H, j.ldw, kBox);
  }
  if (L::kGated) {
    fine = fine && make_map(&maps.b0, j.x, j.T, j.H, j.ldx, n_rows);
    maps.b1 = maps.b0;
  }
  if (!fine) return cudaErrorUnknown;
  const size_t smem = kSmem;  // all, whatever the stages take: no other CTA on its SM
  const auto kernel = ffn_parts_kernel<kProduct>;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
  if (e != cudaSuccess) return e;
  const int64_t tiles = s.m_tiles * s.n_tiles * (kProduct == kDw ? 2 : 1) * s.splits;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2 * static_cast<unsigned>(std::min<int64_t>(tiles, sm_pairs())));
  cfg.blockDim = dim3(kPairThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  count_launch();
  const cudaError_t launched = cudaLaunchKernelEx(&cfg, kernel, maps, j, s);
  if (launched != cudaSuccess || s.splits == 1) return launched;
  if (kProduct == kDx)
    return launch_ffn_sum({s.sums, j.T * j.H, s.splits, static_cast<float*>(j.dx), j.T, j.H, j.lddx, false}, stream);
  const cudaError_t e1 = launch_ffn_sum(
      {s.sums, 2 * j.F * j.H, s.splits, static_cast<float*>(j.dw_gate), j.F, j.H, j.lddw, j.accumulate}, stream);
  if (e1 != cudaSuccess) return e1;
  return launch_ffn_sum(
      {s.sums + j.F * j.H, 2 * j.F * j.H, s.splits, static_cast<float*>(j.dw_up), j.F, j.H, j.lddw, j.accumulate}, stream);
}

int64_t padded(int64_t n) { return (n + 7) / 8 * 8; }

}  // namespace

size_t ffn_parts_workspace(int64_t T, int64_t H, int64_t F, bool grad) {
  size_t values = size_t(T + 2 * F) * size_t(padded(H));
  if (!grad) return 6 * values;
  values += 2 * size_t(T) * size_t(padded(F));
  return (6 * values + 15) / 16 * 16 + 4 * split_values(T, H, F);
}

cudaError_t launch_ffn_parts(FfnJob j, bool grad, void* workspace, cudaStream_t stream) {
  const int64_t pitch = padded(j.H), packs = pitch / 8, runs = (packs + 31) / 32;
  __nv_bfloat16* at = static_cast<__nv_bfloat16*>(workspace);
  Sources s;
  const void** data[3] = {&j.x, &j.w_gate, &j.w_up};
  for (int i = 0; i < 3; ++i) {
    s.from[i] = static_cast<const float*>(*data[i]);
    s.to[i] = at;
    s.rows[i] = i == 0 ? j.T : j.F;
    s.ld[i] = i == 0 ? j.ldx : j.ldw;
    *data[i] = at;
    at += 3 * s.rows[i] * pitch;
  }
  j.ldx = j.ldw = pitch;
  if (grad) {
    j.ldg = padded(j.F);
    j.dg = at;
    j.du = at + 3 * j.T * j.ldg;
    at += 6 * j.T * j.ldg;
  }
  float* sums = reinterpret_cast<float*>(static_cast<char*>(workspace) +
                                         ((reinterpret_cast<char*>(at) - static_cast<char*>(workspace)) + 15) / 16 * 16);
  const int64_t most = (std::max(j.T, j.F) * runs + kThreads / 32 - 1) / (kThreads / 32);
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>(most, int64_t(sm_count()) * 8)), 3);
  count_launch();
  ffn_parts_of_kernel<<<grid, kThreads, 0, stream>>>(s, j.H, static_cast<int>(packs), static_cast<int>(runs));
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  if (!grad) return launch_product<kForward>(j, nullptr, stream);
  e = launch_product<kInner>(j, nullptr, stream);
  if (e == cudaSuccess && j.dx != nullptr) e = launch_product<kDx>(j, sums, stream);
  if (e == cudaSuccess && j.dw_gate != nullptr) e = launch_product<kDw>(j, sums, stream);
  return e;
}

}  // namespace sf
