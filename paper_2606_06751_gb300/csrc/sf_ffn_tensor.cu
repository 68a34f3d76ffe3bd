// sf_ffn_tensor.cu - the products of the gated feed-forward operators on the
// tensor cores (bf16 and f16).
//
// Every product is written as D[m][n] = sum_k A[m][k] B[n][k] with m along the
// rows of what is stored, so that a warp's 32 lanes (rows of D in tensor memory)
// store 32 neighbouring values, whatever the alignment of the output:
//   forward, inner  m: 64 features of Wg and the same 64 of Wu, n: tokens, k: H
//   dx              m: H, n: tokens, k: features of dg with Wg, then of du with Wu
//   dW              m: H, n: features of dg, then of du, k: tokens
// Weights under dx and both operands of dW lie with m or n along their rows; the
// tensor cores take them as they are.
#include <algorithm>

#include "sf_ffn_tensor.h"
#include "sf_ffn_tiles.cuh"

namespace sf {
namespace {

constexpr int kMaxStages = 12;

// The tensor cores cut their f32 sums off instead of rounding them, 16 k at a time, by up to 2^-23
// of the sum: 3.5e-5 of a sum of 8192 products of one sign, 3.7e-7 of 256 (measured).  That is
// little against a result of 16 bits.  Weights' gradients in f32 are summed there in runs of kRun
// blocks of 64 k, which are added up in registers: 3.8e-7 however long the sum.  8192 x 4096 x 12288
// bf16: dW in f32 takes 1170 us so, in bf16 without runs 1100.
constexpr int kRun = 4;

struct Shape {
  int64_t m_tiles, n_tiles;  // dW: n tiles of one of the two matrices
  int N;                     // columns of D
  int stages;
  int blocks, half;          // blocks of 64 k; dx: those of the first half
  uint32_t columns;          // of tensor memory
};

struct Maps {
  CUtensorMap a0, a1, b0, b1;
};

// A tile's sums take this much longer than any other wait, at most: 10 us a block (a third of one is measured).
__device__ __forceinline__ uint64_t sums_limit(const Shape& s) { return kWaitLimitNs + uint64_t(s.blocks) * 10000u; }

__device__ __forceinline__ void prefetch_maps(const Maps& maps) {
  prefetch_tensormap(&maps.a0);
  prefetch_tensormap(&maps.a1);
  prefetch_tensormap(&maps.b0);
  prefetch_tensormap(&maps.b1);
}

// Copies block `kb` of the operands of a CTA's tile; `rows` is the tile's first m, `from` the first n it loads.
template <int kProduct, int kCtas>
__device__ __forceinline__ void copy_block(const Maps& maps, const Shape& s, int kb, int m, int n, int n_rows,
                                           bool second, uint32_t a, uint32_t b, uint32_t bar) {
  if constexpr (Layout<kProduct>::kGated) {
    const int k = kb * kBox;
    tensor_copy<kCtas>(a, &maps.a0, k, m, bar);
    tensor_copy<kCtas>(a + kBoxBytes, &maps.a1, k, m, bar);
    tensor_copy<kCtas>(b, &maps.b0, k, n, bar);
  } else if constexpr (kProduct == kDx) {
    const bool up = kb >= s.half;
    const int k = (up ? kb - s.half : kb) * kBox;
    const CUtensorMap* w = up ? &maps.a1 : &maps.a0;
    tensor_copy<kCtas>(a, w, m, k, bar);
    tensor_copy<kCtas>(a + kBoxBytes, w, m + kBox, k, bar);
    tensor_copy<kCtas>(b, up ? &maps.b1 : &maps.b0, k, n, bar);
  } else {
    const int k = kb * kBox;
    tensor_copy<kCtas>(a, &maps.a0, m, k, bar);
    tensor_copy<kCtas>(a + kBoxBytes, &maps.a0, m + kBox, k, bar);
    for (int i = 0; i < n_rows; i += kBox)
      tensor_copy<kCtas>(b + uint32_t(i / kBox) * kBoxBytes, second ? &maps.b1 : &maps.b0, n + i, k, bar);
  }
}

// The products of one block of 64 k.
template <int kProduct, int kCtas>
__device__ __forceinline__ void multiply_block(uint32_t d, uint32_t a, uint32_t b, uint32_t desc, bool first) {
  using L = Layout<kProduct>;
#pragma unroll
  for (int k = 0; k < kBox / 16; ++k)
    tensor_product<kCtas>(d, operand_of<L::kAAlongK>(a + k * kStepBytes<L::kAAlongK>),
                          operand_of<L::kBAlongK>(b + k * kStepBytes<L::kBAlongK>), desc, !(first && k == 0));
}

// Adds 16 columns of every kStep to `sum`, while they are below `columns`.
template <int kStep, int kChunks>
__device__ __forceinline__ void add_columns(uint32_t at, int columns, float (&sum)[kChunks][16]) {
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    if (kStep * c >= columns) break;
#pragma unroll
    for (int h = 0; h < 16; h += 8) {
      uint32_t v[8];
      tensor_load8(at + kStep * c + h, v);
      tensor_loaded();
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[c][h + i] += __uint_as_float(v[i]);
    }
  }
}

// ---------------------------------------------------------------- large products: a pair of SMs a tile

constexpr int kGroups = 3;
// Groups of store warps; with runs a warp's share of a tile's columns stays in its registers.
template <bool kRuns>
constexpr int kGroupsOf = kRuns ? 4 : kGroups;
template <bool kRuns>
constexpr int kPairThreads = 128 + 128 * kGroupsOf<kRuns>;
constexpr int kSwapBytes = kGroups * 2 * 4 * 8 * 32 * 4;  // groups, parities, quadrants, columns, lanes

// Persistent pairs of CTAs: each pair multiplies 256 rows by N columns, the sums of
// one tile being stored while the next is multiplied.  Warp 0 copies, warp 1 of the
// pair's first CTA multiplies, warps from 4 store.  Bound by the tensor cores where
// the tiles fill the SMs: forward 8192 x 4096 x 12288 bf16 902 us (1.83 PFLOP/s) in a
// burst, 1015 at the power limit; else by the copies from L2 (32 KB of operands a pair's
// SM and block of 64 k, at 48 bytes a clock) and by a launch's first and last tile.
template <typename T, int kProduct, bool kRuns>
__global__ void __launch_bounds__(kPairThreads<kRuns>, 1) __cluster_dims__(2, 1, 1)
    ffn_pair_kernel(const __grid_constant__ Maps maps, const FfnJob j, const Shape s) {
  using L = Layout<kProduct>;
  constexpr int kStoreWarps = 4 * kGroupsOf<kRuns>;
  extern __shared__ unsigned char raw[];
  __shared__ uint64_t full[kMaxStages], empty[kMaxStages], sums_full[2], sums_empty[2];
  __shared__ uint32_t tensor_at;
  __shared__ int abort;
  unsigned char* base = align_1024(raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t rank = cluster_rank();
  const int half_n = s.N / 2;
  const uint32_t stage_bytes = kABytes + uint32_t(half_n) * kDepthBytes;
  const int64_t tiles = s.m_tiles * s.n_tiles * (kProduct == kDw ? 2 : 1);
  const int64_t pairs = gridDim.x / 2;
  const int run = kRuns ? kRun : s.blocks;  // blocks that are summed at once

  if (tid == 0) {
    prefetch_maps(maps);
    abort = 0;
    for (int i = 0; i < s.stages; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sums_full[i], 1);
      mbar_init(&sums_empty[i], 2 * (kStoreWarps + (kProduct == kInner ? 1 : 0)));
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
        tile_of<kProduct>(tile, s.m_tiles, s.n_tiles, s.N, m, n, second);
        for (int kb = 0; kb < s.blocks; ++kb) {
          ok = mbar_wait_bounded(&empty[stage], parity, &abort);
          if (!ok) break;
          const uint32_t a = smem_u32(base) + stage * stage_bytes;
          if (rank == 0) mbar_arrive_expect_tx(&full[stage], 2 * stage_bytes);
          copy_block<kProduct, 2>(maps, s, kb, static_cast<int>(m + rank * L::kRows), static_cast<int>(n + rank * half_n),
                                  half_n, second, a, a + kABytes, at_rank(&full[stage], 0));
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
      const uint32_t desc = product_of(j.dtype == SF_BF16, L::kAAlongK, L::kBAlongK, 256, s.N);
      int stage = 0;
      uint32_t parity = 0;
      int64_t done = 0;
      bool ok = true;
      for (int64_t tile = blockIdx.x / 2; ok && tile < tiles; tile += pairs) {
        for (int kb0 = 0; ok && kb0 < s.blocks; kb0 += run, ++done) {
          const int buf = static_cast<int>(done & 1), end = min(kb0 + run, s.blocks);
          ok = mbar_wait_bounded(&sums_empty[buf], uint32_t(done >> 1 & 1) ^ 1u, &abort);
          if (!ok) break;
          tensor_fence_after();
          for (int kb = kb0; kb < end; ++kb) {
            ok = mbar_wait_bounded(&full[stage], parity, &abort);
            if (!ok) break;
            tensor_fence_after();
            const uint32_t a = smem_u32(base) + stage * stage_bytes;
            multiply_block<kProduct, 2>(sums + buf * 256, a, a + kABytes, desc, kb == kb0);
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
  } else if (kProduct == kInner && warp == 3) {
    // the upstream gradients of the next tile, into L2: their loads come while the copies fill every queue
    const auto fetch = [&](int64_t tile) {
      if (tile >= tiles) return;
      int64_t m, n;
      bool second;
      tile_of<kProduct>(tile, s.m_tiles, s.n_tiles, s.N, m, n, second);
      m += rank * L::kRows;
      if (m >= j.F) return;
      for (int64_t t = n + lane; t < n + s.N && t < j.T; t += 32) {
        const T* p = static_cast<const T*>(j.dh) + t * j.lddh + m;
        prefetch_l2(p);
        prefetch_l2(p + min(int64_t(L::kRows), j.F - m) - 1);
      }
    };
    int64_t done = 0;
    fetch(blockIdx.x / 2);
    for (int64_t tile = blockIdx.x / 2; tile < tiles; tile += pairs, ++done) {
      fetch(tile + pairs);
      mbar_wait_bounded(&sums_full[done & 1], uint32_t(done >> 1 & 1), &abort, sums_limit(s));
      // a warp that waits for every phase of a barrier has to hold back the one after next
      __syncwarp();
      if (lane == 0) arrive_at(at_rank(&sums_empty[done & 1], 0));
    }
  } else if (kRuns && warp >= 4) {
    // as below, but a warp adds its columns of a tile's runs up first
    const int q = warp & 3, group = (warp - 4) >> 2;
    constexpr int kStep = 16 * kGroupsOf<kRuns>, kChunks = 256 / kStep;
    int64_t done = 0;
    for (int64_t tile = blockIdx.x / 2; tile < tiles; tile += pairs) {
      int64_t m, n;
      bool second;
      tile_of<kProduct>(tile, s.m_tiles, s.n_tiles, s.N, m, n, second);
      m += rank * L::kRows;
      float sum[kChunks][16];
#pragma unroll
      for (int c = 0; c < kChunks; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[c][i] = 0.f;
      for (int kb0 = 0; kb0 < s.blocks; kb0 += run, ++done) {
        const int buf = static_cast<int>(done & 1);
        // after a timeout garbage, and a status
        if (!mbar_wait_bounded(&sums_full[buf], uint32_t(done >> 1 & 1), &abort, sums_limit(s)) && lane == 0)
          report(j.status, SF_ST_TIMEOUT);
        tensor_fence_after();
        add_columns<kStep>(sums + buf * 256 + (uint32_t(q) << 21) + 16 * group, s.N - 16 * group, sum);
        tensor_fence_before();
        __syncwarp();
        if (lane == 0) arrive_at(at_rank(&sums_empty[buf], 0));
      }
#pragma unroll
      for (int c = 0; c < kChunks; ++c)
        if (16 * group + kStep * c < s.N)
          store_plain<T, kProduct>(j, second, m + 32 * q + lane, n + 16 * group + kStep * c, 1, 16, sum[c]);
    }
  } else if (warp >= 4) {
    // groups of four warps take chunks of 16 columns in turn; a warp reads the 32 lanes of its quadrant
    const int q = warp & 3, group = (warp - 4) >> 2;
    float* swap = reinterpret_cast<float*>(base + s.stages * stage_bytes) + group * (2 * 4 * 8 * 32);
    int64_t done = 0;
    int turn = 0;
    for (int64_t tile = blockIdx.x / 2; tile < tiles; tile += pairs, ++done) {
      int64_t m, n;
      bool second;
      tile_of<kProduct>(tile, s.m_tiles, s.n_tiles, s.N, m, n, second);
      m += rank * L::kRows;
      const int buf = static_cast<int>(done & 1);
      T dh_next[8];
      if constexpr (kProduct == kInner)
        load_dh<T>(j, n + 16 * group + (q < 2 ? 0 : 8), 1, m + 32 * (q & 1) + lane, dh_next);
      // else garbage, and a status
      const bool ok = mbar_wait_bounded(&sums_full[buf], uint32_t(done >> 1 & 1), &abort, sums_limit(s));
      tensor_fence_after();
      const uint32_t at = sums + buf * 256 + (uint32_t(q) << 21);
      const auto give_back = [&] {  // this warp has read its last columns of the tile
        tensor_fence_before();
        __syncwarp();
        if (lane == 0) arrive_at(at_rank(&sums_empty[buf], 0));
      };
      for (int c = 16 * group; c < s.N; c += 16 * kGroups) {
        uint32_t v[16];
        if constexpr (L::kGated) {
          // quadrants 0 and 1 hold g, 2 and 3 u of the same features: each keeps half of the columns
          // and gets the other factor for them
          const int mine = q < 2 ? 0 : 8;
          const int64_t f = m + 32 * (q & 1) + lane, t0 = n + c + mine;
          float g[8], u[8];
          T dh[8];
          if constexpr (kProduct == kInner) {  // on their way since the chunk before
#pragma unroll
            for (int i = 0; i < 8; ++i) dh[i] = dh_next[i];
            if (c + 16 * kGroups < s.N) load_dh<T>(j, t0 + 16 * kGroups, 1, f, dh_next);
          }
          tensor_load16(at + c, v);
          tensor_loaded();
          if (c + 16 * kGroups >= s.N) give_back();
          float* out = swap + (turn * 4 + q) * 8 * 32 + lane;
          const float* in = swap + (turn * 4 + (q ^ 2)) * 8 * 32 + lane;
#pragma unroll
          for (int i = 0; i < 8; ++i) out[32 * i] = __uint_as_float(q < 2 ? v[8 + i] : v[i]);
          named_barrier(1 + group * 2 + (q & 1), 64);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float own = __uint_as_float(q < 2 ? v[i] : v[8 + i]), other = in[32 * i];
            g[i] = q < 2 ? own : other;
            u[i] = q < 2 ? other : own;
          }
          store_gated<T, kProduct>(j, t0, 1, f, 8, g, u, dh);
          turn ^= 1;
        } else {
          tensor_load16(at + c, v);
          tensor_loaded();
          if (c + 16 * kGroups >= s.N) give_back();
          float x[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) x[i] = __uint_as_float(v[i]);
          store_plain<T, kProduct>(j, second, m + 32 * q + lane, n + c, 1, 16, x);
        }
      }
      if (16 * group >= s.N) give_back();  // no chunk of its own
      if (!ok && lane == 0) report(j.status, SF_ST_TIMEOUT);
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

// ---------------------------------------------------------------- small products: a tile a cluster, k split among its CTAs

constexpr int kSplitThreads = 256;
constexpr int kMostRunN = 128;  // columns of a tile that is summed in runs

// Each CTA of a cluster sums its share of the blocks for the same 128 rows and N
// columns; then CTA r adds up, in the CTAs' order, and stores a share of the columns.
// Tensor memory is given back before the CTAs wait for one another.  Bound by the
// weights' bytes for few tokens: 48 through 4096 x 12288 37 us (81 % of the copy rate),
// through 2048 x 8192 15 us (10 are the bytes').
// With runs every warp adds its columns of a run up before the next is multiplied; the next
// run's first blocks are on their way by then.
template <typename T, int kProduct, bool kRuns>
__global__ void __launch_bounds__(kSplitThreads) ffn_split_kernel(const __grid_constant__ Maps maps, const FfnJob j,
                                                                  const Shape s) {
  using L = Layout<kProduct>;
  extern __shared__ unsigned char raw[];
  __shared__ uint64_t full[kMaxStages], empty[kMaxStages], sums_full;
  __shared__ uint32_t tensor_at;
  __shared__ int abort;
  unsigned char* base = align_1024(raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = static_cast<int>(cluster_rank()), C = static_cast<int>(cluster_size());
  const uint32_t stage_bytes = kABytes + uint32_t(s.N) * kDepthBytes;
  const int64_t tile = blockIdx.x / C;
  const int64_t m = tile % s.m_tiles * L::kRows;
  int64_t n = tile / s.m_tiles;
  const bool second = kProduct == kDw && n >= s.n_tiles;
  if (second) n -= s.n_tiles;
  n *= s.N;
  const int first = static_cast<int>(int64_t(s.blocks) * rank / C), last = static_cast<int>(int64_t(s.blocks) * (rank + 1) / C);

  if (tid == 0) {
    prefetch_maps(maps);
    abort = 0;
    for (int i = 0; i < s.stages; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    mbar_init(&sums_full, 1);
    fence_barrier_init();
  }
  // columns between the kernel before and the one behind: neither can wait for them while this one waits for it
  griddep_wait();
  if (warp == 2) tensor_alloc<1>(&tensor_at, s.columns);
  tensor_fence_before();
  __syncthreads();
  tensor_fence_after();
  griddep_launch_dependents();
  const uint32_t sums = tensor_at;

  constexpr int kWarpStep = 32, kChunks = kRuns ? kMostRunN / kWarpStep : 1;  // of a warp's columns
  float sum[kChunks][16];
#pragma unroll
  for (int c = 0; c < kChunks; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) sum[c][i] = 0.f;
  const int q = warp & 3;
  const uint32_t mine = sums + (uint32_t(q) << 21) + 16 * (warp >> 2);
  bool ok = true;
  if constexpr (kRuns) {
    const uint32_t desc = product_of(j.dtype == SF_BF16, L::kAAlongK, L::kBAlongK, 128, s.N);
    int stage = 0, copied = first;
    uint32_t parity = warp == 0 ? 1 : 0, sums_parity = 0;  // the copies wait for the phase before the first
    for (int kb0 = first; kb0 < last; kb0 += kRun) {
      const int end = min(kb0 + kRun, last);
      if (warp == 0) {
        if (lane == 0) {
          for (const int ahead = min(last, end + s.stages); copied < ahead; ++copied) {
            if (!mbar_wait_bounded(&empty[stage], parity, &abort)) break;
            const uint32_t a = smem_u32(base) + stage * stage_bytes;
            mbar_arrive_expect_tx(&full[stage], stage_bytes);
            copy_block<kProduct, 1>(maps, s, copied, static_cast<int>(m), static_cast<int>(n), s.N, second, a, a + kABytes,
                                    smem_u32(&full[stage]));
            if (++stage == s.stages) {
              stage = 0;
              parity ^= 1;
            }
          }
        }
        __syncwarp();
      } else if (warp == 1) {
        if (lane == 0) {
          for (int kb = kb0; kb < end; ++kb) {
            if (!mbar_wait_bounded(&full[stage], parity, &abort)) break;
            tensor_fence_after();
            const uint32_t a = smem_u32(base) + stage * stage_bytes;
            multiply_block<kProduct, 1>(sums, a, a + kABytes, desc, kb == kb0);
            products_arrive<1>(&empty[stage]);
            if (++stage == s.stages) {
              stage = 0;
              parity ^= 1;
            }
          }
          products_arrive<1>(&sums_full);
        }
        __syncwarp();
      }
      ok = mbar_wait_bounded(&sums_full, sums_parity, &abort, sums_limit(s)) && ok;
      sums_parity ^= 1;
      tensor_fence_after();
      add_columns<kWarpStep>(mine, s.N - 16 * (warp >> 2), sum);
      tensor_fence_before();
      __syncthreads();  // before the next run's products
      tensor_fence_after();
    }
    if (warp == 0) {
      if (lane == 0) {
        for (int i = 0; i < s.stages; ++i) {  // the last products' arrivals, before this CTA may end
          if (!mbar_wait_bounded(&empty[stage], parity, &abort)) break;
          if (++stage == s.stages) {
            stage = 0;
            parity ^= 1;
          }
        }
      }
      __syncwarp();
    }
  } else {
    if (warp == 0) {
      if (lane == 0) {
        int stage = 0;
        uint32_t parity = 1;
        for (int kb = first; kb < last; ++kb) {
          if (!mbar_wait_bounded(&empty[stage], parity, &abort)) break;
          const uint32_t a = smem_u32(base) + stage * stage_bytes;
          mbar_arrive_expect_tx(&full[stage], stage_bytes);
          copy_block<kProduct, 1>(maps, s, kb, static_cast<int>(m), static_cast<int>(n), s.N, second, a, a + kABytes,
                                  smem_u32(&full[stage]));
          if (++stage == s.stages) {
            stage = 0;
            parity ^= 1;
          }
        }
        for (int i = 0; i < s.stages; ++i) {  // the last products' arrivals, before this CTA may end
          if (!mbar_wait_bounded(&empty[stage], parity, &abort)) break;
          if (++stage == s.stages) {
            stage = 0;
            parity ^= 1;
          }
        }
      }
      __syncwarp();
    } else if (warp == 1) {
      if (lane == 0) {
        const uint32_t desc = product_of(j.dtype == SF_BF16, L::kAAlongK, L::kBAlongK, 128, s.N);
        int stage = 0;
        uint32_t parity = 0;
        for (int kb = first; kb < last; ++kb) {
          if (!mbar_wait_bounded(&full[stage], parity, &abort)) break;
          tensor_fence_after();
          const uint32_t a = smem_u32(base) + stage * stage_bytes;
          multiply_block<kProduct, 1>(sums, a, a + kABytes, desc, kb == first);
          products_arrive<1>(&empty[stage]);
          if (++stage == s.stages) {
            stage = 0;
            parity ^= 1;
          }
        }
        products_arrive<1>(&sums_full);
      }
      __syncwarp();
    }
    ok = mbar_wait_bounded(&sums_full, 0, &abort, sums_limit(s));
    tensor_fence_after();
  }
  if (!ok || *static_cast<volatile int*>(&abort)) {  // let copies in flight land
    if (tid == 0) report(j.status, SF_ST_TIMEOUT);
    const uint64_t t0 = global_timer_ns();
    while (global_timer_ns() - t0 < 2000000u) {
    }
  }
  float* partial = reinterpret_cast<float*>(base);  // [column][128 rows], where the stages were
  const bool direct = !L::kGated && C == 1;         // nothing to add up or exchange
  const auto put = [&](int c, const float (&x)[16]) {
    if constexpr (!L::kGated) {
      if (direct) store_plain<T, kProduct>(j, second, m + 32 * q + lane, n + c, 1, 16, x);
    }
    if (!direct) {
#pragma unroll
      for (int i = 0; i < 16; ++i) partial[(c + i) * 128 + 32 * q + lane] = x[i];
    }
  };
  if constexpr (kRuns) {
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
      if (16 * (warp >> 2) + kWarpStep * c < s.N) put(16 * (warp >> 2) + kWarpStep * c, sum[c]);
  } else {
    for (int c = 0; c < s.N - 16 * (warp >> 2); c += kWarpStep) {
      uint32_t v[16];
      float x[16];
      tensor_load16(mine + c, v);
      tensor_loaded();
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = last > first ? __uint_as_float(v[i]) : 0.f;
      put(c + 16 * (warp >> 2), x);
    }
  }
  tensor_fence_before();
  __syncthreads();
  if (warp == 2) tensor_free<1>(sums, s.columns);  // before the CTAs wait for one another
  if (direct) return;
  if (C > 1) cluster_sync();
  const int share = (s.N + C - 1) / C, from = rank * share, count = min(share, s.N - from);
  // a thread a row, K columns at a time
  constexpr int K = 8, kStep = kSplitThreads / L::kRows;
  const int r = tid & (L::kRows - 1);
  const int64_t row = m + r;
  for (int c = tid / L::kRows; c < count; c += K * kStep) {
    float v[K], u[K];
    T dh[K];
    if constexpr (kProduct == kInner) load_dh<T>(j, n + from + c, kStep, row, dh);
#pragma unroll
    for (int i = 0; i < K; ++i) v[i] = u[i] = 0.f;
    for (int k = 0; k < C; ++k) {
      const uint32_t p = at_rank(partial + (from + c) * 128 + r, k);
#pragma unroll
      for (int i = 0; i < K; ++i)
        if (c + i * kStep < count) {
          v[i] += load_at(p + i * kStep * 512);
          if (L::kGated) u[i] += load_at(p + i * kStep * 512 + 256);
        }
    }
    const int most = min(count - c, K * kStep);
    if constexpr (L::kGated)
      store_gated<T, kProduct>(j, n + from + c, kStep, row, most, v, u, dh);
    else
      store_plain<T, kProduct>(j, second, row, n + from + c, kStep, most, v);
  }
  if (C > 1) cluster_sync();  // the others have read this CTA's sums
}

// ---------------------------------------------------------------- host


// A matrix of `rows` rows of `len` values, `ld` apart, read in boxes of 64 x `box_rows`, 128-byte swizzle; what lies
// outside is 0.
bool make_map(CUtensorMap* map, const void* p, int32_t dtype, int64_t rows, int64_t len, int64_t ld, int box_rows) {
  const EncodeFn encode = encode_fn();
  if (encode == nullptr) return false;
  const cuuint64_t dims[2] = {cuuint64_t(len), cuuint64_t(rows)};
  const cuuint64_t strides[1] = {rows > 1 ? cuuint64_t(ld) * 2 : cuuint64_t((len * 2 + 15) / 16 * 16)};
  const cuuint32_t box[2] = {kBox, cuuint32_t(box_rows)}, ones[2] = {1, 1};
  return encode(map, dtype == SF_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2,
                const_cast<void*>(p), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int kProduct>
bool make_maps(Maps& maps, const FfnJob& j, int n_rows) {
  if (Layout<kProduct>::kGated) {
    if (!make_map(&maps.a0, j.w_gate, j.dtype, j.F, j.H, j.ldw, kBox) ||
        !make_map(&maps.a1, j.w_up, j.dtype, j.F, j.H, j.ldw, kBox) ||
        !make_map(&maps.b0, j.x, j.dtype, j.T, j.H, j.ldx, n_rows))
      return false;
    maps.b1 = maps.b0;
    return true;
  }
  const int rows = kProduct == kDx ? n_rows : kBox;
  if (!make_map(&maps.b0, j.dg, j.dtype, j.T, j.F, j.ldg, rows) ||
      !make_map(&maps.b1, j.du, j.dtype, j.T, j.F, j.ldg, rows))
    return false;
  if (kProduct == kDw) {
    if (!make_map(&maps.a0, j.x, j.dtype, j.T, j.H, j.ldx, kBox)) return false;
    maps.a1 = maps.a0;
    return true;
  }
  return make_map(&maps.a0, j.w_gate, j.dtype, j.F, j.H, j.ldw, kBox) &&
         make_map(&maps.a1, j.w_up, j.dtype, j.F, j.H, j.ldw, kBox);
}

constexpr size_t kSmemMost = 227 * 1024, kSmemBarriers = 1024, kSmemFixed = kSmemBarriers + 1024;  // and alignment

// The split kernel's shared memory.
uint32_t columns_of(int N) {
  uint32_t c = 32;
  while (c < uint32_t(N)) c *= 2;
  return c;
}
int split_stages(int N, int C, int blocks) {
  const size_t stage = kABytes + size_t(N) * kDepthBytes;
  const int most = static_cast<int>(std::min<size_t>(kMaxStages, (kSmemMost - kSmemFixed) / stage));
  // four blocks on their way: more CTAs an SM do better than more blocks of one
  return std::min(most, std::min<int>(4, static_cast<int>(ceil_div(blocks, C))));
}
size_t split_smem(int N, int C, int blocks) {
  const size_t sums = size_t(N) * 512;
  // CTAs that share an SM must find room in tensor memory: shared memory allows no more of them than that
  const size_t room = kSmemMost * columns_of(N) / 512;
  return 1024 + std::max({sums, room, split_stages(N, C, blocks) * (kABytes + size_t(N) * kDepthBytes)});
}

int split_per_sm(int N, int C, int blocks) {
  return std::max<int>(1, static_cast<int>(kSmemMost / (split_smem(N, C, blocks) + 2048)));
}
// CTAs that run at once with `per_sm` on an SM: clusters of four and eight do not fill every
// group of some 19 SMs.
int64_t split_slots(int C, int per_sm) {
  return C == 8 ? (per_sm == 1 ? 120 : per_sm * 19 / 8 * 64) : per_sm * (C == 4 ? 144 : sm_count());
}

template <typename T, int kProduct, bool kRuns>
cudaError_t launch_pairs(const FfnJob& j, Shape s, cudaStream_t stream) {
  Maps maps;
  if (!make_maps<kProduct>(maps, j, s.N / 2)) return cudaErrorUnknown;
  const size_t stage = kABytes + size_t(s.N / 2) * kDepthBytes, swap = Layout<kProduct>::kGated ? kSwapBytes : 0;
  s.stages = static_cast<int>(std::min<size_t>(kMaxStages, (kSmemMost - kSmemFixed - swap) / stage));
  const size_t smem = kSmemMost - kSmemBarriers;  // all, whatever the stages take: no other CTA on its SM
  const auto kernel = ffn_pair_kernel<T, kProduct, kRuns>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
  if (e != cudaSuccess) return e;
  const int64_t tiles = s.m_tiles * s.n_tiles * (kProduct == kDw ? 2 : 1);
  const unsigned grid = 2 * static_cast<unsigned>(std::min<int64_t>(tiles, sm_pairs()));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kPairThreads<kRuns>);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  count_launch();
  return cudaLaunchKernelEx(&cfg, kernel, maps, j, s);
}

template <typename T, int kProduct, bool kRuns>
cudaError_t launch_split(const FfnJob& j, Shape s, int C, cudaStream_t stream) {
  Maps maps;
  if (!make_maps<kProduct>(maps, j, s.N)) return cudaErrorUnknown;
  s.columns = columns_of(s.N);
  s.stages = split_stages(s.N, C, s.blocks);
  size_t smem = split_smem(s.N, C, s.blocks);
  const int64_t tiles = s.m_tiles * s.n_tiles * (kProduct == kDw ? 2 : 1);
  if (tiles * C >= int64_t(1) << 31) return cudaErrorInvalidConfiguration;
  // clusters are placed side by side on an SM while it has room: no more room than the fewest
  // that run at once need (100 x 512 x 2048, C = 4: 9.1 -> 8.0 us)
  const int most = split_per_sm(s.N, C, s.blocks);
  int per_sm = 1;
  while (per_sm < most && split_slots(C, per_sm) < tiles * C) ++per_sm;
  if (per_sm < most) smem = std::max(smem, kSmemMost / per_sm - 2048);
  const auto kernel = ffn_split_kernel<T, kProduct, kRuns>;
  // one limit for all sizes: calls from other threads set it too
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             static_cast<int>(kSmemMost - kSmemBarriers));
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(tiles * C));
  cfg.blockDim = dim3(kSplitThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = C;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  count_launch();
  return cudaLaunchKernelEx(&cfg, kernel, maps, j, s);
}

// How a product is cut.  The candidates' times are estimated, in microseconds, from
// what was measured: an SM takes 48 bytes a clock from L2, a launch with its first
// copies and its last sums costs 5 us, a tile's stores what `stores` says.
struct Choice {
  bool pairs;
  int N, n_tiles, C;
  double us;
};
double block_us(int rows_n) { return (kABytes + double(rows_n) * kDepthBytes) / 91200.0; }

template <int kProduct, bool kRuns>
Choice choose(int64_t M, int64_t Nall, int blocks, int64_t bytes) {
  using L = Layout<kProduct>;
  const int two = kProduct == kDw ? 2 : 1, sms = sm_count();
  const auto stores = [](int N) { return kProduct == kInner ? 1.2 + 0.012 * N : 0.8 + 0.006 * N; };
  const double least = double(bytes) / 6.5e6;
  const int64_t few = ceil_div(Nall, 256), most = std::min<int64_t>(ceil_div(Nall, 32), few + 8);
  Choice best = {};
  best.us = 1e30;
  for (int64_t nt = few; nt <= most; ++nt) {
    const auto width = [&](int granule) { return static_cast<int>(ceil_div(ceil_div(Nall, nt), granule) * granule); };
    {
      const int N = width(kProduct == kDw ? 128 : 32);
      const int64_t n_tiles = ceil_div(Nall, N), tiles = ceil_div(M, 2 * L::kRows) * n_tiles * two;
      const double rounds = double(ceil_div(tiles, sm_pairs()));
      const double us = 5.5 + std::max(least, rounds * std::max(blocks * block_us(N / 2), stores(N))) + stores(N);
      if (us < best.us) best = {true, N, static_cast<int>(n_tiles), 1, us};
    }
    const int N = width(kProduct == kDw ? 64 : 16);
    if (kRuns && N > kMostRunN) continue;
    const int64_t n_tiles = ceil_div(Nall, N), tiles = ceil_div(M, L::kRows) * n_tiles * two;
    for (int C = 1; C <= 8 && (C == 1 || blocks >= 2 * C); C *= 2) {
      const int per_sm = split_per_sm(N, C, blocks);
      const double slots = double(split_slots(C, per_sm)), ctas = double(tiles * C), waves = std::ceil(ctas / slots);
      const double share = ctas / sms;  // of an SM, on the average; the fullest has more
      const double at_once = std::min<double>(per_sm, std::max(1.0, (share + std::ceil(share)) / 2));
      const double sum = double(ceil_div(blocks, C)) * block_us(N) * at_once;
      // bytes on their way: 2.3 us of them make the rate of memory
      const double way = std::min(ctas, slots) * split_stages(N, C, blocks) * (kABytes + double(N) * kDepthBytes);
      const double reads = std::max(least, double(bytes) / (way / 2.3));
      const double us = 4.5 + std::max(reads + 4.0 * (waves - 1), waves * (sum + 1.0 + (C > 1 ? 0.015 : 0.008) * N)) +
                        (C == 8 ? 2.4 : C == 4 ? 1.6 : C == 2 ? 0.8 : 0.0);
      if (us < best.us) best = {false, N, static_cast<int>(n_tiles), C, us};
    }
  }
  return best;
}

template <typename T, int kProduct, bool kRuns = false>
cudaError_t launch_product(const FfnJob& j, cudaStream_t stream) {
  using L = Layout<kProduct>;
  const int64_t M = L::kGated ? j.F : j.H, Nall = kProduct == kDw ? j.F : j.T;
  const int64_t k = kProduct == kDx ? j.F : kProduct == kDw ? j.T : j.H;
  Shape s = {};
  s.half = static_cast<int>(ceil_div(k, kBox));
  s.blocks = kProduct == kDx ? 2 * s.half : s.half;
  const int64_t bytes = 2 * (j.T * j.H + 2 * j.F * j.H + (kProduct == kForward ? 1 : 2) * j.T * j.F);
  const Choice c = choose<kProduct, kRuns>(M, Nall, s.blocks, bytes);
  s.N = c.N;
  s.n_tiles = c.n_tiles;
  s.m_tiles = ceil_div(M, c.pairs ? 2 * L::kRows : L::kRows);
  return c.pairs ? launch_pairs<T, kProduct, kRuns>(j, s, stream)
                 : launch_split<T, kProduct, kRuns>(j, s, c.C, stream);
}

template <typename T>
cudaError_t launch_type(const FfnJob& j, bool grad, cudaStream_t stream) {
  if (!grad) return launch_product<T, kForward>(j, stream);
  cudaError_t e = launch_product<T, kInner>(j, stream);
  if (e == cudaSuccess && j.dx != nullptr) e = launch_product<T, kDx>(j, stream);
  if (e == cudaSuccess && j.dw_gate != nullptr)
    e = j.dw_dtype == SF_F32 && j.T > kRun * kBox ? launch_product<T, kDw, true>(j, stream)
                                                  : launch_product<T, kDw>(j, stream);
  return e;
}

}  // namespace

cudaError_t launch_ffn_tensor(const FfnJob& j, bool grad, cudaStream_t stream) {
  return j.dtype == SF_BF16 ? launch_type<__nv_bfloat16>(j, grad, stream) : launch_type<__half>(j, grad, stream);
}

}  // namespace sf
