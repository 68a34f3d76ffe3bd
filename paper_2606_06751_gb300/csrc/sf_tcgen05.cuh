// sf_tcgen05.cuh - tensor-core building blocks for sm_103a: matrices in shared
// memory as 128-byte swizzled tiles, products into tensor memory, and their barriers.
// kCtas is the number of CTAs that work on one product (a pair's SMs share it).
#pragma once

#include "sf_float.cuh"

namespace sf {

constexpr int kDepthBytes = 128;                // of k in a tile's row (or of m, n, in one that has these along the row)
constexpr int kBox = 64;                        // 16-bit values in it
constexpr uint32_t kBoxBytes = kBox * kDepthBytes;  // a square of 64 x 64 values

// A matrix operand in shared memory, 128-byte swizzle.  Along k in the rows: 8-row
// groups follow one another every 1024 bytes.  Along m or n in the rows (a row a k):
// groups of 8 k every 1024 bytes, runs of 64 m or n every 8192.
template <bool kAlongK>
__device__ __forceinline__ uint64_t operand_of(uint32_t at) {
  constexpr uint64_t fixed = (uint64_t(1024 >> 4) << 32) | (uint64_t(kAlongK ? 1 : kBoxBytes >> 4) << 16) |
                             (uint64_t(1) << 46) | (uint64_t(2) << 61);
  return fixed | ((at >> 4) & 0x3fffu);
}
// Bytes from one step of 16 k to the next.
template <bool kAlongK>
constexpr uint32_t kStepBytes = kAlongK ? 32 : 2048;

// Instruction descriptor: f32 sums of f16 or bf16 products.
__device__ __forceinline__ uint32_t product_of(bool bf16, bool a_along_k, bool b_along_k, int M, int N) {
  return (1u << 4) | (bf16 ? (1u << 7) | (1u << 10) : 0u) | (a_along_k ? 0u : 1u << 15) | (b_along_k ? 0u : 1u << 16) |
         (uint32_t(N >> 3) << 17) | (uint32_t(M >> 4) << 24);
}

template <int kCtas>
__device__ __forceinline__ void tensor_product(uint32_t d, uint64_t a, uint64_t b, uint32_t desc, bool add) {
  if constexpr (kCtas == 2)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(desc), "r"(uint32_t(add))
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(desc), "r"(uint32_t(add))
        : "memory");
}

// Arrives on `bar` (of both CTAs of a pair) once the products issued so far are done.
template <int kCtas>
__device__ __forceinline__ void products_arrive(uint64_t* bar) {
  if constexpr (kCtas == 2)
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
            smem_u32(bar)),
        "h"(uint16_t(3))
        : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar))
                 : "memory");
}

// One warp; waits while other CTAs of the SM hold the columns.  So that no two kernels,
// of this library or another, can wait for each other's columns, a CTA either takes all
// shared memory of its SM with them, or waits for no other CTA while it holds some: it
// allocates behind griddep_wait, lets the next kernel start (griddep_launch_dependents)
// when all its warps know that the columns are there, and gives them back before it waits
// for its cluster.
template <int kCtas>
__device__ __forceinline__ void tensor_alloc(uint32_t* at, uint32_t columns) {
  if constexpr (kCtas == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(at)), "r"(columns)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  } else {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(at)), "r"(columns)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
}
template <int kCtas>
__device__ __forceinline__ void tensor_free(uint32_t at, uint32_t columns) {
  if constexpr (kCtas == 2)
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns) : "memory");
  else
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns) : "memory");
}

__device__ __forceinline__ void tensor_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tensor_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 8 or 16 columns of the warp's 32 lanes, in flight until tensor_loaded().
__device__ __forceinline__ void tensor_load8(uint32_t at, uint32_t (&v)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void tensor_load16(uint32_t at, uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, "
      "[%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(at)
      : "memory");
}
__device__ __forceinline__ void tensor_loaded() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// A box of a matrix to this CTA's shared memory; the bytes count on `bar`, an
// address in the cluster's shared memory (a pair's first CTA's).
template <int kCtas>
__device__ __forceinline__ void tensor_copy(uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y, uint32_t bar) {
  if constexpr (kCtas == 2)
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2"
        " [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar)
        : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar)
        : "memory");
}

// Relaxed: what it orders is reads of tensor memory that have completed.  A release
// would also wait for the warp's stores to global memory.
__device__ __forceinline__ void arrive_at(uint32_t bar) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// From the shared memory of a CTA of the cluster.
__device__ __forceinline__ float load_at(uint32_t at) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}

}  // namespace sf
