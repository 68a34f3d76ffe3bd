// sf_float.cuh - building blocks of the training-step kernels: 16-byte packs
// of f32, bf16 or f16 values, rows that start at any element, and sums as pairs.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "sf_device.cuh"

namespace sf {

// Values of type T in 16 bytes, and their conversion; stores round once, to nearest even.
template <typename T>
struct Pack {
  static constexpr int kN = 16 / int(sizeof(T));
};

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }

template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) {
  return v;
}
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) {
  return __float2bfloat16_rn(v);
}
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) {
  return __float2half_rn(v);
}

__device__ __forceinline__ void unpack(const uint4& u, float (&f)[4], float) {
  f[0] = __uint_as_float(u.x);
  f[1] = __uint_as_float(u.y);
  f[2] = __uint_as_float(u.z);
  f[3] = __uint_as_float(u.w);
}
__device__ __forceinline__ void unpack(const uint4& u, float (&f)[8], __nv_bfloat16) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {  // a bf16 is the upper half of an f32
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void unpack(const uint4& u, float (&f)[8], __half) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __half2float(__ushort_as_half(static_cast<unsigned short>(w[i])));
    f[2 * i + 1] = __half2float(__ushort_as_half(static_cast<unsigned short>(w[i] >> 16)));
  }
}

// Two f32 in a 64-bit register: one instruction for both.
__device__ __forceinline__ uint64_t pair_of(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void split(uint64_t r, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(r));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// A pack as pairs of f32.
__device__ __forceinline__ void unpack2(const uint4& u, uint64_t (&z)[2], float) {
  z[0] = pair_of(__uint_as_float(u.x), __uint_as_float(u.y));
  z[1] = pair_of(__uint_as_float(u.z), __uint_as_float(u.w));
}
template <typename T>
__device__ __forceinline__ void unpack2(const uint4& u, uint64_t (&z)[4], T t) {
  float f[8];
  unpack(u, f, t);
#pragma unroll
  for (int i = 0; i < 4; ++i) z[i] = pair_of(f[2 * i], f[2 * i + 1]);
}

// A pack of -inf.
__device__ __forceinline__ uint4 same4(uint32_t w) { return make_uint4(w, w, w, w); }
__device__ __forceinline__ uint4 lowest_pack(float) { return same4(0xff800000u); }
__device__ __forceinline__ uint4 lowest_pack(__nv_bfloat16) { return same4(0xff80ff80u); }
__device__ __forceinline__ uint4 lowest_pack(__half) { return same4(0xfc00fc00u); }

// A pack to an address that is aligned to its elements only.
__device__ __forceinline__ void store_elements(float* p, const uint4& u) {
  p[0] = __uint_as_float(u.x);
  p[1] = __uint_as_float(u.y);
  p[2] = __uint_as_float(u.z);
  p[3] = __uint_as_float(u.w);
}
template <typename T>
__device__ __forceinline__ void store_elements(T* p, const uint4& u) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
  unsigned short* h = reinterpret_cast<unsigned short*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    h[2 * i] = static_cast<unsigned short>(w[i]);
    h[2 * i + 1] = static_cast<unsigned short>(w[i] >> 16);
  }
}

// The largest value of K packs; NaN only if all are.
template <int K>
__device__ __forceinline__ float packs_max(const uint4 (&u)[K], float) {
  float m = __uint_as_float(u[0].x);
#pragma unroll
  for (int k = 0; k < K; ++k)
    m = fmaxf(fmaxf(fmaxf(m, __uint_as_float(u[k].x)), fmaxf(__uint_as_float(u[k].y), __uint_as_float(u[k].z))),
              __uint_as_float(u[k].w));
  return m;
}
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t max_f16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
template <int K>
__device__ __forceinline__ float packs_max(const uint4 (&u)[K], __nv_bfloat16) {
  uint32_t m = u[0].x;
#pragma unroll
  for (int k = 0; k < K; ++k)
    m = max_bf16x2(max_bf16x2(m, u[k].x), max_bf16x2(max_bf16x2(u[k].y, u[k].z), u[k].w));
  return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
}
template <int K>
__device__ __forceinline__ float packs_max(const uint4 (&u)[K], __half) {
  uint32_t m = u[0].x;
#pragma unroll
  for (int k = 0; k < K; ++k)
    m = max_f16x2(max_f16x2(m, u[k].x), max_f16x2(max_f16x2(u[k].y, u[k].z), u[k].w));
  return fmaxf(__half2float(__ushort_as_half(static_cast<unsigned short>(m))),
               __half2float(__ushort_as_half(static_cast<unsigned short>(m >> 16))));
}

__device__ __forceinline__ uint4 pack(const float (&f)[4], float) {
  return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
__device__ __forceinline__ uint4 pack(const float (&f)[8], __nv_bfloat16) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
    w[i] = uint32_t(__bfloat16_as_ushort(h.x)) | (uint32_t(__bfloat16_as_ushort(h.y)) << 16);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 pack(const float (&f)[8], __half) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2 h = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
    w[i] = uint32_t(__half_as_ushort(h.x)) | (uint32_t(__half_as_ushort(h.y)) << 16);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// 16-byte global accesses of data that is read or written once: not kept in
// L1.  Plain (coherent) loads: an output may be the input itself.
__device__ __forceinline__ uint4 load16(const void* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p)
               : "memory");
  return v;
}
__device__ __forceinline__ void store16(void* p, const uint4& v) {
  asm volatile("st.global.L1::no_allocate.v4.u32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z),
               "r"(v.w)
               : "memory");
}

// L2 policies: data that is not used again leaves first.
__device__ __forceinline__ uint64_t policy_evict_first() {
  uint64_t p;
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
  return p;
}
__device__ __forceinline__ void store16(void* p, const uint4& v, uint64_t policy) {
  asm volatile("st.global.L1::no_allocate.L2::cache_hint.v4.u32 [%0], {%1, %2, %3, %4}, %5;" ::"l"(p), "r"(v.x),
               "r"(v.y), "r"(v.z), "r"(v.w), "l"(policy)
               : "memory");
}

// Elements of a run of n at p that lie before its first 16-byte boundary.
template <typename T>
__device__ __forceinline__ int head_of(const T* p, int64_t n) {
  const int off = static_cast<int>((16u - (reinterpret_cast<uintptr_t>(p) & 15u)) & 15u) / int(sizeof(T));
  return n < off ? static_cast<int>(n) : off;
}

__device__ __forceinline__ bool finite(float v) { return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u; }

__device__ __forceinline__ float neg_inf() { return __uint_as_float(0xff800000u); }
__device__ __forceinline__ float quiet_nan() { return __uint_as_float(0x7fffffffu); }

// A sum held as an unevaluated pair of f32, about 48 bits: each addition's
// rounding error is found exactly (Knuth's two-sum) and kept in lo.
struct Sum2 {
  float hi = 0.f, lo = 0.f;
  __device__ __forceinline__ void add(float v) {
    const float s = hi + v, b = s - hi;
    lo += (hi - (s - b)) + (v - b);
    hi = s;
  }
  // rounded; lo is NaN once a sum has overflowed
  __device__ __forceinline__ float value() const { return finite(hi) ? hi + lo : hi; }
};
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
  return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kFull, v, o));
  return v;
}
// In a fixed order.  hi has the same bits in every lane (two-sum does not depend on its terms' order), lo may
// differ in its last ones: one lane's sum is the one to use.
__device__ __forceinline__ Sum2 warp_sum(Sum2 s) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float h = __shfl_xor_sync(kFull, s.hi, o), l = __shfl_xor_sync(kFull, s.lo, o);
    s.add(h);
    s.lo += l;
  }
  return s;
}

// Thread-block clusters.
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
// All threads of the cluster: what was written before (also to another CTA's
// shared memory) is seen after.
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Its two halves, for what only needs the other CTAs to have started: before the first access to
// another CTA's shared memory.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.aligned;" ::: "memory"); }
// The address of `p` in the shared memory of CTA `rank` of the cluster.
__device__ __forceinline__ uint32_t at_rank(const void* p, uint32_t rank) {
  uint32_t at;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
  return at;
}

// Launch `kern`; with `dependent`, as the programmatic dependent of the
// previous launch on `stream`: it may start while that one drains, and waits
// for its end in griddep_wait().
template <typename... KArgs, typename... Args>
cudaError_t launch_after(void (*kern)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t stream,
                         bool dependent, const Args&... args) {
  static_assert(((sizeof(KArgs) == sizeof(Args)) && ...), "arguments of the kernel's own types");
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = dependent ? 1 : 0;
  // parameters by address: a list of tensors is up to 32 KB
  void* params[] = {const_cast<void*>(static_cast<const void*>(&args))...};
  return cudaLaunchKernelExC(&cfg, reinterpret_cast<const void*>(kern), params);
}

}  // namespace sf
