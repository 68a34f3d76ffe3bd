// sf_route.cu - the router of a layer of experts and its gradient
// (sf_route_experts, sf_route_experts_grad).
//
// A token is worked on by 8, 16 or 32 lanes of a warp, each holding NV
// consecutive experts in registers; what it costs is instructions, not memory,
// and what is not done once a value is shared by the tokens of a warp.
//
// Forward: the k-th largest of the lanes' two largest values each bounds the
// k-th largest of all from below.  The values that reach the bound (14 of 128
// for k = 8, as a rule) are gathered, and each counts those that come before
// it.  Sigmoids are first taken from the hardware's approximations, with a
// margin for their error; only the gathered ones are computed as the operator
// defines them, which decides.  Where the margin leaves a group's choice open,
// or more than 32 values are gathered, the token's values are all computed
// exactly, and taken one by one if there are too many equal ones.  65536 tokens
// to 8 of 256 experts in 8 groups, f32: 48 us, 490 instructions a token at 63 % of
// the issue slots (memory would allow 11 us); taking the k largest one by one
// from all values, a warp a token, 150 us.
#include <algorithm>
#include <type_traits>

#include "sf_float.cuh"
#include "sf_launch.h"

namespace sf {
namespace {

constexpr int kWarps = 8, kThreads = kWarps * 32;

__device__ __forceinline__ float sigmoid(float z) { return 1.f / (1.f + expf(-z)); }
// Within kSigmoidError of it: 2 units each of ex2.approx and rcp.approx, and the
// rounding of the product, at most 88 where the sigmoid is not 0 or 1 anyway.
constexpr float kSigmoidError = 2e-6f;
__device__ __forceinline__ float sigmoid_fast(float z) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(z * -1.4426950408889634f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
  return r;
}
// exp(z - m) of an expert that is available, m >= z; NaN stays NaN.
__device__ __forceinline__ float softmax_term(float z, float m) { return z == neg_inf() ? 0.f : expf(z - m); }

// exp(x) for x <= 0 by ex2.approx: within 2.4e-7 + 7.5e-8 |x| of it (the
// instruction's error; the product's rounding and that of log2(e)), as much as the
// rounding of a difference of f32 logits is worth.
__device__ __forceinline__ float exp_fast(float x) {
  float e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x * 1.4426950408889634f));
  return e;
}

// Reductions over the LPT lanes of a token.
template <int LPT>
__device__ __forceinline__ float token_max(float v) {
  if constexpr (LPT == 32) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
  } else {
#pragma unroll
    for (int o = LPT / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kFull, v, o));
    return v;
  }
}
template <int LPT>
__device__ __forceinline__ uint32_t token_max(uint32_t v) {
  if constexpr (LPT == 32) {
    return __reduce_max_sync(kFull, v);
  } else {
#pragma unroll
    for (int o = LPT / 2; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(kFull, v, o));
    return v;
  }
}
template <int LPT>
__device__ __forceinline__ float token_sum(float v) {
#pragma unroll
  for (int o = LPT / 2; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
  return v;
}
// The bits of this token's lanes in a ballot, from bit 0.
template <int LPT>
__device__ __forceinline__ uint32_t token_bits(uint32_t ballot, int lane) {
  if constexpr (LPT == 32) return ballot;
  return (ballot >> (lane & ~(LPT - 1))) & ((1u << (LPT & 31)) - 1u);
}

__device__ __forceinline__ float load_value(const void* p, int64_t i, int dtype) {
  if (dtype == SF_F32) return static_cast<const float*>(p)[i];
  if (dtype == SF_BF16) return to_f32(static_cast<const __nv_bfloat16*>(p)[i]);
  return to_f32(static_cast<const __half*>(p)[i]);
}
__device__ __forceinline__ void store_value(void* p, int64_t i, int dtype, float v) {
  if (dtype == SF_F32)
    static_cast<float*>(p)[i] = v;
  else if (dtype == SF_BF16)
    static_cast<__nv_bfloat16*>(p)[i] = from_f32<__nv_bfloat16>(v);
  else
    static_cast<__half*>(p)[i] = from_f32<__half>(v);
}

// NV values of a row at p[at], a lane's, as packs or one by one: pack q holds the
// lane's values q N .. q N + N - 1 and starts at element first(q, N), value i is
// element first(i, 1); elements from `end` on are 0, and are not written.  Packs
// are whole where they are used (see in_packs).
template <typename T, int NV, typename First>
__device__ __forceinline__ void load_packs(const T* row, int end, const First& first, float (&z)[NV]) {
  constexpr int N = Pack<T>::kN;
  if constexpr (NV % N == 0) {
#pragma unroll
    for (int p = 0; p < NV / N; ++p) {
      float f[N];
      unpack(first(p, N) < end ? *reinterpret_cast<const uint4*>(row + first(p, N)) : same4(0u), f, T());
#pragma unroll
      for (int q = 0; q < N; ++q) z[p * N + q] = f[q];
    }
  }
}
template <int NV, typename First>
__device__ __forceinline__ void load_lane(const void* p, int64_t at, int dtype, int end, bool packs,
                                          const First& first, float (&z)[NV]) {
  if (packs && dtype == SF_F32) return load_packs(static_cast<const float*>(p) + at, end, first, z);
  if (packs && dtype == SF_BF16) return load_packs(static_cast<const __nv_bfloat16*>(p) + at, end, first, z);
  if (packs) return load_packs(static_cast<const __half*>(p) + at, end, first, z);
#pragma unroll
  for (int i = 0; i < NV; ++i) z[i] = first(i, 1) < end ? load_value(p, at + first(i, 1), dtype) : 0.f;
}

template <typename T, int NV, typename First>
__device__ __forceinline__ void store_packs(T* row, int end, const First& first, const float (&v)[NV]) {
  constexpr int N = Pack<T>::kN;
  if constexpr (NV % N == 0) {
#pragma unroll
    for (int p = 0; p < NV / N; ++p) {
      float f[N];
#pragma unroll
      for (int q = 0; q < N; ++q) f[q] = v[p * N + q];
      if (first(p, N) < end) store16(row + first(p, N), pack(f, T()));
    }
  }
}
template <int NV, typename First>
__device__ __forceinline__ void store_lane(void* p, int64_t at, int dtype, int end, bool packs, const First& first,
                                           const float (&v)[NV]) {
  if (packs && dtype == SF_F32) return store_packs(static_cast<float*>(p) + at, end, first, v);
  if (packs && dtype == SF_BF16) return store_packs(static_cast<__nv_bfloat16*>(p) + at, end, first, v);
  if (packs) return store_packs(static_cast<__half*>(p) + at, end, first, v);
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (first(i, 1) < end) store_value(p, at + first(i, 1), dtype, v[i]);
}
// Whether rows of E values, ld apart, are whole packs on their boundaries, for lanes of NV values.
bool in_packs(const void* p, int dtype, int64_t E, int64_t ld, int NV) {
  const int N = dtype == SF_F32 ? 4 : 8;
  return NV % N == 0 && E % N == 0 && ld % N == 0 && reinterpret_cast<uintptr_t>(p) % 16 == 0;
}

// The two largest of a group's choice values.
struct Top2 {
  float a = neg_inf(), b = neg_inf();
  __device__ __forceinline__ void add(float v) {
    b = fmaxf(b, fminf(a, v));
    a = fmaxf(a, v);
  }
  __device__ __forceinline__ void merge(float oa, float ob) {
    b = fmaxf(fminf(a, oa), fmaxf(b, ob));
    a = fmaxf(a, oa);
  }
};

// Values of a token that are ranked, kRounds a lane.
template <int LPT>
struct Gather {
  static constexpr int kRounds = LPT == 8 ? 4 : LPT == 16 ? 3 : 2, kMost = LPT * kRounds;
};

// Larger for the larger choice value, and for the lower of two experts with equal ones (both zeros are).
__device__ __forceinline__ uint64_t rank_key(float u, int e) {
  const uint32_t b = __float_as_uint(u + 0.f);
  return uint64_t((b & 0x80000000u) ? ~b : b | 0x80000000u) << 32 | (0xffffffffu - static_cast<uint32_t>(e));
}

// An ordered integer of a lane's value; -inf is 0 but for the lane's bits.
template <int LPT>
__device__ __forceinline__ uint32_t lane_key(float u, int slot) {
  const uint32_t b = __float_as_uint(u);
  const uint32_t k = u == neg_inf() ? 0u : (b & 0x80000000u) ? ~b : b | 0x80000000u;
  return (k & ~uint32_t(LPT - 1)) | static_cast<uint32_t>(LPT - 1 - slot);
}
// The value of an ordered integer; 0 (no value): -inf.
__device__ __forceinline__ float key_value(uint32_t k) {
  return k == 0 ? neg_inf() : __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k);
}

// How a token's experts lie in its lanes: a group's in `lanes` lanes (a power of
// two), `each` consecutive ones a lane.
struct RouteShape {
  int lanes, each;
  bool packs;
};

template <int NV, int LPT, bool kSigmoid>
__global__ void __launch_bounds__(kThreads, NV > 8 ? 3 : 4) route_kernel(const RouteJob j, const RouteShape shape) {
  constexpr int kTokens = 32 / LPT;  // of a warp
  constexpr int kRounds = Gather<LPT>::kRounds, kGathered = Gather<LPT>::kMost;
  constexpr int kPad = NV % 4 == 0 ? 4 : 0;  // of a lane's biases, which then lie in banks of their own
  extern __shared__ __align__(16) float dynamic[];  // biases, loads [E]
  __shared__ __align__(16) uint64_t all_keys[kWarps][kTokens][kGathered];  // choice value and expert, by rank_key
  __shared__ float2 all_picked[kWarps][kTokens][32];         // (score or weight, expert) of the chosen
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, slot = lane & (LPT - 1), first_lane = lane - slot;
  const int E = static_cast<int>(j.E), k = j.cfg.k, dtype = j.dtype, top_groups = j.cfg.top_groups;
  const bool grouped = top_groups < j.cfg.groups;
  const int G = grouped ? j.cfg.groups : 1, per = E / G;
  const int group = slot / shape.lanes, within = (slot & (shape.lanes - 1)) * shape.each;
  const int e0 = group * per + within;  // this lane's first expert, and how many it has
  const int count = group < G ? max(0, min(shape.each, per - within)) : 0;
  const auto consecutive = [&](int p, int n) { return e0 + p * n; };
  float* biases = dynamic;
  int32_t* hist = reinterpret_cast<int32_t*>(biases + LPT * (NV + kPad));
  uint64_t* keys = all_keys[warp][lane / LPT];
  float2* picked = all_picked[warp][lane / LPT];
  if (threadIdx.x < LPT) {  // a token's lanes, each its own; not available past its last expert
    for (int i = 0; i < NV; ++i)
      biases[slot * (NV + kPad) + i] = i >= count ? neg_inf() : j.bias != nullptr ? j.bias[e0 + i] : 0.f;
  }
  for (int e = threadIdx.x; e < E; e += kThreads) hist[e] = 0;
  __syncthreads();
  const float* bias = biases + slot * (NV + kPad);
  float error = kSigmoidError;
  bool odd_bias = false;  // biases that are not finite
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (i < count) {
      odd_bias |= !finite(bias[i]);
      if (finite(bias[i])) error = fmaxf(error, kSigmoidError + fabsf(bias[i]) * 0x1p-22f);  // its sums' roundings
    }
  error = token_max<LPT>(error);
  odd_bias = __any_sync(kFull, odd_bias);
  uint32_t bits = 0;
  for (int64_t t0 = (blockIdx.x * int64_t(kWarps) + warp) * kTokens; t0 < j.T;
       t0 += int64_t(gridDim.x) * kWarps * kTokens) {
    const int64_t t = t0 + lane / LPT;
    const bool real = t < j.T;
    int found = 0;  // experts chosen
    for (bool exact = !kSigmoid;; exact = true) {
      float u[NV], odd = 0.f;
      Top2 best;
      load_lane<NV>(j.logits, t * j.ld, dtype, real ? e0 + count : 0, shape.packs, consecutive, u);
      if (!exact) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          odd = fmaf(u[i], 0.f, odd);  // NaN for infinities and NaN
          u[i] = sigmoid_fast(u[i]) + bias[i];
          best.add(u[i]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          odd = fmaf(u[i], 0.f, odd);
          u[i] = (kSigmoid ? sigmoid(u[i]) : u[i]) + bias[i];
          best.add(u[i]);
        }
      }
      if (__any_sync(kFull, odd != 0.f || odd_bias)) {  // logits or biases that are not finite, and padding that is -inf
        best = Top2();
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const float z = real && i < count ? load_value(j.logits, t * j.ld + e0 + i, dtype) : neg_inf();
          if (z == neg_inf()) {
            u[i] = neg_inf();
          } else if (u[i] != u[i] || (!kSigmoid && z == -neg_inf())) {
            bits |= SF_ST_NONFINITE;
            u[i] = neg_inf();
          }
          best.add(u[i]);
        }
      }
      const float margin = exact ? 0.f : 2.f * error;  // of two values' difference
      bool open = false;                               // undecided within the margin
      bool live = real;                                // whether this lane's group may be chosen from
      if (grouped) {
        // a group is kept if fewer than top_groups come before it
        Top2 all = best;
        for (int o = 1; o < shape.lanes; o <<= 1)
          all.merge(__shfl_xor_sync(kFull, all.a, o), __shfl_xor_sync(kFull, all.b, o));
        const float value = j.cfg.group_top > 1 && all.b != neg_inf() ? all.a + all.b : all.a;
        int before = 0, close = 0;  // for certain, perhaps
        if (exact) {
          for (int g = 0; g < G; ++g) {
            const float o = __shfl_sync(kFull, value, first_lane + g * shape.lanes);
            before += o > value || (o == value && g < group);
          }
        } else {
          const float above = value + 2.f * margin, near = value - 2.f * margin;
          for (int g = 0; g < G; ++g) {
            const float o = __shfl_sync(kFull, value, first_lane + g * shape.lanes);
            before += o > above;
            close += o >= near;  // itself and equal ones, so that infinite values are told apart exactly
          }
          --close;
        }
        open = value != neg_inf() && before < top_groups && close >= top_groups;
        live &= before < top_groups;
      }
      if (!live) best = Top2();
      // the bound: the k-th largest of the lanes' two largest, as ordered integers whose lowest bits are the
      // lane's, so that no two are equal (and the bound a little lower than it could be)
      uint32_t a = lane_key<LPT>(best.a, slot), b = lane_key<LPT>(best.b, slot), kth = 0;
      for (int c = 0; c < k; ++c) {
        kth = token_max<LPT>(a);
        if (a == kth) {
          a = b;
          b = 0;
        }
      }
      float bound = key_value(kth & ~uint32_t(LPT - 1));
      bound = fmaxf(bound - margin, -3.402823466e38f);  // not -inf: no expert that is not available
      // the values that may be among the k largest
      uint32_t mine = 0;
#pragma unroll
      for (int i = 0; i < NV; ++i) mine |= u[i] >= bound ? 1u << i : 0u;
      if (!live) mine = 0;
      int end = __popc(mine);
      int at = -end;
#pragma unroll
      for (int o = 1; o < LPT; o <<= 1) {
        const int up = __shfl_up_sync(kFull, end, o, LPT);
        if (slot >= o) end += up;
      }
      at += end;
      const int n = __shfl_sync(kFull, end, LPT - 1, LPT);
      if (__any_sync(kFull, open || n > kGathered)) {
        if (!exact) continue;
        // too many equal values: one by one
        for (int c = 0; c < k; ++c) {
          float m = neg_inf();
#pragma unroll
          for (int i = 0; i < NV; ++i) m = fmaxf(m, live ? u[i] : neg_inf());
          const float top = token_max<LPT>(m);
          const uint32_t who = token_bits<LPT>(__ballot_sync(kFull, m == top), lane);
          const int owner = __ffs(static_cast<int>(who)) - 1;
          int taken = -1;
#pragma unroll
          for (int i = 0; i < NV; ++i)
            if (slot == owner && taken < 0 && top != neg_inf() && u[i] == top) {
              taken = e0 + i;
              u[i] = neg_inf();
            }
          taken = __shfl_sync(kFull, taken, owner, LPT);
          if (taken >= 0) {
            if (slot == owner) {
              const float z = load_value(j.logits, t * j.ld + taken, dtype);
              picked[c] = make_float2(kSigmoid ? sigmoid(z) : z, __int_as_float(taken));
            }
            found = c + 1;
          }
        }
        break;
      }
      found = min(n, k);
      for (; mine != 0; mine &= mine - 1) keys[at++] = static_cast<uint32_t>(e0 + __ffs(static_cast<int>(mine)) - 1);
      __syncwarp();
      const int most = kTokens == 1 ? n : __reduce_max_sync(kFull, n);  // of the warp's tokens
      int e[kRounds], rank[kRounds];  // of this lane's gathered values
      float score[kRounds];           // sigmoid or logit
      uint64_t key[kRounds];
#pragma unroll
      for (int r = 0; r < kRounds; ++r) {
        if (r * LPT >= most) break;
        rank[r] = kGathered;
        key[r] = ~uint64_t(0);
        if (r * LPT + slot < n) {
          e[r] = static_cast<int>(keys[r * LPT + slot]);
          score[r] = load_value(j.logits, t * j.ld + e[r], dtype);
          if (kSigmoid) score[r] = sigmoid(score[r]);
          key[r] = rank_key(score[r] + (j.bias != nullptr ? j.bias[e[r]] : 0.f), e[r]);
          keys[r * LPT + slot] = key[r];
          rank[r] = 0;
        }
      }
      __syncwarp();
      for (int i = 0; i < n; i += 2) {
        const ulonglong2 o = *reinterpret_cast<const ulonglong2*>(keys + i);
        const uint64_t second = i + 1 < n ? o.y : 0;
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
          if (r * LPT >= most) break;
          rank[r] += (o.x > key[r]) + (second > key[r]);
        }
      }
#pragma unroll
      for (int r = 0; r < kRounds; ++r) {
        if (r * LPT >= most) break;
        if (rank[r] < k) picked[rank[r]] = make_float2(score[r], __int_as_float(e[r]));
      }
      break;
    }
    __syncwarp();
    // weights, by the order of choice
    float m = neg_inf(), sum = 0.f;
    if (!kSigmoid && j.cfg.renorm) {
      for (int c = slot; c < found; c += LPT) m = fmaxf(m, picked[c].x);
      m = token_max<LPT>(m);
    } else if (!kSigmoid) {
      float z[NV];
      load_lane<NV>(j.logits, t * j.ld, dtype, real ? e0 + count : 0, shape.packs, consecutive, z);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (!(z[i] < -neg_inf()) || i >= count) z[i] = neg_inf();  // faulty ones, and no experts
        m = fmaxf(m, z[i]);
      }
      m = token_max<LPT>(m);
      const float from = m == neg_inf() ? 0.f : m;
#pragma unroll
      for (int i = 0; i < NV; ++i) sum += exp_fast(z[i] - from);
    }
    if (!kSigmoid || j.cfg.renorm) {
      for (int c = slot; c < found; c += LPT) {
        float w = picked[c].x;
        if (!kSigmoid) picked[c].x = w = expf(w - m);
        if (j.cfg.renorm) sum += w;
      }
      sum = token_sum<LPT>(sum);
    } else {
      sum = 1.f;
    }
    if (real)
      for (int c = slot; c < k; c += LPT) {
        const bool is = c < found;  // fewer experts than k: -1
        const float2 o = is ? picked[c] : make_float2(0.f, __int_as_float(-1));
        j.index[t * k + c] = __float_as_int(o.y);
        j.weight[t * k + c] = is && sum > 0.f ? o.x / sum * j.cfg.scale : 0.f;
        if (is) atomicAdd(hist + __float_as_int(o.y), 1);
      }
    __syncwarp();
  }
  report(j.status, bits);
  if (j.load == nullptr) return;
  __syncthreads();
  if (j.only_cta) {  // the totals are this CTA's counts
    for (int e = threadIdx.x; e < E; e += kThreads) j.load[e] = hist[e];
    return;
  }
  griddep_wait();  // the totals have been cleared
  for (int e = threadIdx.x; e < E; e += kThreads)
    if (hist[e] != 0) atomicAdd(j.load + e, hist[e]);
}

// Any number of experts and groups, by a warp a token and from shared memory:
// for shapes whose groups do not lie in whole lanes of up to 32 values (more
// than 32 (32 / groups) experts a group).  The k chosen are taken one by one.
__global__ void __launch_bounds__(kThreads) route_any_kernel(const RouteJob j) {
  extern __shared__ __align__(16) float dynamic[];  // choice values [kWarps][E], loads [E]
  __shared__ float group_values[kWarps][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int E = static_cast<int>(j.E), k = j.cfg.k, G = j.cfg.groups, per = E / G, dtype = j.dtype;
  const bool sigmoids = j.cfg.score == SF_SCORE_SIGMOID;
  float* u = dynamic + warp * E;
  int32_t* hist = reinterpret_cast<int32_t*>(dynamic + kWarps * E);
  for (int e = threadIdx.x; e < E; e += kThreads) hist[e] = 0;
  __syncthreads();
  uint32_t bits = 0;
  for (int64_t t = blockIdx.x * int64_t(kWarps) + warp; t < j.T; t += int64_t(gridDim.x) * kWarps) {
    float m = neg_inf(), sum = 0.f;
    __syncwarp();
    for (int e = lane; e < E; e += 32) {
      const float z = load_value(j.logits, t * j.ld + e, dtype);
      float v = (sigmoids ? sigmoid(z) : z) + (j.bias != nullptr ? j.bias[e] : 0.f);
      if (z == neg_inf()) v = neg_inf();
      if (z != neg_inf() && (v != v || (!sigmoids && z == -neg_inf()))) {
        bits |= SF_ST_NONFINITE;
        v = neg_inf();
      }
      u[e] = v;
      if (z < -neg_inf()) m = fmaxf(m, z);
    }
    __syncwarp();
    Top2 best;
    if (lane < G)
      for (int i = 0; i < per; ++i) best.add(u[lane * per + i]);
    const float value = j.cfg.group_top > 1 && best.b != neg_inf() ? best.a + best.b : best.a;
    if (lane < G) group_values[warp][lane] = value;
    __syncwarp();
    int before = 0;
    for (int g = 0; g < G; ++g) {
      const float o = group_values[warp][g];
      before += o > value || (o == value && g < lane);
    }
    const uint32_t kept = __ballot_sync(kFull, lane < G && before < j.cfg.top_groups);
    int chosen = -1;
    float score = neg_inf();
    for (int c = 0; c < k; ++c) {
      float top = neg_inf();
      int at = E;
      for (int e = lane; e < E; e += 32)
        if (((kept >> (e / per)) & 1u) && u[e] > top) {
          top = u[e];
          at = e;
        }
      const float most = token_max<32>(top);
      if (most == neg_inf()) break;
      at = __reduce_min_sync(kFull, top == most ? at : E);
      if (lane == 0) u[at] = neg_inf();
      __syncwarp();
      if (lane == c) {
        chosen = at;
        score = load_value(j.logits, t * j.ld + at, dtype);
      }
    }
    float w;
    if (sigmoids) {
      w = chosen >= 0 ? sigmoid(score) : 0.f;
      sum = 1.f;
    } else {
      m = token_max<32>(j.cfg.renorm ? score : m);
      w = chosen >= 0 ? expf(score - m) : 0.f;
      if (!j.cfg.renorm)
        for (int e = lane; e < E; e += 32) {
          const float z = load_value(j.logits, t * j.ld + e, dtype);
          if (z < -neg_inf() && z != neg_inf()) sum += exp_fast(z - m);
        }
      sum = token_sum<32>(sum);
    }
    if (j.cfg.renorm) sum = token_sum<32>(w);
    if (lane < k) {
      j.index[t * k + lane] = chosen;
      j.weight[t * k + lane] = chosen >= 0 && sum > 0.f ? w / sum * j.cfg.scale : 0.f;
      if (chosen >= 0) atomicAdd(hist + chosen, 1);
    }
  }
  report(j.status, bits);
  if (j.load == nullptr) return;
  griddep_wait();  // the totals have been cleared
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += kThreads) {
    if (j.only_cta)
      j.load[e] = hist[e];
    else if (hist[e] != 0)
      atomicAdd(j.load + e, hist[e]);
  }
}

template <int NV, int LPT>
cudaError_t launch_route_lanes(const RouteJob& j, const RouteShape& shape, bool after_clear, cudaStream_t stream) {
  constexpr int kTokens = kWarps * 32 / LPT;  // of a CTA
  const size_t smem = (size_t(LPT) * (NV + 4) + size_t(j.E)) * 4;
  const int64_t ctas = (j.T + kTokens - 1) / kTokens;
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>(ctas, int64_t(sm_count()) * 8)));
  count_launch();
  const auto kern = j.cfg.score == SF_SCORE_SIGMOID ? route_kernel<NV, LPT, true> : route_kernel<NV, LPT, false>;
  return launch_after(kern, grid, dim3(kThreads), smem, stream, after_clear, j, shape);
}

template <int LPT>
cudaError_t launch_route_width(const RouteJob& j, RouteShape shape, bool after_clear, cudaStream_t stream) {
  const auto go = [&](auto nv) {
    constexpr int NV = decltype(nv)::value;
    const int N = j.dtype == SF_F32 ? 4 : 8;
    const int64_t per = j.cfg.top_groups < j.cfg.groups ? j.E / j.cfg.groups : j.E;
    shape.packs = shape.each % N == 0 && in_packs(j.logits, j.dtype, per, j.ld, NV);
    return launch_route_lanes<NV, LPT>(j, shape, after_clear, stream);
  };
  if constexpr (LPT == 32) {
    if (shape.each <= 1) return go(std::integral_constant<int, 1>());
    if (shape.each <= 2) return go(std::integral_constant<int, 2>());
  }
  if (shape.each <= 4) return go(std::integral_constant<int, 4>());
  if (shape.each <= 8) return go(std::integral_constant<int, 8>());
  if (shape.each <= 16) return go(std::integral_constant<int, 16>());
  if (shape.each <= 24) return go(std::integral_constant<int, 24>());
  return go(std::integral_constant<int, 32>());
}

// The shape for LPT lanes a token; each = 0: they do not do.
RouteShape shape_of(const RouteJob& j, int LPT) {
  RouteShape s{0, 0, false};
  const bool grouped = j.cfg.top_groups < j.cfg.groups;
  const int G = grouped ? j.cfg.groups : 1, kept = grouped ? j.cfg.top_groups : 1;
  if (G > LPT) return s;
  s.lanes = 1;
  while (s.lanes * 2 * G <= LPT) s.lanes *= 2;
  const int per = static_cast<int>(j.E) / G, N = j.dtype == SF_F32 ? 4 : 8;
  int each = (per + s.lanes - 1) / s.lanes;
  if (per % N == 0 && each > 2) each = (each + N - 1) / N * N;  // whole packs
  // two values each of the lanes that are kept bound the k-th largest; a lane holds up to 32 values, 16
  // of f32 while there are more lanes to have (us, 65536 tokens to 8 of 256 experts with 32 / 16 values:
  // sigmoid f32 50 / 46, in groups 58 / 52; softmax bf16 38 / 44)
  if (each > (LPT < 32 && N == 4 ? 16 : 32) || (LPT < 32 && 2 * s.lanes * kept < j.cfg.k)) return s;
  s.each = each;
  return s;
}

// Gradient: the chosen experts' lanes put their own values (or, where all
// experts have a gradient, their upstream gradients) into a row of zeros in
// shared memory, from which every lane takes its NV.  Several tokens a warp:
// their reads, two of which wait for one another, are in flight together.  Bound
// by the latency of those reads: as many tokens a warp, and warps an SM, as the
// registers allow (100003 x 160 bf16 over all experts: 35 us with two tokens of 16
// lanes, 29 with four of 8).  65536 x 256 f32: 17 us (4.0 TB/s written), over all
// experts 23 us (5.8 TB/s).
template <int NV, int LPT, bool kDense>
__global__ void __launch_bounds__(kThreads, NV > 16 ? 3 : kDense ? 4 : 5) route_grad_kernel(const RouteGradJob j, const bool packs) {
  constexpr int kTokens = 32 / LPT;  // of a warp
  extern __shared__ __align__(16) float rows[];  // [kWarps * 32][NV]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, slot = lane & (LPT - 1);
  const int E = static_cast<int>(j.E), k = j.cfg.k, dtype = j.dtype;
  float* d = rows + (warp * 32 + lane - slot) * NV;
  // a token's lanes take its packs in turn, whether they are read as packs or not: the sums' order is one
  const int width = dtype == SF_F32 ? 4 : 8;
  const auto in_turn = [&](int p, int n) {
    return n == 1 ? (p / width * LPT + slot) * width + p % width : (p * LPT + slot) * n;
  };
  const bool sigmoids = j.cfg.score == SF_SCORE_SIGMOID;
  uint32_t bits = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) d[i * LPT + slot] = 0.f;
  // the slots of the token after this one are read ahead: a logit waits for its index
  const int64_t step = int64_t(gridDim.x) * kWarps * kTokens;
  int64_t t = (blockIdx.x * int64_t(kWarps) + warp) * kTokens + lane / LPT;
  int next_e = -1;
  float next_dw = 0.f;
  if (t < j.T && slot < k) {
    next_e = j.index[t * k + slot];
    next_dw = j.dweight[t * k + slot];
  }
  for (; t - lane / LPT < j.T; t += step) {
    const bool real = t < j.T;
    int e = next_e;
    float dw = next_dw, z = neg_inf();
    if (e < -1 || e >= E) {
      bits |= SF_ST_INDEX;
      e = -1;
    }
    if (e >= 0)
      z = load_value(j.logits, t * j.ld + e, dtype);
    else
      dw = 0.f;
    float all[NV];
    if (kDense) {
      load_lane<NV>(j.logits, t * j.ld, dtype, real ? E : 0, packs, in_turn, all);
      if (in_turn(NV - 1, 1) >= E) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if (in_turn(i, 1) >= E) all[i] = neg_inf();
      }
    }
    next_e = -1;
    if (t + step < j.T && slot < k) {
      next_e = j.index[(t + step) * k + slot];
      next_dw = j.dweight[(t + step) * k + slot];
    }
    float g = 0.f, s, inner;
    if (kDense) {
      float m = all[0];
#pragma unroll
      for (int i = 1; i < NV; ++i) m = fmaxf(m, all[i]);
      m = token_max<LPT>(m);
      if (m == neg_inf()) m = 0.f;  // no expert: a sum of 0, or NaN
      s = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        all[i] = exp_fast(all[i] - m);
        s += all[i];
      }
      s = token_sum<LPT>(s);
      inner = token_sum<LPT>(exp_fast(z - m) * dw);
      const bool sound = finite(s);
      if (!sound) bits |= SF_ST_NONFINITE;
      s = sound && s > 0.f ? 1.f / s : 0.f;  // no gradient without a distribution
      inner *= s;
      if (!sound) {
        inner = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) all[i] = 0.f;
      }
      g = dw;
    } else if (sigmoids) {
      const float p = e >= 0 ? sigmoid(z) : 0.f;
      const float slope = e >= 0 ? p * (1.f / (1.f + expf(z))) : 0.f;
      if (j.cfg.renorm) {
        s = token_sum<LPT>(p);
        inner = token_sum<LPT>(p * dw);
        g = s > 0.f ? slope / s * (dw - inner / s) : 0.f;
      } else {
        g = slope * dw;
      }
    } else {
      const float m = token_max<LPT>(z), q = softmax_term(z, m);
      s = token_sum<LPT>(q);
      inner = token_sum<LPT>(q * dw);
      if (!finite(s)) bits |= SF_ST_NONFINITE;
      s = finite(s) && s > 0.f ? 1.f / s : 0.f;
      g = s > 0.f ? q * s * (dw - inner * s) : 0.f;
    }
    __syncwarp();  // the row is zeros
    if (e >= 0) d[e] = kDense ? g : g * j.cfg.scale;
    __syncwarp();
    float v[NV];
    const float c = kDense ? s * j.cfg.scale : 0.f, shift = kDense ? -inner * c : 0.f;
    const auto take = [&](auto n) {
      constexpr int N = decltype(n)::value;
#pragma unroll
      for (int i = 0; i < NV; ++i) v[i] = d[((i / N) * LPT + slot) * N + i % N];
    };
    if (width == 8)
      take(std::integral_constant<int, 8>());
    else
      take(std::integral_constant<int, 4>());
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (kDense) v[i] = all[i] * fmaf(v[i], c, shift);
    }
    __syncwarp();
    if (e >= 0) d[e] = 0.f;
    store_lane<NV>(j.dlogits, t * j.ldd, dtype, real ? E : 0, packs, in_turn, v);
  }
  report(j.status, bits);
}

template <int NV, int LPT>
cudaError_t launch_grad_lanes(const RouteGradJob& j, cudaStream_t stream) {
  constexpr int kTokens = kWarps * 32 / LPT;
  const int64_t ctas = (j.T + kTokens - 1) / kTokens;
  const int grid = static_cast<int>(std::min<int64_t>(ctas, int64_t(sm_count()) * 8));
  const bool packs = in_packs(j.logits, j.dtype, j.E, j.ld, NV) && in_packs(j.dlogits, j.dtype, j.E, j.ldd, NV);
  const bool dense = j.cfg.score == SF_SCORE_SOFTMAX && !j.cfg.renorm;
  const auto kern = dense ? route_grad_kernel<NV, LPT, true> : route_grad_kernel<NV, LPT, false>;
  count_launch();
  kern<<<grid, kThreads, size_t(kThreads) * NV * 4, stream>>>(j, packs);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_route(RouteJob j, bool accumulate, cudaStream_t stream) {
  bool after_clear = false;
  j.only_cta = !accumulate && j.T <= kWarps;
  if (j.load != nullptr && !accumulate && !j.only_cta) {
    ZeroList z;
    z.add(j.load, size_t(j.E) * sizeof(int32_t));
    const cudaError_t e = launch_zero_many(z, stream, &after_clear);
    if (e != cudaSuccess) return e;
  }
  // as few lanes a token as do: what is not per value is shared by more tokens
  if (const RouteShape s = shape_of(j, 8); s.each > 0) return launch_route_width<8>(j, s, after_clear, stream);
  if (const RouteShape s = shape_of(j, 16); s.each > 0) return launch_route_width<16>(j, s, after_clear, stream);
  if (const RouteShape s = shape_of(j, 32); s.each > 0) return launch_route_width<32>(j, s, after_clear, stream);
  const int64_t ctas = std::min<int64_t>((j.T + kWarps - 1) / kWarps, int64_t(sm_count()) * 4);
  count_launch();
  return launch_after(route_any_kernel, dim3(static_cast<unsigned>(ctas)), dim3(kThreads),
                      size_t(j.E) * 4 * (kWarps + 1), stream, after_clear, j);
}

cudaError_t launch_route_grad(const RouteGradJob& j, cudaStream_t stream) {
  // as few lanes a token as have its k experts one each and its row in 16 to 32 values
  if (j.cfg.k <= 8 && j.E <= 64) return launch_grad_lanes<8, 8>(j, stream);
  if (j.cfg.k <= 8 && j.E <= 128) return launch_grad_lanes<16, 8>(j, stream);
  if (j.cfg.k <= 8 && j.E <= 192) return launch_grad_lanes<24, 8>(j, stream);
  if (j.cfg.k <= 8 && j.E <= 256) return launch_grad_lanes<32, 8>(j, stream);
  if (j.cfg.k <= 16 && j.E <= 128) return launch_grad_lanes<8, 16>(j, stream);
  if (j.cfg.k <= 16 && j.E <= 256) return launch_grad_lanes<16, 16>(j, stream);
  if (j.E <= 256) return launch_grad_lanes<8, 32>(j, stream);
  if (j.E <= 512) return launch_grad_lanes<16, 32>(j, stream);
  return launch_grad_lanes<32, 32>(j, stream);
}

}  // namespace sf
