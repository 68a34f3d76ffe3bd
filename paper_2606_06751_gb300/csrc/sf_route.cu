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
// exactly, and taken one by one if there are too many equal ones.
#include <algorithm>

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

// exp(x) for x <= 0 by ex2.approx, for sums and terms that are good to 1e-6.
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

template <typename T, int NV>
__device__ __forceinline__ void load_packs(const T* row, int e0, int E, float (&z)[NV]) {
  constexpr int N = Pack<T>::kN;
  if constexpr (NV % N == 0) {
#pragma unroll
    for (int p = 0; p < NV / N; ++p) {
      float f[N];
      unpack(e0 + p * N < E ? *reinterpret_cast<const uint4*>(row + e0 + p * N) : same4(0u), f, T());
#pragma unroll
      for (int q = 0; q < N; ++q) z[p * N + q] = f[q];
    }
  }
}
// A lane's NV values of the row that starts at element `at`, from e0; 0 past the
// row's end.  `packs`: in 16-byte packs (see in_packs).
template <int NV>
__device__ __forceinline__ void load_lane(const void* p, int64_t at, int dtype, int e0, int E, bool packs,
                                          float (&z)[NV]) {
  if (packs && dtype == SF_F32) return load_packs(static_cast<const float*>(p) + at, e0, E, z);
  if (packs && dtype == SF_BF16) return load_packs(static_cast<const __nv_bfloat16*>(p) + at, e0, E, z);
  if (packs) return load_packs(static_cast<const __half*>(p) + at, e0, E, z);
#pragma unroll
  for (int i = 0; i < NV; ++i) z[i] = e0 + i < E ? load_value(p, at + e0 + i, dtype) : 0.f;
}

template <typename T, int NV>
__device__ __forceinline__ void store_packs(T* row, int e0, int E, const float (&v)[NV]) {
  constexpr int N = Pack<T>::kN;
  if constexpr (NV % N == 0) {
#pragma unroll
    for (int p = 0; p < NV / N; ++p) {
      float f[N];
#pragma unroll
      for (int q = 0; q < N; ++q) f[q] = v[p * N + q];
      if (e0 + p * N < E) store16(row + e0 + p * N, pack(f, T()));
    }
  }
}
template <int NV>
__device__ __forceinline__ void store_lane(void* p, int64_t at, int dtype, int e0, int E, bool packs,
                                           const float (&v)[NV]) {
  if (packs && dtype == SF_F32) return store_packs(static_cast<float*>(p) + at, e0, E, v);
  if (packs && dtype == SF_BF16) return store_packs(static_cast<__nv_bfloat16*>(p) + at, e0, E, v);
  if (packs) return store_packs(static_cast<__half*>(p) + at, e0, E, v);
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (e0 + i < E) store_value(p, at + e0 + i, dtype, v[i]);
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

constexpr int kGathered = 32;  // values of a token that are ranked

// Shared memory of a warp: a token's gathered values each.
template <int LPT>
struct Gathered {
  float2 key[32 / LPT][kGathered];  // (choice value, expert)
};

template <int NV, int LPT, bool kSigmoid>
__global__ void __launch_bounds__(kThreads, NV > 8 ? 3 : 4) route_kernel(const RouteJob j, const bool packs) {
  constexpr int kTokens = 32 / LPT;  // of a warp
  constexpr int kRounds = kGathered / LPT;
  constexpr int kPad = NV % 4 == 0 ? 4 : 0;  // of a lane's biases, which then lie in banks of their own
  extern __shared__ __align__(16) float dynamic[];  // biases, loads [E]; where needed, choice values [kWarps * kTokens][E]
  __shared__ Gathered<LPT> gathered[kWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, slot = lane & (LPT - 1), first = lane - slot;
  const int E = static_cast<int>(j.E), k = j.cfg.k, e0 = slot * NV, dtype = j.dtype;
  const int G = j.cfg.groups, per = E / G, top_groups = j.cfg.top_groups;
  const bool grouped = top_groups < G;
  // groups of a power of two of whole lanes: by shuffles; others through shared memory
  const int group_lanes = per % NV == 0 ? per / NV : 0;
  const bool shuffles = group_lanes > 0 && (group_lanes & (group_lanes - 1)) == 0;
  float* biases = dynamic;
  int32_t* hist = reinterpret_cast<int32_t*>(biases + LPT * (NV + kPad));
  float* values = reinterpret_cast<float*>(hist + E) + (warp * kTokens + lane / LPT) * E;
  float2* keys = gathered[warp].key[lane / LPT];
  for (int e = threadIdx.x; e < LPT * NV; e += kThreads)  // past the last expert: not available
    biases[e + e / NV * kPad] = e >= E ? neg_inf() : j.bias != nullptr ? j.bias[e] : 0.f;
  for (int e = threadIdx.x; e < E; e += kThreads) hist[e] = 0;
  __syncthreads();
  const float* bias = biases + slot * (NV + kPad);
  float error = kSigmoidError;
  bool odd_bias = false;  // biases that are not finite
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (e0 + i < E) {
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
    int e[kRounds], rank[kRounds];  // of this lane's gathered values
    float score[kRounds];           // sigmoid or logit
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      e[r] = -1;
      rank[r] = kGathered;
      score[r] = 0.f;
    }
    for (bool exact = !kSigmoid;; exact = true) {
      float u[NV], odd = 0.f;
      Top2 best;
      load_lane<NV>(j.logits, t * j.ld, dtype, e0, real ? E : 0, packs, u);
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
          const float z = real && e0 + i < E ? load_value(j.logits, t * j.ld + e0 + i, dtype) : neg_inf();
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
        const auto kept = [&](float value, int mine, const auto& other) {
          int before = 0, close = 0;  // for certain, perhaps
          for (int g = 0; g < G; ++g) {
            const float o = other(g);
            const bool tie = exact && o == value && g < mine;
            before += o > value + 2.f * margin || tie;
            close += (g != mine && o > value - 2.f * margin) || tie;
          }
          open |= value != neg_inf() && before < top_groups && close >= top_groups;
          return before < top_groups;
        };
        if (shuffles) {
          Top2 all = best;
          for (int o = 1; o < group_lanes; o <<= 1)
            all.merge(__shfl_xor_sync(kFull, all.a, o), __shfl_xor_sync(kFull, all.b, o));
          const float value = j.cfg.group_top > 1 && all.b != neg_inf() ? all.a + all.b : all.a;
          live &= kept(value, slot / group_lanes,
                       [&](int g) { return __shfl_sync(kFull, value, first + g * group_lanes); });
        } else {
          __syncwarp();
#pragma unroll
          for (int i = 0; i < NV; ++i)
            if (e0 + i < E) values[e0 + i] = u[i];
          __syncwarp();
          for (int g = slot; g < G; g += LPT) {
            Top2 b;
            for (int i = 0; i < per; ++i) b.add(values[g * per + i]);
            // in the group's first place, which only this lane has read
            values[g * per] = j.cfg.group_top > 1 && b.b != neg_inf() ? b.a + b.b : b.a;
          }
          __syncwarp();
          uint32_t mask = 0;
          for (int r = 0; r < G; r += LPT) {
            const int g = r + slot;
            const bool keep = g < G && kept(values[g * per], g, [&](int o) { return values[o * per]; });
            mask |= token_bits<LPT>(__ballot_sync(kFull, keep), lane) << r;
          }
          best = Top2();
#pragma unroll
          for (int i = 0; i < NV; ++i) {
            if (e0 + i < E && !((mask >> ((e0 + i) / per)) & 1u)) u[i] = neg_inf();
            best.add(u[i]);
          }
        }
      }
      if (!live) best = Top2();
      // the bound: the k-th largest of the lanes' two largest
      float bound = neg_inf();
      for (int c = 0; c < k; ++c) {
        bound = token_max<LPT>(best.a);
        const uint32_t at = token_bits<LPT>(__ballot_sync(kFull, best.a == bound), lane);
        if (slot == __ffs(static_cast<int>(at)) - 1) {
          best.a = best.b;
          best.b = neg_inf();
        }
      }
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
#pragma unroll
          for (int r = 0; r < kRounds; ++r)
            if (r * LPT + slot == c && taken >= 0) {
              e[r] = taken;
              rank[r] = c;
              score[r] = load_value(j.logits, t * j.ld + taken, dtype);
              if (kSigmoid) score[r] = sigmoid(score[r]);
            }
        }
        break;
      }
      for (; mine != 0; mine &= mine - 1) keys[at++].y = __int_as_float(e0 + __ffs(static_cast<int>(mine)) - 1);
      __syncwarp();
      float uc[kRounds];
#pragma unroll
      for (int r = 0; r < kRounds; ++r) {
        uc[r] = neg_inf();
        if (r * LPT + slot < n) {
          e[r] = __float_as_int(keys[r * LPT + slot].y);
          score[r] = load_value(j.logits, t * j.ld + e[r], dtype);
          if (kSigmoid) score[r] = sigmoid(score[r]);
          uc[r] = score[r] + biases[e[r] + e[r] / NV * kPad];
          keys[r * LPT + slot].x = uc[r];
          rank[r] = 0;
        }
      }
      __syncwarp();
      for (int i = 0; i < n; ++i) {
        const float2 o = keys[i];
#pragma unroll
        for (int r = 0; r < kRounds; ++r) rank[r] += o.x > uc[r] || (o.x == uc[r] && __float_as_int(o.y) < e[r]);
      }
      __syncwarp();
      break;
    }
    // weights
    float w[kRounds], sum = 0.f;
    int found = 0;
    if (kSigmoid) {
#pragma unroll
      for (int r = 0; r < kRounds; ++r) w[r] = rank[r] < k ? score[r] : 0.f;
    } else {
      float m = neg_inf();
      float z[NV];
      if (j.cfg.renorm) {
#pragma unroll
        for (int r = 0; r < kRounds; ++r) m = fmaxf(m, rank[r] < k ? score[r] : neg_inf());
      } else {
        load_lane<NV>(j.logits, t * j.ld, dtype, e0, real ? E : 0, packs, z);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          if (!(z[i] < -neg_inf()) || e0 + i >= E) z[i] = neg_inf();  // faulty ones, and no experts
          m = fmaxf(m, z[i]);
        }
      }
      m = token_max<LPT>(m);
#pragma unroll
      for (int r = 0; r < kRounds; ++r) w[r] = rank[r] < k ? expf(score[r] - m) : 0.f;
      if (!j.cfg.renorm) {
        if (m == neg_inf()) m = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) sum += exp_fast(z[i] - m);
        sum = token_sum<LPT>(sum);
      }
    }
    if (j.cfg.renorm) {
#pragma unroll
      for (int r = 0; r < kRounds; ++r) sum += w[r];
      sum = token_sum<LPT>(sum);
    } else if (kSigmoid) {
      sum = 1.f;
    }
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      if (rank[r] < k) {
        j.index[t * k + rank[r]] = e[r];
        j.weight[t * k + rank[r]] = sum > 0.f ? w[r] / sum * j.cfg.scale : 0.f;
        atomicAdd(hist + e[r], 1);
      }
      found += __popc(token_bits<LPT>(__ballot_sync(kFull, rank[r] < k), lane));
    }
    if (real)
      for (int c = found + slot; c < k; c += LPT) {  // fewer experts than k
        j.index[t * k + c] = -1;
        j.weight[t * k + c] = 0.f;
      }
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

template <int NV, int LPT>
cudaError_t launch_route_lanes(const RouteJob& j, bool after_clear, cudaStream_t stream) {
  constexpr int kTokens = kWarps * 32 / LPT;  // of a CTA
  const bool grouped = j.cfg.top_groups < j.cfg.groups;
  const size_t smem = (size_t(LPT) * (NV + 4) + size_t(j.E) * (grouped ? 1 + kTokens : 1)) * 4;
  const int64_t ctas = (j.T + kTokens - 1) / kTokens;
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>(ctas, int64_t(sm_count()) * 8)));
  count_launch();
  const auto kern = j.cfg.score == SF_SCORE_SIGMOID ? route_kernel<NV, LPT, true> : route_kernel<NV, LPT, false>;
  return launch_after(kern, grid, dim3(kThreads), smem, stream, after_clear, j,
                      in_packs(j.logits, j.dtype, j.E, j.ld, NV));
}

// Gradient: the chosen experts' lanes put their own values (or, where all
// experts have a gradient, their upstream gradients) into a row of zeros in
// shared memory, from which every lane takes its NV.  Several tokens a warp:
// their reads, two of which wait for one another, are in flight together.
template <int NV, int LPT, bool kDense>
__global__ void __launch_bounds__(kThreads) route_grad_kernel(const RouteGradJob j, const bool packs) {
  constexpr int kTokens = 32 / LPT;  // of a warp
  extern __shared__ __align__(16) float rows[];  // [kWarps * 32][NV]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, slot = lane & (LPT - 1);
  const int E = static_cast<int>(j.E), k = j.cfg.k, e0 = slot * NV, dtype = j.dtype;
  float* d = rows + (warp * 32 + lane - slot) * NV;
  const bool sigmoids = j.cfg.score == SF_SCORE_SIGMOID;
  uint32_t bits = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) d[e0 + i] = 0.f;
  for (int64_t t0 = (blockIdx.x * int64_t(kWarps) + warp) * kTokens; t0 < j.T; t0 += int64_t(gridDim.x) * kWarps * kTokens) {
    const int64_t t = t0 + lane / LPT;
    const bool real = t < j.T;
    float all[NV];
    if (kDense) {
      load_lane<NV>(j.logits, t * j.ld, dtype, e0, real ? E : 0, packs, all);
      if (e0 + NV > E) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if (e0 + i >= E) all[i] = neg_inf();
      }
    }
    int e = -1;
    float dw = 0.f, z = neg_inf();
    if (real && slot < k) {
      e = j.index[t * k + slot];
      dw = j.dweight[t * k + slot];
      if (e < -1 || e >= E) {
        bits |= SF_ST_INDEX;
        e = -1;
      }
      if (e >= 0)
        z = load_value(j.logits, t * j.ld + e, dtype);
      else
        dw = 0.f;
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
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      v[i] = d[e0 + i];
      if (kDense) v[i] = all[i] * fmaf(v[i], c, shift);
    }
    __syncwarp();
    if (e >= 0) d[e] = 0.f;
    store_lane<NV>(j.dlogits, t * j.ldd, dtype, e0, real ? E : 0, packs, v);
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
  // As few lanes a token as hold its row in 32 values and, two values each, one and a half times k values
  // of the groups that are kept (else the bound is loose, or there is none).
  const int64_t held = int64_t(4) * j.cfg.top_groups, need = int64_t(3) * j.cfg.k * j.cfg.groups;
  if (8 * held >= need) {
    if (j.E <= 32) return launch_route_lanes<4, 8>(j, after_clear, stream);
    if (j.E <= 64) return launch_route_lanes<8, 8>(j, after_clear, stream);
    if (j.E <= 128) return launch_route_lanes<16, 8>(j, after_clear, stream);
    if (j.E <= 256) return launch_route_lanes<32, 8>(j, after_clear, stream);
  }
  if (16 * held >= need) {
    if (j.E <= 64) return launch_route_lanes<4, 16>(j, after_clear, stream);
    if (j.E <= 128) return launch_route_lanes<8, 16>(j, after_clear, stream);
    if (j.E <= 256) return launch_route_lanes<16, 16>(j, after_clear, stream);
    if (j.E <= 512) return launch_route_lanes<32, 16>(j, after_clear, stream);
  }
  if (j.E <= 32) return launch_route_lanes<1, 32>(j, after_clear, stream);
  if (j.E <= 64) return launch_route_lanes<2, 32>(j, after_clear, stream);
  if (j.E <= 128) return launch_route_lanes<4, 32>(j, after_clear, stream);
  if (j.E <= 256) return launch_route_lanes<8, 32>(j, after_clear, stream);
  if (j.E <= 512) return launch_route_lanes<16, 32>(j, after_clear, stream);
  return launch_route_lanes<32, 32>(j, after_clear, stream);
}

cudaError_t launch_route_grad(const RouteGradJob& j, cudaStream_t stream) {
  // as few lanes a token as have its k experts one each and its row in 16 values
  if (j.cfg.k <= 8 && j.E <= 64) return launch_grad_lanes<8, 8>(j, stream);
  if (j.cfg.k <= 8 && j.E <= 128) return launch_grad_lanes<16, 8>(j, stream);
  if (j.cfg.k <= 16 && j.E <= 128) return launch_grad_lanes<8, 16>(j, stream);
  if (j.cfg.k <= 16 && j.E <= 256) return launch_grad_lanes<16, 16>(j, stream);
  if (j.E <= 256) return launch_grad_lanes<8, 32>(j, stream);
  if (j.E <= 512) return launch_grad_lanes<16, 32>(j, stream);
  return launch_grad_lanes<32, 32>(j, stream);
}

}  // namespace sf
