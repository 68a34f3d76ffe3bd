// sf_policy_loss.cu - the clipped policy loss with a KL term, from logits, with
// its gradient (sf_policy_loss).
//
// Per row the softmax statistics m = max x_j and S = sum exp(x_j - m), x = tau z,
// give lp = x_y - m - log S; loss and derivative c follow from a few scalars of
// the row, and the gradient is g w tau c ([j = y] - exp(x_j - m) / S).  One
// exponential an element for the statistics and one for the gradient, against
// an element's bytes in and out: a streaming kernel, bound by memory.
#include <algorithm>

#include "sf_float.cuh"
#include "sf_launch.h"

namespace sf {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// What a row's scalars say: the gradient's factor and the terms of the sums.
struct RowLoss {
  float logp = 0.f, loss = 0.f, factor = 0.f;
  float4 terms = {0.f, 0.f, 0.f, 0.f};  // weight times loss, pg, kl, clipped
  uint32_t bits = 0;
};
// The log-probability of a row that is left out: one that no row has (-0), so
// that the sums can be taken from the log-probabilities.
constexpr uint32_t kLeftOut = 0x80000000u;
__device__ __forceinline__ RowLoss left_out(uint32_t bits) {
  RowLoss r;
  r.bits = bits;
  if (bits != 0) r.logp = __uint_as_float(kLeftOut);
  return r;
}

// A row's scalars, read before its statistics are known.
struct RowIn {
  float zy, w, A, old, ref, g;
};
// One scalar a lane (a register instead of five) until they are needed.
template <typename T>
__device__ __forceinline__ float lane_scalar(const PolicyJob& j, int64_t row, int y, int lane) {
  switch (lane) {
    case 0: return to_f32(static_cast<const T*>(j.logits)[row * j.ld + y]);
    case 1: return j.advantage[row];
    case 2: return j.old_logp[row];
    case 3: return j.ref_logp != nullptr ? j.ref_logp[row] : 0.f;
    case 4: return j.grad_out != nullptr ? *j.grad_out : 1.f;
    default: return 0.f;
  }
}
__device__ __forceinline__ RowIn gather_row(float scalar, float w) {
  RowIn in;
  in.zy = __shfl_sync(kFull, scalar, 0);
  in.w = w;
  in.A = __shfl_sync(kFull, scalar, 1);
  in.old = __shfl_sync(kFull, scalar, 2);
  in.ref = __shfl_sync(kFull, scalar, 3);
  in.g = __shfl_sync(kFull, scalar, 4);
  return in;
}

// The loss of a row from its token's log-probability.
__device__ __forceinline__ RowLoss loss_of(const PolicyJob& j, const RowIn& in, float lp) {
  RowLoss r;
  const float A = in.A, w = in.w;
  const float ratio = expf(lp - in.old);
  const float held = fminf(fmaxf(ratio, 1.f - j.cfg.clip_low), 1.f + j.cfg.clip_high);
  const bool clipped = held * A < ratio * A;
  const float pg = -fminf(ratio * A, held * A);
  float kl = 0.f, loss = pg, c = clipped ? 0.f : -ratio * A;
  if (j.ref_logp != nullptr) {
    const float u = in.ref - lp;
    const float em = expm1f(u);
    kl = em - u;
    if (j.cfg.kl_coef != 0.f) {
      loss += j.cfg.kl_coef * kl;
      c -= j.cfg.kl_coef * em;
    }
  }
  const float f = c * w * in.g * j.cfg.inv_temperature;
  if (!finite(loss) || !finite(w * loss) || !finite(w * kl) || !finite(f) || ratio != ratio)
    return left_out(SF_ST_NONFINITE);
  r.logp = lp + 0.f;  // never -0
  r.loss = loss;
  r.factor = f;
  r.terms = make_float4(w * loss, w * pg, w * kl, clipped ? w : 0.f);
  return r;
}

// m: the row's reference, ty: the chosen token's exponent tau z_y against it, S:
// the sum of the exponentials of all exponents.
__device__ __forceinline__ RowLoss row_loss(const PolicyJob& j, const RowIn& in, float m, float ty, float S) {
  // a NaN logit makes S NaN, a +inf one m, and so does a row without any above -inf
  return finite(m) && finite(S) ? loss_of(j, in, ty - logf(S)) : left_out(SF_ST_NONFINITE);
}

__device__ __forceinline__ void write_row(const PolicyJob& j, int64_t row, const RowLoss& r) {
  if (j.logp != nullptr) j.logp[row] = r.logp;
  if (j.token_loss != nullptr) j.token_loss[row] = r.loss;
  if (j.N == 1) {  // its terms are the sums
    j.stats[0] = r.terms.x;
    j.stats[1] = r.terms.y;
    j.stats[2] = r.terms.z;
    j.stats[3] = r.terms.w;
  } else if (j.terms != nullptr) {
    j.terms[row] = r.terms;
  }
  report(j.status, r.bits);
}

__device__ __forceinline__ float row_weight(const PolicyJob& j, int64_t row) {
  return j.weight != nullptr ? j.weight[row] : j.mean;
}

template <typename T, int kThreads>
__device__ void zero_row(T* d, int64_t V) {
  const int head = head_of(d, V);
  const int64_t nv = (V - head) / Pack<T>::kN;
  for (int64_t i = threadIdx.x; i < head; i += kThreads) d[i] = from_f32<T>(0.f);
  for (int64_t i = threadIdx.x; i < nv; i += kThreads) store16(d + head + i * Pack<T>::kN, make_uint4(0, 0, 0, 0));
  for (int64_t i = head + nv * Pack<T>::kN + threadIdx.x; i < V; i += kThreads) d[i] = from_f32<T>(0.f);
}

// Exponentials of a row against a reference r near its largest logit (which is
// at most kGrow powers of 2 above it, and is r itself if it stands out), as powers
// of 2 with scale = tau log2(e).  f32: r is a logit and the difference is taken
// first, which is exact near r.  16-bit types, two values of which come in the
// bytes of one, take one multiply-add: r is a logit times scale, rounded, and z
// scale - r is then rounded once.  All that meets a row's r, the chosen token's
// own exponent and the sums of other references too, goes by that r, so that its
// rounding does not matter while it is small: |r| <= 2^20 (see slow_row).
template <typename T>
struct Reference {
  static constexpr bool kScaled = sizeof(T) == 2;
  static __device__ __forceinline__ float of(float z, float scale) { return kScaled ? z * scale : z; }
  // what a thread starts from: values far below add nothing
  static __device__ __forceinline__ float floor() { return kScaled ? -1048576.f : -1e30f; }
  // a sum has its largest term's 1 unless all logits are below the floor: there the smallest of them are lost,
  // and a gradient's factor divided by it may not be finite
  static __device__ __forceinline__ bool sound(float r, float S) {
    return !(S < 0.5f) && !(kScaled && r > 1048576.f);
  }
  // the exponent of 2 of a logit, and of another reference
  static __device__ __forceinline__ float exponent(float z, float r, float scale) {
    return kScaled ? fmaf(z, scale, -r) : (z - r) * scale;
  }
  static __device__ __forceinline__ float between(float from, float to, float scale) {
    return kScaled ? from - to : (from - to) * scale;
  }
};

// Reference::exponent of two logits at once.
template <typename T>
struct Exponent {
  uint64_t a, b;
  __device__ __forceinline__ Exponent(float r, float scale) : a(pair_of(scale, scale)), b(pair_of(-r, -r)) {}
  __device__ __forceinline__ uint64_t operator()(uint64_t z) const {
    return Reference<T>::kScaled ? fma2(z, a, b) : mul2(add2(z, b), a);
  }
};

// Running reference r of one thread and sum of the exponentials against it.  What
// a chunk adds is summed by itself (at most 16 terms to each of two sums), and
// the chunks' sums with what each addition rounded off (Kahan): equal terms that
// are small beside the sum round the same way every time, and a plain sum lost
// 1.3e-5 of itself that way at 131072 entries and 1.8e-3 at 2^24.  The reference
// follows a logit that exceeds it by more than kGrow powers of 2, not every larger
// one: each rescaling errs by an exponential and a product, and in a row whose
// logits rise all along there was one a chunk (more than 9e-6 of the sum at 2^24
// entries).  Now what an error counts falls to a 16th from one to the next.
constexpr float kGrow = 4.f;
template <typename T>
struct MaxSum {
  float r = Reference<T>::floor();
  float s = 0.f, lost = 0.f;  // the sum, and what it is short of
  __device__ __forceinline__ void grow(float z, float scale) {
    const float to = Reference<T>::of(z, scale);
    if (Reference<T>::between(to, r, scale) > kGrow) {
      const float f = exp2_fast(Reference<T>::between(r, to, scale));
      s *= f;
      lost *= f;
      r = to;
    }
  }
  __device__ __forceinline__ void add(float v) {
    const float y = v + lost, t = s + y;
    lost = y - (t - s);
    s = t;
  }
  __device__ __forceinline__ float sum() const { return s + lost; }
};

// The exponentials of two logits, added to two sums.
template <typename T>
__device__ __forceinline__ uint64_t add_terms(uint64_t sums, uint64_t z, const Exponent<T>& e) {
  float x, y;
  split(e(z), x, y);
  return add2(sums, pair_of(exp2_fast(x), exp2_fast(y)));
}

// Untiled bulk copy global -> shared; addresses and size multiples of 16 bytes.
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                   smem_u32(dst)),
               "l"(src), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar,
                                          uint64_t policy) {
  asm volatile(
      "cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;" ::"r"(
          smem_u32(dst)),
      "l"(src), "r"(bytes), "r"(smem_u32(bar)), "l"(policy)
      : "memory");
}

__device__ __forceinline__ uint4 load_shared16(const void* p) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "r"(smem_u32(p))
               : "memory");
  return v;
}

// A row as 16-byte packs, with single elements before the first and after the last.
template <typename T>
struct RowPacks {
  int head, packs, tail_at;
  __device__ __forceinline__ RowPacks(const T* z, int V) {
    head = head_of(z, V);
    packs = (V - head) / Pack<T>::kN;
    tail_at = head + packs * Pack<T>::kN;
  }
  // The element that thread i holds of those outside the packs, or -1.
  __device__ __forceinline__ int single(int i, int V) const {
    return i < head ? i : i >= 32 && i - 32 < V - tail_at ? tail_at + i - 32 : -1;
  }
};

// What the warp that puts a row's statistics together hands the others.
struct __align__(16) RowScale {
  float r, p;   // the row's reference; -factor / S
  float chosen; // the chosen token's gradient
  int y;        // the chosen token; -1: write zeros; kSlowRow: not known yet
};
constexpr int kSlowRow = -2;

// ey: the chosen token's exponent of 2.
__device__ __forceinline__ RowScale row_scale(const RowLoss& l, float r, float S, float ey, int y) {
  RowScale o;
  o.r = r;
  o.p = -l.factor / S;
  o.chosen = l.factor + exp2_fast(ey) * o.p;
  o.y = l.bits != 0 ? -1 : y;
  return o;
}

// The statistics of a row whose values lie too far out for Reference, as in a
// row of nothing but masks of the type's lowest value: by a block, with exact
// differences from the maximum.  Every thread gets (maximum, sum).
template <typename T, int kThreads>
__device__ float2 slow_row(const T* z, int V, float scale, float2* stats) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float m = neg_inf();
  for (int i = threadIdx.x; i < V; i += kThreads) m = fmaxf(m, to_f32(z[i]));
  m = warp_max(m);
  named_barrier(1, kThreads);
  if (lane == 0) stats[warp].x = m;
  named_barrier(1, kThreads);
  for (int q = 0; q < kThreads / 32; ++q) m = fmaxf(m, stats[q].x);
  MaxSum<T> a;
  for (int i = threadIdx.x; i < V; i += kThreads) a.add(exp2_fast((to_f32(z[i]) - m) * scale));
  float s = warp_sum(a.sum());
  if (lane == 0) stats[warp].y = s;
  named_barrier(1, kThreads);
  s = 0.f;
  for (int q = 0; q < kThreads / 32; ++q) s += stats[q].y;
  return make_float2(m, s);
}

// Bit l of the result: row first + (i + l) * step (i + l < rows) has a weight and a token that exists.
__device__ __forceinline__ uint32_t active_rows(const PolicyJob& j, int64_t first, int64_t step, int i, int rows) {
  const int l = threadIdx.x & 31;
  bool on = false;
  if (i + l < rows) {
    const int64_t row = first + int64_t(i + l) * step;
    if (row_weight(j, row) != 0.f) {
      const int64_t y = j.target[row];
      on = y >= 0 && y < j.V;
    }
  }
  return __ballot_sync(kFull, on);
}

// Many rows: a CTA a row.  One warp keeps a ring of chunks filled by bulk
// copies, row after row: every row's packs once for its statistics and, for a
// gradient, once more for that, which L2 still holds.  The copies run ahead
// over the ends of passes and rows, so that the reads of the next row go on
// while this one's gradient is written.  What is not used again (the second
// read, the gradient) leaves L2 first: 716 -> 587 us at 6144 x 131072 bf16.
// kThreads consumers take kPacks packs of a chunk each; kPerSm CTAs an SM.
// 6144 x 131072 bf16 with gradients: 587 us, 5.5 TB/s in and out (82 % of the
// copy rate; 72 % of the issue slots); 4095 x 50001 f32 without: 122 us (6.7 TB/s).
constexpr int kMaxSlots = 6, kRingBytes = 192 * 1024;  // of an SM's CTAs

template <typename T, int kThreads, int kPacks, int kPerSm, bool kGrad>
__global__ void __launch_bounds__(kThreads + 32, kPerSm) policy_ring_kernel(const PolicyJob j, const int slots) {
  constexpr int N = Pack<T>::kN, kWarps = kThreads / 32, kChunk = kThreads * kPacks;  // packs
  constexpr int kPasses = kGrad ? 2 : 1;
  using Ref = Reference<T>;
  extern __shared__ __align__(128) unsigned char ring[];
  __shared__ __align__(8) uint64_t full[kMaxSlots], empty[kMaxSlots];
  __shared__ float2 stats[kWarps];
  __shared__ RowScale shared_scale;
  __shared__ int abort_flag;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, V = static_cast<int>(j.V);
  const int64_t first = blockIdx.x, step = gridDim.x;
  const int rows = static_cast<int>((j.N - first + step - 1) / step);  // its row i: first + i * step
  const float scale = j.cfg.inv_temperature * kLog2e;
  if (tid == 0) {
    for (int b = 0; b < slots; ++b) {
      mbar_init(full + b, 1);
      mbar_init(empty + b, kWarps);
    }
    fence_barrier_init();
    abort_flag = 0;
  }
  __syncthreads();

  if (warp == kWarps) {  // the copies
    const uint64_t once = policy_evict_first();
    bool timeout = false;
    uint32_t slot = 0, turn = 0;
    uint64_t issued = 0;
    for (int i = 0; i < rows; i += 32) {
      uint32_t mask = active_rows(j, first, step, i, rows);
      if (lane != 0) continue;
      for (; mask != 0; mask &= mask - 1) {
        const int64_t row = first + int64_t(i + __ffs(static_cast<int>(mask)) - 1) * step;
        const T* z = static_cast<const T*>(j.logits) + row * j.ld;
        const RowPacks<T> rp(z, V);
        for (int pass = 0; pass < kPasses; ++pass)
          for (int c = 0; c < rp.packs; c += kChunk) {
            if (!mbar_wait_bounded(empty + slot, turn ^ 1u, &abort_flag)) timeout = true;
            const uint32_t bytes = uint32_t(min(kChunk, rp.packs - c)) * 16u;
            mbar_arrive_expect_tx(full + slot, bytes);
            if (pass + 1 == kPasses)
              bulk_load(ring + slot * (kChunk * 16), z + rp.head + int64_t(c) * N, bytes, full + slot, once);
            else
              bulk_load(ring + slot * (kChunk * 16), z + rp.head + int64_t(c) * N, bytes, full + slot);
            ++issued;
            if (++slot == uint32_t(slots)) {
              slot = 0;
              turn ^= 1u;
            }
          }
      }
    }
    // the last copies land before the CTA ends, whatever became of the consumers
    const uint64_t n = slots;
    for (uint64_t q = issued > n ? issued - n : 0; q < issued; ++q)
      if (!mbar_wait_timeout(full + q % n, (q / n) & 1u)) timeout = true;
    if (timeout) report(j.status, SF_ST_TIMEOUT);
    return;
  }

  const uint64_t once = policy_evict_first();
  bool timeout = false;
  uint32_t slot = 0, turn = 0, mask = 0;
  // The next chunk's packs at p * kThreads + tid, -inf past the row's `left`.
  const auto next_chunk = [&](int left, uint4 (&u)[kPacks]) {
    if (!mbar_wait_bounded(full + slot, turn, &abort_flag)) timeout = true;
    const unsigned char* src = ring + slot * (kChunk * 16) + tid * 16;
#pragma unroll
    for (int p = 0; p < kPacks; ++p)
      u[p] = p * kThreads + tid < left ? load_shared16(src + p * kThreads * 16) : lowest_pack(T());
  };
  // The slot may be filled again.  After the packs' use, and with a fence: without one nothing orders these
  // reads before the next copy's writes, and packs of the chunk after next came out of reads that went late.
  const auto done_chunk = [&] {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) mbar_arrive(empty + slot);
    if (++slot == uint32_t(slots)) {
      slot = 0;
      turn ^= 1u;
    }
  };
  // warp 0: the row's loss from its statistics (ey: the chosen token's exponent of 2), and what the gradient takes
  const auto finish = [&](int64_t row, int y, float scalar, float r, float S, float ey) {
    const RowLoss l = row_loss(j, gather_row(scalar, row_weight(j, row)), r, ey * kLn2, S);
    if (lane == 0) {
      write_row(j, row, l);
      shared_scale = row_scale(l, r, S, ey, y);
    }
  };
  for (int i = 0; i < rows; ++i) {
    if ((i & 31) == 0) mask = active_rows(j, first, step, i, rows);
    const int64_t row = first + int64_t(i) * step;
    T* d = kGrad ? static_cast<T*>(j.dlogits) + row * j.ldd : nullptr;
    if (!((mask >> (i & 31)) & 1u)) {
      if (kGrad) zero_row<T, kThreads>(d, V);
      if (tid == 0) {
        write_row(j, row, left_out(row_weight(j, row) != 0.f ? SF_ST_INDEX : 0u));
      }
      continue;
    }
    const T* z = static_cast<const T*>(j.logits) + row * j.ld;
    const RowPacks<T> rp(z, V);
    const int single = rp.single(tid, V);
    const float lone = single >= 0 ? to_f32(z[single]) : neg_inf();
    int y = 0;
    float scalar = 0.f;
    if (warp == 0) {
      y = static_cast<int>(j.target[row]);
      scalar = lane_scalar<T>(j, row, y, lane);
    }
    MaxSum<T> a;
    if (single >= 0) {
      a.grow(lone, scale);
      a.add(exp2_fast(Ref::exponent(lone, a.r, scale)));
    }
    for (int c = 0; c < rp.packs; c += kChunk) {
      uint4 u[kPacks];
      next_chunk(rp.packs - c, u);
      a.grow(packs_max(u, T()), scale);
      const Exponent<T> e(a.r, scale);
      uint64_t sums = 0;  // two, of this chunk
#pragma unroll
      for (int p = 0; p < kPacks; ++p) {
        uint64_t z2[N / 2];
        unpack2(u[p], z2, T());
#pragma unroll
        for (int q = 0; q < N / 2; ++q) sums = add_terms(sums, z2[q], e);
      }
      float x, y2;
      split(sums, x, y2);
      a.add(x + y2);
      done_chunk();
    }
    const float wr = warp_max(a.r);
    const float ws = warp_sum(a.sum() * exp2_fast(Ref::between(a.r, wr, scale)));
    if (lane == 0) stats[warp] = make_float2(wr, ws);
    named_barrier(1, kThreads);
    if (warp == 0) {
      const float2 o = lane < kWarps ? stats[lane] : make_float2(Ref::floor(), 0.f);
      const float r = warp_max(o.x);
      const float S = warp_sum(o.y * exp2_fast(Ref::between(o.x, r, scale)));
      if (Ref::sound(r, S))
        finish(row, y, scalar, r, S, Ref::exponent(__shfl_sync(kFull, scalar, 0), r, scale));
      else if (lane == 0)
        shared_scale.y = kSlowRow;
    }
    named_barrier(2, kThreads);
    if (shared_scale.y == kSlowRow) {
      const float2 o = slow_row<T, kThreads>(z, V, scale, stats);
      if (warp == 0) finish(row, y, scalar, o.x, o.y, (__shfl_sync(kFull, scalar, 0) - o.x) * scale);
      named_barrier(2, kThreads);
      if (kGrad) {
        const RowScale r = shared_scale;
        for (int c = 0; c < rp.packs; c += kChunk) {  // copies that are on their way all the same
          uint4 u[kPacks];
          next_chunk(0, u);
          done_chunk();
        }
        for (int q = tid; q < V; q += kThreads) {
          const float g = q == r.y ? r.chosen : r.y < 0 ? 0.f : exp2_fast((to_f32(z[q]) - r.r) * scale) * r.p;
          d[q] = from_f32<T>(g);
        }
        named_barrier(1, kThreads);  // shared_scale is read
      }
      continue;
    }
    if (!kGrad) continue;
    const RowScale o = shared_scale;
    if (o.y < 0) {  // a faulty row
      for (int c = 0; c < rp.packs; c += kChunk) {
        uint4 u[kPacks];
        next_chunk(0, u);
        done_chunk();
      }
      zero_row<T, kThreads>(d, V);
      continue;
    }
    if (single >= 0)
      d[single] = from_f32<T>(single == o.y ? o.chosen : exp2_fast(Ref::exponent(lone, o.r, scale)) * o.p);
    const bool even = (reinterpret_cast<uintptr_t>(d + rp.head) & 15u) == 0;  // both rows at the same offset
    const int chosen = o.y < rp.head ? -1 : (o.y - rp.head) / N;  // the chosen token's pack
    const Exponent<T> e(o.r, scale);
    const uint64_t p2 = pair_of(o.p, o.p);
    T* to = d + rp.head + int64_t(tid) * N;
    for (int c = 0; c < rp.packs; c += kChunk, to += kChunk * N) {
      uint4 u[kPacks];
      next_chunk(rp.packs - c, u);
#pragma unroll
      for (int p = 0; p < kPacks; ++p) {
        const int at = c + p * kThreads + tid;
        uint64_t z2[N / 2];
        unpack2(u[p], z2, T());
        float f[N];
#pragma unroll
        for (int q = 0; q < N / 2; ++q) {
          float x, y2;
          split(e(z2[q]), x, y2);
          split(mul2(pair_of(exp2_fast(x), exp2_fast(y2)), p2), f[2 * q], f[2 * q + 1]);
        }
        const uint4 g = pack(f, T());
        if (at < rp.packs) {
          T* out = to + p * kThreads * N;
          if (even)
            store16(out, g, once);
          else
            store_elements(out, g);
          if (at == chosen) d[o.y] = from_f32<T>(o.chosen);
        }
      }
      done_chunk();
    }
  }
  if (timeout) report(j.status, SF_ST_TIMEOUT);
}

// Few rows: a row by a cluster of C CTAs, read once.  A thread holds up to P
// packs as exponentials relative to its warp's maximum; each warp sends its
// (maximum, sum) to the first CTA's shared memory, whose first warp puts the
// row together and sends the scale back to all.  Latency: one row of 65536 bf16
// 4.2 us (13.4 by one CTA), 32 rows of 131072 with gradients 10.5 us.
constexpr int kClusterThreads = 512, kClusterWarps = kClusterThreads / 32, kMaxCluster = 8;

__device__ __forceinline__ void store_at(uint32_t at, float2 v) {
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(at), "f"(v.x), "f"(v.y) : "memory");
}
__device__ __forceinline__ void store_at(uint32_t at, const RowScale& v) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at), "f"(v.r), "f"(v.p), "f"(v.chosen),
               "f"(__int_as_float(v.y))
               : "memory");
}

template <typename T, int P, bool kGrad>
__global__ void __launch_bounds__(kClusterThreads, 2) policy_cluster_kernel(const PolicyJob j, const int per) {
  constexpr int N = Pack<T>::kN;
  __shared__ float2 pairs[kMaxCluster * kClusterWarps];
  __shared__ RowScale shared_scale;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, V = static_cast<int>(j.V);
  const int C = static_cast<int>(cluster_size()), rank = static_cast<int>(cluster_rank());
  const int64_t row = blockIdx.x / C;
  const float scale = j.cfg.inv_temperature * kLog2e, w = row_weight(j, row);
  const int64_t y64 = w != 0.f ? j.target[row] : 0;
  T* d = kGrad ? static_cast<T*>(j.dlogits) + row * j.ldd : nullptr;
  if (w == 0.f || y64 < 0 || y64 >= V) {  // the same in all CTAs of the cluster
    if (kGrad) {
      const int len = (V + C - 1) / C, from = rank * len;
      if (from < V) zero_row<T, kClusterThreads>(d + from, V - from < len ? V - from : len);
    }
    if (rank == 0 && tid == 0) {
      write_row(j, row, left_out(w != 0.f ? SF_ST_INDEX : 0u));
    }
    return;
  }
  const int y = static_cast<int>(y64);
  const T* z = static_cast<const T*>(j.logits) + row * j.ld;
  const RowPacks<T> rp(z, V);
  const int from_pack = rank * per, packs = min(per, rp.packs - from_pack);  // of this CTA; may be none
  const T* body = z + rp.head + int64_t(from_pack) * N;
  const int single = rank == 0 ? rp.single(tid, V) : -1;
  float lone = single >= 0 ? to_f32(z[single]) : neg_inf();
  float f[P * N];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    float v[N];
    if (p * kClusterThreads + tid < packs) {
      unpack(load16(body + (p * kClusterThreads + tid) * N), v, T());
    } else {
#pragma unroll
      for (int q = 0; q < N; ++q) v[q] = neg_inf();
    }
#pragma unroll
    for (int q = 0; q < N; ++q) f[p * N + q] = v[q];
  }
  float m = lone;
#pragma unroll
  for (int q = 0; q < P * N; ++q) m = fmaxf(m, f[q]);
  m = warp_max(m);
  const float from = m == neg_inf() ? 0.f : m;  // nothing in this warp: sums of 2^-inf, or NaN
  float s = lone = exp2_fast((lone - from) * scale);
#pragma unroll
  for (int q = 0; q < P * N; ++q) {
    f[q] = exp2_fast((f[q] - from) * scale);
    s += f[q];
  }
  s = warp_sum(s);
  float scalar = 0.f;
  if (rank == 0 && warp == 0) scalar = lane_scalar<T>(j, row, y, lane);
  cluster_sync();  // all CTAs have started; the row's reads are done in all (an output may be the input)
  if (lane == 0) store_at(at_rank(&pairs[rank * kClusterWarps + warp], 0), make_float2(m, s));
  cluster_sync();
  if (rank == 0 && warp == 0) {
    float M = neg_inf(), S = 0.f;
#pragma unroll
    for (int q = 0; q < kMaxCluster * kClusterWarps / 32; ++q)
      if (q * 32 + lane < C * kClusterWarps) M = fmaxf(M, pairs[q * 32 + lane].x);
    M = warp_max(M);
#pragma unroll
    for (int q = 0; q < kMaxCluster * kClusterWarps / 32; ++q)
      if (q * 32 + lane < C * kClusterWarps) {
        const float2 o = pairs[q * 32 + lane];
        S += o.x == neg_inf() ? o.y : o.y * exp2_fast((o.x - M) * scale);
      }
    S = warp_sum(S);
    const RowIn in = gather_row(scalar, w);
    const RowLoss l = row_loss(j, in, M, (in.zy - M) * j.cfg.inv_temperature, S);
    if (kGrad && lane < C) store_at(at_rank(&shared_scale, lane), row_scale(l, M, S, (in.zy - M) * scale, y));
    if (lane == 0) write_row(j, row, l);
  }
  if (!kGrad) return;
  __syncwarp();
  cluster_sync();
  const RowScale o = shared_scale;
  const bool zero = o.y < 0;  // a faulty row: what is held may be NaN
  const float p0 = m == neg_inf() ? 0.f : o.p * exp2_fast((m - o.r) * scale);
  if (single >= 0) d[single] = from_f32<T>(zero ? 0.f : single == o.y ? o.chosen : lone * p0);
  T* out = d + rp.head + int64_t(from_pack) * N;
  const bool even = (reinterpret_cast<uintptr_t>(out) & 15u) == 0;  // both rows at the same offset
  const int chosen = o.y < rp.head ? -1 : (o.y - rp.head) / N - from_pack;  // the chosen token's pack
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int at = p * kClusterThreads + tid;
    if (at < packs) {
      float v[N];
#pragma unroll
      for (int q = 0; q < N; ++q) v[q] = zero ? 0.f : f[p * N + q] * p0;
      if (even) {
        store16(out + at * N, pack(v, T()));
      } else {
#pragma unroll
        for (int q = 0; q < N; ++q) out[at * N + q] = from_f32<T>(v[q]);
      }
      if (at == chosen) d[o.y] = from_f32<T>(o.chosen);
    }
  }
}

// The sums over the rows in a fixed order, as pairs of f32 (64-bit additions
// are slow here: 11 us where the pairs take 3): the rows of a block of kSumRows
// by one CTA each, then (where there are several) their sums by one.  The rows'
// terms come from the workspace; of up to SF_POLICY_DIRECT_ROWS rows, whose
// call is host time in the main, they are computed again from the
// log-probabilities, so that no workspace has to be had (loss of 512 rows 34 ->
// 30 us; 8192 rows would take 12 us more that way).
constexpr int kSumThreads = 512, kSumRows = 8192;

// The sum of 4 pairs over the block, in warp 0.
__device__ void sum_block(Sum2 (&a)[4], Sum2 (*buf)[kSumThreads / 32]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    a[q] = warp_sum(a[q]);
    if (lane == 0) buf[q][warp] = a[q];
  }
  __syncthreads();
  if (warp == 0) {
#pragma unroll
    for (int q = 0; q < 4; ++q) a[q] = warp_sum(lane < kSumThreads / 32 ? buf[q][lane] : Sum2());
  }
}

__global__ void __launch_bounds__(kSumThreads) policy_sum_kernel(const PolicyJob j, float2* part) {
  __shared__ Sum2 buf[4][kSumThreads / 32];
  griddep_wait();
  Sum2 a[4];
  const int64_t from = int64_t(blockIdx.x) * kSumRows, to = from + kSumRows < j.N ? from + kSumRows : j.N;
  for (int64_t i = from + threadIdx.x; i < to; i += kSumThreads) {
    float4 t = {0.f, 0.f, 0.f, 0.f};
    if (j.terms != nullptr) {
      t = j.terms[i];
    } else {
      RowIn in;
      in.w = row_weight(j, i);
      const float lp = j.logp[i];
      if (in.w != 0.f && __float_as_uint(lp) != kLeftOut) {
        in.A = j.advantage[i];
        in.old = j.old_logp[i];
        in.ref = j.ref_logp != nullptr ? j.ref_logp[i] : 0.f;
        in.g = in.zy = 0.f;
        t = loss_of(j, in, lp).terms;
      }
    }
    a[0].add(t.x);
    a[1].add(t.y);
    a[2].add(t.z);
    a[3].add(t.w);
  }
  sum_block(a, buf);
  if (threadIdx.x == 0) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (part != nullptr)
        part[int64_t(blockIdx.x) * 4 + q] = make_float2(a[q].hi, finite(a[q].hi) ? a[q].lo : 0.f);
      else
        j.stats[q] = a[q].value();
    }
  }
}

__global__ void __launch_bounds__(128) policy_sum_parts_kernel(const float2* part, int64_t blocks, float* stats) {
  griddep_wait();
  const int q = threadIdx.x >> 5;
  Sum2 s;
  for (int64_t i = threadIdx.x & 31; i < blocks; i += 32) {
    const float2 p = part[i * 4 + q];
    s.add(p.x);
    s.add(p.y);
  }
  s = warp_sum(s);
  if ((threadIdx.x & 31) == 0) stats[q] = s.value();
}

template <typename T, int kThreads, int kPacks, int kPerSm, bool kGrad>
cudaError_t launch_ring(const PolicyJob& j, cudaStream_t stream) {
  constexpr int kSlot = kThreads * kPacks * 16, kSlots = std::min(kMaxSlots, kRingBytes / kPerSm / kSlot);
  const auto kern = policy_ring_kernel<T, kThreads, kPacks, kPerSm, kGrad>;
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kSlots * kSlot);
  if (e != cudaSuccess) return e;
  const int grid = static_cast<int>(std::min<int64_t>(j.N, int64_t(sm_count()) * kPerSm));
  count_launch();
  kern<<<grid, kThreads + 32, kSlots * kSlot, stream>>>(j, kSlots);
  return cudaGetLastError();
}

template <typename T, int P, bool kGrad>
cudaError_t launch_cluster(const PolicyJob& j, int C, cudaStream_t stream) {
  const int per = static_cast<int>(std::max<int64_t>(1, (j.V / Pack<T>::kN + C - 1) / C));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(j.N * C));
  cfg.blockDim = dim3(kClusterThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = C;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  count_launch();
  return cudaLaunchKernelEx(&cfg, policy_cluster_kernel<T, P, kGrad>, j, per);
}

template <typename T, bool kGrad>
cudaError_t launch_rows(const PolicyJob& j, cudaStream_t stream) {
  constexpr int kHeld = sizeof(T) == 4 ? 8 : 4;  // packs a thread: 32 values
  const int64_t packs = j.V / Pack<T>::kN;
  // CTAs a row that hold it, more of them while there are SMs for them and packs for their threads
  int C = 1;
  while (C <= kMaxCluster && int64_t(C) * kClusterThreads * kHeld < packs) C *= 2;
  while (C < kMaxCluster && j.N * C * 2 <= int64_t(sm_count()) * 2 && packs > int64_t(C) * kClusterThreads) C *= 2;
  if (C <= kMaxCluster && j.N * C <= int64_t(sm_count()) * 2) return launch_cluster<T, kHeld, kGrad>(j, C, stream);
  // As many CTAs an SM as leave their rows in L2 (129 MB) until the second read, a row each, with four 76 MB
  // in all, with two 84 (us with 4 / 2 / 1 an SM: 4096 x 32768 bf16, 40 MB with 4, 100 / 117 / 167; 4096 x
  // 65536, 80 MB, 209 / 197; 2048 x 50001 f32, 122 MB, 179 / 153 / 163; 6144 x 131072 bf16, 159 MB, 735 / 587 /
  // 642; 2048 x 131072 f32, 319 MB, 491 / 489 / 389).  With two an SM that is 80 MB as the last gain and 159 as
  // the first loss: nothing between was measured, and 84 is the cautious end.  Without a second read always four.
  const double rows = double(j.V) * sizeof(T) * sm_count();  // bytes of a row on every SM
  if (!kGrad || rows * 4 <= 76e6) return launch_ring<T, 256, 4, 4, kGrad>(j, stream);
  if (rows * 2 <= 84e6) return launch_ring<T, 512, 2, 2, kGrad>(j, stream);
  return launch_ring<T, 992, 2, 1, kGrad>(j, stream);
}

template <typename T>
cudaError_t launch_type(const PolicyJob& j, cudaStream_t stream) {
  return j.dlogits != nullptr ? launch_rows<T, true>(j, stream) : launch_rows<T, false>(j, stream);
}

int64_t sum_blocks(int64_t N) { return (N + kSumRows - 1) / kSumRows; }

}  // namespace

size_t policy_loss_workspace(int64_t N) {
  return size_t(N) * sizeof(float4) + (sum_blocks(N) > 1 ? size_t(sum_blocks(N)) * 4 * sizeof(float2) : 0);
}

bool policy_loss_direct(int64_t N, const float* logp) { return N <= SF_POLICY_DIRECT_ROWS && logp != nullptr; }

cudaError_t launch_policy_loss(PolicyJob j, void* workspace, cudaStream_t stream) {
  j.terms = policy_loss_direct(j.N, j.logp) ? nullptr : static_cast<float4*>(workspace);
  j.mean = 1.f / static_cast<float>(j.N);
  const cudaError_t e = j.dtype == SF_F32    ? launch_type<float>(j, stream)
                        : j.dtype == SF_BF16 ? launch_type<__nv_bfloat16>(j, stream)
                                             : launch_type<__half>(j, stream);
  if (e != cudaSuccess || j.N == 1) return e;
  const int64_t blocks = sum_blocks(j.N);
  float2* part = blocks > 1 ? reinterpret_cast<float2*>(j.terms + j.N) : nullptr;
  count_launch();
  const cudaError_t s = launch_after(policy_sum_kernel, dim3(static_cast<unsigned>(blocks)), dim3(kSumThreads), 0,
                                     stream, true, j, part);
  if (s != cudaSuccess || part == nullptr) return s;
  count_launch();
  return launch_after(policy_sum_parts_kernel, dim3(1), dim3(128), 0, stream, true, part, blocks, j.stats);
}

}  // namespace sf
