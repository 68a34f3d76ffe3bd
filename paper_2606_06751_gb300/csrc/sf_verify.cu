// sf_verify.cu - drafted tokens verified against the policy's rows by given
// random numbers (sf_verify_draft).
//
// A drafted token y is kept while u q(y) < p(y); the first that is not is replaced
// by a draw from max(p - q, 0), as the winner of a race: the entry of largest r_j /
// e_j, e_j exponential, is j with probability r_j / sum r.  Two launches: the
// softmax statistics of all rows, a CTA a piece of a row (the rows' only read but
// one), and then a cluster of CTAs a sequence, each of which decides from the
// statistics where the sequence stops and races a slice of the one row (with its
// draft row and noise) that the next token comes from.  Bound by memory: (2 L + 1)
// rows and a row of noise a sequence.
#include <algorithm>

#include "sf_float.cuh"
#include "sf_launch.h"

namespace sf {

// What a piece of a row says: its largest logit, the sum of the exponentials
// against it and the first place of the largest.
struct __align__(16) VerifyPiece {
  float m, s;
  int at, pad;
};

namespace {

using Piece = VerifyPiece;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxPieces = 64;

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Larger value first, then lower place: one integer order for values above 0 (or any sign by `ordered`).
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);  // -0 as 0
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint64_t place_key(uint32_t value, int at) {
  return uint64_t(value) << 32 | (0xffffffffu - static_cast<uint32_t>(at));
}
__device__ __forceinline__ int place_of(uint64_t key) {
  return static_cast<int>(0xffffffffu - static_cast<uint32_t>(key));
}

__device__ __forceinline__ int drafted(const VerifyJob& j, int64_t b, bool* bad) {
  const int L = static_cast<int>(j.L);
  if (j.length == nullptr) return L;
  const int n = j.length[b];
  *bad = n < 0 || n > L;
  return n < 0 ? 0 : n > L ? L : n;
}

// Statistics of piece blockIdx.x of row blockIdx.y (+ 65535 blockIdx.z): policy
// rows first, then the draft's.
template <typename T, bool kGreedy>
__global__ void __launch_bounds__(kThreads) verify_piece_kernel(const VerifyJob j, const int64_t rows) {
  constexpr int N = Pack<T>::kN;
  __shared__ float sm[kWarps], ss[kWarps];
  __shared__ uint64_t sk[kWarps];
  griddep_launch_dependents();
  const int64_t row = int64_t(blockIdx.z) * 65535 + blockIdx.y;
  if (row >= rows) return;
  const int64_t policy_rows = j.B * (j.L + 1);
  const int64_t of_draft = row - policy_rows;  // >= 0: a draft row
  const int64_t b = of_draft < 0 ? row / (j.L + 1) : of_draft / j.L;
  const int i = static_cast<int>(of_draft < 0 ? row - b * (j.L + 1) : of_draft - b * j.L);
  bool bad;
  const int n = drafted(j, b, &bad);
  if (of_draft < 0 ? i > n : i >= n) return;
  const T* z = of_draft < 0 ? static_cast<const T*>(j.target) + row * j.ldt
                            : static_cast<const T*>(j.draft) + of_draft * j.ldq;
  const int V = static_cast<int>(j.V), tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int from = static_cast<int>(blockIdx.x) * j.piece, to = min(V, from + j.piece);
  const float scale = j.tau * kLog2e;
  float m = neg_inf();
  uint64_t best = 0;
  bool nan = false;
  for (int q = from + tid; q < to; q += kThreads) {
    const float v = to_f32(z[q]);
    nan |= v != v;
    m = fmaxf(m, v);
    if (kGreedy && v == v) {
      const uint64_t k = place_key(ordered(v), q);
      best = k > best ? k : best;
    }
  }
  m = warp_max(m);
  if (lane == 0) sm[warp] = m;
  if (kGreedy) {
    best = warp_max_u64(best);
    if (lane == 0) sk[warp] = best;
  }
  __syncthreads();
  m = sm[0];
#pragma unroll
  for (int w = 1; w < kWarps; ++w) m = fmaxf(m, sm[w]);
  Sum2 a;
  for (int q = from + tid; q < to; q += kThreads)
    if (m != neg_inf()) a.add(exp2_fast((to_f32(z[q]) - m) * scale));
  float s = warp_sum(a.value());
  if (__any_sync(kFull, nan)) s = quiet_nan();
  if (lane == 0) ss[warp] = s;
  __syncthreads();
  if (tid == 0) {
    Piece o;
    o.m = m;
    o.s = 0.f;
    for (int w = 0; w < kWarps; ++w) o.s += ss[w];
    o.at = 0;
    o.pad = 0;
    if (kGreedy) {
      uint64_t k = sk[0];
      for (int w = 1; w < kWarps; ++w) k = sk[w] > k ? sk[w] : k;
      o.at = place_of(k);
    }
    j.pieces[row * j.per_row + blockIdx.x] = o;
  }
}

// A row's statistics from its pieces, in every lane: maximum, sum, first place of
// the maximum.  The sum is NaN where a logit is NaN or +inf or none is above -inf.
struct Row {
  float m, s;
  int at;
};
__device__ __forceinline__ Row row_of(const Piece* p, int pieces, float tau, int lane) {
  float m = neg_inf();
  for (int i = lane; i < pieces; i += 32) m = fmaxf(m, p[i].m);
  m = warp_max(m);
  float s = 0.f;
  uint32_t first = 0xffffffffu;
  for (int i = lane; i < pieces; i += 32) {
    const Piece q = p[i];
    s += q.m == neg_inf() ? q.s : q.s * expf((q.m - m) * tau);
    if (q.m == m) first = min(first, static_cast<uint32_t>(q.at));
  }
  Row r;
  r.m = m;
  r.s = warp_sum(s);
  if (!(r.s > 0.f) || !finite(m)) r.s = quiet_nan();
  r.at = static_cast<int>(__reduce_min_sync(kFull, first));
  return r;
}

// Where a sequence stops.
struct Stop {
  int at;       // accepted tokens
  int from;     // 0: no token; 1: the policy's row alone; 2: less the draft's; 3: without the drafted token
  float m, s, mq, sq;
  int last;     // greedy: the next token; 3: the drafted token
};

template <typename T, bool kGreedy>
__global__ void __launch_bounds__(kThreads) verify_sample_kernel(const VerifyJob j) {
  __shared__ float2 rows[SF_VERIFY_MAX_DRAFT + 1];   // (maximum, sum)
  __shared__ float2 drafts[SF_VERIFY_MAX_DRAFT + 1];
  __shared__ float lps[SF_VERIFY_MAX_DRAFT + 1];
  __shared__ int firsts[SF_VERIFY_MAX_DRAFT + 1];
  __shared__ int takes[SF_VERIFY_MAX_DRAFT + 1];  // 1 accepted, 0 not, -1 a faulty row, -2 no such token
  __shared__ uint64_t warps_best[kWarps];
  __shared__ uint64_t best_of[16];  // of the cluster's CTAs
  __shared__ Stop stop;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int C = static_cast<int>(cluster_size()), rank = static_cast<int>(cluster_rank());
  const int64_t b = blockIdx.x / C;
  const int V = static_cast<int>(j.V), L = static_cast<int>(j.L);
  bool bad_length = false;
  griddep_wait();
  const int n = drafted(j, b, &bad_length);
  const T* target = static_cast<const T*>(j.target) + b * (L + 1) * j.ldt;
  const T* draft = j.draft != nullptr ? static_cast<const T*>(j.draft) + b * L * j.ldq : nullptr;
  const Piece* tp = j.pieces + b * (L + 1) * j.per_row;
  const Piece* dp = j.pieces + (j.B * (L + 1) + b * L) * j.per_row;
  uint32_t bits = bad_length ? SF_ST_INDEX : 0u;
  for (int i = warp; i <= n; i += kWarps) {
    const Row r = row_of(tp + int64_t(i) * j.per_row, j.per_row, j.tau, lane);
    Row q = {0.f, 1.f, 0};
    if (!kGreedy && draft != nullptr && i < n) q = row_of(dp + int64_t(i) * j.per_row, j.per_row, j.tau, lane);
    if (lane == 0) {
      int take = r.s != r.s ? -1 : 0;
      float lp = 0.f;
      if (i < n && take == 0) {
        const int64_t y = j.token[b * L + i];
        if (y < 0 || y >= V) {
          take = -2;
        } else if (kGreedy) {
          take = y == r.at ? 1 : 0;
          lp = (to_f32(target[i * j.ldt + y]) - r.m) * j.tau - logf(r.s);
        } else {
          const float ty = (to_f32(target[i * j.ldt + y]) - r.m) * j.tau;
          const float p = expf(ty) / r.s;
          const float qy = draft != nullptr ? expf((to_f32(draft[i * j.ldq + y]) - q.m) * j.tau) / q.s : 1.f;
          take = q.s != q.s ? -1 : j.uniform[b * L + i] * qy < p ? 1 : 0;
          lp = ty - logf(r.s);
        }
      }
      rows[i] = make_float2(r.m, r.s);
      drafts[i] = make_float2(q.m, q.s);
      firsts[i] = r.at;
      takes[i] = take;
      lps[i] = lp;
    }
  }
  __syncthreads();
  if (tid == 0) {
    int k = 0;
    while (k < n && takes[k] == 1) ++k;
    Stop o;
    o.at = k;
    o.m = rows[k].x;
    o.s = rows[k].y;
    o.mq = drafts[k].x;
    o.sq = drafts[k].y;
    o.last = kGreedy ? firsts[k] : 0;
    o.from = takes[k] == -1 ? 0 : k == n || takes[k] == -2 || kGreedy ? 1 : draft != nullptr ? 2 : 3;
    if (o.from == 3) o.last = static_cast<int>(j.token[b * L + k]);
    stop = o;
  }
  __syncthreads();
  const Stop o = stop;
  int next = -1;
  if (kGreedy) {
    next = o.from == 0 ? -1 : o.last;
  } else if (o.from != 0) {
    const T *z = target + o.at * j.ldt, *zq = draft != nullptr ? draft + min(o.at, L - 1) * j.ldq : nullptr;
    const float* e = j.noise + b * V;
    const int from = static_cast<int>(int64_t(V) * rank / C), to = static_cast<int>(int64_t(V) * (rank + 1) / C);
    uint64_t best = 0;
    int form = o.from;
    for (;;) {
      best = 0;
      for (int q = from + tid; q < to; q += kThreads) {
        float r = expf((to_f32(z[q]) - o.m) * j.tau) / o.s;
        if (form == 2) r -= expf((to_f32(zq[q]) - o.mq) * j.tau) / o.sq;
        if (form == 3 && q == o.last) r = 0.f;
        const float v = r / e[q];
        if (r > 0.f && e[q] > 0.f && v > 0.f) {
          const uint64_t key = place_key(__float_as_uint(v), q);
          best = key > best ? key : best;
        }
      }
      best = warp_max_u64(best);
      if (lane == 0) warps_best[warp] = best;
      __syncthreads();
      if (warp == 0) {
        best = warp_max_u64(lane < kWarps ? warps_best[lane] : 0);
        if (lane < C)
          asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(at_rank(&best_of[rank], lane)), "l"(best) : "memory");
      }
      cluster_sync();
      best = 0;
      for (int c = 0; c < C; ++c) best = best_of[c] > best ? best_of[c] : best;
      cluster_sync();  // all have read before a second race writes
      if (best != 0 || form != 2) break;
      form = 1;  // no residual above 0
    }
    next = best != 0 ? place_of(best) : -1;
  }
  if (rank != 0) return;
  if (next < 0) bits |= SF_ST_NONFINITE;
  for (int i = tid; i <= L; i += kThreads) {
    int64_t t = -1;
    float lp = 0.f;
    if (i < o.at) {
      t = j.token[b * L + i];
      lp = lps[i];
    } else if (i == o.at && next >= 0) {
      t = next;
      lp = (to_f32(target[i * j.ldt + next]) - o.m) * j.tau - logf(o.s);
    }
    j.out_token[b * (L + 1) + i] = t;
    if (j.logp != nullptr) j.logp[b * (L + 1) + i] = lp;
  }
  if (tid == 0) {
    j.accepted[b] = o.at;
    if (o.at < n && takes[o.at] == -2) bits |= SF_ST_INDEX;
    report(j.status, bits);
  }
}

int piece_of(int64_t V) {
  const int64_t p = std::max<int64_t>(4096, (V + kMaxPieces - 1) / kMaxPieces);
  return static_cast<int>((p + 7) / 8 * 8);
}

template <typename T, bool kGreedy>
cudaError_t launch_type(VerifyJob j, cudaStream_t stream) {
  const int64_t rows = j.B * (j.L + 1) + (j.draft != nullptr && !kGreedy ? j.B * j.L : 0);
  const dim3 grid(j.per_row, static_cast<unsigned>(std::min<int64_t>(rows, 65535)),
                  static_cast<unsigned>((rows + 65534) / 65535));
  count_launch();
  verify_piece_kernel<T, kGreedy><<<grid, kThreads, 0, stream>>>(j, rows);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  // CTAs a sequence: while there are SMs for them and entries for their threads
  int C = 1;
  while (!kGreedy && C < 8 && j.B * C * 2 <= int64_t(sm_count()) * 4 && j.V > int64_t(C) * kThreads * 4) C *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(j.B * C));
  cfg.blockDim = dim3(kThreads);
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
  return cudaLaunchKernelEx(&cfg, verify_sample_kernel<T, kGreedy>, j);
}

template <typename T>
cudaError_t launch_mode(const VerifyJob& j, cudaStream_t stream) {
  return j.noise == nullptr ? launch_type<T, true>(j, stream) : launch_type<T, false>(j, stream);
}

}  // namespace

size_t verify_workspace(int64_t B, int64_t L, int64_t V) {
  const int64_t piece = piece_of(V);
  return size_t(B * (2 * L + 1)) * size_t((V + piece - 1) / piece) * sizeof(Piece);
}

cudaError_t launch_verify(VerifyJob j, void* workspace, cudaStream_t stream) {
  j.piece = piece_of(j.V);
  j.per_row = static_cast<int>((j.V + j.piece - 1) / j.piece);
  j.pieces = static_cast<Piece*>(workspace);
  return j.dtype == SF_F32    ? launch_mode<float>(j, stream)
         : j.dtype == SF_BF16 ? launch_mode<__nv_bfloat16>(j, stream)
                              : launch_mode<__half>(j, stream);
}

}  // namespace sf
