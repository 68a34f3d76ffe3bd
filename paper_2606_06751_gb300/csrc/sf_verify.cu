// sf_verify.cu - drafted tokens verified against the policy's rows by given
// random numbers (sf_verify_draft).
//
// A drafted token y is kept while u q(y) < p(y); the first that is not is replaced
// by a draw from max(p - q, 0), as the winner of a race: the entry of largest r_j /
// e_j, e_j exponential, is j with probability r_j / sum r.  One launch: a cluster of
// CTAs a sequence, each with a slice of the vocabulary.  The positions go by in
// groups: each warp streams its part of the group's rows (policy's and draft's) into
// (maximum, sum of exponentials) pairs, the CTAs exchange them, and all decide alike
// whether the sequence stops there.  Rows behind that group are not read.  The slice
// of the one row that the next token comes from is then raced against the noise.
// Bound by memory for many sequences: 64 of 4 tokens over 131072 bf16 entries, 187 MB,
// take 42 us (66 % of the copy rate; the exponentials alone some 16 us of the special
// function units, and the race begins when the rows are done).  One sequence over
// 32768 takes 10 us of latency.  Four CTAs of 256 threads an SM: three take 48 us, two
// with pieces of twice the size 44.  Groups of three positions, which read fewer rows,
// were no faster: another exchange costs what they save.

#include "sf_float.cuh"
#include "sf_launch.h"

namespace sf {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kPacks = 4;       // of 16 bytes that a thread has in flight
constexpr int kPerSm = 4;       // CTAs of an SM
constexpr int kMostCtas = 16;   // of a cluster
constexpr int kGroup = 16;      // positions of a group

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Larger value first, then lower place: one integer order for values above 0.
__device__ __forceinline__ uint64_t place_key(uint32_t value, int at) {
  return uint64_t(value) << 32 | (0xffffffffu - static_cast<uint32_t>(at));
}
constexpr uint64_t kUndrawn = 1;  // below all keys: there are values above 0, but none can be drawn
__device__ __forceinline__ int place_of(uint64_t key) {
  return static_cast<int>(0xffffffffu - static_cast<uint32_t>(key));
}

// 16-byte packs of a row by address: pack 0 holds the row's first value, `off`
// values behind a 16-byte boundary.  Values before the row and behind it are -inf.
template <typename T>
__device__ __forceinline__ uint4 row_pack(const T* z, int off, int pack, int V) {
  constexpr int N = Pack<T>::kN;
  const int at = pack * N - off;
  if (at >= 0 && at + N <= V) return load16(z + at);
  uint4 u = lowest_pack(T());
  T* e = reinterpret_cast<T*>(&u);
#pragma unroll
  for (int q = 0; q < N; ++q)
    if (at + q >= 0 && at + q < V) e[q] = z[at + q];
  return u;
}
template <typename T>
__device__ __forceinline__ int row_offset(const T* z) {
  return static_cast<int>((reinterpret_cast<uintptr_t>(z) & 15u) / sizeof(T));
}

// What part of a row says: its largest logit, the sum of the exponentials against
// it and the first place of the largest.  The sum is NaN with a NaN or +inf logit.
struct Part {
  float m, s;
  int at;
};
constexpr int kNowhere = 0x7fffffff;

__device__ __forceinline__ Part nothing() { return {neg_inf(), 0.f, kNowhere}; }

// The lanes' parts (of `n` lanes, a power of two), in a fixed order.
template <bool kGreedy>
__device__ __forceinline__ Part joined_lanes(Part a, int n, float scale) {
  float top = a.m;
  for (int o = n / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, o));
  if (a.m != neg_inf()) a.s *= exp2_fast((a.m - top) * scale);
  for (int o = n / 2; o > 0; o >>= 1) a.s += __shfl_xor_sync(kFull, a.s, o);
  if (kGreedy) {
    a.at = a.m == top ? a.at : kNowhere;
    for (int o = n / 2; o > 0; o >>= 1) a.at = min(a.at, __shfl_xor_sync(kFull, a.at, o));
  }
  a.m = top;
  return a;
}

// The warp's largest value; NaN only if all are.
__device__ __forceinline__ float warp_top(float v) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}

// kPacks packs a lane of a row.
template <typename T>
struct Piece {
  uint4 u[kPacks];
  int base;  // the place in the row of the lane's first value
  int row;
};
constexpr int kStride = kPacks * 32;  // packs of a piece

// Where a warp is in its run of pieces.
template <typename T>
struct Cursor {
  const T* z;      // the row
  int off, p;      // its distance from a 16-byte boundary; the lane's next pack
  int whole, end;  // packs of the row that end in it; of the CTA's slice
  int row, left;   // pieces left of this row
  // packs p, p + 32, ...; outside the slice -inf
  __device__ __forceinline__ void load(Piece<T>& piece, int V) const {
    constexpr int N = Pack<T>::kN;
    const int p0 = p - static_cast<int>(threadIdx.x & 31);
    piece.base = p * N - off;
    piece.row = row;
    if ((p0 > 0 || off == 0) && p0 + kStride <= min(whole, end)) {
      const T* at = z + piece.base;
#pragma unroll
      for (int k = 0; k < kPacks; ++k) piece.u[k] = load16(at + k * 32 * N);
    } else {
#pragma unroll
      for (int k = 0; k < kPacks; ++k)
        piece.u[k] = p + k * 32 < end ? row_pack(z, off, p + k * 32, V) : lowest_pack(T());
    }
  }
};

// A warp's part of a row, piece by piece: the reference is the largest logit so far,
// the sum each lane's own.
template <typename T, bool kGreedy>
struct Running {
  float m = neg_inf(), scale;
  uint64_t s = 0;  // a pair of sums
  int at = kNowhere;
  __device__ __forceinline__ void add(const Piece<T>& piece) {
    constexpr int N = Pack<T>::kN;
    const float top = warp_top(packs_max(piece.u, T()));
    if (top > m) {  // one branch for the warp
      const float by = exp2_fast((m - top) * scale);
      s = mul2(s, pair_of(by, by));
      m = top;
      at = kNowhere;
    }
    const float ref = m == neg_inf() ? 0.f : m;  // NaN among logits of -inf stays NaN below
    const uint64_t minus = pair_of(-ref, -ref), by = pair_of(scale, scale);
#pragma unroll
    for (int k = 0; k < kPacks; ++k) {
      uint64_t w[N / 2];
      unpack2(piece.u[k], w, T());
#pragma unroll
      for (int q = 0; q < N / 2; ++q) {
        float x, y;
        if (kGreedy) {
          split(w[q], x, y);
          const int place = piece.base + k * 32 * N + 2 * q;
          if (y == m) at = min(at, place + 1);
          if (x == m) at = min(at, place);
        }
        split(mul2(add2(w[q], minus), by), x, y);
        s = add2(s, pair_of(exp2_fast(x), exp2_fast(y)));
      }
    }
  }
  // the lanes' together; then empty
  __device__ __forceinline__ Part take() {
    float x, y;
    split(s, x, y);
    Part a;
    a.m = m;
    a.s = warp_sum(x + y);
    a.at = kGreedy ? static_cast<int>(__reduce_min_sync(kFull, static_cast<uint32_t>(at))) : kNowhere;
    m = neg_inf();
    s = 0;
    at = kNowhere;
    return a;
  }
};

// Where a sequence stops.
struct Stop {
  int at = -1;   // accepted tokens; -1: not yet
  int from;      // 0: no token; 1: the policy's row alone; 2: less the draft's; 3: without the drafted token
  float m, s, mq, sq;
  int last;      // greedy: the next token; 3: the drafted token
};

// The largest r_j / e_j a thread has met, r_j = p_j - q_j as `form` says, and the
// largest r_j; its indices rise, so the first of equal ones stays.
struct Race {
  float best, top;
  int at;
  float m, by, mq, byq, scale;  // maxima, reciprocal sums
  int form, token;
  __device__ __forceinline__ void run(float z, float zq, float e, int j) {
    // products rounded by themselves: equal rows have a difference of 0
    float r = __fmul_rn(exp2_fast((z - m) * scale), by);
    if (form == 2) r = __fsub_rn(r, __fmul_rn(exp2_fast((zq - mq) * scale), byq));
    if (form == 3 && j == token) r = 0.f;
    top = fmaxf(top, r);
    const float v = __fdividef(r, e);
    if (v > best && e > 0.f) {
      best = v;
      at = j;
    }
  }
};

template <typename T, bool kGreedy>
__global__ void __launch_bounds__(kThreads, kPerSm) verify_kernel(const VerifyJob j) {
  __shared__ Part warps[2 * kGroup][kWarps];          // the group's rows: policy's, then draft's
  __shared__ Part ctas[2][2 * kGroup][kMostCtas];     // of the cluster, for this group and the one before
  __shared__ float2 rows[kGroup], drafts[kGroup];  // (maximum, sum)
  __shared__ int firsts[kGroup];
  __shared__ int takes[kGroup];  // 1 accepted, 0 not, -1 a faulty row, -2 no such token
  __shared__ float zs[SF_VERIFY_MAX_DRAFT], zqs[SF_VERIFY_MAX_DRAFT], us[SF_VERIFY_MAX_DRAFT];
  __shared__ int64_t ys[SF_VERIFY_MAX_DRAFT];
  __shared__ float lps[SF_VERIFY_MAX_DRAFT + 1];
  __shared__ uint64_t warps_best[kWarps];
  __shared__ uint64_t best_of[kMostCtas];
  constexpr int N = Pack<T>::kN;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int C = static_cast<int>(cluster_size()), rank = static_cast<int>(cluster_rank());
  cluster_arrive();
  const int64_t b = blockIdx.x / static_cast<unsigned>(C);
  const int V = static_cast<int>(j.V), L = static_cast<int>(j.L);
  const int given = j.length == nullptr ? L : j.length[b], n = min(max(given, 0), L);
  const T* target = static_cast<const T*>(j.target) + b * (L + 1) * j.ldt;
  const T* draft = !kGreedy && j.draft != nullptr ? static_cast<const T*>(j.draft) + b * L * j.ldq : nullptr;
  const float scale = j.tau * kLog2e;
  // packs of a CTA's slice; rows that do not all start on 16 bytes may have one more
  const bool even_rows = ((reinterpret_cast<uintptr_t>(j.target) | uint64_t(j.ldt) * sizeof(T)) & 15u) == 0 &&
                         (draft == nullptr || ((reinterpret_cast<uintptr_t>(j.draft) | uint64_t(j.ldq) * sizeof(T)) & 15u) == 0);
  const int slice = ((V + (even_rows ? 0 : N - 1) + N - 1) / N + C - 1) / C;
  uint32_t bits = given != n ? SF_ST_INDEX : 0u;
  Stop o;
  for (int g0 = 0, turn = 0; o.at < 0; g0 += kGroup, turn ^= 1) {
    const int g = min(kGroup, n + 1 - g0);  // positions; the last may be the one behind the drafted tokens
    const int with_draft = draft != nullptr ? min(g, n - g0) : 0, all = g + with_draft;
    for (int i = lane; i < all; i += 32) warps[i][warp] = nothing();
    __syncwarp();
    // the slices of all rows as one run of pieces, cut evenly among the warps
    const int per_row = (slice + kStride - 1) / kStride;
    const int first = all * per_row * warp / kWarps, last = all * per_row * (warp + 1) / kWarps;
    Cursor<T> at;
    const auto to_row = [&](int row) {
      at.row = row;
      at.z = row < g ? target + (g0 + row) * j.ldt : draft + (g0 + row - g) * j.ldq;
      at.off = row_offset(at.z);
      at.p = rank * slice + lane;
      at.whole = (at.off + V) / N;
      at.end = min((rank + 1) * slice, (at.off + V + N - 1) / N);
      at.left = per_row;
    };
    const auto fetch = [&](Piece<T>& piece) {
      at.load(piece, V);
      if (--at.left > 0)
        at.p += kStride;
      else if (at.row + 1 < all)
        to_row(at.row + 1);
    };
    Piece<T> odd, even;
    if (first < last) {
      const int row = first / per_row, gone = first - row * per_row;
      to_row(row);
      at.p += gone * kStride;
      at.left -= gone;
      fetch(even);
    }
    if (g0 == 0 && tid < n) {  // what the decisions need besides
      const int64_t y = j.token[b * L + tid];
      ys[tid] = y;
      if (y >= 0 && y < V) {
        zs[tid] = to_f32(target[tid * j.ldt + y]);
        if (!kGreedy) {
          zqs[tid] = draft != nullptr ? to_f32(draft[tid * j.ldq + y]) : 0.f;
          us[tid] = j.uniform[b * L + tid];
        }
      }
    }
    Running<T, kGreedy> run;
    run.scale = scale;
    const auto keep = [&](int row) {
      const Part a = run.take();
      if (lane == 0) warps[row][warp] = a;
    };
    for (int item = first; item < last; item += 2) {  // the next piece is on its way while one is summed
      const bool two = item + 1 < last, three = item + 2 < last;
      if (two) fetch(odd);
      run.add(even);
      if (!two || odd.row != even.row) keep(even.row);
      if (!two) break;
      if (three) fetch(even);
      run.add(odd);
      if (!three || even.row != odd.row) keep(odd.row);
    }
    __syncthreads();
    if (g0 == 0) cluster_wait();  // the others have started
    for (int i = warp; i < all; i += kWarps) {
      Part a = joined_lanes<kGreedy>(lane < kWarps ? warps[i][lane] : nothing(), kWarps, scale);
      a.m = __shfl_sync(kFull, a.m, 0);
      a.s = __shfl_sync(kFull, a.s, 0);
      a.at = __shfl_sync(kFull, a.at, 0);
      if (lane < C) {
        const uint32_t to = at_rank(&ctas[turn][i][rank], lane);
        asm volatile("st.shared::cluster.f32 [%0], %1;\n\tst.shared::cluster.f32 [%0 + 4], %2;\n\t"
                     "st.shared::cluster.u32 [%0 + 8], %3;" ::"r"(to),
                     "f"(a.m), "f"(a.s), "r"(a.at)
                     : "memory");
      }
    }
    cluster_sync();
    for (int i = warp; i < g; i += kWarps) {
      const Part r = joined_lanes<kGreedy>(lane < C ? ctas[turn][i][lane] : nothing(), kMostCtas, scale);
      Part q = {0.f, 1.f, 0};
      if (i < with_draft) q = joined_lanes<kGreedy>(lane < C ? ctas[turn][g + i][lane] : nothing(), kMostCtas, scale);
      if (lane == 0) {
        const int at = g0 + i;
        // a NaN sum, no logit above -inf, or +inf
        int take = r.s > 0.f && finite(r.m) ? 0 : -1;
        if (at < n && take == 0) {
          const int64_t y = ys[at];
          if (y < 0 || y >= V) {
            take = -2;
          } else {
            const float ty = (zs[at] - r.m) * j.tau;
            lps[at] = ty - logf(r.s);
            if (kGreedy) {
              take = y == r.at ? 1 : 0;
            } else {
              const float qy = draft != nullptr ? expf((zqs[at] - q.m) * j.tau) / q.s : 1.f;
              take = !(q.s > 0.f && finite(q.m)) ? -1 : us[at] * qy < expf(ty) / r.s ? 1 : 0;
            }
          }
        }
        rows[i] = make_float2(r.m, r.s);
        drafts[i] = make_float2(q.m, q.s);
        firsts[i] = r.at;
        takes[i] = take;
      }
    }
    __syncthreads();
    for (int i = 0; i < g && o.at < 0; ++i) {
      const int at = g0 + i, take = takes[i];
      if (at < n && take == 1) continue;
      o.at = at;
      o.m = rows[i].x;
      o.s = rows[i].y;
      o.mq = drafts[i].x;
      o.sq = drafts[i].y;
      o.from = take == -1 ? 0 : at == n || take == -2 || kGreedy ? 1 : draft != nullptr ? 2 : 3;
      o.last = kGreedy ? firsts[i] : o.from == 3 ? static_cast<int>(ys[at]) : 0;
      if (at < n && take == -2) bits |= SF_ST_INDEX;
    }
  }
  int next = -1;
  if (kGreedy) {
    next = o.from == 0 ? -1 : o.last;
  } else if (o.from != 0) {
    const T *z = target + o.at * j.ldt, *zq = o.from == 2 ? draft + o.at * j.ldq : z;
    const float* e = j.noise + b * V;
    Race race;
    race.m = o.m;
    race.by = 1.f / o.s;
    race.mq = o.mq;
    race.byq = 1.f / o.sq;
    race.scale = j.tau * kLog2e;
    race.form = o.from;
    race.token = o.last;
    const bool even = ((reinterpret_cast<uintptr_t>(z) | reinterpret_cast<uintptr_t>(zq) | reinterpret_cast<uintptr_t>(e)) &
                       15u) == 0;
    uint64_t best = 0;
    for (;;) {
      race.best = race.top = 0.f;
      race.at = -1;
      int rest = 0;
      if (even) {  // whole packs of the three rows side by side
        const int packs = V / N;
        const int from = static_cast<int>(int64_t(packs) * rank / C), to = static_cast<int>(int64_t(packs) * (rank + 1) / C);
#pragma unroll 2
        for (int p = from + tid; p < to; p += kThreads) {
          float f[N], g[N], h[N];
          const uint4 u = load16(z + p * N), v = race.form == 2 ? load16(zq + p * N) : u;
          uint4 w[N / 4];
#pragma unroll
          for (int k = 0; k < N / 4; ++k) w[k] = load16(e + p * N + 4 * k);
          unpack(u, f, T());
          unpack(v, g, T());
#pragma unroll
          for (int k = 0; k < N / 4; ++k) unpack(w[k], reinterpret_cast<float(&)[4]>(h[4 * k]), 0.f);
#pragma unroll
          for (int k = 0; k < N; ++k) race.run(f[k], g[k], h[k], p * N + k);
        }
        rest = packs * N;
      }
      {
        const int left = V - rest;
        const int from = rest + static_cast<int>(int64_t(left) * rank / C), to = rest + static_cast<int>(int64_t(left) * (rank + 1) / C);
#pragma unroll 4
        for (int q = from + tid; q < to; q += kThreads)
          race.run(to_f32(z[q]), race.form == 2 ? to_f32(zq[q]) : 0.f, e[q], q);
      }
      best = race.at >= 0 ? place_key(__float_as_uint(race.best), race.at) : race.top > 0.f ? kUndrawn : 0;
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
      if (best != 0 || race.form == 1) break;
      race.form = 1;  // no residual above 0
    }
    next = best > kUndrawn ? place_of(best) : -1;
  }
  if (rank != 0) return;
  if (next < 0) bits |= SF_ST_NONFINITE;
  for (int i = tid; i <= L; i += kThreads) {
    int64_t t = -1;
    float lp = 0.f;
    if (i < o.at) {
      t = ys[i];
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
    report(j.status, bits);
  }
}

template <typename T, bool kGreedy>
cudaError_t launch_type(const VerifyJob& j, cudaStream_t stream) {
  // CTAs a sequence: while all stay at once and each thread has a pack of a row.
  // 64 sequences of 4 tokens, 131072 bf16 entries: 55, 46, 55 us with 4, 8, 16; one of
  // 32768: 15, 12, 10 us.
  int C = 1;
  while (C < kMostCtas && j.B * C * 2 <= int64_t(sm_count()) * kPerSm && j.V > int64_t(C) * kThreads * Pack<T>::kN) C *= 2;
  const auto kernel = verify_kernel<T, kGreedy>;
  if (C > 8) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(j.B * C));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = C;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  count_launch();
  return cudaLaunchKernelEx(&cfg, kernel, j);
}

template <typename T>
cudaError_t launch_mode(const VerifyJob& j, cudaStream_t stream) {
  return j.noise == nullptr ? launch_type<T, true>(j, stream) : launch_type<T, false>(j, stream);
}

}  // namespace

cudaError_t launch_verify(const VerifyJob& j, cudaStream_t stream) {
  return j.dtype == SF_F32    ? launch_mode<float>(j, stream)
         : j.dtype == SF_BF16 ? launch_mode<__nv_bfloat16>(j, stream)
                              : launch_mode<__half>(j, stream);
}

}  // namespace sf
