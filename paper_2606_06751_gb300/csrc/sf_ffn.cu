// sf_ffn.cu - the gated feed-forward product h = act(x Wg^T) * (x Wu^T) and its
// gradient (sf_gated_ffn, sf_gated_ffn_grad): which form a call takes, and the copy of
// rows that tensor copies cannot read.
//   bf16, f16          the tensor cores (sf_ffn_tensor.cu); rows that do not start
//                      on 16 bytes are copied first, but for a few tokens
//   f32                the tensor cores by parts (sf_ffn_parts.cu), but for a few
//                      tokens' product
//   a few tokens       one read of the weights on the f32 units (sf_ffn_few.cu)
#include <algorithm>

#include "sf_float.cuh"
#include "sf_ffn_tensor.h"

namespace sf {
namespace {

constexpr int kThreads = 256;

// ---------------------------------------------------------------- rows for tensor copies

// Rows of 16-bit values that start anywhere, copied to rows that start on 16 bytes.
struct Spread {
  const unsigned short* from[3];
  uint4* to[3];
  int64_t rows[3], ld[3];
};
// Eight 16-bit values from `off` in two 16-byte words; off is one number for the warp.
__device__ __forceinline__ uint4 eight_from(const uint4& a, const uint4& b, int off) {
  uint32_t w[5];
  switch (off >> 1) {
    case 0: w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x; break;
    case 1: w[0] = a.y, w[1] = a.z, w[2] = a.w, w[3] = b.x, w[4] = b.y; break;
    case 2: w[0] = a.z, w[1] = a.w, w[2] = b.x, w[3] = b.y, w[4] = b.z; break;
    default: w[0] = a.w, w[1] = b.x, w[2] = b.y, w[3] = b.z, w[4] = b.w;
  }
  if (off & 1) {
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = __funnelshift_r(w[k], w[k + 1], 16);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// A warp a run of 128 packs of a row.  A pack's 8 values lie in two of the source's
// 16-byte words; the second is the next lane's first, read once more.  Bound by memory
// with all reads of a run on their way at once.
__global__ void __launch_bounds__(kThreads) ffn_spread_kernel(const __grid_constant__ Spread s, int64_t len, int packs,
                                                              int runs) {
  constexpr int kPacks = 4;
  griddep_launch_dependents();
  const int part = blockIdx.y, lane = threadIdx.x & 31;
  const int64_t rows = s.rows[part], ld = s.ld[part], step = int64_t(gridDim.x) * (kThreads / 32);
  const int64_t first = int64_t(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5);
  const unsigned short *from = s.from[part], *end = from + (rows - 1) * ld + len;  // behind the last value
  int64_t r = first / runs;
  int run = static_cast<int>(first - r * runs);
  const int64_t rows_on = step / runs;
  const int runs_on = static_cast<int>(step - rows_on * runs);
  while (r < rows) {
    const unsigned short* row = from + r * ld;
    const int off = static_cast<int>(reinterpret_cast<uintptr_t>(row) >> 1 & 7u);
    const int p = run * (32 * kPacks) + lane;
    const unsigned short* at = row + int64_t(p) * 8 - off;
    uint4* to = s.to[part] + r * packs + p;
    uint4 a[kPacks], b[kPacks];
    bool whole[kPacks];
#pragma unroll
    for (int k = 0; k < kPacks; ++k) {
      const unsigned short* q = at + k * 256;
      whole[k] = p + k * 32 < packs && q >= from && q + 16 <= end;
      if (whole[k]) {
        a[k] = *reinterpret_cast<const uint4*>(q);
        b[k] = off != 0 ? *reinterpret_cast<const uint4*>(q + 8) : a[k];  // from L1
      }
    }
#pragma unroll
    for (int k = 0; k < kPacks; ++k) {
      if (p + k * 32 >= packs) break;
      uint4 v;
      if (whole[k]) {
        v = eight_from(a[k], b[k], off);
      } else {
        const int64_t c = int64_t(p + k * 32) * 8;
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t lo = c + 2 * i < len ? row[c + 2 * i] : 0u, hi = c + 2 * i + 1 < len ? row[c + 2 * i + 1] : 0u;
          w[i] = lo | hi << 16;
        }
        v = make_uint4(w[0], w[1], w[2], w[3]);
      }
      to[k * 32] = v;
    }
    r += rows_on;
    run += runs_on;
    if (run >= runs) {
      run -= runs;
      ++r;
    }
  }
}

// ---------------------------------------------------------------- host

// Rows of nothing, for weights without tokens.
__global__ void __launch_bounds__(kThreads) ffn_clear_kernel(char* gate, char* up, int64_t rows, int64_t bytes,
                                                             int64_t pitch) {
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
    for (int64_t i = threadIdx.x * int64_t(2); i < bytes; i += kThreads * 2) {
      *reinterpret_cast<unsigned short*>(gate + r * pitch + i) = 0;
      *reinterpret_cast<unsigned short*>(up + r * pitch + i) = 0;
    }
}

size_t value_size(int32_t dtype) { return dtype == SF_F32 ? 4 : 2; }
size_t round16(size_t n) { return (n + 15) & ~size_t(15); }

// Whether a call takes the form for a few tokens.  Products, us here against the tensor cores:
//   f32          512 x 2048: 16 tokens 6.5 / 16, 32 10.5 / 16, 48 14.6 / 16.4; 1024 x 4096: 16 18 / 31,
//                24 24 / 31, 32 30.5 / 31.2, 48 43 / 31.5; 2048 x 8192: 16 55 / 91, 24 77 / 91, 32 96 / 91,
//                48 142 / 94; 4096 x 12288: 12 144 / 306, 16 149 / 305, 24 208 / 305, 32 276 / 306, 48 402 / 307
//   f32 gradient up to 8 tokens, as many as have the form: 24 / 34, 39 / 67, 126 / 177, 280 / 516
//   16 bits      one token through 4096 x 12288  32.7 / 35.2, two 37.0 / 34.7; through 1024 x 2048
//                one 3.7 / 5.4, four 4.4 / 5.4
//   uneven rows  one token through 4097 x 12288  55 / 131 (with the copy of the weights), two 90 / 132
bool few_tokens(int32_t dtype, int64_t T, int64_t H, int64_t F, bool aligned, bool grad) {
  if (F > kFewMostFeatures) return false;
  if (dtype == SF_F32) return T <= (grad ? kFewGradTokens : 32);
  if (grad) return false;
  return aligned ? T == 1 || (T <= 4 && F * H <= int64_t(1) << 22) : T <= 2;
}

}  // namespace

bool ffn_rows_on16(const void* p, int64_t ld, int32_t dtype) {
  return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (ld * int64_t(value_size(dtype))) % 16 == 0;
}

size_t ffn_workspace(int32_t dtype, int64_t T, int64_t H, int64_t F, bool aligned, bool grad) {
  if (few_tokens(dtype, T, H, F, aligned, grad)) return grad ? ffn_few_workspace(T, H, F) : 0;
  if (dtype == SF_F32) return ffn_parts_workspace(T, H, F, grad);
  const size_t inner = grad ? 2 * size_t(T) * round16(size_t(F) * 2) : 0;
  return inner + (aligned ? 0 : size_t(T + 2 * F) * round16(size_t(H) * 2));
}

cudaError_t launch_ffn(FfnJob j, bool grad, void* workspace, cudaStream_t stream) {
  if (j.T == 0) {
    if (j.dw_gate == nullptr || j.accumulate) return cudaSuccess;
    const int64_t size = value_size(j.dw_dtype);
    count_launch();
    ffn_clear_kernel<<<static_cast<unsigned>(std::min<int64_t>(j.F, sm_count() * 8)), kThreads, 0, stream>>>(
        static_cast<char*>(j.dw_gate), static_cast<char*>(j.dw_up), j.F, j.H * size, j.lddw * size);
    return cudaGetLastError();
  }
  const bool even = ffn_rows_on16(j.x, j.T > 1 ? j.ldx : 0, j.dtype) &&
                    ffn_rows_on16(j.w_gate, j.F > 1 ? j.ldw : 0, j.dtype) &&
                    ffn_rows_on16(j.w_up, j.F > 1 ? j.ldw : 0, j.dtype);
  if (few_tokens(j.dtype, j.T, j.H, j.F, even, grad))
    return grad ? launch_ffn_few_grad(j, workspace, stream) : launch_ffn_few(j, even, stream);
  if (j.dtype == SF_F32) return launch_ffn_parts(j, grad, workspace, stream);
  char* at = static_cast<char*>(workspace);
  if (grad) {
    const size_t row = round16(size_t(j.F) * 2);
    j.dg = at;
    j.du = at + size_t(j.T) * row;
    j.ldg = int64_t(row / 2);
    at += 2 * size_t(j.T) * row;
  }
  if (!even) {
    const int64_t packs = int64_t(round16(size_t(j.H) * 2) / 16);
    Spread s;
    const void** data[3] = {&j.x, &j.w_gate, &j.w_up};
    for (int i = 0; i < 3; ++i) {
      s.from[i] = static_cast<const unsigned short*>(*data[i]);
      s.to[i] = reinterpret_cast<uint4*>(at);
      s.rows[i] = i == 0 ? j.T : j.F;
      s.ld[i] = i == 0 ? j.ldx : j.ldw;
      *data[i] = at;
      at += size_t(s.rows[i]) * packs * 16;
    }
    const int64_t runs = (packs + 127) / 128, most = (std::max(j.T, j.F) * runs + kThreads / 32 - 1) / (kThreads / 32);
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>(most, int64_t(sm_count()) * 8)), 3);
    count_launch();
    ffn_spread_kernel<<<grid, kThreads, 0, stream>>>(s, j.H, static_cast<int>(packs), static_cast<int>(runs));
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    j.ldx = j.ldw = packs * 8;
  }
  return launch_ffn_tensor(j, grad, stream);
}

}  // namespace sf
