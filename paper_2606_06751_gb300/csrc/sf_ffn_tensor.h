// sf_ffn_tensor.h - the forms of the gated feed-forward operators.
#pragma once

#include "sf_launch.h"

namespace sf {

// bf16 and f16; rows of x and the weights start on 16 bytes.
cudaError_t launch_ffn_tensor(const FfnJob& job, bool grad, cudaStream_t stream);

// f32, any rows; workspace of ffn_parts_workspace bytes.
size_t ffn_parts_workspace(int64_t T, int64_t H, int64_t F, bool grad);
cudaError_t launch_ffn_parts(FfnJob job, bool grad, void* workspace, cudaStream_t stream);

// A few tokens: products of any type (f32, or up to four tokens), f32 gradients of up to kFewGradTokens.
// even: rows of x and the weights start on 16 bytes.
constexpr int64_t kFewGradTokens = 8, kFewMostFeatures = int64_t(65535) * 8;
cudaError_t launch_ffn_few(const FfnJob& job, bool even, cudaStream_t stream);
size_t ffn_few_workspace(int64_t T, int64_t H, int64_t F);
cudaError_t launch_ffn_few_grad(FfnJob job, void* workspace, cudaStream_t stream);

// The sum of `parts` matrices of rows x len f32, `stride` apart, written or added to rows `ld` apart.
struct FfnSum {
  const float* from;
  int64_t stride;
  int parts;
  float* to;
  int64_t rows, len, ld;
  bool accumulate;
};
cudaError_t launch_ffn_sum(const FfnSum& job, cudaStream_t stream);

}  // namespace sf
