// sf_ffn_tensor.h - the tensor-core form of the gated feed-forward operators.
#pragma once

#include "sf_launch.h"

namespace sf {

// bf16 and f16; rows of x and the weights start on 16 bytes.
cudaError_t launch_ffn_tensor(const FfnJob& job, bool grad, cudaStream_t stream);

}  // namespace sf
