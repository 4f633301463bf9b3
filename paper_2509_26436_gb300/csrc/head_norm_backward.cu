// The gradient of the norm of each head with the rotation (head_norm.cuh).
#include "head_norm.cuh"

namespace quartz {

cudaError_t launch_norm_backward(HeadNormArgs &a, cudaStream_t s) { return launch_norm_mode<kBackward>(a, s); }

}  // namespace quartz
