// Rotary positions of several axes (head_norm.cuh).
#include "head_norm.cuh"

namespace quartz {

cudaError_t launch_norm_rotate(HeadNormArgs &a, cudaStream_t s) { return launch_norm_mode<kRotate>(a, s); }

}  // namespace quartz
