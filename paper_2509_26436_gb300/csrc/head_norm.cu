// The norm of each head with the rotation, and the launches of head_norm.cuh's
// kernels.
#include "head_norm.cuh"

namespace quartz {
namespace {

// dw of side blockIdx.y, 32 elements per CTA: each of its 32 warps sums every 32nd
// of the side's parts, then the warps are added up (8 warps: 6.1 us).
constexpr int kSumThreads = 1024;

__global__ void __launch_bounds__(kSumThreads) head_norm_sum_kernel(HeadNormArgs a)
{
    griddep_wait();
    __shared__ float s_sum[kSumThreads / 32][32];
    const int side = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, d = blockIdx.x * 32 + lane;
    if (!a.side[side].dw) return;
    const float *part = a.part + (side ? static_cast<int64_t>(a.ctas[0]) * a.dim : 0) + d;
    float s = 0.f;
    if (d < a.dim) {
#pragma unroll 8
        for (int i = warp; i < a.ctas[side]; i += kSumThreads / 32) s += part[static_cast<int64_t>(i) * a.dim];
    }
    s_sum[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && d < a.dim) {
#pragma unroll
        for (int w = 1; w < kSumThreads / 32; ++w) s += s_sum[w][lane];
        if (a.w_type == QUARTZ_OUT_F32) static_cast<float *>(a.side[side].dw)[d] = s;
        else if (a.w_type == QUARTZ_OUT_F16) static_cast<__half *>(a.side[side].dw)[d] = __float2half_rn(s);
        else static_cast<__nv_bfloat16 *>(a.side[side].dw)[d] = __float2bfloat16_rn(s);
    }
}

}  // namespace

size_t head_norm_workspace_bytes(int dim) { return (static_cast<size_t>(device_sms()) * kMostBackward + 2) * dim * 4; }

cudaError_t launch_norm_forward(HeadNormArgs &a, cudaStream_t s) { return launch_norm_mode<kForward>(a, s); }

cudaError_t launch_rope_axes(HeadNormArgs a, cudaStream_t s) { return launch_norm_rotate(a, s); }

cudaError_t launch_head_norm(HeadNormArgs a, cudaStream_t s) { return launch_norm_forward(a, s); }

cudaError_t launch_head_norm_backward(HeadNormArgs a, cudaStream_t s)
{
    cudaError_t e = cudaSuccess;
    // sets the CTAs of each side; else both sums are 0
    if (a.tokens > 0 && a.side[0].heads + a.side[1].heads > 0) e = launch_norm_backward(a, s);
    if (e != cudaSuccess || !a.part) return e;
    return launch_pdl(head_norm_sum_kernel, dim3((a.dim + 31) / 32, 2), dim3(kSumThreads), 0, s, a);
}

}  // namespace quartz
