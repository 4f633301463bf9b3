// Attention of several new tokens over a paged cache: heads of 128 with a cap, distances, or a factor that is not positive
// (tokens_attention.cuh).
#include "tokens_attention.cuh"

namespace quartz {

cudaError_t launch_tokens_attn_128_shaped(const TokensArgs &a, const TokensMaps &m, int kind, int tiles, int parts, int ctas, cudaStream_t s)
{
    if (tiles == 1) return launch_tokens_attn<128, 1, true, 2>(a, m, kind, ctas, s);
    return parts == 2 ? launch_tokens_attn<128, 2, true, 2>(a, m, kind, ctas, s) : launch_tokens_attn<128, 2, true, 1>(a, m, kind, ctas, s);
}

}  // namespace quartz
