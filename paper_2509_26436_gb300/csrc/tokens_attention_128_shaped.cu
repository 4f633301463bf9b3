// Attention of several new tokens over a paged cache: heads of 128 with a cap, distances, or a factor that is not positive
// (tokens_attention.cuh).
#include "tokens_attention.cuh"

namespace quartz {

cudaError_t launch_tokens_attn_128_shaped(const TokensArgs &a, const TokensMaps &m, int kind, int tiles, int ctas, cudaStream_t s)
{
    return tiles == 2 ? launch_tokens_attn<128, 2, true>(a, m, kind, ctas, s)
                      : launch_tokens_attn<128, 1, true>(a, m, kind, ctas, s);
}

}  // namespace quartz
