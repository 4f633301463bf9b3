// Attention of several new tokens over a paged cache: heads of 128
// (tokens_attention.cuh).
#include "tokens_attention.cuh"

namespace quartz {

cudaError_t launch_tokens_attn_128(const TokensArgs &a, const TokensMaps &m, int kind, int tiles, int parts, int ctas, cudaStream_t s)
{
    if (tiles == 1) return launch_tokens_attn<128, 1, false, 2>(a, m, kind, ctas, s);
    return parts == 2 ? launch_tokens_attn<128, 2, false, 2>(a, m, kind, ctas, s) : launch_tokens_attn<128, 2, false, 1>(a, m, kind, ctas, s);
}

}  // namespace quartz
