// Attention of several new tokens over a paged cache: heads of 64
// (tokens_attention.cuh).
#include "tokens_attention.cuh"

namespace quartz {

cudaError_t launch_tokens_attn_64(const TokensArgs &a, const TokensMaps &m, int kind, int tiles, int parts, int ctas, cudaStream_t s)
{
    if (tiles == 1) return launch_tokens_attn<64, 1, false, 2>(a, m, kind, ctas, s);
    return parts == 2 ? launch_tokens_attn<64, 2, false, 2>(a, m, kind, ctas, s) : launch_tokens_attn<64, 2, false, 1>(a, m, kind, ctas, s);
}

}  // namespace quartz
