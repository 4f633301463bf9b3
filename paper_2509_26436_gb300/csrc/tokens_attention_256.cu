// Attention of several new tokens over a paged cache: heads of 256
// (tokens_attention.cuh).
#include "tokens_attention.cuh"

namespace quartz {

cudaError_t launch_tokens_attn_256(const TokensArgs &a, const TokensMaps &m, int kind, int, int parts, int ctas, cudaStream_t s)
{
    return parts == 2 ? launch_tokens_attn<256, 1, false, 2>(a, m, kind, ctas, s) : launch_tokens_attn<256, 1, false, 1>(a, m, kind, ctas, s);
}

}  // namespace quartz
