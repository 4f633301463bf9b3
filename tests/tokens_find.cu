// Where each CTA of the attention of several new tokens begins, and how far it goes,
// without the attention: tokens_find alone (test_gpu_tokens_find.py).
#include "tokens_attention.cuh"

namespace {

template <int R>
__global__ void find_kernel(quartz::TokensArgs a, long long *out)
{
    __shared__ quartz::TokensFind f;
    quartz::TokensRun run;
    const bool some = quartz::tokens_find<R>(a, f, run);
    if (threadIdx.x) return;
    long long *o = out + 8 * blockIdx.x;
    o[0] = some, o[1] = run.pos, o[2] = run.end, o[3] = run.edge;
    if (some) o[4] = f.at.b, o[5] = f.at.head, o[6] = f.at.block, o[7] = f.at.off;
}

}  // namespace

// out: 8 numbers a CTA.  err: one word.
extern "C" int find(int rows, const int *lens, const int *starts, int seqs, int tokens, int max_len, int max_new, int heads,
                    int group, int ctas, long long *out, int *err)
{
    quartz::TokensArgs a{};
    a.lens = lens, a.starts = starts, a.seqs = seqs, a.tokens = tokens, a.max_len = max_len, a.max_new = max_new;
    a.kv_heads = heads, a.group = group, a.dev_err = err;
    if (rows == 256) find_kernel<256><<<ctas, 512>>>(a, out);
    else find_kernel<128><<<ctas, 512>>>(a, out);
    return cudaDeviceSynchronize();
}
