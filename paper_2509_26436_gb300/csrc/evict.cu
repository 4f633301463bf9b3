// Eviction by accumulated attention weight, the choice, for sm_103a: per
// sequence and key / value head the first `sinks`, the last `recent` and of
// the tokens between the `want` with the largest weights, equal weights by the
// lowest index, as ascending indices.
//
// A radix select: each weight becomes a 32-bit key that orders like it, and
// four passes count the keys that share the digits found so far by their next
// eight bits, from the top, until the `want`-th largest key is known.  Two
// more passes count and write what stays, in order.  The work is a few reads
// of 4 bytes per token, so latency of the passes counts: the keys are read
// from global memory once and held in shared memory where they fit.
#include "quartz_internal.h"

namespace quartz {
namespace {

constexpr int kThreads = 1024;
constexpr int kWarps = kThreads / 32;
constexpr int kDigits = 256;

struct SelectArgs {
    const float *w;
    int64_t w_sb, w_sh;
    const int32_t *lens;
    int heads;
    int32_t max_len, budget, recent, sinks;
    int32_t *kept, *new_lens;
    int *dev_err;
};

// Unsigned keys in the order of the weights: -0 is 0, NaN below everything.
__device__ __forceinline__ uint32_t order_key(float f)
{
    if (!(f == f)) return 0u;
    const uint32_t u = __float_as_uint(f + 0.0f);  // -0 + 0 = 0
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

template <bool HELD>
__global__ void __launch_bounds__(kThreads, 1) evict_select_kernel(SelectArgs a)
{
    griddep_wait();
    extern __shared__ uint32_t s_keys[];
    __shared__ uint32_t s_hist[kDigits];
    __shared__ uint32_t s_above[kWarps], s_equal[kWarps];
    __shared__ uint32_t s_digit, s_left;
    const int64_t bh = blockIdx.x;
    const int64_t b = bh / a.heads;
    const int h = static_cast<int>(bh - b * a.heads);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int len = a.lens[b];
    if (len < 0 || len > a.max_len) {
        if (tid == 0) atomicExch(a.dev_err, QUARTZ_DEV_INDEX);
        len = len < 0 ? 0 : a.max_len;
    }
    int32_t *kept = a.kept + bh * a.budget;
    const int rows = min(len, a.budget);
    if (h == 0 && tid == 0) a.new_lens[b] = rows;
    for (int j = rows + tid; j < a.budget; j += kThreads) kept[j] = -1;
    if (len <= a.budget) {
        for (int j = tid; j < rows; j += kThreads) kept[j] = j;
        return;
    }
    const float *w = a.w + b * a.w_sb + h * a.w_sh;
    const int lo = a.sinks, hi = len - a.recent;  // the tokens between
    uint32_t want = static_cast<uint32_t>(a.budget - a.sinks - a.recent);  // < hi - lo
    if (HELD) {
        for (int t = lo + tid; t < hi; t += kThreads) s_keys[t - lo] = order_key(w[t]);
        __syncthreads();
    }
    auto key_at = [&](int t) { return HELD ? s_keys[t - lo] : order_key(w[t]); };

    // the want-th largest key: `prefix` holds its digits found so far
    uint32_t prefix = 0, mask = 0;
    for (int shift = 24; shift >= 0 && want > 0; shift -= 8) {
        for (int i = tid; i < kDigits; i += kThreads) s_hist[i] = 0;
        __syncthreads();
        for (int t0 = lo + warp * 32; t0 < hi; t0 += kThreads) {
            const int t = t0 + lane;
            const uint32_t key = t < hi ? key_at(t) : 0u;
            const bool mine = t < hi && (key & mask) == prefix;
            const uint32_t digit = mine ? (key >> shift) & 255u : kDigits;
            // sums of attention weights share few leading digits: one addition
            // for all lanes with the same
            const uint32_t same = __match_any_sync(0xffffffffu, digit);
            if (mine && lane == __ffs(same) - 1) atomicAdd(&s_hist[digit], __popc(same));
        }
        __syncthreads();
        if (warp == 0) {  // eight digits per lane, from the top
            uint32_t c[8], sum = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                c[i] = s_hist[kDigits - 1 - (lane * 8 + i)];
                sum += c[i];
            }
            uint32_t before = sum;
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const uint32_t v = __shfl_up_sync(0xffffffffu, before, d);
                if (lane >= d) before += v;
            }
            before -= sum;
            if (before < want && want <= before + sum) {  // one lane
                int i = 0;
                while (want > before + c[i]) before += c[i++];
                s_digit = kDigits - 1 - (lane * 8 + i);
                s_left = want - before;
            }
        }
        __syncthreads();
        prefix |= s_digit << shift;
        mask |= 255u << shift;
        want = s_left;  // of those with this prefix
    }
    // now: keys above `prefix` stay, and the first `want` that equal it (none
    // where only sinks and recent tokens stay: mask is still 0)
    const bool none = mask == 0;

    // each warp takes a run of consecutive tokens
    const int per = ((len + kWarps - 1) / kWarps + 31) & ~31;
    const int from = min(len, warp * per), to = min(len, from + per);
    uint32_t above = 0, equal = 0;
    for (int t0 = from; t0 < to; t0 += 32) {
        const int t = t0 + lane;
        const bool middle = t >= lo && t < hi;
        const uint32_t key = middle && t < to ? key_at(t) : 0u;
        const bool always = t < to && !middle;
        above += __popc(__ballot_sync(0xffffffffu, always || (t < to && middle && !none && key > prefix)));
        equal += __popc(__ballot_sync(0xffffffffu, t < to && middle && !none && key == prefix));
    }
    if (lane == 0) s_above[warp] = above, s_equal[warp] = equal;
    __syncthreads();
    uint32_t stay = 0, seen = 0;  // kept and equal ones before this warp's run
    for (int i = 0; i < warp; ++i) {
        const uint32_t e = s_equal[i];
        stay += s_above[i] + (seen < want ? min(e, want - seen) : 0u);
        seen += e;
    }
    const uint32_t before = (1u << lane) - 1;
    for (int t0 = from; t0 < to; t0 += 32) {
        const int t = t0 + lane;
        const bool middle = t >= lo && t < hi;
        const uint32_t key = middle && t < to ? key_at(t) : 0u;
        const bool same = t < to && middle && !none && key == prefix;
        const uint32_t eq = __ballot_sync(0xffffffffu, same);
        const bool keep = t < to && (!middle || (!none && key > prefix) || (same && seen + __popc(eq & before) < want));
        const uint32_t kp = __ballot_sync(0xffffffffu, keep);
        if (keep) kept[stay + __popc(kp & before)] = t;
        stay += __popc(kp);
        seen += __popc(eq);
    }
}

constexpr int64_t kHeldKeys = 48 * 1024;  // 192 KB of the 227 a CTA may have

}  // namespace

cudaError_t launch_evict_select(const float *w, int64_t w_sb, int64_t w_sh, const int32_t *lens, int64_t seqs, int heads,
                                int64_t max_len, int64_t budget, int64_t recent, int64_t sinks, int32_t *kept,
                                int32_t *new_lens, int *dev_err, cudaStream_t s)
{
    SelectArgs a{w, w_sb, w_sh, lens, heads, static_cast<int32_t>(max_len), static_cast<int32_t>(budget),
                 static_cast<int32_t>(recent), static_cast<int32_t>(sinks), kept, new_lens, dev_err};
    const dim3 grid(static_cast<unsigned>(seqs * heads));
    if (max_len <= kHeldKeys) {
        const int bytes = static_cast<int>(max_len) * 4;
        const cudaError_t e = cudaFuncSetAttribute(evict_select_kernel<true>,
                                                   cudaFuncAttributeMaxDynamicSharedMemorySize, kHeldKeys * 4);
        if (e != cudaSuccess) return e;
        return launch_pdl(evict_select_kernel<true>, grid, dim3(kThreads), bytes, s, a);
    }
    return launch_pdl(evict_select_kernel<false>, grid, dim3(kThreads), 0, s, a);
}

}  // namespace quartz
