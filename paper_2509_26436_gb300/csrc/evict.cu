// Eviction by accumulated attention weight, the choice, for sm_103a: per
// sequence and key / value head the first `sinks`, the last `recent` and of
// the tokens between the `want` with the largest weights, equal weights by the
// lowest index, as ascending indices.
//
// Each weight becomes a 32-bit key that orders like it.  The range of the keys
// is cut into 2048 equal buckets, their populations counted, and the bucket
// that holds the `want`-th largest key becomes the next range, until a bucket
// is one key: three passes at most, the later ones over the few keys that are
// left.  (Cut by the range, not by fixed digits: sums of attention weights
// share their leading bits, and as keys, which grow with the logarithm, they
// spread evenly; lanes that meet in a bucket wait for each other.)  Two more
// passes count and write what stays, in order.  The work is a few reads of 4
// bytes per token, so the latency of the passes counts: the keys are read from
// global memory once and held in shared memory where they fit.  16 x 8 heads of
// up to 16384 tokens: 13.4 us in a graph, 15.4 to 17 with cold caches (26.5 with
// four passes over 8-bit digits, whose equal leading digits had to be matched
// across the lanes first).
#include "quartz_internal.h"

namespace quartz {
namespace {

constexpr int kBuckets = 2048;

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

template <bool HELD, int kThreads>
__global__ void __launch_bounds__(kThreads, kThreads == 1024 ? 1 : 6) evict_select_kernel(SelectArgs a)
{
    griddep_wait();
    constexpr int kWarps = kThreads / 32;
    extern __shared__ uint32_t s_keys[];
    __shared__ uint32_t s_hist[kBuckets];
    __shared__ uint32_t s_above[kWarps], s_equal[kWarps];
    __shared__ uint32_t s_bucket, s_left;
    const int64_t bh = blockIdx.x;
    const int64_t b = bh / a.heads;
    const int h = static_cast<int>(bh - b * a.heads);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int len = a.lens[b];
    if (len < 0 || len > a.max_len) {
        if (tid == 0) atomicOr(a.dev_err, QUARTZ_DEV_INDEX);
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
    const bool none = want == 0;  // only sinks and recent tokens stay
    uint32_t top = 0, bottom = 0xffffffffu;
    for (int t0 = lo + tid; t0 < hi; t0 += 16 * kThreads) {
        float f[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) f[i] = t0 + i * kThreads < hi ? w[t0 + i * kThreads] : 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (t0 + i * kThreads < hi) {
                const uint32_t key = order_key(f[i]);
                if (HELD) s_keys[t0 + i * kThreads - lo] = key;
                top = max(top, key);
                bottom = min(bottom, key);
            }
    }
    top = __reduce_max_sync(0xffffffffu, top);
    bottom = __reduce_min_sync(0xffffffffu, bottom);
    if (lane == 0) s_above[warp] = top, s_equal[warp] = bottom;
    __syncthreads();
    top = __reduce_max_sync(0xffffffffu, s_above[lane % kWarps]);
    bottom = __reduce_min_sync(0xffffffffu, s_equal[lane % kWarps]);
    // The warps' counts go to the same places, and where all keys are equal no barrier
    // of the loop lies between.  (Places of their own instead: 64 x 32 heads of up to
    // 4096 tokens 44.8 us, 37.1 with the barrier.)
    __syncthreads();
    auto key_at = [&](int t) { return HELD ? s_keys[t - lo] : order_key(w[t]); };

    // the want-th largest key is in [bottom, bottom + span]
    uint32_t span = top - bottom;
    while (span > 0 && !none) {
        const int shift = max(0, 21 - __clz(span));  // span >> shift < 2048
        for (int i = tid; i < kBuckets; i += kThreads) s_hist[i] = 0;
        __syncthreads();
#pragma unroll 4
        for (int t = lo + tid; t < hi; t += kThreads) {
            const uint32_t off = key_at(t) - bottom;
            if (off <= span) atomicAdd(&s_hist[off >> shift], 1u);
        }
        __syncthreads();
        // kEach buckets per thread, from the top: how many keys lie above them
        constexpr int kEach = kBuckets / kThreads;
        const int high = kBuckets - 1 - kEach * tid;
        uint32_t c[kEach], mine = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) c[i] = s_hist[high - i], mine += c[i];
        uint32_t upto = mine;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const uint32_t v = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += v;
        }
        if (lane == 31) s_above[warp] = upto;
        __syncthreads();
        uint32_t warps = lane < kWarps ? s_above[lane] : 0u;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const uint32_t v = __shfl_up_sync(0xffffffffu, warps, d);
            if (lane >= d) warps += v;
        }
        upto += warp ? __shfl_sync(0xffffffffu, warps, (warp + 31) & 31) : 0u;
        uint32_t before = upto - mine;
        if (before < want && want <= upto) {  // one thread
            int i = 0;
#pragma unroll
            for (int k = 0; k < kEach - 1; ++k)
                if (i == k && want > before + c[k]) before += c[k], ++i;
            s_bucket = high - i;
            s_left = want - before;
        }
        __syncthreads();
        want = s_left;  // of those in the bucket
        bottom += s_bucket << shift;
        span = min((1u << shift) - 1, top - bottom);
        __syncthreads();
    }
    const uint32_t prefix = bottom;  // keys above stay, and the first `want` that equal it

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
    // kept and equal ones before this warp's run: lane i adds up the warps to i
    uint32_t n_above = lane < kWarps ? s_above[lane] : 0u, n_equal = lane < kWarps ? s_equal[lane] : 0u;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, n_above, d), y = __shfl_up_sync(0xffffffffu, n_equal, d);
        if (lane >= d) n_above += x, n_equal += y;
    }
    uint32_t stay = __shfl_sync(0xffffffffu, n_above, (warp + 31) & 31), seen = __shfl_sync(0xffffffffu, n_equal, (warp + 31) & 31);
    if (warp == 0) stay = seen = 0;
    stay += min(seen, want);  // the first `want` equal ones stay
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
constexpr int64_t kSmallKeys = 8 * 1024;

}  // namespace

cudaError_t launch_evict_select(const float *w, int64_t w_sb, int64_t w_sh, const int32_t *lens, int64_t seqs, int heads,
                                int64_t max_len, int64_t budget, int64_t recent, int64_t sinks, int32_t *kept,
                                int32_t *new_lens, int *dev_err, cudaStream_t s)
{
    SelectArgs a{w, w_sb, w_sh, lens, heads, static_cast<int32_t>(max_len), static_cast<int32_t>(budget),
                 static_cast<int32_t>(recent), static_cast<int32_t>(sinks), kept, new_lens, dev_err};
    const dim3 grid(static_cast<unsigned>(seqs * heads));
    const int bytes = max_len <= kHeldKeys ? static_cast<int>(max_len) * 4 : 0;
    // More CTAs than SMs, of keys that leave room for several: CTAs of 256 threads,
    // up to six of which share an SM (64 x 32 heads of 4096 tokens: 40.8 us, 94.8
    // with 1024 threads; 32 x 8 of 8192: 16.3, 18.3; of 16384: 28.4, 26.2).
    if (grid.x > static_cast<unsigned>(device_sms()) && max_len <= kSmallKeys) {
        const cudaError_t e = allow_shared<evict_select_kernel<true, 256>>(kSmallKeys * 4);
        if (e != cudaSuccess) return e;
        return launch_pdl(evict_select_kernel<true, 256>, grid, dim3(256), bytes, s, a);
    }
    if (max_len <= kHeldKeys) {
        const cudaError_t e = allow_shared<evict_select_kernel<true, 1024>>(kHeldKeys * 4);
        if (e != cudaSuccess) return e;
        return launch_pdl(evict_select_kernel<true, 1024>, grid, dim3(1024), bytes, s, a);
    }
    return launch_pdl(evict_select_kernel<false, 1024>, grid, dim3(1024), 0, s, a);
}

}  // namespace quartz
