// Attention of one new token over a paged cache, for sm_103a: the kernel for
// 16-bit pages, the join of the splits, the sums of attention weights and the
// plan (paged_attention.cuh has the scheme; paged_attention_lzs.cu the kernel
// for encoded pages).
#include <atomic>

#include "paged_attention.cuh"

namespace quartz {
namespace {

// Query rows of the CTA's heads, 16 bits, rows of D + 8: the 16-byte reads of
// the eight heads' lanes then fall into different banks.
template <int D, int NT, bool BF, int MINB>
__global__ void __launch_bounds__(kPagedThreads, MINB) paged_attn_kernel(PagedArgs a)
{
    griddep_wait();
    constexpr int TILE = 8 * NT, KC = D / 32, VC = D / 64;
    constexpr bool kQRegs = D <= 128;  // wider heads read the query from shared memory again for each tile
    constexpr float kUp = BF ? 0.f : 13.f, kSlack = BF ? 8.f : 2.f;  // 2^(up + slack) fits fp16
    __shared__ __align__(16) uint16_t s_q[kPagedHeads][D + 8];
    __shared__ PagedJoin s_join;
    __shared__ __align__(16) uint8_t s_o[kPagedWarps][kPagedJoinBytes<D>];

    const int head_block = blockIdx.x % a.head_blocks, split = blockIdx.x / a.head_blocks;
    const int kv_head = blockIdx.y, b = blockIdx.z, head0 = head_block * kPagedHeads;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = lane >> 2, q = lane & 3;
    const PagedRange range = paged_range(a.lens, b, a.max_len, a.window, a.dev_err);
    const int begin = split * a.chunk;
    if (a.part_o && begin >= range.count()) return;
    const int end = range.base + min(begin + a.chunk, range.count());  // first token behind the split

    for (int e = threadIdx.x; e < kPagedHeads * (D / 8); e += kPagedThreads) {
        const int h = e / (D / 8), d = (e - h * (D / 8)) * 8;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (head0 + h < a.group)
            v = *reinterpret_cast<const uint4 *>(a.q + b * a.q_sb + (static_cast<int64_t>(kv_head) * a.group + head0 + h) * a.q_sh + d);
        *reinterpret_cast<uint4 *>(&s_q[h][d]) = v;
    }
    __syncthreads();
    uint4 qf[kQRegs ? KC : 1];
    if (kQRegs)
#pragma unroll
        for (int c = 0; c < KC; ++c) qf[c] = *reinterpret_cast<const uint4 *>(&s_q[n][(c * 4 + q) * 8]);

    const int32_t *table = a.table + b * a.table_stride;
    const int mask = (1 << a.page_shift) - 1;
    const uint16_t *kbase = reinterpret_cast<const uint16_t *>(a.k.data) + kv_head * a.k.stride_head + q * 8;
    const uint16_t *vbase = reinterpret_cast<const uint16_t *>(a.v.data) + kv_head * a.v.stride_head + n * 8;
    bool bad = false;
    // page of token base + (lane mod TILE); past the end: the last token's
    auto page_of = [&](int base) {
        const int t = min(base + (lane & (TILE - 1)), end - 1);
        const uint32_t page = static_cast<uint32_t>(table[t >> a.page_shift]);
        bad |= page >= a.num_pages;
        return page < a.num_pages ? page : 0u;
    };
    auto row_of = [&](const uint16_t *p, const PagedSide &s, uint32_t pages, int base, int i) {
        const uint32_t page = __shfl_sync(0xffffffffu, pages, i);
        const uint32_t slot = static_cast<uint32_t>(min(base + i, end - 1)) & mask;
        return p + (static_cast<uint64_t>(page) * s.stride_page + static_cast<uint64_t>(slot) * s.stride_slot);
    };
    uint4 kf[NT][KC];
    auto load_k = [&](uint32_t pages, int base) {
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const uint16_t *p = row_of(kbase, a.k, pages, base, (n >> 1) * 2 * NT + 2 * i + (n & 1));
#pragma unroll
            for (int c = 0; c < KC; ++c) kf[i][c] = __ldg(reinterpret_cast<const uint4 *>(p + c * 32));
        }
    };

    PagedState<D> st;
    st.init();
    int base = range.base + begin + warp * TILE;
    uint32_t pages = 0, next_pages = 0;
    if (base < end) {
        pages = page_of(base);
        load_k(pages, base);
        if (base + kPagedWarps * TILE < end) next_pages = page_of(base + kPagedWarps * TILE);
    }
    float *score_row = a.scores && head0 + n < a.group
                           ? a.scores + ((static_cast<int64_t>(b) * a.kv_heads + kv_head) * a.group + head0 + n) * a.score_stride
                           : nullptr;
    while (base < end) {
        uint4 vf[2 * NT][VC];
#pragma unroll
        for (int j = 0; j < 2 * NT; ++j) {
            const uint16_t *p = row_of(vbase, a.v, pages, base, 2 * NT * q + j);
#pragma unroll
            for (int c = 0; c < VC; ++c) vf[j][c] = __ldg(reinterpret_cast<const uint4 *>(p + c * 64));
        }
        float s[NT][4];
#pragma unroll
        for (int i = 0; i < NT; ++i) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.f;
#pragma unroll
        for (int c = 0; c < KC; ++c) {
            const uint4 w = kQRegs ? qf[kQRegs ? c : 0] : *reinterpret_cast<const uint4 *>(&s_q[n][(c * 4 + q) * 8]);
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                mma16<BF>(s[i], w.x, w.x, w.y, w.y, kf[i][c].x, kf[i][c].y);
                mma16<BF>(s[i], w.z, w.z, w.w, w.w, kf[i][c].z, kf[i][c].w);
            }
        }
        const int next = base + kPagedWarps * TILE;
        if (next < end) {
            load_k(next_pages, next);
            pages = next_pages;
            if (next + kPagedWarps * TILE < end) next_pages = page_of(next + kPagedWarps * TILE);
        }
        float sc[NT][2];
#pragma unroll
        for (int i = 0; i < NT; ++i) sc[i][0] = s[i][0] * a.scale_log2, sc[i][1] = s[i][1] * a.scale_log2;
        if (base + TILE > end || base < range.first) {
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int t = base + 2 * NT * q + 2 * i + x;
                    if (t >= end || t < range.first) sc[i][x] = -INFINITY;
                }
        }
        if (score_row) {
            float *to = score_row + (base - range.base) + 2 * NT * q;
#pragma unroll
            for (int i = 0; i < NT; ++i) *reinterpret_cast<float2 *>(to + 2 * i) = make_float2(sc[i][0], sc[i][1]);
        }
        st.template weigh<NT>(sc, kUp, kSlack);
        uint32_t hi[NT], lo[NT];
#pragma unroll
        for (int i = 0; i < NT; ++i) split_pair<BF>(sc[i][0], sc[i][1], hi[i], lo[i]);
#pragma unroll
        for (int c = 0; c < VC; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                auto word = [&](int j) { return reinterpret_cast<const uint32_t *>(&vf[j][c])[e]; };
                float(&o0)[4] = st.o[c * 8 + 2 * e], (&o1)[4] = st.o[c * 8 + 2 * e + 1];
                if (NT == 2) {
                    mma16<BF>(o0, hi[0], lo[0], hi[NT - 1], lo[NT - 1], permute(word(0), word(1), 0x5410),
                              permute(word(2 * NT - 2), word(2 * NT - 1), 0x5410));
                    mma16<BF>(o1, hi[0], lo[0], hi[NT - 1], lo[NT - 1], permute(word(0), word(1), 0x7632),
                              permute(word(2 * NT - 2), word(2 * NT - 1), 0x7632));
                } else {
                    mma8<BF>(o0, hi[0], lo[0], permute(word(0), word(1), 0x5410));
                    mma8<BF>(o1, hi[0], lo[0], permute(word(0), word(1), 0x7632));
                }
            }
        base = next;
    }
    if (bad) atomicExch(a.dev_err, QUARTZ_DEV_INDEX);
    st.l += __shfl_xor_sync(0xffffffffu, st.l, 1);
    st.l += __shfl_xor_sync(0xffffffffu, st.l, 2);
    if (q == 0) s_join.m[warp][n] = st.m, s_join.l[warp][n] = st.l;
    paged_finish<D>(s_join, s_o[0], sizeof(s_o[0]), st, a, b, kv_head, head0, split, kUp);
}

template <int D, bool BF>
struct Kernel16 {
    static constexpr int NT = D <= 128 ? 2 : 1, MINB = D <= 128 ? 3 : 2;
    static int occupancy()
    {
        static std::atomic<int> cache{0};
        int occ = cache.load(std::memory_order_relaxed);
        if (occ == 0) {
            int k = 0;
            if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&k, paged_attn_kernel<D, NT, BF, MINB>, kPagedThreads, 0) !=
                cudaSuccess)
                return 1;
            occ = k > 0 ? k : 1;
            cache.store(occ, std::memory_order_relaxed);
        }
        return occ;
    }
    static cudaError_t launch(const PagedArgs &a, dim3 grid, cudaStream_t s)
    {
        return launch_pdl(paged_attn_kernel<D, NT, BF, MINB>, grid, dim3(kPagedThreads), 0, s, a);
    }
};

// ---------------------------------------------------------------------------
// Join of the splits, and the sums of weights
// ---------------------------------------------------------------------------
constexpr int kMaxSplits = 1024;

// One CTA per (sequence, query head), a thread per 4 elements and group of
// splits; the splits that hold tokens follow from the length.
template <int D>
__global__ void __launch_bounds__(256) paged_join_kernel(PagedArgs a)
{
    griddep_wait();
    constexpr int kLanes = D / 4, kGroups = 256 / kLanes;
    __shared__ float s_f[kMaxSplits];
    __shared__ float4 s_o[kGroups][kLanes];
    __shared__ float s_red[8], s_inv;
    const int64_t row = blockIdx.x;
    const int b = static_cast<int>(row / (a.kv_heads * a.group));
    const PagedRange range = paged_range(a.lens, b, a.max_len, a.window, a.dev_err);
    const int splits = (range.count() + a.chunk - 1) / a.chunk;
    const float *ml = a.part_ml + 2 * row * a.n_split;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    float m = -INFINITY;
    for (int i = tid; i < splits; i += 256) m = fmaxf(m, ml[2 * i]);
#pragma unroll
    for (int d = 16; d; d /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    if (lane == 0) s_red[warp] = m;
    __syncthreads();
    m = s_red[0];
#pragma unroll
    for (int w = 1; w < 8; ++w) m = fmaxf(m, s_red[w]);
    __syncthreads();
    float sum = 0.f;
    for (int i = tid; i < splits; i += 256) {
        const float f = m == -INFINITY ? 0.f : ex2(ml[2 * i] - m);
        s_f[i] = f;
        sum += f * ml[2 * i + 1];
    }
#pragma unroll
    for (int d = 16; d; d /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if (lane == 0) s_red[warp] = sum;
    __syncthreads();
    if (tid == 0) {
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) t += s_red[w];
        s_inv = t > 0.f ? 1.f / t : 0.f;
        if (a.lse) a.lse[row] = m + log2f(t);
    }
    const int g = tid / kLanes, c = tid - g * kLanes;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (g < kGroups) {
        const float4 *o = reinterpret_cast<const float4 *>(a.part_o + row * a.n_split * D) + c;
#pragma unroll 4
        for (int i = g; i < splits; i += kGroups) {
            const float4 u = o[static_cast<int64_t>(i) * kLanes];
            const float f = s_f[i];
            v.x += f * u.x, v.y += f * u.y, v.z += f * u.z, v.w += f * u.w;
        }
        s_o[g][c] = v;
    }
    __syncthreads();
    if (g == 0) {
#pragma unroll
        for (int k = 1; k < kGroups; ++k) {
            const float4 u = s_o[k][c];
            v.x += u.x, v.y += u.y, v.z += u.z, v.w += u.w;
        }
        const float r = s_inv;
        paged_store4(a.o, a.o_type, row * D + c * 4, make_float4(v.x * r, v.y * r, v.z * r, v.w * r));
    }
}

// weights[b, h, t] += sum over the head's query heads of 2^(score - lse), in
// head order: four tokens per thread.
__global__ void __launch_bounds__(256) paged_weights_kernel(PagedArgs a, float *weights, int64_t w_sb, int64_t w_sh)
{
    griddep_wait();
    const int h = blockIdx.y, b = blockIdx.z;
    const PagedRange range = paged_range(a.lens, b, a.max_len, a.window, a.dev_err);
    const int t = (blockIdx.x * 256 + threadIdx.x) * 4;
    if (t >= range.count()) return;
    const int64_t row0 = (static_cast<int64_t>(b) * a.kv_heads + h) * a.group;
    float p[4] = {0.f, 0.f, 0.f, 0.f};
    for (int g = 0; g < a.group; ++g) {
        const float4 s = *reinterpret_cast<const float4 *>(a.scores + (row0 + g) * a.score_stride + t);
        const float lse = a.lse[row0 + g];
        p[0] += ex2(s.x - lse), p[1] += ex2(s.y - lse), p[2] += ex2(s.z - lse), p[3] += ex2(s.w - lse);
    }
    float *w = weights + b * w_sb + h * w_sh + range.base + t;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (t + i < range.count() && range.base + t + i >= range.first) w[i] += p[i];
}

int log2_of(int v)
{
    int n = 0;
    while ((1 << n) < v) ++n;
    return n;
}

// Splits per sequence and tokens per split.  A split is a multiple of one tile
// of each of the CTA's warps.  Long sequences are cut to pieces that keep the
// SMs evenly loaded when lengths differ; short ones only as far as SMs are
// free.
struct PagedPlan {
    int n_split, chunk;
    int64_t tokens, score_stride;
};

PagedPlan paged_plan(const quartz_paged_cache_t *c, int64_t seqs, int q_heads, int64_t max_len, int64_t window)
{
    PagedPlan p;
    // a window's first tile may hold 15 tokens before it
    p.tokens = window > 0 && window + 15 < max_len ? window + 15 : max_len;
    const int group = q_heads / c->heads;
    const int64_t ctas = seqs * c->heads * ((group + kPagedHeads - 1) / kPagedHeads);
    const int occ = c->type == QUARTZ_PAGES_ENCODED ? paged_kernel_occupancy_encoded(c->dim, c->k.enc.p.group_s)
                                                    : paged_kernel_occupancy_16bit(c->type, c->dim);
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
        sms <= 0)
        sms = 152;
    const int64_t slots = static_cast<int64_t>(sms) * occ;
    int64_t n = (4 * slots + ctas - 1) / ctas;
    const int64_t most = (p.tokens + 255) / 256;
    if (n > most) n = most;
    if (n * ctas < slots) {
        const int64_t fill = (slots + ctas - 1) / ctas, tiles = (p.tokens + 63) / 64;
        n = fill < tiles ? fill : tiles;
    }
    if (n > kMaxSplits) n = kMaxSplits;
    if (n < 1) n = 1;
    const int64_t chunk = ((p.tokens + n - 1) / n + 63) / 64 * 64;
    p.chunk = static_cast<int>(chunk);
    p.n_split = static_cast<int>((p.tokens + chunk - 1) / chunk);
    if (p.n_split < 1) p.n_split = 1;
    p.score_stride = (p.tokens + 63) / 64 * 64;
    return p;
}

size_t up256(size_t n) { return (n + 255) & ~size_t(255); }

}  // namespace

int paged_kernel_occupancy_16bit(int type, int dim)
{
    const bool bf = type == QUARTZ_PAGES_BF16;
    switch (dim) {
        case 64: return bf ? Kernel16<64, true>::occupancy() : Kernel16<64, false>::occupancy();
        case 128: return bf ? Kernel16<128, true>::occupancy() : Kernel16<128, false>::occupancy();
        case 192: return bf ? Kernel16<192, true>::occupancy() : Kernel16<192, false>::occupancy();
        default: return bf ? Kernel16<256, true>::occupancy() : Kernel16<256, false>::occupancy();
    }
}

cudaError_t launch_paged_16bit(int type, int dim, const PagedArgs &a, dim3 grid, cudaStream_t s)
{
    const bool bf = type == QUARTZ_PAGES_BF16;
    switch (dim) {
        case 64: return bf ? Kernel16<64, true>::launch(a, grid, s) : Kernel16<64, false>::launch(a, grid, s);
        case 128: return bf ? Kernel16<128, true>::launch(a, grid, s) : Kernel16<128, false>::launch(a, grid, s);
        case 192: return bf ? Kernel16<192, true>::launch(a, grid, s) : Kernel16<192, false>::launch(a, grid, s);
        default: return bf ? Kernel16<256, true>::launch(a, grid, s) : Kernel16<256, false>::launch(a, grid, s);
    }
}

size_t paged_attention_workspace_bytes(const quartz_paged_cache_t *c, int64_t seqs, int q_heads, int64_t max_len,
                                       int64_t window, bool with_weights)
{
    const PagedPlan p = paged_plan(c, seqs, q_heads, max_len, window);
    const size_t rows = static_cast<size_t>(seqs) * q_heads;
    size_t n = 256;
    if (p.n_split > 1) n += up256(rows * p.n_split * c->dim * 4) + up256(rows * p.n_split * 8);
    if (with_weights) n += up256(rows * 4) + up256(rows * static_cast<size_t>(p.score_stride) * 4);
    return n;
}

cudaError_t launch_paged_attention(const quartz_paged_cache_t *c, const PagedAttnCall &call, cudaStream_t s)
{
    const PagedPlan p = paged_plan(c, call.seqs, call.q_heads, call.max_len, call.window);
    PagedArgs a{};
    a.q = static_cast<const uint16_t *>(call.q);
    a.q_sb = call.q_sb, a.q_sh = call.q_sh;
    a.table = call.table, a.table_stride = call.table_stride;
    a.lens = call.lens;
    const quartz_pages_t *pages[2] = {&c->k, &c->v};
    PagedSide *side[2] = {&a.k, &a.v};
    for (int i = 0; i < 2; ++i) {
        side[i]->data = static_cast<const uint8_t *>(pages[i]->data);
        side[i]->stride_page = static_cast<uint32_t>(pages[i]->stride_page);
        side[i]->stride_slot = static_cast<uint32_t>(pages[i]->stride_slot);
        side[i]->stride_head = pages[i]->stride_head;
        side[i]->codes = pages[i]->enc.codes;
        side[i]->flags = pages[i]->enc.flags;
        side[i]->scales = reinterpret_cast<const __half *>(pages[i]->enc.scales);
    }
    a.num_pages = static_cast<uint32_t>(c->num_pages);
    a.page_shift = log2_of(c->page_size);
    a.kv_heads = c->heads;
    a.group = call.q_heads / c->heads;
    a.head_blocks = (a.group + kPagedHeads - 1) / kPagedHeads;
    a.max_len = static_cast<int>(call.max_len);
    a.window = static_cast<int>(call.window < call.max_len ? call.window : 0);
    a.n_split = p.n_split, a.chunk = p.chunk;
    a.scale_log2 = call.scale * kPagedLog2e;
    a.o = call.o, a.o_type = call.o_type;
    a.dev_err = call.dev_err;
    uint8_t *ws = static_cast<uint8_t *>(call.workspace);
    const size_t rows = static_cast<size_t>(call.seqs) * call.q_heads;
    if (p.n_split > 1) {
        a.part_o = reinterpret_cast<float *>(ws);
        ws += up256(rows * p.n_split * c->dim * 4);
        a.part_ml = reinterpret_cast<float *>(ws);
        ws += up256(rows * p.n_split * 8);
    }
    if (call.weights) {
        a.lse = reinterpret_cast<float *>(ws);
        ws += up256(rows * 4);
        a.scores = reinterpret_cast<float *>(ws);
        a.score_stride = p.score_stride;
    }
    const dim3 grid(static_cast<unsigned>(p.n_split * a.head_blocks), static_cast<unsigned>(c->heads),
                    static_cast<unsigned>(call.seqs));
    cudaError_t e = c->type == QUARTZ_PAGES_ENCODED ? launch_paged_encoded(c->dim, c->k.enc.p.group_s, a, grid, s)
                                                    : launch_paged_16bit(c->type, c->dim, a, grid, s);
    if (e == cudaSuccess && p.n_split > 1) {
        const dim3 join(static_cast<unsigned>(rows));
        switch (c->dim) {
            case 64: e = launch_pdl(paged_join_kernel<64>, join, dim3(256), 0, s, a); break;
            case 128: e = launch_pdl(paged_join_kernel<128>, join, dim3(256), 0, s, a); break;
            case 192: e = launch_pdl(paged_join_kernel<192>, join, dim3(256), 0, s, a); break;
            default: e = launch_pdl(paged_join_kernel<256>, join, dim3(256), 0, s, a); break;
        }
    }
    if (e == cudaSuccess && call.weights) {
        const dim3 g(static_cast<unsigned>((p.tokens + 1023) / 1024), static_cast<unsigned>(c->heads),
                     static_cast<unsigned>(call.seqs));
        e = launch_pdl(paged_weights_kernel, g, dim3(256), 0, s, a, call.weights, call.w_sb, call.w_sh);
    }
    return e;
}

}  // namespace quartz
