// Attention of one new token over a paged cache, for sm_103a: the kernel for
// 16-bit pages, the join of the splits, the sums of attention weights and the
// plan (paged_attention.cuh has the scheme; paged_attention_lzs.cu the kernel
// for encoded pages).
#include <atomic>

#include "paged_attention.cuh"

namespace quartz {
namespace {

// A warp's ring of tiles: 16 rows of keys, then of values, D elements each, as
// 16-byte chunks.  Chunk c of row t sits at c ^ (t % 8) (in its group of 8), so
// that the matrix loads, which read one chunk of 8 rows, hit all banks.
template <int D>
struct Tile16 {
    static constexpr int kChunks = D / 8, kRow = D * 2, kSide = 16 * kRow, kBytes = 2 * kSide;
    static constexpr int kPerLane = 16 * kChunks / 32;  // chunks a lane copies, each side
    // Stages and CTAs per SM so that some 128 KB per SM are on their way.
    static constexpr int kStages = D == 192 ? 4 : 3, kCtas = D == 64 ? 4 : D == 128 ? 2 : 1;
    __device__ static constexpr int at(int t, int c) { return t * kRow + (((c & ~7) | ((c ^ t) & 7)) << 4); }
};

__device__ __forceinline__ void ldmatrix4(uint32_t a, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(a));
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t a, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(a));
}

template <int D, bool BF, bool SHARE>
__global__ void __launch_bounds__(kPagedThreads, Tile16<D>::kCtas) paged_attn_kernel(PagedArgs a)
{
    griddep_wait();
    using Tile = Tile16<D>;
    constexpr int kStages = Tile::kStages, kWarpBytes = kStages * Tile::kBytes;
    constexpr bool kQRegs = D <= 128;  // wider heads read the query from shared memory again for each tile
    constexpr float kUp = BF ? 0.f : 13.f, kSlack = BF ? 8.f : 2.f;  // 2^(up + slack) fits fp16
    static_assert(kWarpBytes >= kPagedJoinBytes<D>, "the join uses the ring");
    extern __shared__ __align__(16) uint8_t s_ring[];
    __shared__ __align__(16) uint16_t s_q[kPagedHeads][D + 8];
    __shared__ PagedJoin s_join;

    const int head_block = blockIdx.x / a.n_split, split = blockIdx.x - head_block * a.n_split;
    const int kv_head = blockIdx.y, head0 = head_block * kPagedHeads;
    int b, begin, chunk;
    if (!paged_place<SHARE>(a, split, b, begin, chunk)) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = lane >> 2, q = lane & 3;
    const PagedRange range = paged_range(a.lens, b, a.max_len, a.window, a.dev_err);
    if (a.part_o && begin >= range.count()) return;
    const int end = range.base + min(begin + chunk, range.count());  // first token behind the split
    const int base0 = range.base + begin + warp * 16;
    const int tiles = base0 < end ? (end - base0 + kPagedWarps * 16 - 1) / (kPagedWarps * 16) : 0;
    const uint32_t ring = smem_u32(s_ring) + warp * kWarpBytes;

    // --- copies of a tile: a lane takes chunks lane + 32 k.  Tokens that are not
    // seen repeat the nearest that is: nothing of theirs, which may be infinite
    // or NaN, meets a weight of 0.
    const int32_t *table = a.table + b * a.table_stride;
    const uint32_t page_mask = (1u << a.page_shift) - 1;
    const uint16_t *kbase = reinterpret_cast<const uint16_t *>(a.k.data) + kv_head * a.k.stride_head;
    const uint16_t *vbase = reinterpret_cast<const uint16_t *>(a.v.data) + kv_head * a.v.stride_head;
    bool bad = false;
    auto seen = [&](int t) { return max(min(t, end - 1), range.first); };
    // page of token base + lane % 16
    auto pages_of = [&](int base) {
        const uint32_t page = static_cast<uint32_t>(__ldg(table + (seen(base + (lane & 15)) >> a.page_shift)));
        bad |= page >= a.num_pages;
        return page < a.num_pages ? page : 0u;
    };
    auto fetch = [&](int base, uint32_t pages, int stage) {
        const uint32_t to = ring + stage * Tile::kBytes;
#pragma unroll
        for (int k = 0; k < Tile::kPerLane; ++k) {
            const int i = lane + 32 * k, t = i / Tile::kChunks, c = i % Tile::kChunks;
            const uint64_t page = __shfl_sync(0xffffffffu, pages, t);
            const uint64_t slot = static_cast<uint32_t>(seen(base + t)) & page_mask;
            cp_async16(to + Tile::at(t, c), kbase + (page * a.k.stride_page + slot * a.k.stride_slot) + c * 8);
            cp_async16(to + Tile::kSide + Tile::at(t, c), vbase + (page * a.v.stride_page + slot * a.v.stride_slot) + c * 8);
        }
    };
    uint32_t next_pages = 0;  // of the next tile to fetch
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) {
        if (s < tiles) fetch(base0 + s * kPagedWarps * 16, pages_of(base0 + s * kPagedWarps * 16), s);
        cp_async_commit();
    }
    if (kStages - 1 < tiles) next_pages = pages_of(base0 + (kStages - 1) * kPagedWarps * 16);

    // --- the query: per 16 elements, lane q of a head holds 2 q, 2 q + 1 and 2 q
    // + 8, 2 q + 9, which are stored side by side
    for (int e = threadIdx.x; e < kPagedHeads * (D / 16); e += kPagedThreads) {
        const int h = e / (D / 16), d = (e - h * (D / 16)) * 16;
        uint4 v = make_uint4(0, 0, 0, 0), w = v;
        if (head0 + h < a.group) {
            const uint4 *p = reinterpret_cast<const uint4 *>(a.q + b * a.q_sb + (static_cast<int64_t>(kv_head) * a.group + head0 + h) * a.q_sh + d);
            v = p[0], w = p[1];
        }
        *reinterpret_cast<uint4 *>(&s_q[h][d]) = make_uint4(v.x, w.x, v.y, w.y);
        *reinterpret_cast<uint4 *>(&s_q[h][d + 8]) = make_uint4(v.z, w.z, v.w, w.w);
    }
    __syncthreads();
    auto query = [&](int c) { return *reinterpret_cast<const uint2 *>(&s_q[n][c * 16 + q * 4]); };
    uint2 qf[kQRegs ? D / 16 : 1];
    if (kQRegs)
#pragma unroll
        for (int c = 0; c < D / 16; ++c) qf[c] = query(c);

    // matrix loads: lane l gives the address of row l % 8 of block l / 8; keys:
    // blocks (tokens 0-7, 8-15) x (first, second 8 of 16 dimensions), values:
    // the same blocks, transposed
    const int ld_row = lane & 15, ld_col = lane >> 4;
    PagedState<D> st;
    st.init();
    const int64_t score_row = ((static_cast<int64_t>(b) * a.kv_heads + kv_head) * a.group + head0 + 2 * q) * a.score_stride;
    int stage = 0;
    for (int it = 0; it < tiles; ++it) {
        const int base = base0 + it * kPagedWarps * 16;
        cp_async_wait<kStages - 2>();
        __syncwarp();
        {
            const int ahead = it + kStages - 1;
            if (ahead < tiles) {
                fetch(base0 + ahead * kPagedWarps * 16, next_pages, stage == 0 ? kStages - 1 : stage - 1);
                if (ahead + 1 < tiles) next_pages = pages_of(base0 + (ahead + 1) * kPagedWarps * 16);
            }
            cp_async_commit();
        }
        const uint32_t tile = ring + stage * Tile::kBytes;
        stage = stage == kStages - 1 ? 0 : stage + 1;

        float s[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};  // two chains
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
            uint32_t k[4];
            ldmatrix4(tile + Tile::at(ld_row, 2 * c + ld_col), k);
            const uint2 w = kQRegs ? qf[kQRegs ? c : 0] : query(c);
            mma16<BF>(s[c & 1], k[0], k[1], k[2], k[3], w.x, w.y);
        }
        float sc[2][2];  // tokens n and n + 8, heads 2 q and 2 q + 1
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int x = 0; x < 2; ++x) sc[i][x] = (s[0][2 * i + x] + s[1][2 * i + x]) * a.scale_log2;
        if (base + 16 > end || base < range.first) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (base + n + 8 * i >= end || base + n + 8 * i < range.first) sc[i][0] = sc[i][1] = -INFINITY;
        }
        if (a.scores) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int x = 0; x < 2; ++x)
                    if (head0 + 2 * q + x < a.group)
                        a.scores[score_row + x * a.score_stride + (base - range.base) + n + 8 * i] = sc[i][x];
        }
        float p[2][2];
        st.weigh(sc, p, kUp, kSlack);
        uint32_t hi[2], lo[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            split_pair<BF>(p[i][0], p[i][1], hi[i], lo[i], true);
            hi[i] = transposed(hi[i]);
            lo[i] = transposed(lo[i]);
        }
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
            uint32_t v[4];
            ldmatrix4_trans(tile + Tile::kSide + Tile::at(ld_row, 2 * c + ld_col), v);
            mma16<BF>(st.o[2 * c], hi[0], lo[0], hi[1], lo[1], v[0], v[1]);
            mma16<BF>(st.o[2 * c + 1], hi[0], lo[0], hi[1], lo[1], v[2], v[3]);
        }
        if (BF && a.o_type == QUARTZ_OUT_F32) {
            const uint32_t r0 = transposed(bf16_pair(p[0][0], p[0][1])), r1 = transposed(bf16_pair(p[1][0], p[1][1]));
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                uint32_t v[4];
                ldmatrix4_trans(tile + Tile::kSide + Tile::at(ld_row, 2 * c + ld_col), v);
                mma16<BF>(st.o[2 * c], r0, 0u, r1, 0u, v[0], v[1]);
                mma16<BF>(st.o[2 * c + 1], r0, 0u, r1, 0u, v[2], v[3]);
            }
        }
    }
    cp_async_wait<0>();
    __syncwarp();
    if (bad) atomicOr(a.dev_err, QUARTZ_DEV_INDEX);
    paged_finish<D, false, SHARE>(s_join, s_ring, kWarpBytes, st, a, b, kv_head, head0, split, kUp);
}

template <int D, bool BF>
struct Kernel16 {
    static constexpr int kSmem = kPagedWarps * Tile16<D>::kStages * Tile16<D>::kBytes;
    static int occupancy()
    {
        static std::atomic<int> cache{0};
        int occ = cache.load(std::memory_order_relaxed);
        if (occ == 0) {
            int k = 0;
            if (allow_shared<paged_attn_kernel<D, BF, false>>(kSmem) != cudaSuccess ||
                cudaOccupancyMaxActiveBlocksPerMultiprocessor(&k, paged_attn_kernel<D, BF, false>, kPagedThreads, kSmem) != cudaSuccess)
                return 1;
            occ = k > 0 ? k : 1;
            cache.store(occ, std::memory_order_relaxed);
        }
        return occ;
    }
    static cudaError_t launch(const PagedArgs &a, dim3 grid, cudaStream_t s)
    {
        return a.share ? launch_as<true>(a, grid, s) : launch_as<false>(a, grid, s);
    }
    template <bool SHARE>
    static cudaError_t launch_as(const PagedArgs &a, dim3 grid, cudaStream_t s)
    {
        const cudaError_t e = allow_shared<paged_attn_kernel<D, BF, SHARE>>(kSmem);
        if (e != cudaSuccess) return e;
        if (a.cluster) return launch_pdl_cluster(paged_attn_kernel<D, BF, SHARE>, a.n_split, grid, dim3(kPagedThreads), kSmem, s, a);
        return launch_pdl(paged_attn_kernel<D, BF, SHARE>, grid, dim3(kPagedThreads), kSmem, s, a);
    }
};

// ---------------------------------------------------------------------------
// Join of the splits, and the sums of weights
// ---------------------------------------------------------------------------
constexpr int kMaxSplits = 1024;
constexpr int kJoinThreads = 256;
constexpr int kJoinHeads = 64;  // query heads whose sums are held at a time

// CTA (x, key / value head, sequence).  Join of the splits: head x of the key
// head's query heads (and x + gridDim.x, ...), a thread per 4 elements and
// group of splits.  Sums of weights: 1024 tokens from 1024 x on, four per
// thread, weights[b, h, t] += sum over the query heads of 2^(score - m) / l, in
// head order; every CTA finds the heads' m and l from the splits itself, which
// is less than another launch.
template <int D>
__global__ void __launch_bounds__(kJoinThreads) paged_join_kernel(PagedArgs a, float *weights, int64_t w_sb, int64_t w_sh)
{
    griddep_wait();
    constexpr int kLanes = D / 4, kGroups = kJoinThreads / kLanes;
    __shared__ float s_f[kMaxSplits];
    __shared__ float4 s_o[kGroups][kLanes];
    __shared__ float s_red[8], s_inv;
    __shared__ float2 s_ml[kJoinHeads];  // m and log2 l: apart, since together they would lose l where m is large
    const int b = blockIdx.z;
    const PagedRange range = paged_range(a.lens, b, a.max_len, a.window, a.dev_err);
    const int64_t row0 = (static_cast<int64_t>(b) * a.kv_heads + blockIdx.y) * a.group;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int splits = (range.count() + a.chunk - 1) / a.chunk;  // that hold tokens
    int64_t part0 = row0 * a.n_split;                      // of the key head's first query head
    if (a.share) {
        const PagedShare s = paged_share(a);
        splits = __shfl_sync(0xffffffffu, s.count, b);
        part0 = static_cast<int64_t>(blockIdx.y) * a.group * a.n_split + __shfl_sync(0xffffffffu, s.first, b);
    }

    for (int head = blockIdx.x; a.part_o && head < a.group; head += gridDim.x) {
        const int64_t row = row0 + head;
        const int64_t part = part0 + static_cast<int64_t>(head) * a.n_split;
        const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml) + part;
        float m = kPagedLow;
        for (int i = tid; i < splits; i += kJoinThreads) m = fmaxf(m, ml[i].x);
#pragma unroll
        for (int d = 16; d; d /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
        if (lane == 0) s_red[warp] = m;
        __syncthreads();
        m = s_red[0];
#pragma unroll
        for (int w = 1; w < 8; ++w) m = fmaxf(m, s_red[w]);
        __syncthreads();
        float sum = 0.f;
        for (int i = tid; i < splits; i += kJoinThreads) {
            const float2 v = ml[i];
            const float f = ex2(v.x - m);
            s_f[i] = f;
            sum += f * v.y;
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
        }
        const int g = tid / kLanes, c = tid - g * kLanes;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (g < kGroups) {
            const float4 *o = reinterpret_cast<const float4 *>(a.part_o + part * D) + c;
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
        __syncthreads();  // shared memory serves the next head
    }
    if (!weights) return;

    float *w = weights + b * w_sb + blockIdx.y * w_sh + range.base;
    bool held = false;
    for (int t0 = blockIdx.x * 4 * kJoinThreads; t0 < range.count(); t0 += gridDim.x * 4 * kJoinThreads) {
        const int t = t0 + 4 * tid;
        float p[4] = {0.f, 0.f, 0.f, 0.f};
        for (int g0 = 0; g0 < a.group; g0 += kJoinHeads) {
            const int heads = min(kJoinHeads, a.group - g0);
            if (!held) {  // m and log2 l of each head, a warp each
                __syncthreads();
                for (int g = warp; g < heads; g += kJoinThreads / 32) {
                    const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml) + part0 + static_cast<int64_t>(g0 + g) * a.n_split;
                    float m = kPagedLow, sum = 0.f;
                    for (int i = lane; i < splits; i += 32) m = fmaxf(m, ml[i].x);
#pragma unroll
                    for (int d = 16; d; d /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
                    for (int i = lane; i < splits; i += 32) {
                        const float2 v = ml[i];
                        sum += ex2(v.x - m) * v.y;
                    }
#pragma unroll
                    for (int d = 16; d; d /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
                    if (lane == 0) s_ml[g] = make_float2(m, log2f(sum));
                }
                __syncthreads();
                held = a.group <= kJoinHeads;
            }
            if (t < range.count()) {
                const float *score = a.scores + (row0 + g0) * a.score_stride + t;
#pragma unroll 4
                for (int g = 0; g < heads; ++g) {
                    const float4 s = *reinterpret_cast<const float4 *>(score + g * a.score_stride);
                    const float m = s_ml[g].x, l = s_ml[g].y;
                    p[0] += ex2(s.x - m - l), p[1] += ex2(s.y - m - l), p[2] += ex2(s.z - m - l), p[3] += ex2(s.w - m - l);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (t + i < range.count() && range.base + t + i >= range.first) w[t + i] += p[i];
    }
}

// Splits per sequence and tokens per split (a multiple of one tile of each of
// the CTA's warps).  Where lengths differ, many CTAs are empty or short: four
// times as many as the SMs hold keep them loaded, of 256 tokens at least (a CTA
// costs some 5 us besides its tiles); where sequences and heads alone are twice
// what they hold, none is cut for that (128 x 8 heads of up to 1000 tokens, bf16:
// 47.6 us whole, 60.4 in two).  Long sequences are cut to 1024 tokens,
// up to 16 times what the SMs hold: 8 sequences of up to 65536 tokens, encoded,
// 100.9 us (2048 102.3, 512 110.0, 4096 122.9); 32 of up to 8192, bf16, 98.6
// (2048 100.6, 512 104.8, 256 113.8).  A few short ones are cut only as far as
// SMs are free, or, to few enough splits for a cluster, two thirds of them.
struct PagedPlan {
    int n_split, chunk;
    int share;
    bool cluster;
    int64_t tokens, score_stride;
};

PagedPlan paged_plan(const quartz_paged_cache_t *c, int64_t seqs, int q_heads, int64_t max_len, int64_t window,
                     bool with_weights)
{
    PagedPlan p;
    // a window's first tile may hold 15 tokens before it; a table without room
    // for any token is planned as for one
    p.tokens = window > 0 && window < max_len - 15 ? window + 15 : max_len;
    if (p.tokens < 1) p.tokens = 1;
    const int group = q_heads / c->heads;
    const int64_t ctas = (seqs > 0 ? seqs : 1) * c->heads * ((group + kPagedHeads - 1) / kPagedHeads);
    const int occ = c->type == QUARTZ_PAGES_ENCODED ? paged_kernel_occupancy_encoded(c->dim, c->k.enc.p.group_s)
                                                    : paged_kernel_occupancy_16bit(c->type, c->dim);
    const int64_t slots = static_cast<int64_t>(device_sms()) * occ;
    int64_t n = ctas < 2 * slots ? (4 * slots + ctas - 1) / ctas : 1;
    const int64_t most = (p.tokens + 255) / 256, by_length = (p.tokens + 1023) / 1024, full = 16 * slots / ctas;
    if (n < by_length && n < full) n = by_length < full ? by_length : full;
    if (n > most) n = most;
    if (n * ctas < slots) {
        const int64_t fill = (slots + ctas - 1) / ctas, tiles = (p.tokens + 63) / 64, loose = 2 * slots / (3 * ctas);
        n = fill < tiles ? fill : tiles;
        if (n <= kPagedCluster && loose >= 2 && n > loose) n = loose;
    }
    if (n > kMaxSplits) n = kMaxSplits;
    if (n < 1) n = 1;
    const int64_t chunk = ((p.tokens + n - 1) / n + 63) / 64 * 64;
    p.chunk = static_cast<int>(chunk);
    p.n_split = static_cast<int>((p.tokens + chunk - 1) / chunk);
    if (p.n_split < 1) p.n_split = 1;
    // At most 8 splits and two thirds of the SMs' places taken: a head's splits
    // are a cluster and join themselves, which saves the join's launch (40
    // heads, 777 tokens, encoded: 5.9 us against 6.7; 200 tokens, fp16: 4.6
    // against 5.7).  With the SMs nearly full, clusters wait for places next to
    // each other (777 tokens, fp16, 7 splits: 8.8 against 7.0).
    p.cluster = p.n_split > 1 && p.n_split <= kPagedCluster && 3 * p.n_split * ctas <= 2 * slots && !with_weights;
    // Few sequences (what rounding to whole places loses is an eighth at most):
    // one wave, shared out by the lengths.  Against the splits above, 8 heads,
    // encoded: one of 131072 tokens 48.1 us (60.3), 2 and 4 of 32768 each 27.5 and
    // 50.0 (34.0, 54.6), of up to 32768 19.3 and 32.0 (23.9, 36.5); 8 of up to
    // 65536, a wave of 7 places each, 98.1 (96.4).  bf16: one of 131072 89.2 (93.4).
    const int64_t wave = slots / (ctas / (seqs > 0 ? seqs : 1)), units = (p.tokens + kShareUnit - 1) / kShareUnit;
    p.share = 0;
    if (!p.cluster && p.n_split > 1 && seqs <= kShareSeqs && wave >= 8 * seqs) {
        p.share = static_cast<int>(wave < kMaxSplits ? wave : kMaxSplits);
        p.n_split = static_cast<int>(p.share < seqs * units ? p.share : seqs * units);
    }
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
    const PagedPlan p = paged_plan(c, seqs, q_heads, max_len, window, with_weights);
    const size_t rows = static_cast<size_t>(seqs) * q_heads;
    size_t n = 256;
    const bool join = p.n_split > 1 && !p.cluster;
    const size_t parts = (p.share ? q_heads : rows) * p.n_split;
    if (join) n += up256(parts * c->dim * 4);
    if (join || with_weights) n += up256(parts * 8);
    if (with_weights) n += up256(rows * static_cast<size_t>(p.score_stride) * 4);
    return n;
}

cudaError_t launch_paged_attention(const quartz_paged_cache_t *c, const PagedAttnCall &call, cudaStream_t s)
{
    const PagedPlan p = paged_plan(c, call.seqs, call.q_heads, call.max_len, call.window, call.weights != nullptr);
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
    a.share = p.share, a.seqs = static_cast<int>(call.seqs);
    a.scale_log2 = call.scale * kPagedLog2e;
    a.o = call.o, a.o_type = call.o_type;
    a.dev_err = call.dev_err;
    uint8_t *ws = static_cast<uint8_t *>(call.workspace);
    const size_t rows = static_cast<size_t>(call.seqs) * call.q_heads;
    const size_t parts = (p.share ? call.q_heads : rows) * p.n_split;
    const bool join = p.n_split > 1 && !p.cluster;
    a.cluster = p.cluster;
    if (join) {
        a.part_o = reinterpret_cast<float *>(ws);
        ws += up256(parts * c->dim * 4);
    }
    if (join || call.weights) {
        a.part_ml = reinterpret_cast<float *>(ws);
        ws += up256(parts * 8);
    }
    if (call.weights) {
        a.scores = reinterpret_cast<float *>(ws);
        a.score_stride = p.score_stride;
    }
    const dim3 grid(static_cast<unsigned>(p.n_split * a.head_blocks), static_cast<unsigned>(c->heads),
                    static_cast<unsigned>(p.share ? 1 : call.seqs));
    cudaError_t e = c->type == QUARTZ_PAGES_ENCODED ? launch_paged_encoded(c->dim, c->k.enc.p.group_s, a, grid, s)
                                                    : launch_paged_16bit(c->type, c->dim, a, grid, s);
    if (e == cudaSuccess && (join || call.weights)) {
        int64_t x = join ? a.group : 1;
        if (call.weights && (p.tokens + 4 * kJoinThreads - 1) / (4 * kJoinThreads) > x) x = (p.tokens + 4 * kJoinThreads - 1) / (4 * kJoinThreads);
        const dim3 g(static_cast<unsigned>(x), static_cast<unsigned>(c->heads), static_cast<unsigned>(call.seqs));
        switch (c->dim) {
            case 64: e = launch_pdl(paged_join_kernel<64>, g, dim3(kJoinThreads), 0, s, a, call.weights, call.w_sb, call.w_sh); break;
            case 128: e = launch_pdl(paged_join_kernel<128>, g, dim3(kJoinThreads), 0, s, a, call.weights, call.w_sb, call.w_sh); break;
            case 192: e = launch_pdl(paged_join_kernel<192>, g, dim3(kJoinThreads), 0, s, a, call.weights, call.w_sb, call.w_sh); break;
            default: e = launch_pdl(paged_join_kernel<256>, g, dim3(kJoinThreads), 0, s, a, call.weights, call.w_sb, call.w_sh); break;
        }
    }
    return e;
}

}  // namespace quartz
