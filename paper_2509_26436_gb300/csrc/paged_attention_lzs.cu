// Attention of one new token over QuaRTZ-encoded pages, for sm_103a
// (paged_attention.cuh has the scheme).
//
// A code c with FLAG F stands for c 2^F (Eq. 2), at most 3 significant bits
// and |c 2^F| <= 112: exact in fp16 and in bf16, so the codes of a group
// multiply on the tensor cores as what they stand for and the group's 16-bit
// scale is applied to the group's sum (keys), or to the softmax weight
// (values):
//   score_t = scale sum_g s_k[t,g] (q . v_k[t])_g,
//   o[g]    = sum_t (p_t s_v[t,g]) v_v[t,g].
// A 4-bit code becomes a 16-bit float without a conversion: the nibble with
// its sign bit flipped (c + 8) in the mantissa of a constant 2^n, and one fused
// multiply-add that takes 2^n + 8 off and multiplies by 2^F, exactly.
//   keys (fp16, 10 mantissa bits):  nibbles at bits 0 and 4 both fit, so a
//     word of 8 codes takes one shift, four and-xor and four fma;
//   values (bf16, so that a weight times a scale, whatever its size, keeps its
//     8 bits; with the remainder 16): words of two tokens are paired by halves
//     first, since an operand register holds two tokens of one column.
#include <atomic>

#include "paged_attention.cuh"

namespace quartz {
namespace {

__device__ __forceinline__ uint32_t fma_f16x2(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t d;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}

__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}

// (x & mask) ^ flip in one instruction.
__device__ __forceinline__ uint32_t and_xor(uint32_t x, uint32_t mask, uint32_t flip)
{
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, 0x6A;" : "=r"(d) : "r"(x), "r"(mask), "r"(flip));
    return d;
}

// The eight codes of a word (code k in bits 4k ..) times 2^F as fp16 pairs
// (k, k + 4): f = 1024 + (c + 8), or 1024 + 16 (c + 8) for the odd nibbles of
// each byte; f 2^F - 1032 2^F, f 2^F / 16 - 72 2^F.  `flag4` = F in the
// exponent fields of a pair (F * 0x04000400).
__device__ __forceinline__ void key_codes(uint32_t w, uint32_t flag4, uint32_t (&k)[4])
{
    const uint32_t m0 = 0x3C003C00u + flag4, m1 = 0x2C002C00u + flag4;  // 2^F, 2^F / 16
    const uint32_t a0 = 0xE408E408u + flag4, a1 = 0xD480D480u + flag4;  // -1032 2^F, -72 2^F
    const uint32_t w8 = w >> 8;
    k[0] = fma_f16x2(and_xor(w, 0x000F000Fu, 0x64086408u), m0, a0);
    k[1] = fma_f16x2(and_xor(w, 0x00F000F0u, 0x64806480u), m1, a1);
    k[2] = fma_f16x2(and_xor(w8, 0x000F000Fu, 0x64086408u), m0, a0);
    k[3] = fma_f16x2(and_xor(w8, 0x00F000F0u, 0x64806480u), m1, a1);
}

// The eight codes of a word of token 0 and of token 1, times 2^F0 and 2^F1, as
// bf16 pairs (token 0, token 1): f = 128 + (c + 8), f 2^F - 136 2^F.  `flags`
// = F0 + (F1 << 16).
__device__ __forceinline__ void value_codes(uint32_t w0, uint32_t w1, uint32_t flags, uint32_t (&v)[8])
{
    const uint32_t f = flags << 7;
    const uint32_t m = 0x3F803F80u + f, a = 0xC308C308u + f;  // 2^F, -136 2^F
    const uint32_t lo = permute(w0, w1, 0x5410), hi = permute(w0, w1, 0x7632);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[j] = fma_bf16x2(and_xor(lo >> (4 * j), 0x000F000Fu, 0x43084308u), m, a);
        v[4 + j] = fma_bf16x2(and_xor(hi >> (4 * j), 0x000F000Fu, 0x43084308u), m, a);
    }
}

// The G scales of a row (2 G bytes, aligned to their largest power of two).
template <int G>
__device__ __forceinline__ void load_scales(const __half *p, float (&s)[G])
{
    if (G == 1) {
        s[0] = __half2float(__ldg(p));
    } else if (G == 2 || G == 4) {
#pragma unroll
        for (int i = 0; i < G; i += 2) {
            const float2 f = __half22float2(__ldg(reinterpret_cast<const __half2 *>(p + i)));
            s[i] = f.x, s[i + (G > 1)] = f.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < G; ++i) s[i] = __half2float(__ldg(p + i));
    }
}

template <int D, int GS, int NT, int MINB>
__global__ void __launch_bounds__(kPagedThreads, MINB) paged_attn_lzs_kernel(PagedArgs a)
{
    griddep_wait();
    constexpr int TILE = 8 * NT, G = D / 64, FPR = D / GS;  // FLAGs per row
    constexpr bool kQRegs = D <= 128;
    __shared__ __align__(16) uint16_t s_q[kPagedHeads][D + 8];
    __shared__ __align__(16) PagedJoin<D> s_join;

    const int head_block = blockIdx.x % a.head_blocks, split = blockIdx.x / a.head_blocks;
    const int kv_head = blockIdx.y, b = blockIdx.z, head0 = head_block * kPagedHeads;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = lane >> 2, q = lane & 3;
    const PagedRange range = paged_range(a.lens, b, a.max_len, a.window, a.dev_err);
    const int begin = split * a.chunk;
    if (a.part_o && begin >= range.count) return;
    const int end = range.first + min(begin + a.chunk, range.count);

    // the query, in the order the keys' codes unpack to: pairs (k, k + 4) of
    // each 8 elements
    for (int e = threadIdx.x; e < kPagedHeads * (D / 8); e += kPagedThreads) {
        const int h = e / (D / 8), d = (e - h * (D / 8)) * 8;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (head0 + h < a.group)
            v = *reinterpret_cast<const uint4 *>(a.q + b * a.q_sb + (static_cast<int64_t>(kv_head) * a.group + head0 + h) * a.q_sh + d);
        *reinterpret_cast<uint4 *>(&s_q[h][d]) = make_uint4(permute(v.x, v.z, 0x5410), permute(v.x, v.z, 0x7632),
                                                            permute(v.y, v.w, 0x5410), permute(v.y, v.w, 0x7632));
    }
    __syncthreads();
    // lane q of a token holds codes 16 q .. 16 q + 15 of each group
    auto query = [&](int g, int half) { return *reinterpret_cast<const uint4 *>(&s_q[n][g * 64 + q * 16 + half * 8]); };
    uint4 qf[kQRegs ? G : 1][2];
    if (kQRegs)
#pragma unroll
        for (int g = 0; g < G; ++g) qf[g][0] = query(g, 0), qf[g][1] = query(g, 1);

    const int32_t *table = a.table + b * a.table_stride;
    const int mask = (1 << a.page_shift) - 1;
    bool bad = false;
    auto page_of = [&](int base) {
        const int t = min(base + (lane & (TILE - 1)), end - 1);
        const uint32_t page = static_cast<uint32_t>(table[t >> a.page_shift]);
        bad |= page >= a.num_pages;
        return page < a.num_pages ? page : 0u;
    };
    // cache row (below 2^31) of token base + i
    auto row_of = [&](uint32_t pages, int base, int i) {
        const uint32_t page = __shfl_sync(0xffffffffu, pages, i);
        const uint32_t slot = static_cast<uint32_t>(min(base + i, end - 1)) & mask;
        return ((page * a.kv_heads + kv_head) << a.page_shift) + slot;
    };

    uint2 kc[NT][G];
    uint32_t kfl[NT][G];  // FLAG of the lane's 16 codes (G_s = 8: two bytes)
    auto load_k = [&](uint32_t pages, int base) {
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const uint32_t row = row_of(pages, base, (n >> 1) * 2 * NT + 2 * i + (n & 1));
            const uint8_t *c = a.k.codes + static_cast<uint64_t>(row) * (D / 2) + q * 8;
            const uint8_t *f = a.k.flags + static_cast<uint64_t>(row) * FPR + (q * 16) / GS;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                kc[i][g] = __ldg(reinterpret_cast<const uint2 *>(c + g * 32));
                kfl[i][g] = GS == 8 ? __ldg(reinterpret_cast<const uint16_t *>(f + g * 8)) : __ldg(f + g * (64 / GS));
            }
        }
    };
    uint32_t vc[2 * NT][G], vfl[2 * NT][G];
    float ks[2 * NT][G], vs[2 * NT][G];
    auto load_v = [&](uint32_t pages, int base) {
#pragma unroll
        for (int j = 0; j < 2 * NT; ++j) {
            const uint32_t row = row_of(pages, base, 2 * NT * q + j);
            const uint8_t *c = a.v.codes + static_cast<uint64_t>(row) * (D / 2) + n * 4;
            const uint8_t *f = a.v.flags + static_cast<uint64_t>(row) * FPR + (n * 8) / GS;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                vc[j][g] = __ldg(reinterpret_cast<const uint32_t *>(c + g * 32));
                vfl[j][g] = __ldg(f + g * (64 / GS));
            }
            load_scales<G>(a.k.scales + static_cast<uint64_t>(row) * G, ks[j]);
            load_scales<G>(a.v.scales + static_cast<uint64_t>(row) * G, vs[j]);
        }
    };

    PagedState<D> st;
    st.init();
    int base = range.first + begin + warp * TILE;
    uint32_t pages = 0;
    if (base < end) {
        pages = page_of(base);
        load_k(pages, base);
        load_v(pages, base);
        if (base + kPagedWarps * TILE < end) pages = page_of(base + kPagedWarps * TILE);
    }
    float *score_row = a.scores && head0 + n < a.group
                           ? a.scores + ((static_cast<int64_t>(b) * a.kv_heads + kv_head) * a.group + head0 + n) * a.score_stride
                           : nullptr;
    while (base < end) {
        // scores: a sum per group, times the group's scale
        float sc[NT][2];
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            sc[i][0] = sc[i][1] = 0.f;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                float s[4] = {0.f, 0.f, 0.f, 0.f};
                const uint32_t f0 = (GS == 8 ? kfl[i][g] & 0xFFu : kfl[i][g]) * 0x04000400u;
                const uint32_t f1 = GS == 8 ? (kfl[i][g] >> 8) * 0x04000400u : f0;
                uint32_t k[4];
                uint4 w = kQRegs ? qf[kQRegs ? g : 0][0] : query(g, 0);
                key_codes(kc[i][g].x, f0, k);
                mma16<false>(s, w.x, w.x, w.y, w.y, k[0], k[1]);
                mma16<false>(s, w.z, w.z, w.w, w.w, k[2], k[3]);
                w = kQRegs ? qf[kQRegs ? g : 0][1] : query(g, 1);
                key_codes(kc[i][g].y, f1, k);
                mma16<false>(s, w.x, w.x, w.y, w.y, k[0], k[1]);
                mma16<false>(s, w.z, w.z, w.w, w.w, k[2], k[3]);
                sc[i][0] += s[0] * ks[2 * i][g];
                sc[i][1] += s[1] * ks[2 * i + 1][g];
            }
        }
        const int next = base + kPagedWarps * TILE;
        if (next < end) load_k(pages, next);
#pragma unroll
        for (int i = 0; i < NT; ++i) sc[i][0] *= a.scale_log2, sc[i][1] *= a.scale_log2;
        if (base + TILE > end) {
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                if (base + 2 * NT * q + 2 * i >= end) sc[i][0] = -INFINITY;
                if (base + 2 * NT * q + 2 * i + 1 >= end) sc[i][1] = -INFINITY;
            }
        }
        if (score_row) {
            float *to = score_row + (base - range.first) + 2 * NT * q;
#pragma unroll
            for (int i = 0; i < NT; ++i) *reinterpret_cast<float2 *>(to + 2 * i) = make_float2(sc[i][0], sc[i][1]);
        }
        st.template weigh<NT>(sc, 0.f);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            uint32_t hi[NT], lo[NT], v0[8], v1[8];
#pragma unroll
            for (int i = 0; i < NT; ++i)
                split_pair<true>(sc[i][0] * vs[2 * i][g], sc[i][1] * vs[2 * i + 1][g], hi[i], lo[i]);
            value_codes(vc[0][g], vc[1][g], vfl[0][g] | (vfl[1][g] << 16), v0);
            if (NT == 2) value_codes(vc[2 * NT - 2][g], vc[2 * NT - 1][g], vfl[2 * NT - 2][g] | (vfl[2 * NT - 1][g] << 16), v1);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (NT == 2) mma16<true>(st.o[g * 8 + j], hi[0], lo[0], hi[NT - 1], lo[NT - 1], v0[j], v1[j]);
                else mma8<true>(st.o[g * 8 + j], hi[0], lo[0], v0[j]);
            }
        }
        if (next < end) {
            load_v(pages, next);
            if (next + kPagedWarps * TILE < end) pages = page_of(next + kPagedWarps * TILE);
        }
        base = next;
    }
    if (bad) atomicExch(a.dev_err, QUARTZ_DEV_INDEX);
    paged_finish<D>(s_join, st, a, b, kv_head, head0, split, 0.f);
}

template <int D, int GS>
struct KernelLzs {
    static constexpr int NT = D <= 192 ? 2 : 1, MINB = D <= 64 ? 4 : D <= 128 ? 3 : 2;
    static int occupancy()
    {
        static std::atomic<int> cache{0};
        int occ = cache.load(std::memory_order_relaxed);
        if (occ == 0) {
            int k = 0;
            if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&k, paged_attn_lzs_kernel<D, GS, NT, MINB>, kPagedThreads, 0) !=
                cudaSuccess)
                k = 1;
            occ = k > 0 ? k : 1;
            cache.store(occ, std::memory_order_relaxed);
        }
        return occ;
    }
    static cudaError_t launch(const PagedArgs &a, dim3 grid, cudaStream_t s)
    {
        return launch_pdl(paged_attn_lzs_kernel<D, GS, NT, MINB>, grid, dim3(kPagedThreads), 0, s, a);
    }
};

template <int D, class F>
auto with_group(int group_s, F f)
{
    switch (group_s) {
        case 8: return f(KernelLzs<D, 8>());
        case 16: return f(KernelLzs<D, 16>());
        case 32: return f(KernelLzs<D, 32>());
        default: return f(KernelLzs<D, 64>());
    }
}

template <class F>
auto with_kernel(int dim, int group_s, F f)
{
    switch (dim) {
        case 64: return with_group<64>(group_s, f);
        case 128: return with_group<128>(group_s, f);
        case 192: return with_group<192>(group_s, f);
        default: return with_group<256>(group_s, f);
    }
}

}  // namespace

int paged_kernel_occupancy_encoded(int dim, int group_s)
{
    return with_kernel(dim, group_s, [](auto k) { return k.occupancy(); });
}

cudaError_t launch_paged_encoded(int dim, int group_s, const PagedArgs &a, dim3 grid, cudaStream_t s)
{
    return with_kernel(dim, group_s, [&](auto k) { return k.launch(a, grid, s); });
}

}  // namespace quartz
