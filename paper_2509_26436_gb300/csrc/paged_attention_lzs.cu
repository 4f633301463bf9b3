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
// The contraction over the head dimension may take it in any order, so a
// lane's 8 consecutive bytes of codes go into the operand's registers as they
// unpack, and the query is permuted to match, once.
// What bounds it: latency, not HBM.  A tile of 16 tokens of 128 dimensions takes
// 466 instructions of a warp, 172 of them logic and 152 of the half-rate
// multiply-add pipe, whose pipes they hold for two cycles each: 466, 344 and 304
// cycles side by side, of the 818 that it takes.  Meanwhile 2.8 warps per
// scheduler (168 registers) wait for their own dependent instructions: issue slots
// 62% busy, the logic pipe 47%, multiply-add 41%, tensor 25%.  8 sequences of up to 65536 tokens, 64 / 8
// heads, G_s = 16: 96.0 us, 51% of the copy rate (245 us with tiles in
// registers, 125 with the query as the first operand of the keys' product, whose
// duplicated rows had to be copied for every tile).
#include <atomic>

#include "lzs_f16.cuh"
#include "paged_attention.cuh"

namespace quartz {
namespace {

__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}

__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

// The eight codes of a word of token 0 and of token 1, times 2^F0 and 2^F1, as
// bf16 pairs (token 0, token 1): f = 128 + (c + 8), f 2^F - 136 2^F.  `flags`
// = F0 + (F1 << 16).
__device__ __forceinline__ void value_codes(uint32_t w0, uint32_t w1, uint32_t flags, uint32_t (&v)[8])
{
    const uint32_t m = flags * 128u + 0x3F803F80u, a = mul_bf16x2(m, 0xC308C308u);  // 2^F, -136 2^F
    const uint32_t lo = prmt(w0, w1, 0x5410), hi = prmt(w0, w1, 0x7632);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[j] = fma_bf16x2(and_xor(lo >> (4 * j), 0x000F000Fu, 0x43084308u), m, a);
        v[4 + j] = fma_bf16x2(and_xor(hi >> (4 * j), 0x000F000Fu, 0x43084308u), m, a);
    }
}

// A warp's tile of 16 tokens in shared memory, keys and values: codes, FLAGs
// and scales.  Rows and 16-byte chunks of the codes are permuted so that the
// reads below hit different banks: 8-byte reads of one chunk pair of tokens 0,
// 1, 4, 5 (keys), 4-byte reads of tokens 0, 4, 8, 12 (values).
template <int D, int GS>
struct LzsTile {
    static constexpr int kTokens = 16, kChunks = D / 32;  // 16-byte chunks of codes per row
    static constexpr int kCodes = kTokens * D / 2, kFlags = kTokens * D / GS, kScales = kTokens * D / 32;
    static constexpr int kSide = kCodes + kFlags + kScales, kBytes = 2 * kSide;
    static constexpr int kStages = 5;
    // The small planes of both sides as 16-byte chunks: FLAGs, scales, FLAGs, scales.
    static constexpr int kSmall = 2 * (kFlags + kScales) / 16, kSmallPerLane = (kSmall + 31) / 32;
    static constexpr int kCodesPerLane = kCodes / 16 / 32 > 0 ? kCodes / 16 / 32 : 1;

    __host__ __device__ static constexpr int key_at(int t, int c)
    {
        const int odd = (t >> 2) & 1;
        const int r = D == 64 || D == 192 ? t ^ (odd << 1) : t;
        const int x = D == 128 ? odd * 2 : D == 256 ? ((t & 1) + 2 * odd) * 2 : 0;
        return (r * kChunks + (c ^ x)) * 16;
    }
    __host__ __device__ static constexpr int value_at(int t, int c)
    {
        const int q = t >> 2, r = (t & 3) * 4 + q;
        const int x = D == 128 ? (q >> 1) * 2 : D == 256 ? q * 2 : 0;
        return (r * kChunks + (c ^ x)) * 16;
    }
};

// Loads of a tile that has arrived: free to move, from the point on where its
// address was made (`fixed`, after the wait).
__device__ __forceinline__ uint32_t lds32(uint32_t a)
{
    uint32_t v;
    asm("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a));
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a)
{
    uint2 v;
    asm("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
    return v;
}
__device__ __forceinline__ uint4 lds128(uint32_t a)
{
    uint4 v;
    asm("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
    return v;
}
__device__ __forceinline__ uint32_t lds16(uint32_t a)
{
    uint16_t v;
    asm("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(a));
    return v;
}
__device__ __forceinline__ uint32_t lds8(uint32_t a)
{
    uint32_t v;
    asm("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(a));
    return v;
}

// An opaque copy: what follows from it is not recomputed from the lane.
__device__ __forceinline__ uint32_t fixed(uint32_t v)
{
    asm volatile("" : "+r"(v));
    return v;
}

// The G scales of a row of the tile.
template <int G>
__device__ __forceinline__ void lds_scales(uint32_t a, float (&s)[G])
{
    if (G == 1) {
        s[0] = __half2float(__ushort_as_half(static_cast<unsigned short>(lds16(a))));
    } else if (G == 4) {
        const uint2 v = lds64(a);
        const float2 x = __half22float2(*reinterpret_cast<const __half2 *>(&v.x)), y = __half22float2(*reinterpret_cast<const __half2 *>(&v.y));
        s[0] = x.x, s[1 % G] = x.y, s[2 % G] = y.x, s[3 % G] = y.y;
    } else if (G == 2) {
        const uint32_t v = lds32(a);
        const float2 x = __half22float2(*reinterpret_cast<const __half2 *>(&v));
        s[0] = x.x, s[1 % G] = x.y;
    } else {
#pragma unroll
        for (int i = 0; i < G; ++i) s[i] = __half2float(__ushort_as_half(static_cast<unsigned short>(lds16(a + 2 * i))));
    }
}

// GENERAL: pages below 16 tokens, scores for the sums of weights, or binary32
// results; the other instance is for pages of 16 and more, 16-bit results and
// no scores.
template <int D, int GS, bool GENERAL, bool SHARE, int MINB>
__global__ void __launch_bounds__(kPagedThreads, MINB) paged_attn_lzs_kernel(PagedArgs a)
{
    griddep_wait();
    using Tile = LzsTile<D, GS>;
    constexpr int G = D / 64, FPR = D / GS;  // groups and FLAGs per row
    constexpr int kStages = Tile::kStages, kWarpBytes = kStages * Tile::kBytes;
    constexpr bool kQRegs = D <= 128;  // wider heads read the query from shared memory again for each tile
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
    const int end = range.base + min(begin + chunk, range.count());
    // a warp's tiles are consecutive, so that most follow the one before in its page
    const int all_tiles = max(0, end - range.base - begin + 15) >> 4, warp_tiles = (all_tiles + kPagedWarps - 1) / kPagedWarps;
    const int tiles = max(0, min(warp_tiles, all_tiles - warp * warp_tiles));
    const int base0 = range.base + begin + warp * warp_tiles * 16;
    const uint32_t ring = smem_u32(s_ring) + warp * kWarpBytes;

    // --- copies of a tile -------------------------------------------------
    const int32_t *table = a.table + b * a.table_stride;
    const uint32_t page_mask = (1u << a.page_shift) - 1;
    bool bad = false;
    // lane's part of the codes: chunk i = lane + 32 k of the tile
    int key_dst[Tile::kCodesPerLane], value_dst[Tile::kCodesPerLane];
#pragma unroll
    for (int k = 0; k < Tile::kCodesPerLane; ++k) {
        const int i = lane + 32 * k, t = i / Tile::kChunks, c = i % Tile::kChunks;
        key_dst[k] = Tile::key_at(t, c);
        value_dst[k] = Tile::kSide + Tile::value_at(t, c);
    }
    // and of the small planes
    const uint8_t *small_src[Tile::kSmallPerLane];
    int small_row[Tile::kSmallPerLane], small_dst[Tile::kSmallPerLane];
#pragma unroll
    for (int k = 0; k < Tile::kSmallPerLane; ++k) {
        int i = lane + 32 * k;
        const bool in = i < Tile::kSmall;
        const int side = i >= Tile::kSmall / 2;
        i -= side * (Tile::kSmall / 2);
        const bool flag = i < Tile::kFlags / 16;
        const PagedSide &ps = side ? a.v : a.k;
        small_src[k] = (flag ? ps.flags : reinterpret_cast<const uint8_t *>(ps.scales) - Tile::kFlags) + i * 16;
        small_row[k] = in ? (flag ? FPR : 2 * G) : -1;
        small_dst[k] = side * Tile::kSide + Tile::kCodes + i * 16;
    }
    auto checked = [&](int32_t page) {
        bad |= static_cast<uint32_t>(page) >= a.num_pages;
        return static_cast<uint32_t>(page) < a.num_pages ? static_cast<uint32_t>(page) : 0u;
    };
    auto row_of = [&](uint32_t page, int t) {
        return ((page * a.kv_heads + kv_head) << a.page_shift) + (static_cast<uint32_t>(t) & page_mask);
    };
    const bool small_pages = GENERAL && a.page_shift < 4;
    // The next tile to fetch: its first token and cache row; the table's entry
    // for the page behind, read a page ahead.
    int at = base0;
    uint32_t at_row = 0;
    int32_t page_behind = 0;
    const int last_page = (end - 1) >> a.page_shift;
    auto enter = [&](int32_t page) {
        at_row = row_of(checked(page), at);
        const int behind = (at >> a.page_shift) + 1;
        if (behind <= last_page) page_behind = __ldg(table + behind);
    };
    if (tiles > 0 && !small_pages) enter(__ldg(table + (at >> a.page_shift)));
    // Pages of 16 or more: 16 consecutive rows.  Smaller ones: row by row; the
    // small planes' rows are then below the 16 bytes of a copy and go through
    // registers.  There a token that is not seen repeats the nearest that is.
    auto fetch = [&](int stage) {
        const uint32_t to = ring + stage * Tile::kBytes;
        if (!small_pages) {
            const uint64_t row = at_row;
            const uint8_t *kc = a.k.codes + row * (D / 2) + lane * 16, *vc = a.v.codes + row * (D / 2) + lane * 16;
#pragma unroll
            for (int k = 0; k < Tile::kCodesPerLane; ++k) {
                cp_async16(to + key_dst[k], kc + k * 512);
                cp_async16(to + value_dst[k], vc + k * 512);
            }
#pragma unroll
            for (int k = 0; k < Tile::kSmallPerLane; ++k)
                if (small_row[k] >= 0) cp_async16(to + small_dst[k], small_src[k] + row * small_row[k]);
            at += 16;
            at_row += 16;
            if ((at & page_mask) == 0 && at < end) enter(page_behind);
        } else {
            const int mine = max(min(at + (lane & 15), end - 1), range.first);
            const uint32_t my_row = row_of(checked(__ldg(table + (mine >> a.page_shift))), mine);
#pragma unroll
            for (int k = 0; k < Tile::kCodesPerLane; ++k) {
                const int i = lane + 32 * k, t = i / Tile::kChunks, c = i % Tile::kChunks;
                const uint64_t row = __shfl_sync(0xffffffffu, my_row, t);
                cp_async16(to + key_dst[k], a.k.codes + row * (D / 2) + c * 16);
                cp_async16(to + value_dst[k], a.v.codes + row * (D / 2) + c * 16);
            }
            const PagedSide &ps = lane < 16 ? a.k : a.v;  // a lane per row and side
            uint8_t *dst = s_ring + warp * kWarpBytes + stage * Tile::kBytes + (lane < 16 ? 0 : Tile::kSide) + Tile::kCodes;
            const uint8_t *fl = ps.flags + static_cast<uint64_t>(my_row) * FPR;
#pragma unroll
            for (int i = 0; i < FPR; ++i) dst[(lane & 15) * FPR + i] = __ldg(fl + i);
            const __half *sc = ps.scales + static_cast<uint64_t>(my_row) * G;
#pragma unroll
            for (int i = 0; i < G; ++i)
                reinterpret_cast<__half *>(dst + Tile::kFlags)[(lane & 15) * G + i] = __ldg(sc + i);
            at += 16;
        }
    };
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) {
        if (s < tiles) fetch(s);
        cp_async_commit();
    }

    // --- the query, in the order the keys' codes unpack to: pairs (k, k + 4) of
    // each 8 elements
    for (int e = threadIdx.x; e < kPagedHeads * (D / 8); e += kPagedThreads) {
        const int h = e / (D / 8), d = (e - h * (D / 8)) * 8;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (head0 + h < a.group)
            v = *reinterpret_cast<const uint4 *>(a.q + b * a.q_sb + (static_cast<int64_t>(kv_head) * a.group + head0 + h) * a.q_sh + d);
        *reinterpret_cast<uint4 *>(&s_q[h][d]) = make_uint4(prmt(v.x, v.z, 0x5410), prmt(v.x, v.z, 0x7632),
                                                            prmt(v.y, v.w, 0x5410), prmt(v.y, v.w, 0x7632));
    }
    __syncthreads();
    // lane q of a token holds codes 16 q .. 16 q + 15 of each group
    auto query = [&](int g, int half) { return *reinterpret_cast<const uint4 *>(&s_q[n][g * 64 + q * 16 + half * 8]); };
    uint4 qf[kQRegs ? G : 1][2];
    if (kQRegs)
#pragma unroll
        for (int g = 0; g < G; ++g) qf[g][0] = query(g, 0), qf[g][1] = query(g, 1);

    // --- places of the lane's pieces in a tile: keys of tokens (n / 2) 4 + n % 2
    // + 2 i, values of tokens 4 q + j.  Bases that differ between lanes are
    // held in registers (`fixed` keeps the compiler from recomputing them for
    // every tile), the rest are immediate offsets.
    const int key_token = (n >> 1) * 4 + (n & 1);
    constexpr int kRow = Tile::kChunks * 16;
    constexpr int KB = D == 256 ? 4 : 2, VB = D == 256 ? 4 : D == 128 ? 2 : 1;
    uint32_t kb[KB], vb[VB];
#pragma unroll
    for (int i = 0; i < KB; ++i)  // 64, 192: per token i; else per group
        kb[i] = fixed(Tile::key_at(key_token + (D == 64 || D == 192 ? 2 * i : 0), (D == 128 || D == 256 ? 2 * i : 0) + (q >> 1)) + (q & 1) * 8);
#pragma unroll
    for (int i = 0; i < VB; ++i) vb[i] = fixed(Tile::kSide + Tile::value_at(4 * q, 2 * i + (n >> 2)) + (n & 3) * 4);
    auto key_off = [&](int i, int g) { return D == 64 || D == 192 ? kb[i] + g * 32 : kb[g] + i * 2 * kRow; };
    auto value_off = [&](int j, int g) { return (VB > 1 ? vb[VB > 1 ? g : 0] : vb[0] + g * 32) + j * 4 * kRow; };
    const uint32_t kfb = fixed(Tile::kCodes + key_token * FPR + (q * 16) / GS);
    const uint32_t ksb = fixed(Tile::kCodes + Tile::kFlags + key_token * 2 * G);
    const uint32_t vfb = fixed(Tile::kSide + Tile::kCodes + 4 * q * FPR + (n * 8) / GS);

    // Scores of a tile's tokens i and heads x: a sum per group, times the
    // group's scale.
    auto score = [&](uint32_t tile, int base, float (&sc)[2][2]) {
        float ks[2][G];
        lds_scales<G>(tile + ksb, ks[0]);
        lds_scales<G>(tile + ksb + 4 * G, ks[1]);
        sc[0][0] = sc[0][1] = sc[1][0] = sc[1][1] = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            uint32_t k[2][2][4];  // token, word
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint2 c = lds64(tile + key_off(i, g));
                const uint32_t f = GS == 8 ? lds16(tile + kfb + 2 * i * FPR + g * 8) : lds8(tile + kfb + 2 * i * FPR + g * (64 / GS));
                const KeyFlag f0(GS == 8 ? f & 0xFFu : f);
                key_codes(c.x, f0, k[i][0]);
                if (GS == 8) key_codes(c.y, KeyFlag(f >> 8), k[i][1]);
                else key_codes(c.y, f0, k[i][1]);
            }
            float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const uint4 qw = kQRegs ? qf[kQRegs ? g : 0][w] : query(g, w);
                mma16<false>(s, k[0][w][0], k[1][w][0], k[0][w][1], k[1][w][1], qw.x, qw.y);
                mma16<false>(s, k[0][w][2], k[1][w][2], k[0][w][3], k[1][w][3], qw.z, qw.w);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) sc[i][0] += s[2 * i] * ks[i][g], sc[i][1] += s[2 * i + 1] * ks[i][g];
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int t = base + key_token + 2 * i;
            const bool hidden = t >= end || t < range.first;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                sc[i][x] = hidden ? -INFINITY : sc[i][x] * a.scale_log2;
                if (GENERAL && a.scores && head0 + 2 * q + x < a.group)
                    a.scores[(((static_cast<int64_t>(b) * a.kv_heads + kv_head) * a.group + head0 + 2 * q) + x) * a.score_stride +
                             (t - range.base)] = sc[i][x];
            }
        }
    };
    PagedState<D> st;
    st.init();
    // The weighted values of a tile.
    auto add_values = [&](uint32_t tile, int base, const float (&p)[2][2]) {
        float vs[2][G];
        lds_scales<G>(tile + ksb + Tile::kSide, vs[0]);
        lds_scales<G>(tile + ksb + Tile::kSide + 4 * G, vs[1]);
        uint32_t vf[2][G];  // FLAGs of token pairs 4 q, 4 q + 1 and 4 q + 2, 4 q + 3
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int g = 0; g < G; ++g)
                vf[i][g] = lds8(tile + vfb + 2 * i * FPR + g * (64 / GS)) + (lds8(tile + vfb + (2 * i + 1) * FPR + g * (64 / GS)) << 16);
        if (base + 16 > end || base < range.first) {
            // tokens that are not seen have no weight, and nothing of what
            // their slots happen to hold may meet it (a scale may be NaN)
            auto hidden = [&](int t) { return base + t >= end || base + t < range.first; };
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    if (hidden(key_token + 2 * i)) vs[i][g] = 0.f;
                    if (hidden(4 * q + 2 * i)) vf[i][g] &= 0xFFFF0000u;
                    if (hidden(4 * q + 2 * i + 1)) vf[i][g] &= 0x0000FFFFu;
                }
        }
#pragma unroll
        for (int g = 0; g < G; ++g) {
            uint32_t hi[2], lo[2], rest[2], v0[8], v1[8], c[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) c[j] = lds32(tile + value_off(j, g));
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float p0 = p[i][0] * vs[i][g], p1 = p[i][1] * vs[i][g];
                split_pair<true>(p0, p1, hi[i], lo[i], GENERAL);
                if (GENERAL) rest[i] = transposed(bf16_pair(p0, p1));
                hi[i] = transposed(hi[i]);
                lo[i] = transposed(lo[i]);
            }
            value_codes(c[0], c[1], vf[0][g], v0);
            value_codes(c[2], c[3], vf[1][g], v1);
#pragma unroll
            for (int j = 0; j < 8; ++j) mma16<true>(st.o[g * 8 + j], hi[0], lo[0], hi[1], lo[1], v0[j], v1[j]);
            if (GENERAL && a.o_type == QUARTZ_OUT_F32) {
#pragma unroll
                for (int j = 0; j < 8; ++j) mma16<true>(st.o[g * 8 + j], rest[0], 0u, rest[1], 0u, v0[j], v1[j]);
            }
        }
    };

    // A tile's values and the next one's scores side by side: one run of
    // instructions without a branch, in which the one's tensor instructions
    // overlap the other's unpacking.
    float sc[2][2], p[2][2];
    if (tiles > 0) {
        cp_async_wait<kStages - 2>();
        __syncwarp();
        score(fixed(ring), base0, sc);
        st.weigh(sc, p, 0.f, 8.f);
    }
    int stage = 0;
    for (int it = 0; it < tiles; ++it) {
        const int base = base0 + it * 16;
        cp_async_wait<kStages - 3>();
        __syncwarp();
        if (it + kStages - 1 < tiles) fetch(stage == 0 ? kStages - 1 : stage - 1);
        cp_async_commit();
        const uint32_t tile = fixed(ring + stage * Tile::kBytes);
        stage = stage == kStages - 1 ? 0 : stage + 1;
        if (it + 1 < tiles) {
            const uint32_t next = fixed(ring + stage * Tile::kBytes);
            add_values(tile, base, p);
            score(next, base + 16, sc);
            st.weigh(sc, p, 0.f, 8.f);
        } else {
            add_values(tile, base, p);
        }
    }
    cp_async_wait<0>();
    __syncwarp();
    if (bad) atomicOr(a.dev_err, QUARTZ_DEV_INDEX);
    paged_finish<D, true, SHARE>(s_join, s_ring, kWarpBytes, st, a, b, kv_head, head0, split, 0.f);
}

template <int D, int GS>
struct KernelLzs {
    static constexpr int MINB = D <= 64 ? 4 : D <= 128 ? 3 : 2;
    static constexpr int kSmem = kPagedWarps * LzsTile<D, GS>::kStages * LzsTile<D, GS>::kBytes;
    static int occupancy()
    {
        static std::atomic<int> cache{0};
        int occ = cache.load(std::memory_order_relaxed);
        if (occ == 0) {
            int k = 0;
            if (allow_shared<paged_attn_lzs_kernel<D, GS, false, false, MINB>>(kSmem) != cudaSuccess ||
                cudaOccupancyMaxActiveBlocksPerMultiprocessor(&k, paged_attn_lzs_kernel<D, GS, false, false, MINB>, kPagedThreads,
                                                              kSmem) != cudaSuccess)
                return 1;
            occ = k > 0 ? k : 1;
            cache.store(occ, std::memory_order_relaxed);
        }
        return occ;
    }
    static cudaError_t launch(const PagedArgs &a, dim3 grid, cudaStream_t s)
    {
        if (a.scores || a.page_shift < 4 || a.o_type == QUARTZ_OUT_F32)
            return a.share ? launch_as<true, true>(a, grid, s) : launch_as<true, false>(a, grid, s);
        return a.share ? launch_as<false, true>(a, grid, s) : launch_as<false, false>(a, grid, s);
    }
    template <bool GENERAL, bool SHARE>
    static cudaError_t launch_as(const PagedArgs &a, dim3 grid, cudaStream_t s)
    {
        const cudaError_t e = allow_shared<paged_attn_lzs_kernel<D, GS, GENERAL, SHARE, MINB>>(kSmem);
        if (e != cudaSuccess) return e;
        if (a.cluster)
            return launch_pdl_cluster(paged_attn_lzs_kernel<D, GS, GENERAL, SHARE, MINB>, a.n_split, grid, dim3(kPagedThreads), kSmem, s, a);
        return launch_pdl(paged_attn_lzs_kernel<D, GS, GENERAL, SHARE, MINB>, grid, dim3(kPagedThreads), kSmem, s, a);
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
