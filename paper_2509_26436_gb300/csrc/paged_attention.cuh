// Attention of one new token over a paged cache: what the kernels for 16-bit
// and for encoded pages share.
//
// A CTA takes one sequence, one key / value head, up to 8 of the query heads
// that share it and one split (a run of consecutive tokens; for few sequences
// given out by their lengths, PagedShare); its 4 warps take tiles of 16 tokens
// in turn, each through a ring in shared memory of its own that asynchronous
// copies fill some tiles ahead, so no warp waits for another.  The products run
// on the warp-level tensor instruction m16n8k16
// with fp32 accumulators:
//   S' = K Q':  rows: 16 tokens, columns: 8 heads;
//   O += P V:   rows 0-7: the upper 16 bits of the heads' softmax weights, rows
//               8-15: what is left of them, rounded again; the accumulator's
//               lower half, added at the end, makes the weights good to twice
//               the 16-bit type's precision, in rows that eight heads leave
//               free anyway: 2^-22 with fp16, 2^-17 with bf16, for which
//               binary32 results take the rest of the weights in a third part.
// The scores arrive transposed to what the second product takes: one register
// transpose (movmatrix) per 8 x 8 block of 16-bit weights, nothing through
// shared memory.  Legacy tensor instructions are enough here: the step is
// bound by HBM (or, encoded, waits in the decoding), and the tensor pipe has to keep
// up with one pair of products per loaded row only (13% busy on 16-bit pages).
// Measured (32 sequences of up to 8192 tokens, 32 / 8 heads of 128, bf16): 98.6
// us, 88% of the copy rate; with tiles in registers instead of a ring 162 us,
// since a warp then holds one tile's loads in flight.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "ptx.cuh"
#include "quartz_internal.h"

namespace quartz {

constexpr int kPagedWarps = 4;
constexpr int kPagedThreads = kPagedWarps * 32;
constexpr int kPagedHeads = 8;  // query heads per CTA
constexpr int kPagedCluster = 8;  // most splits joined within a cluster (the portable size)
constexpr float kPagedLog2e = 1.4426950408889634f;
constexpr float kPagedLow = -3.402823466e38f;  // a maximum before any score: finite, and no finite score is below it

struct PagedSide {
    const uint8_t *data;  // 16-bit pages
    uint32_t stride_page, stride_slot;  // elements
    int64_t stride_head;
    const uint8_t *codes;  // encoded pages
    const uint8_t *flags;
    const __half *scales;
};

struct PagedArgs {
    const uint16_t *q;
    int64_t q_sb, q_sh;
    const int32_t *table;
    int64_t table_stride;
    const int32_t *lens;
    PagedSide k, v;
    uint32_t num_pages;
    int page_shift, kv_heads, group, head_blocks;  // query heads per key head; CTAs they take
    int max_len, window, n_split, chunk;
    int share, seqs;  // share > 0: as many CTAs, at most, share the tokens of all sequences (PagedShare)
    float scale_log2;
    float *part_o;   // NULL, or [seqs * q_heads, share: q_heads][n_split][dim]: splits for the join; NULL: o is written
    float *part_ml;  // NULL, or as many [2]: maximum and sum (with part_o or scores)
    int cluster;     // the splits of a head are one cluster, which joins them itself
    float *scores;   // NULL, or [seqs * q_heads][score_stride], log2 domain
    int64_t score_stride;
    void *o;
    int o_type;
    int *dev_err;
};

// The tokens a sequence's new token sees: [first, end).  Splits and tiles are
// counted from `base`, the multiple of 16 at or below `first`, so that a tile
// of 16 tokens lies in one page of 16 or more and at an aligned place.
struct PagedRange {
    int base, first, end;
    __device__ __forceinline__ int count() const { return end - base; }
};

__device__ __forceinline__ PagedRange paged_range(const int32_t *lens, int b, int max_len, int window, int *dev_err)
{
    int len = lens[b];
    if (len < 0 || len > max_len) {
        if (threadIdx.x == 0) atomicOr(dev_err, QUARTZ_DEV_INDEX);
        len = len < 0 ? 0 : max_len;
    }
    PagedRange r;
    r.first = window > 0 && len > window ? len - window : 0;
    r.base = r.first & ~15;
    r.end = len;
    return r;
}

// Few sequences: `share` places per key head and block of query heads, one wave
// of CTAs, go to the sequences by their lengths.  In units of 64 tokens (a tile
// of each warp), a place takes `each` = ceil(all / (share - seqs)), a sequence
// ceil(its units / each) places in a row, which is at most `share` together.
// (All lanes of a warp; of lane's sequence.)
constexpr int kShareSeqs = 32;
constexpr int kShareUnit = 64;

struct PagedShare {
    int first, count;  // places
    int chunk;         // tokens of a place
};

__device__ __forceinline__ PagedShare paged_share(const PagedArgs &a)
{
    const int lane = threadIdx.x & 31;
    int units = 0;
    if (lane < a.seqs) units = (paged_range(a.lens, lane, a.max_len, a.window, a.dev_err).count() + kShareUnit - 1) / kShareUnit;
    const int all = __reduce_add_sync(0xffffffffu, units), left = a.share - a.seqs;
    const int each = max(1, (all + left - 1) / left);
    PagedShare s;
    s.count = (units + each - 1) / each;
    s.chunk = each * kShareUnit;
    s.first = s.count;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const int v = __shfl_up_sync(0xffffffffu, s.first, d);
        if (lane >= d) s.first += v;
    }
    s.first -= s.count;
    return s;
}

// What a CTA takes: tokens [begin, begin + chunk) of a sequence, counted from the
// range's base.  False: nothing.  (SHARE is an instance of its own: as a branch
// it cost the other calls 1%, 0.1 us at the start of each of their CTAs.)
template <bool SHARE>
__device__ __forceinline__ bool paged_place(const PagedArgs &a, int place, int &b, int &begin, int &chunk)
{
    b = blockIdx.z;
    chunk = a.chunk;
    begin = place * chunk;
    if (SHARE) {
        const PagedShare s = paged_share(a);
        const unsigned behind = __ballot_sync(0xffffffffu, place < s.first + s.count);
        if (!behind) return false;
        b = __ffs(behind) - 1;
        chunk = s.chunk;
        begin = (place - __shfl_sync(0xffffffffu, s.first, b)) * chunk;
    }
    return true;
}

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// d += A B, 16 x 8 x 16.
template <bool BF>
__device__ __forceinline__ void mma16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                      uint32_t b1)
{
    if (BF)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Two weights as a 16-bit pair and the pair of what the rounding left; what
// that leaves stays in p0 and p1 where it is asked for.
template <bool BF>
__device__ __forceinline__ void split_pair(float &p0, float &p1, uint32_t &hi, uint32_t &lo, bool rest = false)
{
    if (BF) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(p0, p1);
        hi = *reinterpret_cast<const uint32_t *>(&h);
        const float r0 = p0 - __uint_as_float(hi << 16), r1 = p1 - __uint_as_float(hi & 0xFFFF0000u);
        const __nv_bfloat162 l = __floats2bfloat162_rn(r0, r1);
        lo = *reinterpret_cast<const uint32_t *>(&l);
        if (rest) p0 = r0 - __uint_as_float(lo << 16), p1 = r1 - __uint_as_float(lo & 0xFFFF0000u);
    } else {
        const __half2 h = __floats2half2_rn(p0, p1);
        const float2 f = __half22float2(h);
        const __half2 l = __floats2half2_rn(p0 - f.x, p1 - f.y);
        hi = *reinterpret_cast<const uint32_t *>(&h);
        lo = *reinterpret_cast<const uint32_t *>(&l);
    }
}

// What split_pair left, in bf16.
__device__ __forceinline__ uint32_t bf16_pair(float p0, float p1)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(p0, p1);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// A warp's accumulators (rows: heads; 8 columns of the head dimension per
// entry) and its running softmax.  A lane holds the scores of two tokens and
// heads 2 q and 2 q + 1 (q = lane % 4): m are their maxima so far (log2 domain),
// which all lanes of a head share, l this lane's part of the sums of weights.
template <int D>
struct PagedState {
    float o[D / 8][4];
    float m[2], l[2];

    __device__ __forceinline__ void init()
    {
#pragma unroll
        for (int i = 0; i < D / 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][j] = 0.f;
        m[0] = m[1] = kPagedLow;
        l[0] = l[1] = 0.f;
    }

    // Scores sc[token][head] (log2 domain, -inf where masked) to weights
    // p = 2^(sc - m + up).  The maximum follows only when a score passes it by
    // more than `slack`: a weight of 2^slack does no harm, and then no lane
    // has to hear of the others' scores, and no accumulator to be rescaled, in
    // most tiles.  `up` keeps small weights of fp16 normal.
    __device__ __forceinline__ void weigh(const float (&sc)[2][2], float (&p)[2][2], float up, float slack)
    {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int x = 0; x < 2; ++x) p[i][x] = sc[i][x] - m[x];
        if (__any_sync(0xffffffffu, fmaxf(fmaxf(p[0][0], p[0][1]), fmaxf(p[1][0], p[1][1])) > slack)) {
            const int n = (threadIdx.x & 31) >> 2;
            float f[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                float top = fmaxf(m[x], fmaxf(sc[0][x], sc[1][x]));
#pragma unroll
                for (int d = 4; d < 32; d *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                f[x] = ex2(m[x] - top);
                m[x] = top;
                l[x] *= f[x];
#pragma unroll
                for (int i = 0; i < 2; ++i) p[i][x] = sc[i][x] - top;
            }
            const float f0 = __shfl_sync(0xffffffffu, f[0], n >> 1), f1 = __shfl_sync(0xffffffffu, f[1], n >> 1);
            const float fn = n & 1 ? f1 : f0;  // of head n, the accumulators' row
#pragma unroll
            for (int i = 0; i < D / 8; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[i][j] *= fn;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                p[i][x] = ex2(up == 0.f ? p[i][x] : p[i][x] + up);
                l[x] += p[i][x];
            }
    }
};

// The transpose of an 8 x 8 block of 16-bit values, lane = row lane / 4,
// columns 2 (lane % 4) and the next.
__device__ __forceinline__ uint32_t transposed(uint32_t v)
{
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
    return d;
}

template <typename T> __device__ __forceinline__ void paged_store4(void *o, int64_t at, float4 v);
template <> __device__ __forceinline__ void paged_store4<float>(void *o, int64_t at, float4 v)
{
    *reinterpret_cast<float4 *>(static_cast<float *>(o) + at) = v;
}
template <> __device__ __forceinline__ void paged_store4<__half>(void *o, int64_t at, float4 v)
{
    const __half2 a = __floats2half2_rn(v.x, v.y), b = __floats2half2_rn(v.z, v.w);
    *reinterpret_cast<uint2 *>(static_cast<__half *>(o) + at) =
        make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
}
template <> __device__ __forceinline__ void paged_store4<__nv_bfloat16>(void *o, int64_t at, float4 v)
{
    const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
    *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(o) + at) =
        make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
}
__device__ __forceinline__ void paged_store4(void *o, int type, int64_t at, float4 v)
{
    if (type == QUARTZ_OUT_F16) paged_store4<__half>(o, at, v);
    else if (type == QUARTZ_OUT_BF16) paged_store4<__nv_bfloat16>(o, at, v);
    else paged_store4<float>(o, at, v);
}

// Join the warps of a CTA in a fixed order and write the split's result: the
// output itself where there is one split; o (relative to the split's maximum)
// with maximum and sum for the join kernel; or, where the splits of a head are
// a cluster, the output of all of them, each CTA its share of the elements.
struct PagedJoin {
    float m[kPagedWarps][kPagedHeads], l[kPagedWarps][kPagedHeads];
    float all_m[kPagedHeads], all_l[kPagedHeads];  // of the CTA
};

// `smem` + warp * warp_bytes is the warp's own shared memory, at least
// kPagedJoinBytes<D>, free by now.
template <int D>
constexpr int kPagedJoinBytes = kPagedHeads * (D + 4) * 4;

//
// The accumulators' column 2 q + x of entry i is dimension 8 i + 2 q + x, or
// (STRIDED) (i / 8) 64 + (2 q + x) 8 + i % 8.
template <int D, bool STRIDED, bool SHARE>
__device__ __forceinline__ void paged_finish(PagedJoin &s, uint8_t *smem, int warp_bytes, PagedState<D> &st,
                                             const PagedArgs &a, int b, int kv_head, int head0, int split, float up)
{
    auto so = [&](int w, int h, int d) {
        return reinterpret_cast<float4 *>(smem + w * warp_bytes + (h * (D + 4) + d) * 4);
    };
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = lane >> 2, q = lane & 3;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
        for (int d = 4; d < 32; d *= 2) st.l[x] += __shfl_xor_sync(0xffffffffu, st.l[x], d);
        if (n == 0) s.m[warp][2 * q + x] = st.m[x], s.l[warp][2 * q + x] = st.l[x];
    }
    if constexpr (STRIDED) {
#pragma unroll
        for (int hv = 0; hv < D / 64; ++hv)
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int j = 0; j < 8; j += 4) {
                    const float(*o)[4] = &st.o[hv * 8 + j];
                    *so(warp, n, hv * 64 + (2 * q + x) * 8 + j) =
                        make_float4(o[0][x] + o[0][x + 2], o[1][x] + o[1][x + 2], o[2][x] + o[2][x + 2], o[3][x] + o[3][x + 2]);
                }
    } else {
#pragma unroll
        for (int i = 0; i < D / 8; ++i)
            *reinterpret_cast<float2 *>(so(warp, n, 8 * i + 2 * q)) =
                make_float2(st.o[i][0] + st.o[i][2], st.o[i][1] + st.o[i][3]);
    }
    __syncthreads();
    const int64_t row0 = (static_cast<int64_t>(b) * a.kv_heads + kv_head) * a.group + head0;
    for (int e = threadIdx.x; e < kPagedHeads * (D / 4); e += kPagedThreads) {
        const int h = e / (D / 4), d = (e - h * (D / 4)) * 4;
        if (head0 + h >= a.group) break;
        float m = s.m[0][h];
#pragma unroll
        for (int w = 1; w < kPagedWarps; ++w) m = fmaxf(m, s.m[w][h]);
        float sum = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kPagedWarps; ++w) {
            const float f = ex2(s.m[w][h] - m - up);
            const float4 u = *so(w, h, d);
            sum += f * s.l[w][h];
            v.x += f * u.x, v.y += f * u.y, v.z += f * u.z, v.w += f * u.w;
        }
        const int64_t row = row0 + h;
        const int64_t at = (SHARE ? row - static_cast<int64_t>(b) * a.kv_heads * a.group : row) * a.n_split + split;
        if (a.part_ml && d == 0) *reinterpret_cast<float2 *>(a.part_ml + 2 * at) = make_float2(m, sum);
        if (a.cluster) {
            *so(0, h, d) = v;  // read by this thread only, above
            if (d == 0) s.all_m[h] = m, s.all_l[h] = sum;
        } else if (a.part_o) {
            *reinterpret_cast<float4 *>(a.part_o + at * D + d) = v;
        } else {
            const float r = sum > 0.f ? 1.f / sum : 0.f;
            paged_store4(a.o, a.o_type, row * D + d, make_float4(v.x * r, v.y * r, v.z * r, v.w * r));
        }
    }
    if (!a.cluster) return;
    __syncwarp();
    cluster_arrive();
    cluster_wait();
    const uint32_t s_m = smem_u32(s.all_m);
    const uint32_t s_l = smem_u32(s.all_l);
    for (int e = split * kPagedThreads + threadIdx.x; e < kPagedHeads * (D / 4); e += a.n_split * kPagedThreads) {
        const int h = e / (D / 4), d = (e - h * (D / 4)) * 4;
        if (head0 + h >= a.group) break;
        const uint32_t mine = smem_u32(so(0, h, d));
        float ms[kPagedCluster], ls[kPagedCluster];  // all loads before their first use
        float4 us[kPagedCluster];
#pragma unroll
        for (int c = 0; c < kPagedCluster; ++c) {
            const int from = min(c, a.n_split - 1);
            ms[c] = ld_cluster_f32(mapa(s_m + 4 * h, from));
            ls[c] = ld_cluster_f32(mapa(s_l + 4 * h, from));
            us[c] = ld_cluster_f4(mapa(mine, from));
        }
        float m = ms[0], sum = 0.f;
#pragma unroll
        for (int c = 1; c < kPagedCluster; ++c) m = fmaxf(m, ms[c]);
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int c = 0; c < kPagedCluster; ++c) {
            const float f = c < a.n_split ? ex2(ms[c] - m) : 0.f;
            sum += f * ls[c];
            v.x += f * us[c].x, v.y += f * us[c].y, v.z += f * us[c].z, v.w += f * us[c].w;
        }
        const float r = sum > 0.f ? 1.f / sum : 0.f;
        paged_store4(a.o, a.o_type, (row0 + h) * D + d, make_float4(v.x * r, v.y * r, v.z * r, v.w * r));
    }
    __syncwarp();
    cluster_arrive();
    cluster_wait();  // no CTA leaves while another reads its shared memory
}

// CTAs resident per SM of the kernel that serves this cache.
int paged_kernel_occupancy_16bit(int type, int dim);
int paged_kernel_occupancy_encoded(int dim, int group_s);
cudaError_t launch_paged_16bit(int type, int dim, const PagedArgs &a, dim3 grid, cudaStream_t s);
cudaError_t launch_paged_encoded(int dim, int group_s, const PagedArgs &a, dim3 grid, cudaStream_t s);

}  // namespace quartz
