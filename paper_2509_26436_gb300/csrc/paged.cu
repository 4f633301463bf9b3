// Paged cache, the writers, for sm_103a: the append of new tokens into their
// slots (rotation of the keys and Eq. 1 + Eq. 2 fused) and the closing-up of a
// cache after an eviction.  Both are HBM-bound copies.
#include "lzs_encode.cuh"
#include "quartz_internal.h"
#include "rope.cuh"

namespace quartz {
namespace {

// ---------------------------------------------------------------------------
// Append
// ---------------------------------------------------------------------------
constexpr int kAppendThreads = 256;
constexpr int kAppendTokens = 8;                       // most tokens per CTA
constexpr int kAngles = kAppendTokens * 128;           // dim <= 256: 128 pairs

struct AppendDst {
    uint8_t *data;  // 16-bit pages
    int64_t stride_page, stride_slot, stride_head;
    uint2 *codes;  // encoded pages
    uint8_t *flags;
    __half *scales;
};

struct AppendCall {
    AppendArgs a;
    AppendDst dst[2];
    int64_t slots_total;
    int page_shift, heads, units;    // units per row, of half a row with BOTH
    int tokens_here, groups, each;   // per CTA; head groups; heads per thread
};

// Elements a thread takes at a time (a unit): as much of a 64-element group as
// the encoder's lanes hold, or 16 bytes.
constexpr int unit_size(bool encoded) { return encoded ? 16 : 8; }

// The angles of a CTA's tokens in shared memory, (cos, -sin) for the first
// element of a pair and, unless a thread turns both elements of its pairs,
// behind them (sin, cos) for the second: both are m a + n b with (a, b) =
// (first, second).  Neighbouring units, which neighbouring lanes hold, side by
// side.
template <int E>
struct AngleTable {
    const float2 *cs;
    static constexpr int kStride = kAngles / E;
    __device__ __forceinline__ float2 operator()(int i) const { return cs[(i % E) * kStride + i / E]; }
};

// rope_turn's two results from the table: the same operations.
__device__ __forceinline__ float rope_first(float2 v, float x1, float x2) { return __fmaf_rn(v.x, x1, __fmul_rn(v.y, x2)); }
__device__ __forceinline__ float rope_second(float2 v, float x1, float x2) { return __fmaf_rn(-v.y, x1, __fmul_rn(v.x, x2)); }

template <int E>
struct Unit {
    uint32_t w[E / 2];
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < E / 2; ++i) w[i] = 0;
    }
    __device__ __forceinline__ void load8(int i, const void *from)
    {
        const uint4 v = *static_cast<const uint4 *>(from);
        w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
    }
    __device__ __forceinline__ void load(const void *from)
    {
#pragma unroll
        for (int i = 0; i < E / 8; ++i) load8(i, static_cast<const uint4 *>(from) + i);
    }
    __device__ __forceinline__ uint4 quad(int i) const { return make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]); }
    template <typename T>
    __device__ __forceinline__ float get(int e) const { return to_f32<T>(reinterpret_cast<const T *>(&w[e / 2])[e % 2]); }
};

// A unit and its partner, turned: E angles for 2 E elements.
template <typename T, int E>
__device__ __forceinline__ void rotate_both(int d0, const AngleTable<E> &cs, Unit<E> &a, Unit<E> &b)
{
#pragma unroll
    for (int i = 0; i < E / 2; ++i) {
        float y1[2], y2[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const float x1 = a.template get<T>(2 * i + x), x2 = b.template get<T>(2 * i + x);
            const float2 v = cs.cs[(2 * i + x) * AngleTable<E>::kStride + d0 / E];
            y1[x] = rope_first(v, x1, x2);
            y2[x] = rope_second(v, x1, x2);
        }
        a.w[i] = pack_pair<T>(y1[0], y1[1]);
        b.w[i] = pack_pair<T>(y2[0], y2[1]);
    }
}

// The E elements from d0 on of a key row, rotated, in the type of the row (one
// rounding, as the rotation by itself gives).  Pairs of halves take their
// partners from the row again: as vectors of 8 (p) where those lie in one half,
// else one by one.
template <typename T, int E>
__device__ __forceinline__ void rotate_unit(const T *row, int d0, const quartz_rope_t &rope, const AngleTable<E> &cs,
                                            Unit<E> &u, const Unit<E> &p)
{
    const int pairs = rope.rotary / 2;
    float y[E];
    if (rope.interleaved) {
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            const float x1 = u.template get<T>(e), x2 = u.template get<T>(e + 1);
            y[e] = x1, y[e + 1] = x2;
            if (d0 + e < rope.rotary) {
                const float2 v = cs((d0 + e) / 2);
                y[e] = rope_first(v, x1, x2);
                y[e + 1] = rope_second(v, x1, x2);
            }
        }
    } else if (pairs % 8 == 0) {
        // one form for both halves: lanes of both share a warp
#pragma unroll
        for (int g = 0; g < E; g += 8) {
            const bool second = d0 + g >= pairs, turn = d0 + g < rope.rotary;
            const int i0 = second ? d0 + g - pairs : d0 + g;
            const float2 *mn = cs.cs + (second ? kAngles : 0) + (turn ? (i0 % E) * AngleTable<E>::kStride + i0 / E : 0);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float mine = u.template get<T>(g + e), other = p.template get<T>(g + e);
                const float r = rope_first(mn[e * AngleTable<E>::kStride], second ? other : mine, second ? mine : other);
                y[g + e] = turn ? r : mine;
            }
        }
    } else {
#pragma unroll 1
        for (int e = 0; e < E; ++e) {
            const int d = d0 + e;
            float v = to_f32<T>(row[d]);
            if (d < pairs) v = rope_first(cs(d), v, to_f32<T>(row[d + pairs]));
            else if (d < rope.rotary) v = rope_second(cs(d - pairs), to_f32<T>(row[d - pairs]), v);
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (i == e) y[i] = v;
        }
    }
#pragma unroll
    for (int i = 0; i < E / 2; ++i) u.w[i] = pack_pair<T>(y[2 * i], y[2 * i + 1]);
}

// A thread takes a unit of one token's keys and values in several heads, or
// (BOTH) a unit and the one half a row behind, its partners where whole heads
// are turned in halves; the head groups of a CTA share its tokens' angles.  Few
// tokens: keys and values by different CTAs (blockIdx.y).
// GS = 0: 16-bit pages of type T; else encoded pages (T = __half, four
// neighbouring lanes per 64-element group: dim is a multiple of 64, of 128 with
// BOTH).
// BOTH reads a pair's angle and elements once for both results instead of once
// for each, and keeps twice the bytes under way.  16384 tokens of 8 heads of
// 128, rotated: bf16 pages 23.1 us, 86% of the copy rate (36.9 without BOTH and
// with units of 16, whose 32 bytes per lane split every line between two
// loads; 24.2 with 5 CTAs per SM, 26.5 with 4; not rotated 20.0, 25.6 without
// BOTH); encoded 26.4 us (38.8 without BOTH; 10% more with 3 CTAs per SM, 7%
// with 5; 12.9 us of bytes), where warps wait in the encoder's chains: issue slots
// 72% busy, the logic pipe 57%.  64 registers leave 12 to 36 bytes of addresses
// spilled in the encoded instances, 40 up to 28 in the 16-bit ones without BOTH.
template <typename T, int GS, bool BOTH>
__global__ void __launch_bounds__(kAppendThreads, GS == 0 ? 6 : 4) paged_append_kernel(AppendCall c, int tokens)
{
    griddep_wait();
    constexpr int E = unit_size(GS != 0), N = BOTH ? 2 : 1;
    __shared__ float2 s_cs[(BOTH ? 1 : 2) * kAngles];
    const bool keys = gridDim.y == 1 || blockIdx.y == 0, values = gridDim.y == 1 || blockIdx.y == 1;
    const bool rope = c.a.rope.positions != nullptr && keys;
    const int pairs = rope ? c.a.rope.rotary / 2 : 0, per = (pairs + E - 1) / E;  // of the table's E lines, per token
    const int first = blockIdx.x * c.tokens_here;
    if (rope) {
        for (int i = threadIdx.x; i < c.tokens_here * pairs; i += blockDim.x) {
            const int n = i / pairs, j = i - n * pairs;
            if (first + n < tokens) {
                const float2 v = rope_cos_sin(c.a.rope.positions[first + n], rope_unit(c.a.rope.freqs[j]), c.a.rope.scale);
                float2 *to = s_cs + (j % E) * AngleTable<E>::kStride + n * per + j / E;
                to[0] = make_float2(v.x, -v.y);
                if (!BOTH) to[kAngles] = make_float2(v.y, v.x);
            }
        }
        __syncthreads();
    }
    const int places = c.tokens_here * c.units;
    const int group = threadIdx.x / places, place = threadIdx.x - group * places;
    const int n = place / c.units, u = place - n * c.units, lane = threadIdx.x & 31;
    const int t = first + n;
    int64_t slot = t < tokens && group < c.groups ? c.a.slots[t] : -1;
    if (slot >= c.slots_total) {
        atomicOr(c.a.dev_err, QUARTZ_DEV_INDEX);
        slot = -1;
    }
    const AngleTable<E> cs{s_cs + n * per};
    const int64_t page = slot >> c.page_shift, in_page = slot - (page << c.page_shift);
    const bool turn = E * u < 2 * pairs;
    const bool partners = turn && !c.a.rope.interleaved && pairs % 8 == 0;
    const T *k_row = static_cast<const T *>(c.a.k) + t * c.a.k_st + E * u, *v_row = static_cast<const T *>(c.a.v) + t * c.a.v_st + E * u;
    // encoded pages: unit of head 0; heads are page_size rows apart
    const int64_t unit0 = (((page * c.heads) << c.page_shift) + in_page) * (N * c.units) + u;
    auto store = [&](int side, int h, bool in, const Unit<E> &x, int i) {
        const AppendDst &d = c.dst[side];
        if constexpr (GS == 0) {
            if (in)
                *reinterpret_cast<uint4 *>(reinterpret_cast<T *>(d.data) + page * d.stride_page + in_page * d.stride_slot +
                                           h * d.stride_head + E * (u + i * c.units)) = x.quad(0);
        } else {
            const UnitCodes e = encode_unit_sym<GS>(x.quad(0), x.quad(1));
            if (in)
                store_unit_sym<GS>(e, unit0 + i * c.units + (static_cast<int64_t>(h * N * c.units) << c.page_shift), lane, d.codes,
                                   d.flags, d.scales, false);
        }
    };
    for (int k = 0; k < c.each; ++k) {  // the same trips for all lanes: encoding takes them together
        const int h = group + k * c.groups;
        const bool in = slot >= 0 && h < c.heads;
        const T *row = k_row + h * c.a.k_sh;
        Unit<E> x[2], y[N];
        x[0].clear(), x[1].clear(), y[0].clear(), y[N - 1].clear();
        if (keys && in) {
            x[0].load(row);
            if (BOTH) x[1].load(row + E * c.units);
            if (!BOTH && partners) {
#pragma unroll
                for (int i = 0; i < E / 8; ++i) {
                    const int d = E * u + 8 * i;
                    if (d < 2 * pairs) x[1].load8(i, row + 8 * i + (d < pairs ? pairs : -pairs));
                }
            }
        }
        if (values && in) {
#pragma unroll
            for (int i = 0; i < N; ++i) y[i].load(v_row + h * c.a.v_sh + i * E * c.units);
        }
        if (keys) {
            if (in && BOTH && rope) rotate_both<T, E>(E * u, cs, x[0], x[1]);
            if (in && !BOTH && turn) rotate_unit<T, E>(row - E * u, E * u, c.a.rope, cs, x[0], x[1]);
#pragma unroll
            for (int i = 0; i < N; ++i) store(0, h, in, x[i], i);
        }
        if (values) {
#pragma unroll
            for (int i = 0; i < N; ++i) store(1, h, in, y[i], i);
        }
    }
}

template <typename T, int GS>
cudaError_t launch_append(bool both, dim3 grid, dim3 block, cudaStream_t s, const AppendCall &c, int tokens)
{
    return both ? launch_pdl(paged_append_kernel<T, GS, true>, grid, block, 0, s, c, tokens)
                : launch_pdl(paged_append_kernel<T, GS, false>, grid, block, 0, s, c, tokens);
}

// ---------------------------------------------------------------------------
// Closing up
// ---------------------------------------------------------------------------

constexpr int kMoveThreads = 256;
constexpr int kMovePieces = 8;                       // pieces in flight per thread
constexpr int kMoveTile = 512;                       // most rows of a tile

// One array of the cache: a row of `row_bytes` per (page, slot, head), moved in
// pieces of `piece` bytes (1, 2, 4, 8 or 16).
struct Plane {
    uint8_t *base;
    int64_t stride_page, stride_slot, stride_head;  // bytes
    int piece, pieces;                               // pieces per slice of a row
    int slices;
};

struct MoveCall {
    Plane plane[6];
    int planes, parts, heads, page_shift;
    int64_t num_pages;
    bool in_place;
    CompactCall c;
};

__device__ __forceinline__ uint4 load_piece(const uint8_t *p, int bytes)
{
    uint4 v = make_uint4(0, 0, 0, 0);
    switch (bytes) {
        case 16: v = *reinterpret_cast<const uint4 *>(p); break;
        case 8: { const uint2 w = *reinterpret_cast<const uint2 *>(p); v.x = w.x, v.y = w.y; break; }
        case 4: v.x = *reinterpret_cast<const uint32_t *>(p); break;
        case 2: v.x = *reinterpret_cast<const uint16_t *>(p); break;
        default: v.x = *p; break;
    }
    return v;
}

__device__ __forceinline__ void store_piece(uint8_t *p, const uint4 v, int bytes)
{
    switch (bytes) {
        case 16: *reinterpret_cast<uint4 *>(p) = v; break;
        case 8: *reinterpret_cast<uint2 *>(p) = make_uint2(v.x, v.y); break;
        case 4: *reinterpret_cast<uint32_t *>(p) = v.x; break;
        case 2: *reinterpret_cast<uint16_t *>(p) = static_cast<uint16_t>(v.x); break;
        default: *p = static_cast<uint8_t>(v.x); break;
    }
}

// blockIdx.x = (sequence x head) * parts + part, blockIdx.y = plane (the one
// behind the last is the weights').  A tile of rows at a time: first a thread
// per row follows its kept index and the tables to the two addresses, then all
// threads move pieces, eight loads in flight each; so the dependent reads are
// paid once per tile and row, not per piece, and for the next tile while this
// one's loads are under way (16 x 8 heads, up to 4096 rows of 2 x 256 bytes:
// 77 us, 91% of the copy rate; followed per piece 97).  Into new pages, a part is a
// range of rows; in place it is a slice of every row, and the CTA goes through
// the rows in order: row j is written after all rows up to its tile's last are
// read (a barrier per tile), and rows after them come from places behind the
// tile (the kept indices ascend, so kept[j] >= j), which no earlier tile
// writes.
__global__ void __launch_bounds__(kMoveThreads) cache_compact_kernel(MoveCall m)
{
    griddep_wait();
    __shared__ uint8_t *s_from[2][kMoveTile], *s_to[2][kMoveTile];
    const int64_t bh = blockIdx.x / m.parts;
    const int part = static_cast<int>(blockIdx.x - bh * m.parts);
    const int64_t b = bh / m.heads;
    const int h = static_cast<int>(bh - b * m.heads);
    int64_t len = m.c.lens[b];
    if (len < 0 || len > m.c.max_len) {
        if (threadIdx.x == 0) atomicOr(m.c.dev_err, QUARTZ_DEV_INDEX);
        len = len < 0 ? 0 : m.c.max_len;
    }
    const int64_t rows = len < m.c.budget ? len : m.c.budget;
    const int32_t *kept = m.c.kept + bh * m.c.budget;
    const int32_t *from_table = m.c.table + b * m.c.table_stride;
    const int32_t *to_table = m.c.new_table ? m.c.new_table + b * m.c.new_table_stride : from_table;
    const int64_t page_mask = (int64_t(1) << m.page_shift) - 1;

    if (blockIdx.y == m.planes) {  // the sums of attention weights, in place
        if (part != 0) return;
        float *w = m.c.weights + b * m.c.w_sb + h * m.c.w_sh;
        for (int64_t j0 = 0; j0 < rows; j0 += kMoveThreads * kMovePieces) {
            float v[kMovePieces];
#pragma unroll
            for (int r = 0; r < kMovePieces; ++r) {
                const int64_t j = j0 + r * kMoveThreads + threadIdx.x;
                v[r] = 0.f;
                if (j < rows) {
                    const int64_t src = kept[j];
                    if (src >= 0 && src < len) v[r] = w[src];
                }
            }
            __syncthreads();
#pragma unroll
            for (int r = 0; r < kMovePieces; ++r) {
                const int64_t j = j0 + r * kMoveThreads + threadIdx.x;
                if (j < rows) w[j] = v[r];
            }
        }
        __syncthreads();
        for (int64_t j = rows + threadIdx.x; j < len; j += kMoveThreads) w[j] = 0.f;
        return;
    }

    const Plane &p = m.plane[blockIdx.y];
    int64_t first = 0, last = rows;
    int slice = 0;
    if (m.in_place) {
        if (part >= p.slices) return;
        slice = part;
    } else {
        const int64_t per = (rows + m.parts - 1) / m.parts;
        first = per * part;
        last = first + per < rows ? first + per : rows;
    }
    uint8_t *base = p.base + h * p.stride_head + static_cast<int64_t>(slice) * p.pieces * p.piece;
    const int tile_rows = min(kMoveTile, kMoveThreads * kMovePieces / p.pieces);
    // a thread's places in a tile, the same in all of them
    int row[kMovePieces], at[kMovePieces];
#pragma unroll
    for (int r = 0; r < kMovePieces; ++r) {
        const int i = r * kMoveThreads + threadIdx.x;
        row[r] = i / p.pieces;
        at[r] = (i - row[r] * p.pieces) * p.piece;
    }
    bool bad = false;
    auto addresses = [&](int64_t j0, int buffer) {
        for (int i = threadIdx.x; i < tile_rows && j0 + i < last; i += kMoveThreads) {
            const int64_t j = j0 + i, src = kept[j];
            uint8_t *from = nullptr, *to = nullptr;
            if (src < 0 || src >= len) {
                bad = true;
            } else if (!(m.in_place && src == j)) {
                const int64_t sp = from_table[src >> m.page_shift], dp = to_table[j >> m.page_shift];
                if (sp < 0 || sp >= m.num_pages || dp < 0 || dp >= m.num_pages) {
                    bad = true;
                } else {
                    from = base + sp * p.stride_page + (src & page_mask) * p.stride_slot;
                    to = base + dp * p.stride_page + (j & page_mask) * p.stride_slot;
                }
            }
            s_from[buffer][i] = from;
            s_to[buffer][i] = to;
        }
    };
    addresses(first, 0);
    __syncthreads();
    int buffer = 0;
    for (int64_t j0 = first; j0 < last; j0 += tile_rows, buffer ^= 1) {
        const int n = last - j0 < tile_rows ? static_cast<int>(last - j0) : tile_rows;
        uint4 v[kMovePieces];
#pragma unroll
        for (int r = 0; r < kMovePieces; ++r)
            if (row[r] < n && s_from[buffer][row[r]]) v[r] = load_piece(s_from[buffer][row[r]] + at[r], p.piece);
        addresses(j0 + tile_rows, buffer ^ 1);  // the next tile's, while the loads are under way
        if (m.in_place) __syncthreads();
#pragma unroll
        for (int r = 0; r < kMovePieces; ++r)
            if (row[r] < n && s_to[buffer][row[r]]) store_piece(s_to[buffer][row[r]] + at[r], v[r], p.piece);
        __syncthreads();
    }
    if (bad) atomicOr(m.c.dev_err, QUARTZ_DEV_INDEX);
}

int piece_of(int64_t row_bytes)
{
    int p = 16;
    while (row_bytes % p != 0) p /= 2;
    return p;
}

}  // namespace

cudaError_t launch_paged_append(const quartz_paged_cache_t *c, const AppendArgs &a, int64_t tokens, cudaStream_t s)
{
    AppendCall call;
    call.a = a;
    const quartz_pages_t *side[2] = {&c->k, &c->v};
    for (int i = 0; i < 2; ++i) {
        AppendDst &d = call.dst[i];
        d.data = static_cast<uint8_t *>(side[i]->data);
        d.stride_page = side[i]->stride_page;
        d.stride_slot = side[i]->stride_slot;
        d.stride_head = side[i]->stride_head;
        d.codes = reinterpret_cast<uint2 *>(side[i]->enc.codes);
        d.flags = side[i]->enc.flags;
        d.scales = reinterpret_cast<__half *>(side[i]->enc.scales);
    }
    call.page_shift = log2_of(c->page_size);
    call.slots_total = c->num_pages << call.page_shift;
    call.heads = c->heads;
    const bool encoded = c->type == QUARTZ_PAGES_ENCODED;
    call.units = c->dim / unit_size(encoded);
    // By the elements per SM.  Few: keys and values by different CTAs, a token
    // each.  2048: both by one, and BOTH, and several tokens where they leave four
    // CTAs per SM (a power of two of them times 4 to 32 units keeps a CTA's warps
    // full).  32768: a thread takes two heads.  In a graph, heads of 128, encoded /
    // bf16: 16384 tokens of one head 11.6 / 9.1 us (39.7 / 28.3 as few), 4096 of 8
    // 7.7 / 6.2 (13.4 / 12.3; with two CTAs per SM 8.5 / 6.2), 4096 of one 6.8 / 4.8
    // (11.8 / 8.6, and the same from 4096 elements on), 256 of 8 3.1 / 2.9.
    const int sms = device_sms();
    const int64_t per_sm = tokens * call.heads * c->dim / sms;
    const bool some = per_sm >= 2048, many = per_sm >= 32768;
    const bool both = some && (!a.rope.positions || (!a.rope.interleaved && a.rope.rotary == c->dim)) && (!encoded || c->dim % 128 == 0);
    if (both) call.units /= 2;
    int groups = many ? (call.heads + 1) / 2 : call.heads;
    if (groups > kAppendThreads / call.units) groups = kAppendThreads / call.units;
    int n = 1;
    while (some && 2 * n <= kAppendTokens && 2 * n * call.units * groups <= kAppendThreads && tokens >= 2 * n * 4 * sms) n *= 2;
    call.tokens_here = n;
    call.groups = groups;
    call.each = (call.heads + groups - 1) / groups;
    const int threads = n * call.units * groups;  // a multiple of 4
    const dim3 grid(static_cast<unsigned>((tokens + n - 1) / n), some ? 1 : 2), block((threads + 31) & ~31);
    const int total = static_cast<int>(tokens);
    if (c->type == QUARTZ_PAGES_F16) return launch_append<__half, 0>(both, grid, block, s, call, total);
    if (c->type == QUARTZ_PAGES_BF16) return launch_append<__nv_bfloat16, 0>(both, grid, block, s, call, total);
    switch (c->k.enc.p.group_s) {
        case 8: return launch_append<__half, 8>(both, grid, block, s, call, total);
        case 16: return launch_append<__half, 16>(both, grid, block, s, call, total);
        case 32: return launch_append<__half, 32>(both, grid, block, s, call, total);
        default: return launch_append<__half, 64>(both, grid, block, s, call, total);
    }
}

cudaError_t launch_cache_compact(const quartz_paged_cache_t *c, const CompactCall &a, cudaStream_t s)
{
    MoveCall m;
    m.c = a;
    m.heads = c->heads;
    m.page_shift = log2_of(c->page_size);
    m.num_pages = c->num_pages;
    m.in_place = a.new_table == nullptr;
    m.planes = 0;
    const int64_t bh = a.seqs * c->heads, sms = device_sms();
    const quartz_pages_t *side[2] = {&c->k, &c->v};
    auto add = [&](void *base, int64_t row_bytes, int64_t sp, int64_t ss, int64_t sh) {
        Plane &p = m.plane[m.planes++];
        p.base = static_cast<uint8_t *>(base);
        p.stride_page = sp, p.stride_slot = ss, p.stride_head = sh;
        p.piece = piece_of(row_bytes);
        p.pieces = static_cast<int>(row_bytes / p.piece);
        p.slices = 1;
        // in place, slices of a row (of 64 bytes or more) are what there is to
        // spread over the SMs beside sequences and heads
        if (m.in_place)
            while (bh * 2 * p.slices < 2 * sms && p.pieces % 2 == 0 && p.pieces * p.piece > 64) p.pieces /= 2, p.slices *= 2;
    };
    for (int i = 0; i < 2; ++i) {
        if (c->type == QUARTZ_PAGES_ENCODED) {
            const quartz_encoded_t &e = side[i]->enc;
            const int64_t bytes[3] = {c->dim / 2, c->dim / e.p.group_s, c->dim / 32};
            void *base[3] = {e.codes, e.flags, e.scales};
            for (int j = 0; j < 3; ++j)
                add(base[j], bytes[j], bytes[j] * c->heads * c->page_size, bytes[j], bytes[j] * c->page_size);
        } else {
            add(side[i]->data, 2 * c->dim, 2 * side[i]->stride_page, 2 * side[i]->stride_slot, 2 * side[i]->stride_head);
        }
    }
    m.parts = 1;
    if (m.in_place) {
        for (int i = 0; i < m.planes; ++i) m.parts = m.plane[i].slices > m.parts ? m.plane[i].slices : m.parts;
    } else {
        const int64_t rows = a.budget < a.max_len ? a.budget : a.max_len;
        const int64_t tile = kMoveThreads * kMovePieces * 16 / (2 * c->dim), most = (rows + tile - 1) / tile;
        int64_t want = (8 * sms + bh * 2 - 1) / (bh * 2);
        if (want > most) want = most;
        m.parts = want < 1 ? 1 : static_cast<int>(want);
    }
    const dim3 grid(static_cast<unsigned>(bh * m.parts), static_cast<unsigned>(m.planes + (a.weights ? 1 : 0)));
    return launch_pdl(cache_compact_kernel, grid, dim3(kMoveThreads), 0, s, m);
}

}  // namespace quartz
