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
constexpr int kMaxPairs = 128;  // dim <= 256

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
    int page_shift, heads, units;  // units of 16 elements per row
};

template <typename T>
__device__ __forceinline__ void unpack16(const uint4 lo, const uint4 hi, float (&f)[16])
{
    const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const T *p = reinterpret_cast<const T *>(&w[i]);
        f[2 * i] = to_f32<T>(p[0]);
        f[2 * i + 1] = to_f32<T>(p[1]);
    }
}

template <typename T>
__device__ __forceinline__ void pack16(const float (&f)[16], uint4 &lo, uint4 &hi)
{
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        T *p = reinterpret_cast<T *>(&w[i]);
        p[0] = from_f32<T>(f[2 * i]);
        p[1] = from_f32<T>(f[2 * i + 1]);
    }
    lo = make_uint4(w[0], w[1], w[2], w[3]);
    hi = make_uint4(w[4], w[5], w[6], w[7]);
}

// A lane's unit of a row: 16 elements, and for keys that are rotated in halves
// their 16 partners (read again as vectors where the unit lies in one half).
struct RawUnit {
    uint4 lo, hi, plo, phi;
};

// The 16 elements d0 .. d0 + 15 of a key row, rotated, in the type of the row
// (one rounding, as the rotation by itself gives).
template <typename T>
__device__ __forceinline__ void rotate_unit(const T *row, int d0, const quartz_rope_t &rope, const float2 *cs, RawUnit &r)
{
    const int pairs = rope.rotary / 2;
    float x[16], y[16];
    unpack16<T>(r.lo, r.hi, x);
    if (rope.interleaved) {
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            y[e] = x[e], y[e + 1] = x[e + 1];
            if (d0 + e < rope.rotary) {
                const float2 v = rope_turn(x[e], x[e + 1], cs[(d0 + e) / 2]);
                y[e] = v.x, y[e + 1] = v.y;
            }
        }
    } else if (pairs % 16 == 0) {
        float p[16];
        unpack16<T>(r.plo, r.phi, p);
        if (d0 < pairs) {
#pragma unroll
            for (int e = 0; e < 16; ++e) y[e] = rope_turn(x[e], p[e], cs[d0 + e]).x;
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) y[e] = rope_turn(p[e], x[e], cs[d0 - pairs + e]).y;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int d = d0 + e;
            y[e] = x[e];
            if (d < pairs) y[e] = rope_turn(x[e], to_f32<T>(row[d + pairs]), cs[d]).x;
            else if (d < rope.rotary) y[e] = rope_turn(to_f32<T>(row[d - pairs]), x[e], cs[d - pairs]).y;
        }
    }
    pack16<T>(y, r.lo, r.hi);
}

// A CTA goes through tokens; a lane has the same 16 elements of a key or value
// row in all of them (blockIdx.y: further rows), and loads the next token's
// while it works on this one's.  GS = 0: 16-bit pages of type T; else encoded
// pages (T = __half, four lanes per 64-element group, which never cross a row:
// dim is a multiple of 64).
template <typename T, int GS>
__global__ void __launch_bounds__(kAppendThreads) paged_append_kernel(AppendCall c, int tokens)
{
    griddep_wait();
    __shared__ float2 s_cs[2][kMaxPairs];
    __shared__ uint64_t s_unit[kMaxPairs];
    const bool rope = c.a.rope.positions != nullptr;
    const int pairs = rope ? c.a.rope.rotary / 2 : 0;
    for (int i = threadIdx.x; i < pairs; i += blockDim.x) s_unit[i] = rope_unit(c.a.rope.freqs[i]);

    const int side_units = c.heads * c.units, lane = threadIdx.x & 31;
    const int item = blockIdx.y * blockDim.x + threadIdx.x;
    const bool in = item < 2 * side_units;
    const int side = in && item >= side_units;
    const int r = in ? item - side * side_units : 0;
    const int h = r / c.units, u = r - h * c.units;
    const T *src = side ? static_cast<const T *>(c.a.v) + h * c.a.v_sh : static_cast<const T *>(c.a.k) + h * c.a.k_sh;
    const int64_t st = side ? c.a.v_st : c.a.k_st;
    const bool turn = rope && !side && 16 * u < 2 * pairs;
    const bool partners = turn && !c.a.rope.interleaved && pairs % 16 == 0;
    const int partner = 16 * u < pairs ? pairs : -pairs;
    const AppendDst &d = c.dst[side];

    RawUnit next;
    auto load = [&](int64_t t) {
        const T *row = src + t * st + 16 * u;
        next.lo = reinterpret_cast<const uint4 *>(row)[0];
        next.hi = reinterpret_cast<const uint4 *>(row)[1];
        if (partners) {
            next.plo = reinterpret_cast<const uint4 *>(row + partner)[0];
            next.phi = reinterpret_cast<const uint4 *>(row + partner)[1];
        }
    };
    int64_t t = blockIdx.x;
    int64_t slot = c.a.slots[t], pos = rope ? c.a.rope.positions[t] : 0;
    load(t);
    __syncthreads();  // s_unit
    for (int buffer = 0; t < tokens; buffer ^= 1) {
        for (int i = threadIdx.x; i < pairs; i += blockDim.x) s_cs[buffer][i] = rope_cos_sin(pos, s_unit[i], c.a.rope.scale);
        RawUnit now = next;
        const int64_t to = slot;
        const T *row = src + t * st;
        t += gridDim.x;
        if (t < tokens) {
            slot = c.a.slots[t];
            if (rope) pos = c.a.rope.positions[t];
            load(t);
        }
        if (rope) __syncthreads();  // the angles; the other buffer's readers are past the barrier before
        if (to < 0) continue;
        if (to >= c.slots_total) {
            if (threadIdx.x == 0) atomicExch(c.a.dev_err, QUARTZ_DEV_INDEX);
            continue;
        }
        if (turn) rotate_unit<T>(row, 16 * u, c.a.rope, s_cs[buffer], now);
        const int64_t page = to >> c.page_shift, in_page = to - (page << c.page_shift);
        if constexpr (GS == 0) {
            if (in) {
                T *p = reinterpret_cast<T *>(d.data) + page * d.stride_page + in_page * d.stride_slot + h * d.stride_head;
                reinterpret_cast<uint4 *>(p)[2 * u] = now.lo;
                reinterpret_cast<uint4 *>(p)[2 * u + 1] = now.hi;
            }
        } else {
            const UnitCodes e = encode_unit_sym<GS>(now.lo, now.hi);
            const int64_t dst_row = ((page * c.heads + h) << c.page_shift) + in_page;
            if (in) store_unit_sym<GS>(e, dst_row * c.units + u, lane, d.codes, d.flags, d.scales, false);
        }
    }
}

int log2_of(int v)
{
    int n = 0;
    while ((1 << n) < v) ++n;
    return n;
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
// paid once per tile and row, not per piece.  Into new pages, a part is a
// range of rows; in place it is a slice of every row, and the CTA goes through
// the rows in order: row j is written after all rows up to its tile's last are
// read (a barrier per tile), and rows after them come from places behind the
// tile (the kept indices ascend, so kept[j] >= j), which no earlier tile
// writes.
__global__ void __launch_bounds__(kMoveThreads) cache_compact_kernel(MoveCall m)
{
    griddep_wait();
    __shared__ uint8_t *s_from[kMoveTile], *s_to[kMoveTile];
    const int64_t bh = blockIdx.x / m.parts;
    const int part = static_cast<int>(blockIdx.x - bh * m.parts);
    const int64_t b = bh / m.heads;
    const int h = static_cast<int>(bh - b * m.heads);
    int64_t len = m.c.lens[b];
    if (len < 0 || len > m.c.max_len) {
        if (threadIdx.x == 0) atomicExch(m.c.dev_err, QUARTZ_DEV_INDEX);
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
    for (int64_t j0 = first; j0 < last; j0 += tile_rows) {
        const int n = last - j0 < tile_rows ? static_cast<int>(last - j0) : tile_rows;
        for (int i = threadIdx.x; i < n; i += kMoveThreads) {
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
            s_from[i] = from;
            s_to[i] = to;
        }
        __syncthreads();
        uint4 v[kMovePieces];
#pragma unroll
        for (int r = 0; r < kMovePieces; ++r)
            if (row[r] < n && s_from[row[r]]) v[r] = load_piece(s_from[row[r]] + at[r], p.piece);
        if (m.in_place) __syncthreads();
#pragma unroll
        for (int r = 0; r < kMovePieces; ++r)
            if (row[r] < n && s_to[row[r]]) store_piece(s_to[row[r]] + at[r], v[r], p.piece);
        __syncthreads();  // the next tile's addresses
    }
    if (bad) atomicExch(m.c.dev_err, QUARTZ_DEV_INDEX);
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
    call.units = c->dim / 16;
    const int total = 2 * call.heads * call.units;
    const int threads = total < kAppendThreads ? (total + 31) & ~31 : kAppendThreads;
    const int y = (total + threads - 1) / threads;
    int64_t x = (152 * (2048 / threads) + y - 1) / y;  // what fits the SMs; each CTA has several tokens where there are more
    if (x > tokens) x = tokens;
    const dim3 grid(static_cast<unsigned>(x), static_cast<unsigned>(y)), block(threads);
    const int n = static_cast<int>(tokens);
    if (c->type == QUARTZ_PAGES_F16) return launch_pdl(paged_append_kernel<__half, 0>, grid, block, 0, s, call, n);
    if (c->type == QUARTZ_PAGES_BF16) return launch_pdl(paged_append_kernel<__nv_bfloat16, 0>, grid, block, 0, s, call, n);
    switch (c->k.enc.p.group_s) {
        case 8: return launch_pdl(paged_append_kernel<__half, 8>, grid, block, 0, s, call, n);
        case 16: return launch_pdl(paged_append_kernel<__half, 16>, grid, block, 0, s, call, n);
        case 32: return launch_pdl(paged_append_kernel<__half, 32>, grid, block, 0, s, call, n);
        default: return launch_pdl(paged_append_kernel<__half, 64>, grid, block, 0, s, call, n);
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
    const int64_t bh = a.seqs * c->heads;
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
            while (bh * 2 * p.slices < 304 && p.pieces % 2 == 0 && p.pieces * p.piece > 64) p.pieces /= 2, p.slices *= 2;
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
        int64_t want = (152 * 8 + bh * 2 - 1) / (bh * 2), most = (rows + 127) / 128;
        if (want > most) want = most;
        m.parts = want < 1 ? 1 : static_cast<int>(want);
    }
    const dim3 grid(static_cast<unsigned>(bh * m.parts), static_cast<unsigned>(m.planes + (a.weights ? 1 : 0)));
    return launch_pdl(cache_compact_kernel, grid, dim3(kMoveThreads), 0, s, m);
}

}  // namespace quartz
