// Attention of several new tokens per sequence (prompts, chunks of prompts,
// trees of drafted tokens) over a paged cache, on the 5th-generation tensor
// cores:
//   s = scale q . k, capped, less slope x distance;  p = softmax over the tokens
//   seen;  o = sum p v
// in one pass over the keys with the running maximum m and sum l.
//
// Rows are (new token, query head) pairs of one key / value head, 128 to a tile:
// the query heads that share a key head share its loads and fill the tile when
// tokens are few.  A CTA takes one tile, or two side by side, and goes over the
// sequence's keys 128 at a time:
//   S = Q K'    tcgen05.mma from shared memory, 128 x 128 binary32 in TMEM
//   P           by the softmax warps, in one or two parts of 16 bits, over S in TMEM
//   O += P V    tcgen05.mma, P from TMEM, V as it lies (MN-major)
// While the softmax warps work on one S the tensor cores make the other.  There
// are two softmax warpgroups, a thread per row: two tiles have one each; with one
// tile they take its keys in turn and hand the maximum on as soon as it is known.
// O stays in TMEM; it is rescaled only when a maximum rises by more than `slack`,
// so hardly ever.
//
// Warps: 8 softmax; 4 or 8 that fill a ring of [128 tokens x 64 or 128 dimensions]
// units, keys and values in turn, from the pages (TMA or 16-byte copies, into the
// 128-byte swizzle; encoded pages: decoded to fp16 on the way); one that issues
// the products; three that load queries.
//
// The keys of all rows' tiles, one behind the other, are cut into one run of
// equal work per CTA (one CTA per SM), so that lengths, windows and the causal
// edge leave no SM idle; a block of rows counts some tiles more than it has, for
// its queries, masks and results.  Blocks that a cut goes through are joined by
// a second kernel, in the order of the keys.
//
// What bounds it, and what was measured.  Two tiles of 128 keys and dimensions take
// the tensor cores 2048 cycles and the exponentials, at 4 cycles a warp and
// instruction, 1024 of each scheduler; in long runs an iteration takes some 2700
// (1024 tokens over 65536, 32 / 8 heads, bf16: 735-753 us, 1450-1480 TFLOP/s of
// 1950), the rest waits between product, softmax and product.  Causal prompts of
// 8192: 380-400 us, their ends of blocks among it, and the join 15 (a call 400-425,
// 1320 TFLOP/s).  Steps on the kernel (us): 637 with
// 16-byte copies and scores read twice; 556 by TMA; 474 with queries by TMA and
// instances without what plain scores do not need (code for it in the same loop:
// 556, a quarter of the active time waiting for instructions); 457 with results
// through shared memory; 379 with blocks' ends counted in the cut.  Heads of 256
// (128 KB of keys and values for 128 rows): 749 us for 1024 tokens over 32768 with
// whole units in the order keys, values; 516 in the order of the products.
// Encoded pages wait for what is decoded: 100 instructions for 32 elements of a row
// (in four warps 255 us where eight take 217, trees of 61 over up to 65536), but issue
// slots are half busy only; codes on their way, a unit ahead, are waited for most.
// Every instance spills, 260 to 510 bytes of stores a thread: some 0.6% of the
// instructions that run.
#pragma once

#include <cuda.h>

#include "lzs_f16.cuh"
#include "paged_attention.cuh"

namespace quartz {

constexpr int kTokSoftmaxWarps = 8;
constexpr int kTokQueryWarps = 3;
constexpr int kTokMostWarps = 20;
constexpr int kTokKeys = 128;  // keys of a tile
constexpr int kTokTreeMost = 64;

struct TokensArgs {
    const uint16_t *q;
    int64_t q_st, q_sh;
    const int32_t *table;
    int64_t table_stride;
    const int32_t *lens, *starts;
    const uint64_t *tree;    // NULL: causal
    const int32_t *prefix;   // NULL: none
    const float *slopes;     // NULL: none
    PagedSide k, v;
    uint32_t num_pages;
    int page_shift, kv_heads, group, seqs, tokens, max_len, max_new, window, gs_shift;
    // 16-bit pages of 8 tokens or more that a tensor map describes: rows of a box
    // (0: none), and which of the map's dimensions 1 .. 3 head, slot and page are
    int box_rows;
    int k_order, v_order;
    int q_box;  // a box of the queries' map is a tile's rows and 64 dimensions
    int single;              // no sequence has more rows than one CTA takes
    int uncut;               // a CTA per block of rows: no block is cut, and nothing joined
    int cap_near;            // the powers of to_cap fit binary32: the cap's short polynomial may be used
    float scale_log2;
    float cap_log2, to_cap;  // cap > 0: cap log2 e and scale / cap; else 0
    void *o;
    int o_type;
    float *part_o;           // [CTA][2][rows][dim]: first (0) or last (1) tile of a CTA, cut
    float2 *part_ml;         // [CTA][2][rows]: maximum (log2 domain) and sum
    struct TokensJoin *joins;  // [CTA]
    int *dev_err;
};

// A CTA whose last tile goes on in the next CTAs: what the join needs.
struct TokensJoin {
    int parts;  // 0: nothing to join
    int token0, row0, rows, head0;  // rows row0 .. + rows of tokens from token0 on
};

struct TokensSeq {
    int n, m, start, base, pre;  // cached, new (0: nothing to do), first row of q, n - m, prefix
};

__device__ __forceinline__ TokensSeq tokens_seq(const TokensArgs &a, int b)
{
    TokensSeq s;
    const int s1 = a.starts[b + 1];
    s.start = a.starts[b];
    s.n = a.lens[b];
    s.m = s1 - s.start;
    if (s.start < 0 || s1 < s.start || s1 > a.tokens || s.m > a.max_new || s.n > a.max_len || s.n < s.m) {
        atomicOr(a.dev_err, QUARTZ_DEV_INDEX);
        s.n = s.m = s.start = 0;
    }
    s.base = s.n - s.m;
    s.pre = a.prefix ? max(0, min(a.prefix[b], s.n)) : 0;
    return s;
}

// What the rows of a block see: [0, pre) and [lo, hi], as `lead` tiles from 0
// and the rest from tile `first`.
struct TokensTiles {
    int lo, hi, lead, first, count;
    __device__ __forceinline__ int at(int i) const { return i < lead ? i : first + i - lead; }
};

template <int R>
__device__ __forceinline__ TokensTiles tokens_tiles(const TokensArgs &a, const TokensSeq &s, int block)
{
    TokensTiles t;
    const int j0 = block * R / a.group, j1 = min(s.m - 1, (block * R + (R - 1)) / a.group);
    t.lo = a.window > 0 ? max(0, s.base + (a.tree ? 0 : j0) - a.window + 1) : 0;
    t.hi = s.base + (a.tree ? s.m - 1 : j1);
    t.lead = (s.pre + kTokKeys - 1) / kTokKeys;
    t.first = max(t.lead, t.lo / kTokKeys);
    t.count = t.lead + max(0, t.hi / kTokKeys - t.first + 1);
    return t;
}

template <int R>
__device__ __forceinline__ int tokens_blocks(const TokensArgs &a, const TokensSeq &s) { return (s.m * a.group + R - 1) / R; }

// Tiles and row blocks of one key head of 32 sequences from b0 on (to b1), each
// in its lane.  Tiles of a sequence pass 32 bits: m tokens of `group` heads have some
// m^2 group / 2^16 (2^15 where a CTA takes one tile).
struct TokensCount {
    long long tiles;
    int blocks;
};

template <int R>
__device__ __forceinline__ TokensCount tokens_seq_tiles(const TokensArgs &a, int b0, int b1)
{
    const int lane = threadIdx.x & 31;
    TokensSeq s{};
    if (b0 + lane < b1) s = tokens_seq(a, b0 + lane);
    if (a.single) return s.m > 0 ? TokensCount{tokens_tiles<R>(a, s, 0).count, 1} : TokensCount{0, 0};
    TokensCount mine{0, tokens_blocks<R>(a, s)};
    for (int i = 0; i < min(32, b1 - b0); ++i) {
        TokensSeq t;
        t.n = __shfl_sync(0xffffffffu, s.n, i), t.m = __shfl_sync(0xffffffffu, s.m, i);
        t.pre = __shfl_sync(0xffffffffu, s.pre, i), t.base = t.n - t.m, t.start = 0;
        long long sum = 0;
        for (int r = lane; r < tokens_blocks<R>(a, t); r += 32) sum += tokens_tiles<R>(a, t, r).count;
#pragma unroll
        for (int d = 16; d; d /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (lane == i) mine.tiles = sum;
    }
    return mine;
}

struct TokensPlace {
    int b, head, block, off;
};

struct TokensFind {
    long long tiles[kTokMostWarps], blocks[kTokMostWarps];
    TokensPlace at;
};

// What a CTA takes: [pos, end) of all work, in tiles.
struct TokensRun {
    long long pos, end, chunk;
    int edge;  // tiles that a block of rows counts for besides its own
};

// Most of a block's edge: it costs as much as 3 tiles.  Less where a CTA has few
// tiles (a quarter of them), so that none has edges alone.
constexpr int kTokEdge = 3;

// Of all tiles of all sequences, heads and row blocks, in that order, this CTA's
// run, which begins at `at`.  (All threads of the CTA.)  False: none.
template <int R>
__device__ bool tokens_find(const TokensArgs &a, TokensFind &f, TokensRun &run)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    const int share = (a.seqs + warps - 1) / warps;
    const int b0 = min(a.seqs, warp * share), b1 = min(a.seqs, b0 + share);
    long long tiles = 0, blocks = 0;
    for (int b = b0; b < b1; b += 32) {
        const TokensCount n = tokens_seq_tiles<R>(a, b, b1);
        long long t = n.tiles, k = n.blocks;
#pragma unroll
        for (int d = 16; d; d /= 2) t += __shfl_xor_sync(0xffffffffu, t, d), k += __shfl_xor_sync(0xffffffffu, k, d);
        tiles += t, blocks += k;
    }
    if (lane == 0) f.tiles[warp] = tiles * a.kv_heads, f.blocks[warp] = blocks * a.kv_heads;
    __syncthreads();
    long long all_tiles = 0, all_blocks = 0, before = 0;
    for (int w = 0; w < warps; ++w) all_tiles += f.tiles[w], all_blocks += f.blocks[w];
    run.edge = static_cast<int>(min(static_cast<long long>(kTokEdge), all_tiles / (4 * gridDim.x)));
    const int each = a.uncut ? 0 : 1;  // what a tile counts; uncut: blocks are counted instead
    if (a.uncut) run.edge = 1;
    for (int w = 0; w < warp; ++w) before += each * f.tiles[w] + run.edge * f.blocks[w];
    const long long all = each * all_tiles + run.edge * all_blocks, mine_all = (each * tiles + run.edge * blocks) * a.kv_heads;
    run.chunk = (all + gridDim.x - 1) / gridDim.x;
    const long long pos = run.pos = run.chunk * blockIdx.x;
    run.end = min(pos + run.chunk, all);
    if (pos < run.end && pos >= before && pos < before + mine_all) {
        for (int b = b0; b < b1; b += 32) {
            const TokensCount n = tokens_seq_tiles<R>(a, b, b1);
            const long long mine = each * n.tiles + static_cast<long long>(run.edge) * n.blocks;
            long long incl = mine;
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const long long v = __shfl_up_sync(0xffffffffu, incl, d);
                if (lane >= d) incl += v;
            }
            const unsigned behind = __ballot_sync(0xffffffffu, pos < before + incl * a.kv_heads);
            if (!behind) {
                before += __shfl_sync(0xffffffffu, incl, 31) * a.kv_heads;
                continue;
            }
            const int i = __ffs(behind) - 1;
            const long long per_head = __shfl_sync(0xffffffffu, mine, i);
            const long long in = pos - before - (__shfl_sync(0xffffffffu, incl, i) - per_head) * a.kv_heads;
            TokensPlace p;
            p.b = b + i;
            p.head = static_cast<int>(in / per_head);
            long long rest = in - p.head * per_head;
            const TokensSeq s = tokens_seq(a, p.b);
            const int blocks = tokens_blocks<R>(a, s);  // of this sequence
            for (int r0 = 0; r0 < blocks; r0 += 32) {
                const int n = r0 + lane < blocks ? each * tokens_tiles<R>(a, s, r0 + lane).count + run.edge : 0;
                int sums = n;
#pragma unroll
                for (int d = 1; d < 32; d *= 2) {
                    const int v = __shfl_up_sync(0xffffffffu, sums, d);
                    if (lane >= d) sums += v;
                }
                const unsigned here = __ballot_sync(0xffffffffu, rest < sums);
                if (here) {
                    const int j = __ffs(here) - 1;
                    p.block = r0 + j;
                    p.off = static_cast<int>(rest) - __shfl_sync(0xffffffffu, sums - n, j);
                    break;
                }
                rest -= __shfl_sync(0xffffffffu, sums, 31);
            }
            if (lane == 0) f.at = p;
            break;
        }
    }
    __syncthreads();
    return pos < run.end;
}

// A CTA's way over its run: one row block and tiles [first, first + count) of it
// at a time.  Every warp goes it for itself.
template <int R>
struct TokensWalk {
    const TokensArgs &a;
    const TokensRun &run;
    long long pos;
    TokensPlace p;
    TokensSeq s;
    TokensTiles t;
    int span, first, count;

    __device__ __forceinline__ TokensWalk(const TokensArgs &args, const TokensPlace &at, const TokensRun &r)
        : a(args), run(r), pos(r.pos), p(at)
    {
        s = tokens_seq(a, p.b);
        enter();
    }
    // The block's edge comes before its tiles.
    __device__ __forceinline__ void enter()
    {
        t = tokens_tiles<R>(a, s, p.block);
        if (a.uncut) {
            span = 1, first = 0, count = t.count;
            return;
        }
        const long long left = run.end - pos;
        const int most = t.count + run.edge - p.off;
        span = left < most ? static_cast<int>(left) : most;
        first = max(0, p.off - run.edge);
        count = max(0, p.off + span - run.edge) - first;
        if (count == 0) pos = run.end;  // the run ends within the edge: the next CTA's
    }
    __device__ __forceinline__ bool more() const { return pos < run.end; }
    __device__ __forceinline__ bool begins() const { return first == 0; }
    __device__ __forceinline__ bool ends() const { return first + count == t.count; }
    // CTAs that the block goes on in
    __device__ __forceinline__ int behind() const
    {
        return static_cast<int>((t.count + run.edge - p.off - span + run.chunk - 1) / run.chunk);
    }
    __device__ __forceinline__ int tile(int i) const { return t.at(first + i); }
    __device__ __forceinline__ int rows() const { return min(R, s.m * a.group - p.block * R); }
    __device__ __forceinline__ void next()
    {
        pos += span;
        if (pos >= run.end) return;
        p.off = 0;  // only the last block may be left before its end
        if (++p.block >= tokens_blocks<R>(a, s)) {
            p.block = 0;
            if (++p.head >= a.kv_heads) {
                p.head = 0;
                do s = tokens_seq(a, ++p.b);
                while (s.m == 0);
            }
        }
        enter();
    }
};

// LZS: encoded pages, whose decoding pays for every unit, not for its size alone.
template <int D, int TILES, bool LZS>
struct TokensShape {
    static constexpr int kRows = 128 * TILES;
    static constexpr int kUnitDims = D == 128 || (LZS && D == 256) ? 128 : 64, kUnits = D / kUnitDims;  // units of a tile's side
    // Units that one product of the weights takes: next to each other in the ring
    static constexpr int kTogether = kUnitDims == 128 ? 1 : D == 256 ? 2 : kUnits;
    static constexpr int kPanel = kTokKeys * 128;  // 64 dimensions, 128 bytes a row
    static constexpr int kUnitBytes = kTokKeys * kUnitDims * 2, kQTile = 128 * D * 2, kQBytes = TILES * kQTile;
    static constexpr int kMisc = 3 * 1024;  // static shared memory, with its padding
    // Results on their way out, 32 rows x 64 bytes a warp.  Heads of 256 have none: the
    // ring holds two units more than a tile's keys and values instead, which are under
    // way while those are used.
    static constexpr int kOutWarp = D == 256 ? 0 : 2048, kOut = kTokSoftmaxWarps * kOutWarp;
    static constexpr int kFit = (232448 - kMisc - kQBytes - kOut) / kUnitBytes;
    static constexpr int kRing = (kFit < 12 ? kFit : 12) / kTogether * kTogether;
    static constexpr int kSmem = kQBytes + kRing * kUnitBytes + kOut;
    static_assert(kRing >= 2 * kUnits, "the values of a tile and the next keys are held together");
    static_assert(256 + TILES * D <= 512, "TMEM: two S, and O");
};

struct TokensShared {
    uint64_t full[12], empty[12];
    uint64_t q_full, q_free, s_full[2], p_ready[2], pv_done[2], swap[4], hand[8], o_done, o_free, drain;
    uint32_t tmem;
    int abort;
    TokensFind find;
    float m[2][128], l[2][128];  // one tile: a row's maximum and sum, by warpgroup
};
static_assert(sizeof(TokensShared) <= 3 * 1024, "");

// tanh of u, |u| <= 1, good to 3 half steps of binary32: an odd polynomial fitted
// to the least largest relative error (6.7e-8 with these coefficients, before it is
// evaluated); above, 1 - 2 / (1 + e^2|u|).
__device__ __forceinline__ constexpr float tokens_tanh_term(int i)
{
    constexpr float c[7] = {0.99999994f, -0.3333284f, 0.13325204f, -0.05345702f, 0.020289967f, -0.006203367f, 0.0010410185f};
    return c[i];
}

__device__ __forceinline__ float tokens_tanh(float u)
{
    const float q = u * u, size = fabsf(u);
    float p = tokens_tanh_term(6);
#pragma unroll
    for (int i = 5; i >= 0; --i) p = fmaf(p, q, tokens_tanh_term(i));
    const float big = 1.f - __fdividef(2.f, 1.f + ex2(size * 2.8853901f));
    return size <= 1.f ? p * u : copysignf(big, u);
}

// Bits 0 .. 31: columns [a, b] of the 32.
__device__ __forceinline__ uint32_t tokens_bits(int a, int b)
{
    if (a > 31 || b < 0 || a > b) return 0u;
    const uint32_t up = a <= 0 ? ~0u : ~0u << a, down = b >= 31 ? ~0u : (2u << b) - 1u;
    return up & down;
}

// What a row sees of the keys, and how it weighs them.
struct TokensRow {
    int lo, hi, pre, pos, base;
    uint64_t own;  // tree: bits of the new tokens
    float slope;   // log2 domain
    const uint64_t *tree;
    uint64_t some;  // the sequence's new tokens

    // Columns [t0, t0 + 32).
    __device__ __forceinline__ uint32_t seen(int t0) const
    {
        uint32_t v = tokens_bits(lo - t0, hi - t0) | tokens_bits(0, pre - 1 - t0);
        const int d = t0 - base;
        if (own && d > -32 && d < 64) v |= static_cast<uint32_t>(d >= 0 ? own >> d : own << -d);
        return v;
    }
    // The others that drafted token i sees, whether it sees itself or not.
    __device__ __forceinline__ int depth(int i) const { return __popcll(tree[i] & some & ~(1ull << i)); }
    __device__ __forceinline__ int place(int t) const
    {
        return tree && t >= base && t - base < 64 && (some >> (t - base) & 1) ? base + depth(t - base) : t;
    }
};

// Masks of 32 scores of columns t0 ..: -inf where the row does not see.
__device__ __forceinline__ void tokens_mask(uint32_t seen, uint32_t (&s)[32])
{
#pragma unroll
    for (int j = 0; j < 32; ++j)
        if (!(seen >> j & 1)) s[j] = 0xFF800000u;
}

// Their factor or cap, and distance: to the log2 domain.
__device__ __forceinline__ void tokens_shape(const TokensArgs &a, const TokensRow &row, bool valid, int t0, uint32_t (&s)[32])
{
    const float by = a.cap_log2 > 0.f ? a.to_cap : a.scale_log2;
    const uint64_t factor = pack2(by, by);
    uint64_t v[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] = mul2(pack2(__uint_as_float(s[2 * j]), __uint_as_float(s[2 * j + 1])), factor);
    if (a.cap_log2 > 0.f) {
        float most = 0.f;
#pragma unroll
        for (int j = 0; j < 16; ++j) most = max3(most, fabsf(unpack2(v[j]).x), fabsf(unpack2(v[j]).y));
        const uint64_t cap = pack2(a.cap_log2, a.cap_log2);
        if (__all_sync(0xffffffffu, !valid || most <= 1.f)) {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const uint64_t q = mul2(v[j], v[j]);
                uint64_t p = pack2(tokens_tanh_term(6), tokens_tanh_term(6));
#pragma unroll
                for (int i = 5; i >= 0; --i) p = fma2(p, q, pack2(tokens_tanh_term(i), tokens_tanh_term(i)));
                v[j] = mul2(mul2(p, v[j]), cap);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = mul2(pack2(tokens_tanh(unpack2(v[j]).x), tokens_tanh(unpack2(v[j]).y)), cap);
        }
    }
    if (a.slopes) {
        const bool drafted = row.tree && t0 + 31 >= row.base;
        if (!drafted) {
            const int d = row.pos - t0;
            const float far = static_cast<float>(d);
            const uint64_t from = pack2(far, far), slope = pack2(-row.slope, -row.slope);
            const bool behind = __all_sync(0xffffffffu, d >= 31);  // no sign to take off
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                uint64_t dist = add2(from, pack2(-2.f * j, -2.f * j - 1.f));
                if (!behind) dist &= 0x7FFFFFFF7FFFFFFFull;
                v[j] = fma2(dist, slope, v[j]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const float2 dist = make_float2(fabsf(static_cast<float>(row.pos - row.place(t0 + 2 * j))),
                                                fabsf(static_cast<float>(row.pos - row.place(t0 + 2 * j + 1))));
                v[j] = fma2(pack2(dist.x, dist.y), pack2(-row.slope, -row.slope), v[j]);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        const float2 f = unpack2(v[j]);
        s[2 * j] = __float_as_uint(f.x), s[2 * j + 1] = __float_as_uint(f.y);
    }
}

// Two values rounded to the pages' type, and what that left of them.
template <bool BF>
__device__ __forceinline__ uint32_t pair_of(float2 v)
{
    if (BF) return bf16_pair(v.x, v.y);
    const __half2 h = __floats2half2_rn(v.x, v.y);
    return *reinterpret_cast<const uint32_t *>(&h);
}
template <bool BF>
__device__ __forceinline__ float2 left_of(float2 v, uint32_t pair)
{
    const float2 f = BF ? make_float2(__uint_as_float(pair << 16), __uint_as_float(pair & 0xFFFF0000u))
                        : __half22float2(*reinterpret_cast<const __half2 *>(&pair));
    return make_float2(v.x - f.x, v.y - f.y);
}

// PARTS: of a weight, one (rounded to the pages' type), or two (that, and what it
// left, rounded); tokens_plan chooses.
// SHAPED: scores need more than a positive factor.  (An instance of its own: the
// code for it in the others' loop cost them 14%, waiting for instructions.)
template <int D, int KIND, int TILES, bool SHAPED, int PARTS>
struct TokensKernel {
    using Shape = TokensShape<D, TILES, KIND == QUARTZ_PAGES_ENCODED>;
    static constexpr int R = Shape::kRows;
    static constexpr bool kBf = KIND == QUARTZ_PAGES_BF16, kLzs = KIND == QUARTZ_PAGES_ENCODED;
    // Weights are 2^(score - m + up) up to 2^(up + slack): fp16 keeps those down
    // to 2^-22 of the largest in full.
    static constexpr float kUp = kBf ? 0.f : 8.f, kSlack = kBf ? 8.f : 7.f;
    using Walk = TokensWalk<R>;
    // Filling warps: decoding takes twice as many.  Then registers a thread of the
    // softmax, the filling and the last warps, together what the CTA is launched with
    // (encoded, trees of 61 over up to 65536: 214 us; 144, 72, 48 225; 144, 64, 64 219).
    static constexpr int kFillWarps = kLzs ? 8 : 4, kWarps = kTokSoftmaxWarps + kFillWarps + 1 + kTokQueryWarps, kThreads = kWarps * 32;
    static constexpr int kLaunchRegs = kLzs ? 96 : 128;
    static constexpr int kSoftmaxRegs = kLzs ? 136 : 160, kFillRegs = kLzs ? 72 : 96, kLastRegs = kLzs ? 64 : 96;
    static_assert(kTokSoftmaxWarps * kSoftmaxRegs + kFillWarps * kFillRegs + 4 * kLastRegs <= kWarps * kLaunchRegs, "");
    static_assert(kWarps <= kTokMostWarps, "");

    const TokensArgs &a;
    TokensShared &sh;
    const TokensPlace at;
    const TokensRun &run;
    const uint32_t q_smem, ring, tmem;
    volatile int *abort;
    const void *k_map, *v_map, *q_map;

    __device__ __forceinline__ bool wait(const uint64_t &bar, int phase) const
    {
        return mbar_wait_warp(smem_u32(&bar), static_cast<uint32_t>(phase) & 1u, abort, a.dev_err, kWaitLimitNs);
    }
    __device__ __forceinline__ uint32_t unit_at(int u) const { return ring + (u % Shape::kRing) * Shape::kUnitBytes; }
    __device__ __forceinline__ bool wait_full(int u) const { return wait(sh.full[u % Shape::kRing], u / Shape::kRing); }
    // of the ring's place of unit u, freed by unit u - kRing
    __device__ __forceinline__ bool wait_empty(int u) const
    {
        return u < Shape::kRing || wait(sh.empty[u % Shape::kRing], u / Shape::kRing - 1);
    }

    // --- queries --------------------------------------------------------------
    // A box per tile and 64 dimensions where the heads of a token fill a tile in
    // whole tokens (rows behind the sequence's are others' or zeros, and weigh on
    // nothing); else 16 bytes a lane.
    __device__ __forceinline__ void load_queries(int warp)
    {
        constexpr int kChunks = D / 8, kEach = kChunks >= 32 || kChunks == 24 ? 1 : 32 / kChunks;  // rows at a time
        constexpr int kStep = kEach * kTokQueryWarps;
        const int lane = threadIdx.x & 31, c = kEach == 1 ? lane : lane % kChunks;
        const int r_first = warp * kEach + (kEach == 1 ? 0 : lane / kChunks);
        const int dt = kStep / a.group, dg = kStep - dt * a.group;
        int seg = 0;
        for (Walk w(a, at, run); w.more(); w.next(), ++seg) {
            if (seg > 0 && !wait(sh.q_free, seg - 1)) break;
            const int rows = w.rows();
            if (!kLzs && a.q_box) {
                const int boxes = (rows + 127) / 128 * (D / 64), tile = lane / (D / 64), panel = lane - tile * (D / 64);
                const uint32_t bar = smem_u32(&sh.q_full);
                if (lane == 0) {
                    if (warp == 0) mbar_arrive_expect_tx(bar, boxes * Shape::kPanel);
                    else mbar_arrive(bar);
                }
                __syncwarp();
                if (warp == 0 && lane < boxes)
                    tma_load_4d(q_smem + tile * Shape::kQTile + panel * Shape::kPanel, q_map, panel * 64, w.p.head * a.group,
                                w.s.start + (w.p.block * R + tile * 128) / a.group, 0, bar);
                continue;
            }
            const int first = w.p.block * R + r_first;
            int token = first / a.group, g = first - token * a.group;
            const uint16_t *q = a.q + w.s.start * a.q_st + static_cast<int64_t>(w.p.head) * a.group * a.q_sh + c * 8;
            auto to = [&](int r) {
                return q_smem + (r / 128) * Shape::kQTile + (c / 8) * Shape::kPanel + (r % 128) * 128 + (((c ^ r) & 7) << 4);
            };
            auto step = [&] {
                token += dt, g += dg;
                if (g >= a.group) g -= a.group, ++token;
            };
            if (c < kChunks) {
                if constexpr (!kLzs) {
#pragma unroll 4
                    for (int r = r_first; r < rows; r += kStep, step()) cp_async16(to(r), q + token * a.q_st + g * a.q_sh);
                } else {
                    // the eight elements of a chunk in the order of the decoded keys
                    for (int r0 = r_first; r0 < rows; r0 += 4 * kStep) {
                        uint4 v[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if (r0 + i * kStep < rows) v[i] = *reinterpret_cast<const uint4 *>(q + token * a.q_st + g * a.q_sh);
                            step();
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (r0 + i * kStep < rows)
                                sts_b128(to(r0 + i * kStep),
                                         make_uint4(prmt(v[i].x, v[i].z, 0x5410), prmt(v[i].x, v[i].z, 0x7632),
                                                    prmt(v[i].y, v[i].w, 0x5410), prmt(v[i].y, v[i].w, 0x7632)));
                    }
                }
            }
            cp_async_commit();
            cp_async_wait<0>();
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.q_full));
        }
        if (!kLzs && a.q_box && warp == 0 && *abort) {  // as in fill_16bit
            volatile int zero = 0;
            if (seg > 0) mbar_wait_bounded(smem_u32(&sh.q_full), (seg - 1) & 1, &zero, a.dev_err, kWaitLimitNs);
        }
    }

    // --- keys and values ------------------------------------------------------
    // The cached tokens that some new token of the sequence sees: those before
    // `pre`, and from `lo` on to base (causal: to n); of a tree's drafted ones those
    // in `own`.
    struct Loaded {
        int pre, lo, hi, base;
        uint64_t own;
        __device__ __forceinline__ bool all(int t0) const { return t0 + kTokKeys <= pre || (t0 >= lo && t0 + kTokKeys <= hi); }
        __device__ __forceinline__ bool has(int t) const
        {
            return t < pre || (t >= lo && t < hi) || (t >= base && t - base < kTokTreeMost && (own >> (t - base) & 1));
        }
    };
    __device__ __forceinline__ Loaded loaded(const Walk &w) const
    {
        Loaded l;
        l.pre = w.s.pre, l.base = w.s.base, l.hi = w.s.n, l.own = 0;
        l.lo = a.window > 0 ? max(0, w.s.base - a.window + 1) : 0;
        if (a.tree) {
            const int lane = threadIdx.x & 31;
            const uint64_t *tree = a.tree + w.s.start;
            uint64_t bits = (lane < w.s.m ? tree[lane] : 0) | (lane + 32 < w.s.m ? tree[lane + 32] : 0);
            if (w.s.m < kTokTreeMost) bits &= (1ull << w.s.m) - 1;
            const uint32_t low = __reduce_or_sync(0xffffffffu, static_cast<uint32_t>(bits));
            l.own = static_cast<uint64_t>(__reduce_or_sync(0xffffffffu, static_cast<uint32_t>(bits >> 32))) << 32 | low;
            l.hi = l.base;
        }
        return l;
    }

    // Place of token t's page in the table, asked for some time before it is used.
    __device__ __forceinline__ uint32_t page_entry(const Walk &w, int t, bool there) const
    {
        return there ? static_cast<uint32_t>(__ldg(a.table + (w.p.b * a.table_stride + (t >> a.page_shift)))) : 0u;
    }
    __device__ __forceinline__ int checked(uint32_t page, bool &bad) const
    {
        bad |= page >= a.num_pages;
        return page < a.num_pages ? static_cast<int>(page) : 0;
    }

    __device__ __forceinline__ void arrive_full(int u)
    {
        fence_proxy_async();
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(smem_u32(&sh.full[u % Shape::kRing]));
    }

    // 16-bit pages.  Tiles that are seen whole come by TMA, a box per page and 64
    // dimensions, dealt to the warps; the others (a sequence's end, a window's
    // begin; pages that are no boxes) by 16-byte copies with zeros in the rest.
    // Units in the order of the products: keys, values, keys, .. with two tiles; with
    // one the next keys before these values.
    static constexpr int kSkew = TILES == 1;

    __device__ __forceinline__ void fill_16bit(int warp)
    {
        constexpr int kLag = Shape::kRing / 2, kLanes = Shape::kUnitDims / 8, kRowsEach = 32 / kLanes;
        constexpr int kPanels = Shape::kUnitDims / 64;
        const int lane = threadIdx.x & 31, c = lane % kLanes, r_lane = lane / kLanes;
        const uint32_t mask = (1u << a.page_shift) - 1;
        const int boxes = a.box_rows ? kPanels * (kTokKeys / a.box_rows) : 0, box = warp + 4 * lane;
        const int box_row = box / kPanels * a.box_rows, panel = box % kPanels;
        const uint32_t box_to = panel * Shape::kPanel + box_row * 128;
        const uint32_t box_bytes = static_cast<uint32_t>(max(0, (boxes - warp + 3) / 4) * a.box_rows * 128);
        int u = 0, arrived = 0;
        bool bad = false, ok = true;
        auto flush = [&] {
            cp_async_wait<0>();
            while (arrived < u) arrive_full(arrived++);
        };
        for (Walk w(a, at, run); ok && w.more(); w.next()) {
            const Loaded l = loaded(w);
            // of a box, or of this lane's token (not there: none sees it; zeros take its
            // place, so that nothing of it, which may be infinite or NaN, meets a weight of 0)
            auto lookup = [&](int i, bool &there) {
                const int t0 = w.tile(i) * kTokKeys;
                const bool boxed = boxes && l.all(t0);
                const int t = t0 + (boxed ? box_row : warp * 32 + lane);
                there = boxed ? box < boxes : l.has(t);
                return page_entry(w, t, there);
            };
            bool there_k, there_v = false, there_next = false;
            uint32_t page_k = lookup(0, there_k), page_v = 0, page_next = 0;
            for (int i = -kSkew; ok && i < w.count; ++i) {
                if (i + kSkew + 1 < w.count) page_next = lookup(i + kSkew + 1, there_next);
                if (kSkew == 0) page_v = page_k, there_v = there_k;
#pragma unroll 1
                for (int side = 0; ok && side < 2; ++side) {
                    const int tile = side ? i : i + kSkew;
                    if (tile < 0 || tile >= w.count) continue;
                    const int t0 = w.tile(tile) * kTokKeys, here = checked(side ? page_v : page_k, bad);
                    const PagedSide &p = side ? a.v : a.k;
                    if (boxes && l.all(t0)) {
                        if (arrived < u) flush();
                        const int slot = static_cast<int>(static_cast<uint32_t>(t0 + box_row) & mask);
                        const int order = side ? a.v_order : a.k_order;  // 2 bits each: head, slot, page
                        const int c1 = (order & 3) == 1 ? w.p.head : (order >> 2 & 3) == 1 ? slot : here;
                        const int c2 = (order & 3) == 2 ? w.p.head : (order >> 2 & 3) == 2 ? slot : here;
                        const int c3 = (order & 3) == 3 ? w.p.head : (order >> 2 & 3) == 3 ? slot : here;
#pragma unroll 1
                        for (int k = 0; k < Shape::kUnits; ++k, ++u) {
                            if (!(ok = wait_empty(u))) break;
                            const uint32_t bar = smem_u32(&sh.full[u % Shape::kRing]);
                            if (lane == 0) mbar_arrive_expect_tx(bar, box_bytes);
                            __syncwarp();
                            if (box < boxes)
                                tma_load_4d(unit_at(u) + box_to, side ? v_map : k_map, k * Shape::kUnitDims + panel * 64, c1, c2, c3, bar);
                        }
                        arrived = u;
                        continue;
                    }
                    const unsigned there = __ballot_sync(0xffffffffu, side ? there_v : there_k);
                    const int64_t slot = static_cast<uint32_t>(t0 + warp * 32 + lane) & mask;
                    // element offset of this lane's token
                    const int64_t off = static_cast<int64_t>(here) * p.stride_page + slot * p.stride_slot;
                    const uint16_t *base = reinterpret_cast<const uint16_t *>(p.data) + w.p.head * p.stride_head + c * 8;
#pragma unroll 1
                    for (int k = 0; k < Shape::kUnits; ++k) {
                        if (u >= Shape::kRing &&
                            !__all_sync(0xffffffffu, mbar_try_wait(smem_u32(&sh.empty[u % Shape::kRing]), (u / Shape::kRing - 1) & 1))) {
                            flush();  // what it waits for may wait for these
                            if (!(ok = wait_empty(u))) break;
                        }
                        const uint32_t to = unit_at(u) + (c / 8) * Shape::kPanel;
                        const uint16_t *from = base + k * Shape::kUnitDims;
#pragma unroll 4
                        for (int j = 0; j < 32 / kRowsEach; ++j) {
                            const int src = j * kRowsEach + r_lane, r = warp * 32 + src;
                            const int64_t o = __shfl_sync(0xffffffffu, off, src);
                            const bool is = there >> src & 1;
                            cp_async16_or_zero(to + r * 128 + (((c ^ r) & 7) << 4), is ? from + o : from, is ? 16 : 0);
                        }
                        cp_async_commit();
                        ++u;
                        if (u - arrived > kLag) {
                            cp_async_wait<kLag>();
                            arrive_full(arrived++);
                        }
                    }
                }
                page_v = page_k, there_v = there_k;
                page_k = page_next, there_k = there_next;
            }
        }
        flush();
        if (!ok) {  // a role gave up: no box is left under way when the CTA ends
            volatile int zero = 0;
            for (int v = max(0, u - Shape::kRing); v < u; ++v)
                mbar_wait_bounded(smem_u32(&sh.full[v % Shape::kRing]), (v / Shape::kRing) & 1, &zero, a.dev_err, kWaitLimitNs);
        }
        if (bad) atomicOr(a.dev_err, QUARTZ_DEV_INDEX);
    }

    // A lane's piece of a unit of encoded rows: half a row's elements of it.  A warp
    // has 16 rows.
    static constexpr int kWarpRows = kTokKeys / kFillWarps, kPiece = Shape::kUnitDims / 2;
    struct Piece {
        uint4 codes[kPiece / 32];
        uint32_t flags[kPiece / 32];  // bytes; G_s = 8: 4 or 8 of them, 16: 2 or 4, 32: 1 or 2, 64: 1
        uint16_t scale;
    };

    // Lane / 2 of this warp's rows; `row` is that of lane's token (-1: zeros).
    __device__ __forceinline__ void load_piece(const PagedSide &p, int row, int dim0, Piece &to) const
    {
        const int lane = threadIdx.x & 31, e = dim0 + (lane & 1) * kPiece;
        const int64_t r = __shfl_sync(0xffffffffu, row, lane >> 1);
#pragma unroll
        for (int i = 0; i < kPiece / 32; ++i) to.codes[i] = make_uint4(0u, 0u, 0u, 0u), to.flags[i] = 0;
        to.scale = 0;
        if (r < 0) return;
        const uint4 *c = reinterpret_cast<const uint4 *>(p.codes + r * (D / 2) + e / 2);
#pragma unroll
        for (int i = 0; i < kPiece / 32; ++i) to.codes[i] = __ldg(c + i);
        const uint8_t *f = p.flags + r * (D >> a.gs_shift) + (e >> a.gs_shift);
        if constexpr (kPiece == 64) {
            if (a.gs_shift == 3) {
                const uint2 two = __ldg(reinterpret_cast<const uint2 *>(f));
                to.flags[0] = two.x, to.flags[1] = two.y;
            } else if (a.gs_shift == 4) {
                to.flags[0] = __ldg(reinterpret_cast<const uint32_t *>(f));
            } else if (a.gs_shift == 5) {
                to.flags[0] = __ldg(reinterpret_cast<const uint16_t *>(f));
            } else {
                to.flags[0] = __ldg(f);
            }
        } else {
            if (a.gs_shift == 3) to.flags[0] = __ldg(reinterpret_cast<const uint32_t *>(f));
            else if (a.gs_shift == 4) to.flags[0] = __ldg(reinterpret_cast<const uint16_t *>(f));
            else to.flags[0] = __ldg(f);
        }
        to.scale = __ldg(reinterpret_cast<const uint16_t *>(p.scales) + r * (D / 64) + e / 64);
    }

    // Decoded to fp16, elements (0, 4), (1, 5), (2, 6), (3, 7) of each eight side
    // by side.  Codes times 2^FLAG are exact; the product with the scale is
    // rounded once.
    __device__ __forceinline__ void store_piece(const Piece &p, uint32_t unit, int warp) const
    {
        constexpr int kWords = kPiece / 8;
        const int lane = threadIdx.x & 31, c = lane & 1, r = warp * kWarpRows + (lane >> 1);
        const uint32_t scale = prmt(p.scale, 0, 0x1010);
        // a byte per 8 elements
        uint32_t f[kPiece / 32];
        if (a.gs_shift == 3) {
            for (int i = 0; i < kPiece / 32; ++i) f[i] = p.flags[i];
        } else {
            f[0] = prmt(p.flags[0], 0, a.gs_shift == 4 ? 0x1100 : 0x0000);
            if (kPiece == 64) f[kPiece / 32 - 1] = prmt(p.flags[0], 0, a.gs_shift == 4 ? 0x3322 : a.gs_shift == 5 ? 0x1111 : 0x0000);
        }
        uint32_t w[kWords];
#pragma unroll
        for (int i = 0; i < kPiece / 32; ++i) w[4 * i] = p.codes[i].x, w[4 * i + 1] = p.codes[i].y, w[4 * i + 2] = p.codes[i].z, w[4 * i + 3] = p.codes[i].w;
        // The lanes of a row write to other banks at a time: 128 dimensions, two panels,
        // the second begins with its other half; 64, one panel, a half each.
        const bool flip = kPiece == 64 && c;
        if (flip) {
#pragma unroll
            for (int i = 0; i < kWords / 2; ++i) {
                const uint32_t t = w[i];
                w[i] = w[i + kWords / 2], w[i + kWords / 2] = t;
            }
            const uint32_t t = f[0];
            f[0] = f[kPiece / 32 - 1], f[kPiece / 32 - 1] = t;
        }
        const uint32_t to = unit + (kPiece == 64 ? c * Shape::kPanel : 0) + r * 128;
        const int first = kPiece == 64 ? (flip ? 4 : 0) : c * 4;  // chunk of the first word
        KeyFlag flag(0);
#pragma unroll
        for (int j = 0; j < kWords; ++j) {
            if (j % 2 == 0 || a.gs_shift == 3) flag = KeyFlag(f[j / 4] >> (j % 4 * 8) & 255);
            uint32_t k[4];
            key_codes(w[j], flag, k);
#pragma unroll
            for (int x = 0; x < 4; ++x) k[x] = mul_f16x2(k[x], scale);
            sts_b128(to + ((((j ^ first) ^ r) & 7) << 4), make_uint4(k[0], k[1], k[2], k[3]));
        }
    }

    __device__ __forceinline__ void fill_encoded(int warp)
    {
        const int lane = threadIdx.x & 31;
        const int mask = (1 << a.page_shift) - 1;
        Piece now, next;  // the next unit's is on its way while one is decoded
        bool held = false, ok = true, bad = false;
        int u = 0;
        auto decode = [&] {
            if (!held) return true;
            if (!wait_empty(u)) return false;
            store_piece(now, unit_at(u), warp);
            arrive_full(u++);
            return true;
        };
        for (Walk w(a, at, run); ok && w.more(); w.next()) {
            const Loaded l = loaded(w);
            auto lookup = [&](int i, bool &there) {
                const int t = w.tile(i) * kTokKeys + warp * kWarpRows + lane % kWarpRows;
                there = l.has(t);
                return page_entry(w, t, there);
            };
            bool there_k, there_next = false;
            uint32_t page_k = lookup(0, there_k), page_next = 0;
            int row_v = -1;
            for (int i = -kSkew; ok && i < w.count; ++i) {
                int row_k = -1;
                if (i + kSkew < w.count) {
                    const int t = w.tile(i + kSkew) * kTokKeys + warp * kWarpRows + lane % kWarpRows, page = checked(page_k, bad);
                    if (there_k) row_k = ((page * a.kv_heads + w.p.head) << a.page_shift) + (t & mask);
                }
                if (i + kSkew + 1 < w.count) page_next = lookup(i + kSkew + 1, there_next);
                if (kSkew == 0) row_v = row_k;
#pragma unroll 1
                for (int k = 0; k < 2 * Shape::kUnits; ++k) {
                    const bool side = k >= Shape::kUnits;
                    const int tile = side ? i : i + kSkew;
                    if (tile < 0 || tile >= w.count) continue;
                    load_piece(side ? a.v : a.k, side ? row_v : row_k, k % Shape::kUnits * Shape::kUnitDims, next);
                    if (!(ok = decode())) break;
                    now = next;
                    held = true;
                }
                row_v = row_k;
                page_k = page_next, there_k = there_next;
            }
        }
        if (ok) decode();
        if (bad) atomicOr(a.dev_err, QUARTZ_DEV_INDEX);
    }

    // --- products -------------------------------------------------------------
    static constexpr uint32_t kIdescS = idesc_16_f32(kBf, false, 128, kTokKeys);
    static constexpr uint32_t kIdescO = idesc_16_f32(kBf, true, 128, Shape::kTogether * Shape::kUnitDims);

    // S[buf] = Q[tile] K', the keys in units u .., each when it is there.  `last`:
    // its place is free again.  (All lanes; false: gave up.)
    __device__ __forceinline__ bool issue_s(int tile, int buf, int u, bool leader, bool last) const
    {
        const uint32_t q_low = sdesc_low(sdesc_k_major_sw128(q_smem + tile * Shape::kQTile));
#pragma unroll
        for (int k = 0; k < Shape::kUnits; ++k) {
            if (!wait_full(u + k)) return false;
            if (!leader) continue;
            const uint32_t k_low = sdesc_low(sdesc_k_major_sw128(unit_at(u + k)));
#pragma unroll
            for (int i = 0; i < Shape::kUnitDims / 16; ++i) {
                const uint32_t in = (i / 4) * Shape::kPanel + (i % 4) * 32;
                mma_f16_ss(tmem + buf * 128, sdesc_sw128_at(q_low, k * (Shape::kUnitDims / 64) * Shape::kPanel + in),
                           sdesc_sw128_at(k_low, in), kIdescS, k + i > 0);
            }
            if (last) mma_commit(smem_u32(&sh.empty[(u + k) % Shape::kRing]));
        }
        if (leader) mma_commit(smem_u32(&sh.s_full[buf]));
        return true;
    }
    // Column of S that the weight of key t is written over (two weights to a column):
    // one after the other; two parts: those of 64 keys, then the second parts of these,
    // over the scores that both are from.
    __device__ __forceinline__ static constexpr int weights_at(int t) { return PARTS == 1 ? t / 2 : t / 64 * 64 + t % 64 / 2; }

    // O[tile] (+)= P[buf] V, the values in units u ..
    __device__ __forceinline__ bool issue_o(int tile, int buf, int u, bool add, bool leader, bool last) const
    {
#pragma unroll
        for (int k = 0; k < Shape::kUnits; k += Shape::kTogether) {
            for (int x = 0; x < Shape::kTogether; ++x)
                if (!wait_full(u + k + x)) return false;
            if (!leader) continue;
            const uint32_t v_low = sdesc_low(sdesc_mn_major_sw128(unit_at(u + k), Shape::kPanel));
#pragma unroll
            for (int i = 0; i < kTokKeys / 16; ++i)
#pragma unroll
                for (int part = 0; part < PARTS; ++part)
                    mma_f16_ts(tmem + 256 + tile * D + k * Shape::kUnitDims, tmem + buf * 128 + weights_at(16 * i) + 32 * part,
                               sdesc_sw128_at(v_low, i * 2048), kIdescO, add || i + part > 0);
            if (last)
                for (int x = 0; x < Shape::kTogether; ++x) mma_commit(smem_u32(&sh.empty[(u + k + x) % Shape::kRing]));
        }
        if (leader) mma_commit(smem_u32(&sh.pv_done[tile]));
        return true;
    }

    __device__ __forceinline__ void products()
    {
        const bool leader = elect_one();
        int it = 0, seg = 0, u = 0;  // tiles, blocks and units so far
        bool ok = true;
        for (Walk w(a, at, run); ok && w.more(); w.next(), ++seg) {
            if (!(ok = wait(sh.q_full, seg))) break;
            tc_fence_after();
#pragma unroll
            for (int t = 0; ok && t < TILES; ++t) ok = issue_s(t, TILES == 2 ? t : it & 1, u, leader, t + 1 == TILES);
            if (!ok) break;
            u += Shape::kUnits;
            if (leader && w.count == 1) mma_commit(smem_u32(&sh.q_free));
            for (int i = 0; i < w.count; ++i, ++it) {
                const bool again = i + 1 < w.count, last = i + 2 == w.count;
                if constexpr (TILES == 2) {
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        if (!(ok = wait(sh.p_ready[t], it))) break;
                        tc_fence_after();
                        if (!(ok = issue_o(t, t, u, i > 0, leader, t == 1))) break;
                        if (again && !(ok = issue_s(t, t, u + Shape::kUnits, leader, t == 1))) break;
                    }
                    if (!ok) break;
                    u += again ? 2 * Shape::kUnits : Shape::kUnits;
                    if (leader && last) mma_commit(smem_u32(&sh.q_free));
                } else {
                    if (again) {
                        if (!(ok = issue_s(0, (it + 1) & 1, u, leader, true))) break;
                        u += Shape::kUnits;
                        if (leader && last) mma_commit(smem_u32(&sh.q_free));
                    }
                    if (!(ok = wait(sh.p_ready[it & 1], it >> 1))) break;
                    if (i == 0 && seg > 0 && !(ok = wait(sh.o_free, seg - 1))) break;
                    tc_fence_after();
                    if (!(ok = issue_o(0, it & 1, u, i > 0, leader, true))) break;
                    u += Shape::kUnits;
                    if (leader && !again) mma_commit(smem_u32(&sh.o_done));
                }
            }
        }
        // every product is done before the CTA gives its memory up
        if (leader) mma_commit(smem_u32(&sh.drain));
        volatile int zero = 0;
        mbar_wait_bounded(smem_u32(&sh.drain), 0, &zero, a.dev_err, kWaitLimitNs);
    }

    // --- softmax --------------------------------------------------------------
    // One tile: the two warps that have a row's sums add them up.  The barrier's
    // phases are in turn: written, read.
    __device__ __forceinline__ bool add_sums(int row, int wg, float &l, int &count) const
    {
        const uint64_t &bar = sh.swap[(threadIdx.x >> 5) & 3];
        if (count > 0 && !wait(bar, 2 * count - 1)) return false;
        sh.l[wg][row] = l;
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(smem_u32(&bar));
        if (!wait(bar, 2 * count)) return false;
        const volatile float *both = &sh.l[0][row];
        l = both[0] + both[128];
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(smem_u32(&bar));
        ++count;
        return true;
    }

    __device__ __forceinline__ void softmax(int warp)
    {
        constexpr int kDims = TILES == 2 ? D : D / 2;  // of O, per thread, when a block is done
        const int lane = threadIdx.x & 31, wg = warp >> 2, quad = warp & 3, row = quad * 32 + lane;
        const int tile = TILES == 2 ? wg : 0, half = TILES == 2 ? 0 : wg;
        const uint32_t mine = tmem + (static_cast<uint32_t>(quad * 32) << 16);
        const uint32_t o_at = mine + 256 + tile * D, s_at = mine + wg * 128;
        int it = 0, seg = 0, swaps = 0;
        TokensJoin join{};
        for (Walk w(a, at, run); w.more(); w.next(), ++seg) {
            const int r = w.p.block * R + tile * 128 + row;
            const bool valid = r < w.s.m * a.group;
            const int j = valid ? r / a.group : 0, g = valid ? r - j * a.group : 0;
            TokensRow see;
            see.base = w.s.base, see.pre = w.s.pre, see.tree = nullptr, see.own = see.some = 0;
            see.hi = see.pos = w.s.base + j;
            if (a.tree) {
                see.tree = a.tree + w.s.start;
                see.some = w.s.m >= 64 ? ~0ull : (1ull << w.s.m) - 1;
                see.own = see.tree[j] & see.some;
                see.pos = w.s.base + see.depth(j);
                see.hi = w.s.base - 1;
            }
            see.lo = a.window > 0 ? max(0, see.pos - a.window + 1) : 0;
            if (a.tree && a.window > 0 && a.window < kTokTreeMost)
                for (int i = 0; i < w.s.m; ++i)
                    if (see.base + see.depth(i) < see.lo) see.own &= ~(1ull << i);
            see.slope = SHAPED && a.slopes ? a.slopes[w.p.head * a.group + g] * kPagedLog2e : 0.f;
            float m = kPagedLow, l = 0.f;
            for (int i = 0; i < w.count; ++i, ++it) {
                if (TILES == 1 && (it & 1) != wg) continue;
                const int t0 = w.tile(i) * kTokKeys;
                const bool all = !valid || (t0 >= see.lo && t0 + kTokKeys - 1 <= see.hi) || t0 + kTokKeys <= see.pre;
                const bool masked = !__all_sync(0xffffffffu, all);
                if (!wait(sh.s_full[wg], TILES == 2 ? it : it >> 1)) return;
                tc_fence_after();
                // What the scores need beside their factor.  On the way, in registers: a factor
                // and distances of tokens behind the row (whose sign is known); a cap that all
                // are far below.  Masks, and the rest, 32 columns at a time in TMEM.
                const bool ahead = SHAPED && __any_sync(0xffffffffu, valid && see.pre > see.pos + 1 && t0 < see.pre && t0 + kTokKeys > see.pos + 1);
                const bool drafted = see.tree && t0 + kTokKeys > see.base;
                bool far = SHAPED && a.slopes && a.cap_log2 == 0.f && a.scale_log2 > 0.f && !ahead && !drafted;
                bool near = SHAPED && a.cap_near && !a.slopes && !masked;
                auto prepare = [&](bool shape) {
#pragma unroll 1
                    for (int c = 0; c < kTokKeys; c += 32) {
                        const uint32_t seen = valid && masked ? see.seen(t0 + c) : ~0u;
                        const bool mask = masked && __any_sync(0xffffffffu, seen != ~0u);
                        if (!shape && !mask) continue;
                        uint32_t x[32];
                        tmem_ld_row(s_at + c, x);
                        if (SHAPED && shape) tokens_shape(a, see, valid, t0 + c, x);
                        if (mask) tokens_mask(seen, x);
                        tmem_st_row(s_at + c, x);
                    }
                    tmem_wait_st();
                };
                bool done = SHAPED && !far && !near;  // the scores are in the log2 domain
                if (done || masked) prepare(done);
                // The maximum, of the upper 64 columns, then of the lower, which stay in
                // registers.  (Loops over the halves, since code for all 128 runs out of the
                // instruction cache, and all 128 out of registers.)
                uint32_t s[64];
                const uint64_t factor = pack2(a.scale_log2, a.scale_log2), slope = pack2(see.slope, see.slope);
                // -slope (d - c) of column c, to which slope j is added: scale s - slope (d - c - j)
                auto origin = [&](int c) { return -see.slope * static_cast<float>(see.pos - t0 - c); };
                float top, least;
                auto range = [&] {
                    float t[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY}, l[4] = {INFINITY, INFINITY, INFINITY, INFINITY};
#pragma unroll 1
                    for (int c = 64; c >= 0; c -= 64) {
                        tmem_ld_row(s_at + c, s);
                        if (far) {
                            const float from = origin(c);
#pragma unroll
                            for (int x = 0; x < 64; x += 2) {
                                const uint64_t v = fma2(pack2(__uint_as_float(s[x]), __uint_as_float(s[x + 1])), factor, pack2(from, from));
                                const float2 f = unpack2(fma2(slope, pack2(1.f * x, 1.f * x + 1.f), v));
                                t[x / 2 & 3] = max3(t[x / 2 & 3], f.x, f.y);
                            }
                            continue;
                        }
#pragma unroll
                        for (int x = 0; x < 64; x += 2) t[x / 2 & 3] = max3(t[x / 2 & 3], __uint_as_float(s[x]), __uint_as_float(s[x + 1]));
                        if (near)
#pragma unroll
                            for (int x = 0; x < 64; x += 2) l[x / 2 & 3] = min3(l[x / 2 & 3], __uint_as_float(s[x]), __uint_as_float(s[x + 1]));
                    }
                    top = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
                    least = fminf(fminf(l[0], l[1]), fminf(l[2], l[3]));
                };
                range();
                if (near) {
                    near = __all_sync(0xffffffffu, !valid || fmaxf(fabsf(top * a.to_cap), fabsf(least * a.to_cap)) <= 0.5f);
                    if (near) {
                        top = a.cap_log2 * fmaxf(tokens_tanh(top * a.to_cap), tokens_tanh(least * a.to_cap));
                    } else {
                        done = true;
                        prepare(true);
                        range();
                    }
                } else if (!SHAPED) {
                    top *= a.scale_log2;
                }
                if (TILES == 1 && i > 0) {  // the maximum as the tile before left it
                    if (!wait(sh.hand[quad * 2 + (wg ^ 1)], (it - 1) >> 1)) return;
                    const float now = *reinterpret_cast<volatile float *>(&sh.m[wg ^ 1][row]);
                    l *= ex2(m - now);
                    m = now;
                }
                const bool rises = i > 0 && __any_sync(0xffffffffu, valid && top > m + kSlack);
                const float before = m;
                if (i == 0 || rises) m = fmaxf(m, top);
                if (TILES == 1) {
                    sh.m[wg][row] = m;
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&sh.hand[quad * 2 + wg]));
                }
                if (rises) {
                    const float f = ex2(before - m);
                    l *= f;
                    if (!wait(sh.pv_done[tile], it - 1)) return;
                    tc_fence_after();
#pragma unroll 1
                    for (int c = 0; c < D; c += 32) {
                        uint32_t o[32];
                        tmem_ld_row(o_at + c, o);
#pragma unroll
                        for (int x = 0; x < 32; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * f);
                        tmem_st_row(o_at + c, o);
                    }
                }
                // Pairs at a time: shaped scores in two parts run out of registers with 16 (900
                // bytes of spills; 512 new tokens over 4096 encoded ones, a cap: 189 us, 8: 149).
                // Plain ones do not (110, 8: 117).
                constexpr int kPairs = PARTS == 2 && SHAPED ? 8 : 16;
                uint64_t sum[2] = {0, 0};
                // Weights; `exponent` gives those of a pair, column x of the 64 from c on
                auto weigh = [&](auto exponent) {
#pragma unroll 1
                    for (int c = 0; c < kTokKeys; c += 64) {
                        if (c) tmem_ld_row(s_at + c, s);
                        const auto of = exponent(c);
#pragma unroll
                        for (int y = 0; y < 64; y += 2 * kPairs) {
                            uint32_t p[kPairs], second[PARTS == 1 ? 1 : kPairs];
#pragma unroll
                            for (int x = 0; x < kPairs; ++x) {
                                float2 e = unpack2(of(pack2(__uint_as_float(s[y + 2 * x]), __uint_as_float(s[y + 2 * x + 1])), y + 2 * x));
                                e.x = ex2(e.x), e.y = ex2(e.y);
                                sum[x & 1] = add2(sum[x & 1], pack2(e.x, e.y));
                                p[x] = pair_of<kBf>(e);
                                if constexpr (PARTS == 2) second[x] = pair_of<kBf>(left_of<kBf>(e, p[x]));
                            }
                            tmem_st_row(s_at + weights_at(c + y), p);
                            if constexpr (PARTS == 2) tmem_st_row(s_at + weights_at(c + y) + 32, second);
                        }
                    }
                };
                const uint64_t shift = pack2(kUp - m, kUp - m);
                if (near) {
                    // cap tanh(s / cap) by an odd polynomial, good to 11 half steps up to cap / 2
                    // (9.3 before it is evaluated)
                    const float by = a.cap_log2 * a.to_cap, q = a.to_cap * a.to_cap;
                    const uint64_t c0 = pack2(0.99999946f * by, 0.99999946f * by), c1 = pack2(-0.3332632f * by * q, -0.3332632f * by * q),
                                   c2 = pack2(0.13190296f * by * q * q, 0.13190296f * by * q * q),
                                   c3 = pack2(-0.04440222f * by * q * q * q, -0.04440222f * by * q * q * q);
                    weigh([&](int) {
                        return [&](uint64_t v, int) {
                            const uint64_t w = mul2(v, v);
                            return fma2(fma2(fma2(fma2(c3, w, c2), w, c1), w, c0), v, shift);
                        };
                    });
                } else if (far) {
                    weigh([&](int c) {
                        const float from = origin(c) + (kUp - m);
                        return [=](uint64_t v, int x) { return fma2(slope, pack2(1.f * x, 1.f * x + 1.f), fma2(v, factor, pack2(from, from))); };
                    });
                } else {
                    const float by = SHAPED ? 1.f : a.scale_log2;  // done, or plain
                    const uint64_t f = pack2(by, by);
                    weigh([&](int) { return [&](uint64_t v, int) { return fma2(v, f, shift); }; });
                }
                const float2 sums = unpack2(add2(sum[0], sum[1]));
                l += sums.x + sums.y;
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh.p_ready[wg]));
            }
            if (TILES == 1) {
                const int last = (it - 1) & 1;
                if (wg != last) {
                    if (!wait(sh.hand[quad * 2 + last], (it - 1) >> 1)) return;
                    const float now = *reinterpret_cast<volatile float *>(&sh.m[last][row]);
                    l *= ex2(m - now);
                    m = now;
                }
                if (!add_sums(row, wg, l, swaps)) return;
            }
            // the block's result, or this CTA's part of it
            if (!(TILES == 2 ? wait(sh.pv_done[tile], it - 1) : wait(sh.o_done, seg))) return;
            tc_fence_after();
            const bool whole = w.begins() && w.ends();
            const int slot = 2 * blockIdx.x + w.begins();
            const int64_t part = static_cast<int64_t>(slot) * R + tile * 128 + row;
            if (!whole && w.begins()) {
                join.parts = 1 + w.behind();
                join.token0 = w.s.start, join.row0 = w.p.block * R, join.rows = w.rows(), join.head0 = w.p.head * a.group;
            }
            if (!whole && valid && half == 0) a.part_ml[part] = make_float2(m, l);
            const float inv = whole ? (l > 0.f ? 1.f / l : l == 0.f ? 0.f : l) : 1.f;  // NaN stays
            const int64_t out = (static_cast<int64_t>(w.s.start + j) * a.kv_heads * a.group + w.p.head * a.group + g) * D + half * kDims;
            const unsigned rows = __ballot_sync(0xffffffffu, valid);
            const int64_t part0 = (part - lane) * D + half * kDims;  // of the warp's first row
            const uint32_t stage = q_smem + Shape::kQBytes + Shape::kRing * Shape::kUnitBytes + warp * Shape::kOutWarp;
            // 32 columns at a time through shared memory, so that the lanes of a row write
            // side by side: a row's store for itself takes as many steps as there are rows.
#pragma unroll 1
            for (int c = 0; rows && c < kDims; c += 32) {
                uint32_t s[32];
                tmem_ld_row(o_at + half * kDims + c, s);
                float v[32];
#pragma unroll
                for (int x = 0; x < 32; ++x) {
                    // encoded: dimension x is where the decoding puts it
                    const int from = kLzs ? (x & ~7) + (x & 3) * 2 + (x >> 2 & 1) : x;
                    v[x] = __uint_as_float(s[from]) * inv;
                }
                auto halves = [&](int x) {  // elements x and x + 1 in the result's type
                    if (a.o_type == QUARTZ_OUT_BF16) return bf16_pair(v[x], v[x + 1]);
                    const __half2 h = __floats2half2_rn(v[x], v[x + 1]);
                    return *reinterpret_cast<const uint32_t *>(&h);
                };
                if constexpr (Shape::kOut == 0) {
                    if (valid && (!whole || a.o_type == QUARTZ_OUT_F32)) {
                        float *to = whole ? static_cast<float *>(a.o) + out + c : a.part_o + part0 + lane * D + c;
#pragma unroll
                        for (int x = 0; x < 32; x += 4) *reinterpret_cast<float4 *>(to + x) = make_float4(v[x], v[x + 1], v[x + 2], v[x + 3]);
                    } else if (valid) {
#pragma unroll
                        for (int x = 0; x < 32; x += 8)
                            *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(a.o) + out + c + x) =
                                make_uint4(halves(x), halves(x + 2), halves(x + 4), halves(x + 6));
                    }
                } else if (!whole || a.o_type == QUARTZ_OUT_F32) {
#pragma unroll
                    for (int y = 0; y < 32; y += 16) {
#pragma unroll
                        for (int x = 0; x < 4; ++x)
                            sts_b128(stage + lane * 64 + (((x ^ lane >> 1) & 3) << 4),
                                     make_uint4(__float_as_uint(v[y + 4 * x]), __float_as_uint(v[y + 4 * x + 1]),
                                                __float_as_uint(v[y + 4 * x + 2]), __float_as_uint(v[y + 4 * x + 3])));
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int to = i * 8 + lane / 4, x = lane % 4;
                            const float4 f = lds_f4(stage + to * 64 + (((x ^ to >> 1) & 3) << 4));
                            const int64_t at_row = __shfl_sync(0xffffffffu, out, to);
                            if (rows >> to & 1) {
                                if (whole) *reinterpret_cast<float4 *>(static_cast<float *>(a.o) + at_row + c + y + x * 4) = f;
                                else *reinterpret_cast<float4 *>(a.part_o + part0 + to * D + c + y + x * 4) = f;
                            }
                        }
                        __syncwarp();
                    }
                } else {
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        sts_b128(stage + lane * 64 + (((x ^ lane >> 1) & 3) << 4),
                                 make_uint4(halves(8 * x), halves(8 * x + 2), halves(8 * x + 4), halves(8 * x + 6)));
                    }
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int to = i * 8 + lane / 4, x = lane % 4;
                        const float4 f = lds_f4(stage + to * 64 + (((x ^ to >> 1) & 3) << 4));
                        const int64_t at_row = __shfl_sync(0xffffffffu, out, to);
                        if (rows >> to & 1) *reinterpret_cast<float4 *>(static_cast<uint16_t *>(a.o) + at_row + c + x * 8) = f;
                    }
                }
                __syncwarp();
            }
            tc_fence_before();
            if (TILES == 1) {  // O may be written again when both warpgroups have read it
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh.o_free));
            }
        }
        if (threadIdx.x == 0 && !a.uncut) a.joins[blockIdx.x] = join;
    }
};

template <int D, int KIND, int TILES, bool SHAPED, int PARTS>
__global__ void __launch_bounds__(TokensKernel<D, KIND, TILES, SHAPED, PARTS>::kThreads, 1)
    tokens_attn_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
                       const __grid_constant__ CUtensorMap q_map, TokensArgs a)
{
    griddep_wait();
    using K = TokensKernel<D, KIND, TILES, SHAPED, PARTS>;
    using Shape = typename K::Shape;
    extern __shared__ __align__(1024) uint8_t s_tokens[];
    __shared__ TokensShared sh;
    const int warp = threadIdx.x >> 5;
    TokensRun run;
    if (!tokens_find<Shape::kRows>(a, sh.find, run)) {
        if (threadIdx.x == 0 && !a.uncut) a.joins[blockIdx.x] = TokensJoin{};
        return;
    }
    if (threadIdx.x == 0) {
        if (!a.uncut) a.joins[blockIdx.x] = TokensJoin{};  // for a CTA that gives up
        for (int i = 0; i < Shape::kRing; ++i) {
            mbar_init(smem_u32(&sh.full[i]), K::kFillWarps);
            mbar_init(smem_u32(&sh.empty[i]), 1);
        }
        mbar_init(smem_u32(&sh.q_full), kTokQueryWarps);
        mbar_init(smem_u32(&sh.q_free), 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&sh.s_full[i]), 1);
            mbar_init(smem_u32(&sh.p_ready[i]), 4);
            mbar_init(smem_u32(&sh.pv_done[i]), 1);
        }
        for (int i = 0; i < 4; ++i) mbar_init(smem_u32(&sh.swap[i]), 2);
        for (int i = 0; i < 8; ++i) mbar_init(smem_u32(&sh.hand[i]), 1);
        mbar_init(smem_u32(&sh.o_done), 1);
        mbar_init(smem_u32(&sh.o_free), kTokSoftmaxWarps);
        mbar_init(smem_u32(&sh.drain), 1);
        sh.abort = 0;
        fence_mbar_init();
    }
    if (warp == 0) {
        tmem_alloc(smem_u32(&sh.tmem), 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t q_smem = smem_u32(s_tokens), tmem = *reinterpret_cast<volatile uint32_t *>(&sh.tmem);
    K k{a, sh, sh.find.at, run, q_smem, q_smem + Shape::kQBytes, tmem, &sh.abort, &k_map, &v_map, &q_map};
    if (warp < kTokSoftmaxWarps) {
        regs_increase<K::kSoftmaxRegs>();
        k.softmax(warp);
    } else if (warp < kTokSoftmaxWarps + K::kFillWarps) {
        regs_decrease<K::kFillRegs>();
        if constexpr (K::kLzs) k.fill_encoded(warp - kTokSoftmaxWarps);
        else k.fill_16bit(warp - kTokSoftmaxWarps);
    } else {
        regs_decrease<K::kLastRegs>();
        if (warp == kTokSoftmaxWarps + K::kFillWarps) k.products();
        else k.load_queries(warp - kTokSoftmaxWarps - K::kFillWarps - 1);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 0) tmem_dealloc(tmem, 512);
}

struct TokensMaps {
    CUtensorMap k, v, q;
};

// `shaped`: scores need more than a positive factor.
cudaError_t launch_tokens_attn_64(const TokensArgs &a, const TokensMaps &m, int kind, int tiles, int parts, int ctas, cudaStream_t s);
cudaError_t launch_tokens_attn_64_shaped(const TokensArgs &a, const TokensMaps &m, int kind, int tiles, int parts, int ctas, cudaStream_t s);
cudaError_t launch_tokens_attn_128(const TokensArgs &a, const TokensMaps &m, int kind, int tiles, int parts, int ctas, cudaStream_t s);
cudaError_t launch_tokens_attn_128_shaped(const TokensArgs &a, const TokensMaps &m, int kind, int tiles, int parts, int ctas, cudaStream_t s);
cudaError_t launch_tokens_attn_192(const TokensArgs &a, const TokensMaps &m, int kind, int tiles, int parts, int ctas, cudaStream_t s);
cudaError_t launch_tokens_attn_192_shaped(const TokensArgs &a, const TokensMaps &m, int kind, int tiles, int parts, int ctas, cudaStream_t s);
cudaError_t launch_tokens_attn_256(const TokensArgs &a, const TokensMaps &m, int kind, int tiles, int parts, int ctas, cudaStream_t s);
cudaError_t launch_tokens_attn_256_shaped(const TokensArgs &a, const TokensMaps &m, int kind, int tiles, int parts, int ctas, cudaStream_t s);

template <int D, int KIND, int TILES, bool SHAPED, int PARTS>
cudaError_t launch_tokens_attn(const TokensArgs &a, const TokensMaps &m, int ctas, cudaStream_t s)
{
    constexpr int kSmem = TokensKernel<D, KIND, TILES, SHAPED, PARTS>::Shape::kSmem;
    const cudaError_t e = allow_shared<tokens_attn_kernel<D, KIND, TILES, SHAPED, PARTS>>(kSmem);
    if (e != cudaSuccess) return e;
    return launch_pdl(tokens_attn_kernel<D, KIND, TILES, SHAPED, PARTS>, dim3(static_cast<unsigned>(ctas)), dim3(TokensKernel<D, KIND, TILES, SHAPED, PARTS>::kThreads), kSmem, s,
                      m.k, m.v, m.q, a);
}

template <int D, int TILES, bool SHAPED, int PARTS>
cudaError_t launch_tokens_attn(const TokensArgs &a, const TokensMaps &m, int kind, int ctas, cudaStream_t s)
{
    if (kind == QUARTZ_PAGES_F16) return launch_tokens_attn<D, QUARTZ_PAGES_F16, TILES, SHAPED, PARTS>(a, m, ctas, s);
    if (kind == QUARTZ_PAGES_BF16) return launch_tokens_attn<D, QUARTZ_PAGES_BF16, TILES, SHAPED, PARTS>(a, m, ctas, s);
    return launch_tokens_attn<D, QUARTZ_PAGES_ENCODED, TILES, SHAPED, PARTS>(a, m, ctas, s);
}

}  // namespace quartz
