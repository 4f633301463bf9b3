// Attention of several new tokens over a paged cache: the plan, and the join of
// tiles that were cut (tokens_attention.cuh has the scheme).
#include <cmath>
#include <utility>

#include "tokens_attention.cuh"

namespace quartz {
namespace {

constexpr int kJoinThreads = 256, kJoinRows = 8;

// CTA (x, y): rows 8 y .. of the block that CTA x of the attention began and the
// next ones went on with, a thread per 4 elements, the parts in the keys' order.
template <int D>
__global__ void __launch_bounds__(kJoinThreads) tokens_join_kernel(TokensArgs a, int R)
{
    griddep_wait();
    constexpr int kLanes = D / 4, kGroups = kJoinThreads / kLanes;
    const TokensJoin j = a.joins[blockIdx.x];
    if (j.parts < 2) return;
    const int group = threadIdx.x / kLanes, d = (threadIdx.x - group * kLanes) * 4;
    if (group >= kGroups) return;
    const int end = min(j.rows, (static_cast<int>(blockIdx.y) + 1) * kJoinRows);
    for (int r = blockIdx.y * kJoinRows + group; r < end; r += kGroups) {
        auto at = [&](int p) {
            const int64_t cta = blockIdx.x + p;
            return (2 * cta + (p == 0)) * R + r;
        };
        float m = kPagedLow;
#pragma unroll 4
        for (int p = 0; p < j.parts; ++p) m = fmaxf(m, a.part_ml[at(p)].x);
        float sum = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int p = 0; p < j.parts; ++p) {
            const float2 ml = a.part_ml[at(p)];
            const float4 u = *reinterpret_cast<const float4 *>(a.part_o + at(p) * D + d);
            const float f = ex2(ml.x - m);
            sum += f * ml.y;
            v.x += f * u.x, v.y += f * u.y, v.z += f * u.z, v.w += f * u.w;
        }
        const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;  // NaN stays
        const int row = j.row0 + r, token = row / a.group;
        const int64_t out = (static_cast<int64_t>(j.token0 + token) * a.kv_heads * a.group + j.head0 + row - token * a.group) * D + d;
        paged_store4(a.o, a.o_type, out, make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv));
    }
}

struct TokensPlan {
    int tiles, ctas, parts;
    bool uncut;
    int64_t each;  // tiles of keys a CTA, at most
};

// Two tiles side by side where a sequence may have more rows than one holds and
// TMEM has room for them; a CTA per SM, as long as there may be so many tiles of
// keys.  Blocks that all have an SM, of 8 tiles of keys at most, stay whole: the
// join, and its workspace, cost the host some 5 us and the GPU about what they take
// from a CTA.  Tiles of encoded pages and of wider heads take twice as long: 4 of
// them, unless blocks fill half the SMs.  Whole and cut, us a call (8 new tokens,
// 1 to 40 heads of 128, bf16): 256 keys 13 and 18, 777 18.6 and 17.6 to 21, 1024 19.2
// and 18.6 to 20; heads of 256: 512 18.5 and 18.3, 1024 29 and 20 to 25; encoded: 512
// 18.3 and 16.7, 1024 28 and 17.4 to 24; 128 blocks 29 and 34.
//
// Weights enter the value product in two parts, so that only the result's rounding
// is left of the error (relative to 64 bits, bf16 pages and results: 0.0016; in one
// part 0.0021).  Few rows are bound by the pages, not by products (16 trees of 16
// over up to 8192: 65.4 us, in one part 63.1), with a cap or distances by the softmax
// as well (16 x 16 tokens over 8192, fp16: 104 us, 101; a cap 136, 117; distances 160,
// 121), where one rule for all few rows was kept.  Sequences with more rows than a tile
// are bound by products and the softmax (8192 causal tokens: 513 us, in one part
// 400; trees of 61 over up to 65536 encoded tokens 280, 211; heads of 256 in a
// window 164, 144): one part, unless the result is binary32.
TokensPlan tokens_plan(const quartz_paged_cache_t *c, int64_t tokens, int64_t seqs, int q_heads, int64_t max_len, int64_t max_new,
                       int o_type)
{
    const int64_t group = q_heads / c->heads;
    TokensPlan p;
    p.tiles = c->dim <= 128 && max_new * group > 128 ? 2 : 1;
    p.parts = max_new * group <= 128 || o_type == QUARTZ_OUT_F32 ? 2 : 1;
    const int64_t blocks = (tokens * group / (128 * p.tiles) + seqs) * c->heads, most = blocks * (max_len / kTokKeys + 2);
    const bool dear = (c->type == QUARTZ_PAGES_ENCODED || c->dim > 128) && blocks <= device_sms() / 2;
    p.uncut = blocks <= device_sms() && max_len <= (dear ? 4 : 8) * kTokKeys;
    if (p.uncut) {
        p.ctas = static_cast<int>(blocks > 0 ? blocks : 1);
        p.each = max_len / kTokKeys + 2;
        return p;
    }
    p.ctas = static_cast<int>(most < device_sms() ? (most > 0 ? most : 1) : device_sms());
    p.each = (most + p.ctas - 1) / p.ctas;
    return p;
}

// A side of 16-bit pages as boxes of `rows` slots x 64 dimensions: dimensions 1
// to 3 are head, slot and page in the order of their strides; `order` says which
// is which.  False: the map cannot describe it (a stride of 0, say).
bool pool_map(CUtensorMap *map, const quartz_paged_cache_t *c, const quartz_pages_t &p, int rows, int &order)
{
    struct {
        int64_t stride;
        uint64_t n;
        int what;
    } dim[3] = {{p.stride_head, static_cast<uint64_t>(c->heads), 0},
                {p.stride_slot, static_cast<uint64_t>(c->page_size), 1},
                {p.stride_page, static_cast<uint64_t>(c->num_pages), 2}};
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2 - i; ++j)
            if (dim[j].stride > dim[j + 1].stride) std::swap(dim[j], dim[j + 1]);
    uint64_t dims[4] = {static_cast<uint64_t>(c->dim), 0, 0, 0}, strides[3];
    uint32_t box[4] = {64, 1, 1, 1};
    order = 0;
    for (int i = 0; i < 3; ++i) {
        if (dim[i].stride < c->dim) return false;
        dims[i + 1] = dim[i].n;
        strides[i] = static_cast<uint64_t>(dim[i].stride) * 2;
        if (dim[i].what == 1) box[i + 1] = static_cast<uint32_t>(rows);
        order |= (i + 1) << (2 * dim[i].what);
    }
    return make_pool_map(map, c->type == QUARTZ_PAGES_BF16, p.data, dims, strides, box);
}

size_t up256(size_t n) { return (n + 255) & ~size_t(255); }

}  // namespace

// A CTA counts its tiles, and the up to 8 units of each, in 32 bits.
bool paged_tokens_countable(const quartz_paged_cache_t *c, int64_t tokens, int64_t seqs, int q_heads, int64_t max_len, int64_t max_new)
{
    return tokens_plan(c, tokens, seqs, q_heads, max_len, max_new, QUARTZ_OUT_F16).each <= (int64_t(1) << 28) - 64;
}

size_t paged_tokens_workspace_bytes(const quartz_paged_cache_t *c, int64_t tokens, int64_t seqs, int q_heads, int64_t max_len,
                                    int64_t max_new)
{
    const TokensPlan p = tokens_plan(c, tokens, seqs, q_heads, max_len, max_new, QUARTZ_OUT_F16);  // the same for every result
    if (p.uncut) return 256;  // nothing is written to it
    const size_t rows = static_cast<size_t>(p.ctas) * 2 * 128 * p.tiles;
    return up256(rows * c->dim * 4) + up256(rows * 8) + up256(p.ctas * sizeof(TokensJoin));
}

cudaError_t launch_paged_tokens(const quartz_paged_cache_t *c, const PagedTokensCall &call, cudaStream_t s)
{
    const TokensPlan p = tokens_plan(c, call.tokens, call.seqs, call.q_heads, call.max_len, call.max_new, call.o_type);
    TokensArgs a{};
    a.q = static_cast<const uint16_t *>(call.q);
    a.q_st = call.q_st, a.q_sh = call.q_sh;
    a.table = call.table, a.table_stride = call.table_stride;
    a.lens = call.lens, a.starts = call.starts;
    a.tree = call.mask.tree, a.prefix = call.mask.prefix_lens, a.slopes = call.mask.slopes;
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
    a.seqs = static_cast<int>(call.seqs), a.tokens = static_cast<int>(call.tokens);
    a.max_len = static_cast<int>(call.max_len), a.max_new = static_cast<int>(call.max_new);
    a.window = static_cast<int>(call.mask.window < call.max_len ? call.mask.window : 0);
    a.gs_shift = c->type == QUARTZ_PAGES_ENCODED ? log2_of(c->k.enc.p.group_s) : 0;
    a.uncut = p.uncut;
    a.single = call.max_new * a.group <= 128 * p.tiles;
    a.scale_log2 = call.scale * kPagedLog2e;
    if (call.mask.cap > 0.f) a.cap_log2 = call.mask.cap * kPagedLog2e, a.to_cap = call.scale / call.mask.cap;
    a.cap_near = std::fabs(a.to_cap) > 1e-4f && std::fabs(a.to_cap) < 1e3f;
    a.o = call.o, a.o_type = call.o_type;
    a.dev_err = call.dev_err;
    uint8_t *ws = static_cast<uint8_t *>(call.workspace);
    const size_t rows = static_cast<size_t>(p.ctas) * 2 * 128 * p.tiles;
    a.part_o = reinterpret_cast<float *>(ws);
    ws += up256(rows * c->dim * 4);
    a.part_ml = reinterpret_cast<float2 *>(ws);
    ws += up256(rows * 8);
    a.joins = reinterpret_cast<TokensJoin *>(ws);
    TokensMaps m{};
    if (c->type != QUARTZ_PAGES_ENCODED && c->page_size >= 8) {
        const int rows = c->page_size < kTokKeys ? c->page_size : kTokKeys;
        if (pool_map(&m.k, c, c->k, rows, a.k_order) && pool_map(&m.v, c, c->v, rows, a.v_order)) a.box_rows = rows;
    }
    // (a map costs the host 1 us, which few queries do not save)
    if (c->type != QUARTZ_PAGES_ENCODED && 128 % a.group == 0 && call.max_new * a.group > 32 && call.q_sh >= c->dim && call.q_st >= c->dim) {
        const uint64_t dims[4] = {static_cast<uint64_t>(c->dim), static_cast<uint64_t>(call.q_heads), static_cast<uint64_t>(call.tokens), 1};
        const uint64_t strides[3] = {static_cast<uint64_t>(call.q_sh) * 2, static_cast<uint64_t>(call.q_st) * 2, static_cast<uint64_t>(call.q_st) * 2};
        const uint32_t box[4] = {64, static_cast<uint32_t>(a.group), static_cast<uint32_t>(128 / a.group), 1};
        a.q_box = make_pool_map(&m.q, c->type == QUARTZ_PAGES_BF16, call.q, dims, strides, box);
    }
    const dim3 grid(static_cast<unsigned>(p.ctas), static_cast<unsigned>(128 / kJoinRows * p.tiles)), block(kJoinThreads);
    const int R = 128 * p.tiles;
    const bool shaped = call.mask.cap > 0.f || call.mask.slopes || !(call.scale > 0.f);
    cudaError_t e;
    switch (c->dim) {
        case 64:
            e = (shaped ? launch_tokens_attn_64_shaped : launch_tokens_attn_64)(a, m, c->type, p.tiles, p.parts, p.ctas, s);
            return e != cudaSuccess || p.uncut ? e : launch_pdl(tokens_join_kernel<64>, grid, block, 0, s, a, R);
        case 128:
            e = (shaped ? launch_tokens_attn_128_shaped : launch_tokens_attn_128)(a, m, c->type, p.tiles, p.parts, p.ctas, s);
            return e != cudaSuccess || p.uncut ? e : launch_pdl(tokens_join_kernel<128>, grid, block, 0, s, a, R);
        case 192:
            e = (shaped ? launch_tokens_attn_192_shaped : launch_tokens_attn_192)(a, m, c->type, p.tiles, p.parts, p.ctas, s);
            return e != cudaSuccess || p.uncut ? e : launch_pdl(tokens_join_kernel<192>, grid, block, 0, s, a, R);
        default:
            e = (shaped ? launch_tokens_attn_256_shaped : launch_tokens_attn_256)(a, m, c->type, p.tiles, p.parts, p.ctas, s);
            return e != cudaSuccess || p.uncut ? e : launch_pdl(tokens_join_kernel<256>, grid, block, 0, s, a, R);
    }
}

}  // namespace quartz
