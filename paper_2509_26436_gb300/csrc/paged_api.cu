// Host side of the paged cache's C ABI (include/quartz.h): argument validation
// and launches.  As in api.cu, nothing here allocates or synchronises.
#include <cmath>

#include "quartz_internal.h"

using namespace quartz;

namespace {

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int32_t map_cuda(cudaError_t e) { return e == cudaSuccess ? QUARTZ_OK : QUARTZ_ERR_CUDA; }

constexpr float kLog2e = 1.4426950408889634f;
constexpr int64_t kMaxLen = int64_t(1) << 30;
constexpr int64_t kMaxRowStride = int64_t(1) << 40;  // of tables, weights, q, k, v, x, y: products stay below 2^63

bool stride_ok(int64_t s, int64_t multiple) { return s >= 0 && s <= kMaxRowStride && s % multiple == 0; }

// A stride that puts several written elements in one place.
bool repeats(int64_t stride, int64_t n) { return stride == 0 && n > 1; }

bool type_ok(int32_t t) { return t == QUARTZ_OUT_F16 || t == QUARTZ_OUT_BF16 || t == QUARTZ_OUT_F32; }

int32_t check_side(const quartz_paged_cache_t *c, const quartz_pages_t *p)
{
    if (c->type == QUARTZ_PAGES_ENCODED) {
        const quartz_encoded_t &e = p->enc;
        if (e.p.group_s != 8 && e.p.group_s != 16 && e.p.group_s != 32 && e.p.group_s != 64) return QUARTZ_ERR_INVALID_ARG;
        if (e.p.mode != QUARTZ_SYMMETRIC && e.p.mode != QUARTZ_ASYMMETRIC) return QUARTZ_ERR_INVALID_ARG;
        if (e.p.mode != QUARTZ_SYMMETRIC || e.p.group_q != 64 || (e.p.flag_bits != 0 && e.p.flag_bits != 8) ||
            (e.p.code_bits != 0 && e.p.code_bits != 8))
            return QUARTZ_ERR_UNSUPPORTED;
        if (e.K != c->dim || e.rows != c->num_pages * c->heads * c->page_size) return QUARTZ_ERR_INVALID_ARG;
        if (e.rows > (int64_t(1) << 31)) return QUARTZ_ERR_UNSUPPORTED;
        if (!e.codes || !e.flags || !e.scales) return QUARTZ_ERR_INVALID_ARG;
        if (!aligned16(e.codes) || !aligned16(e.flags) || !aligned16(e.scales)) return QUARTZ_ERR_ALIGNMENT;
        return QUARTZ_OK;
    }
    if (!p->data) return QUARTZ_ERR_INVALID_ARG;
    if (!aligned16(p->data)) return QUARTZ_ERR_ALIGNMENT;
    const int64_t s[3] = {p->stride_page, p->stride_slot, p->stride_head};
    for (int64_t v : s) {
        if (v < 0 || v >= (int64_t(1) << 31)) return QUARTZ_ERR_INVALID_ARG;
        if (v % 8 != 0) return QUARTZ_ERR_ALIGNMENT;
    }
    return QUARTZ_OK;
}

int32_t check_cache(const quartz_paged_cache_t *c)
{
    if (!c) return QUARTZ_ERR_INVALID_ARG;
    if (c->type != QUARTZ_PAGES_F16 && c->type != QUARTZ_PAGES_BF16 && c->type != QUARTZ_PAGES_ENCODED)
        return QUARTZ_ERR_INVALID_ARG;
    if (c->page_size < 1 || c->page_size > 4096 || (c->page_size & (c->page_size - 1))) return QUARTZ_ERR_INVALID_ARG;
    if (c->heads < 1 || c->heads > 1024 || c->num_pages < 1 || c->num_pages >= (int64_t(1) << 31) || c->dim < 1)
        return QUARTZ_ERR_INVALID_ARG;
    if (c->dim != 64 && c->dim != 128 && c->dim != 192 && c->dim != 256) return QUARTZ_ERR_UNSUPPORTED;
    int32_t rc = check_side(c, &c->k);
    if (rc == QUARTZ_OK) rc = check_side(c, &c->v);
    if (rc == QUARTZ_OK && c->type == QUARTZ_PAGES_ENCODED && c->k.enc.p.group_s != c->v.enc.p.group_s)
        return QUARTZ_ERR_INVALID_ARG;
    return rc;
}

// Pages that are written hold each row once (attention may read repeated ones).
int32_t check_written(const quartz_paged_cache_t *c)
{
    if (c->type == QUARTZ_PAGES_ENCODED) return QUARTZ_OK;
    for (const quartz_pages_t *p : {&c->k, &c->v})
        if (repeats(p->stride_page, c->num_pages) || repeats(p->stride_slot, c->page_size) || repeats(p->stride_head, c->heads))
            return QUARTZ_ERR_INVALID_ARG;
    return QUARTZ_OK;
}

int32_t check_rope(const quartz_rope_t *r, int32_t dim)
{
    if (!r->positions || !r->freqs) return QUARTZ_ERR_INVALID_ARG;
    if (r->rotary < 2 || r->rotary % 2 || r->rotary > dim || r->rotary > 512) return QUARTZ_ERR_INVALID_ARG;
    if ((r->interleaved & ~1) || (r->backward & ~1) || !std::isfinite(r->scale)) return QUARTZ_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(r->positions) | reinterpret_cast<uintptr_t>(r->freqs)) & 7) return QUARTZ_ERR_ALIGNMENT;
    return QUARTZ_OK;
}

int32_t check_attention(const quartz_paged_cache_t *c, int64_t seqs, int32_t q_heads, int64_t max_len, int64_t window)
{
    const int32_t rc = check_cache(c);
    if (rc) return rc;
    if (seqs < 0 || seqs > 65535 || q_heads < 1 || q_heads > 65536 || q_heads % c->heads) return QUARTZ_ERR_INVALID_ARG;
    if (max_len < 0 || max_len > kMaxLen || window < 0) return QUARTZ_ERR_INVALID_ARG;
    return QUARTZ_OK;
}

}  // namespace

int32_t quartz::check_paged_cache(const quartz_paged_cache_t *c) { return check_cache(c); }

extern "C" {

int32_t quartz_rope(const void *x, int64_t x_stride_token, int64_t x_stride_head, void *y, int64_t y_stride_token,
                    int64_t y_stride_head, int32_t type, int64_t tokens, int32_t heads, int32_t dim,
                    const quartz_rope_t *rope, void *stream)
{
    if (!rope || !type_ok(type) || tokens < 0 || tokens > kMaxLen || heads < 0 || heads > 65535 || dim < 2 ||
        dim > 1024)
        return QUARTZ_ERR_INVALID_ARG;
    if (!stride_ok(x_stride_token, 1) || !stride_ok(x_stride_head, 1) || !stride_ok(y_stride_token, 1) ||
        !stride_ok(y_stride_head, 1))
        return QUARTZ_ERR_INVALID_ARG;
    if (tokens == 0 || heads == 0) return QUARTZ_OK;
    const int32_t rc = check_rope(rope, dim);
    if (rc) return rc;
    if (!x || !y) return QUARTZ_ERR_INVALID_ARG;
    const uintptr_t m = type == QUARTZ_OUT_F32 ? 3 : 1;
    if ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(y)) & m) return QUARTZ_ERR_ALIGNMENT;
    if (repeats(y_stride_token, tokens) || repeats(y_stride_head, heads)) return QUARTZ_ERR_INVALID_ARG;
    RopeArgs a{x, y, x_stride_token, x_stride_head, y_stride_token, y_stride_head, type, heads, dim, *rope};
    return map_cuda(launch_rope(a, tokens, static_cast<cudaStream_t>(stream)));
}

int32_t quartz_paged_append(const quartz_paged_cache_t *cache, const void *k, int64_t k_stride_token,
                            int64_t k_stride_head, const void *v, int64_t v_stride_token, int64_t v_stride_head,
                            int64_t tokens, const int64_t *slots, const quartz_rope_t *rope, void *stream)
{
    int32_t rc = check_cache(cache);
    if (rc) return rc;
    if (tokens < 0 || tokens > kMaxLen) return QUARTZ_ERR_INVALID_ARG;
    const int64_t s[4] = {k_stride_token, k_stride_head, v_stride_token, v_stride_head};
    for (int64_t i : s) {
        if (!stride_ok(i, 1)) return QUARTZ_ERR_INVALID_ARG;
        if (i % 8) return QUARTZ_ERR_ALIGNMENT;
    }
    if (tokens == 0) return QUARTZ_OK;
    if (rope && (rc = check_rope(rope, cache->dim)) != QUARTZ_OK) return rc;
    if (rope && rope->backward) return QUARTZ_ERR_INVALID_ARG;
    if (!k || !v || !slots) return QUARTZ_ERR_INVALID_ARG;
    if (!aligned16(k) || !aligned16(v) || (reinterpret_cast<uintptr_t>(slots) & 7)) return QUARTZ_ERR_ALIGNMENT;
    if ((rc = check_written(cache)) != QUARTZ_OK) return rc;
    AppendArgs a{k, v, k_stride_token, k_stride_head, v_stride_token, v_stride_head, slots, {}, device_error_word()};
    if (!a.dev_err) return QUARTZ_ERR_CUDA;
    if (rope) a.rope = *rope;
    return map_cuda(launch_paged_append(cache, a, tokens, static_cast<cudaStream_t>(stream)));
}

size_t quartz_paged_attention_workspace_size(const quartz_paged_cache_t *cache, int64_t seqs, int32_t q_heads,
                                             int64_t max_len, int64_t window, int32_t with_weights)
{
    if (check_attention(cache, seqs, q_heads, max_len, window) != QUARTZ_OK) return 0;
    return paged_attention_workspace_bytes(cache, seqs, q_heads, max_len, window, with_weights != 0);
}

int32_t quartz_paged_attention(const void *q, int64_t q_stride_seq, int64_t q_stride_head, int64_t seqs,
                               int32_t q_heads, const quartz_paged_cache_t *cache, const int32_t *block_table,
                               int64_t table_stride, const int32_t *seq_lens, int64_t max_len, int64_t window,
                               float scale, void *o, int32_t o_type, float *weights, int64_t weights_stride_seq,
                               int64_t weights_stride_head, void *workspace, size_t workspace_bytes, void *stream)
{
    const int32_t rc = check_attention(cache, seqs, q_heads, max_len, window);
    if (rc) return rc;
    // the kernels multiply by scale log2 e
    if (!type_ok(o_type) || !std::isfinite(scale * kLog2e)) return QUARTZ_ERR_INVALID_ARG;
    if (!stride_ok(q_stride_seq, 1) || !stride_ok(q_stride_head, 1) || !stride_ok(table_stride, 1) ||
        (weights && (!stride_ok(weights_stride_seq, 1) || !stride_ok(weights_stride_head, 1))))
        return QUARTZ_ERR_INVALID_ARG;
    if (q_stride_seq % 8 || q_stride_head % 8) return QUARTZ_ERR_ALIGNMENT;
    if (seqs == 0) return QUARTZ_OK;
    if (!q || !o || !seq_lens || (max_len > 0 && !block_table)) return QUARTZ_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(o) || (reinterpret_cast<uintptr_t>(block_table) & 3) ||
        (reinterpret_cast<uintptr_t>(seq_lens) & 3) || (reinterpret_cast<uintptr_t>(weights) & 3))
        return QUARTZ_ERR_ALIGNMENT;
    if (weights && (repeats(weights_stride_seq, seqs) || repeats(weights_stride_head, cache->heads))) return QUARTZ_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < paged_attention_workspace_bytes(cache, seqs, q_heads, max_len, window, weights != nullptr))
        return QUARTZ_ERR_WORKSPACE;
    if (!aligned16(workspace)) return QUARTZ_ERR_ALIGNMENT;
    PagedAttnCall a{q, q_stride_seq, q_stride_head, seqs, q_heads, block_table, table_stride, seq_lens, max_len, window,
                    scale, o, o_type, weights, weights_stride_seq, weights_stride_head, workspace, device_error_word()};
    if (!a.dev_err) return QUARTZ_ERR_CUDA;
    return map_cuda(launch_paged_attention(cache, a, static_cast<cudaStream_t>(stream)));
}

int32_t quartz_evict_select(const float *weights, int64_t weights_stride_seq, int64_t weights_stride_head,
                            const int32_t *seq_lens, int64_t seqs, int32_t heads, int64_t max_len, int64_t budget,
                            int64_t recent, int64_t sinks, int32_t *kept, int32_t *new_lens, void *stream)
{
    if (seqs < 0 || seqs > 65535 || heads < 1 || heads > 1024 || max_len < 0 || max_len > kMaxLen || budget < 1 ||
        budget > kMaxLen || recent < 0 || sinks < 0 || recent > budget || sinks > budget - recent)
        return QUARTZ_ERR_INVALID_ARG;
    if (!stride_ok(weights_stride_seq, 1) || !stride_ok(weights_stride_head, 1)) return QUARTZ_ERR_INVALID_ARG;
    if (seqs == 0) return QUARTZ_OK;
    if ((max_len > 0 && !weights) || !seq_lens || !kept || !new_lens) return QUARTZ_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(weights) | reinterpret_cast<uintptr_t>(seq_lens) | reinterpret_cast<uintptr_t>(kept) |
         reinterpret_cast<uintptr_t>(new_lens)) & 3)
        return QUARTZ_ERR_ALIGNMENT;
    // every head's CTA reads its sequence's length, which the first head's replaces
    if (new_lens < seq_lens + seqs && seq_lens < new_lens + seqs) return QUARTZ_ERR_INVALID_ARG;
    int *err = device_error_word();
    if (!err) return QUARTZ_ERR_CUDA;
    return map_cuda(launch_evict_select(weights, weights_stride_seq, weights_stride_head, seq_lens, seqs, heads, max_len,
                                        budget, recent, sinks, kept, new_lens, err, static_cast<cudaStream_t>(stream)));
}

int32_t quartz_cache_compact(const quartz_paged_cache_t *cache, int64_t seqs, const int32_t *block_table,
                             int64_t table_stride, const int32_t *new_table, int64_t new_table_stride,
                             const int32_t *seq_lens, int64_t max_len, const int32_t *kept, int64_t budget,
                             float *weights, int64_t weights_stride_seq, int64_t weights_stride_head, void *stream)
{
    const int32_t rc = check_cache(cache);
    if (rc) return rc;
    if (seqs < 0 || seqs > 65535 || max_len < 0 || max_len > kMaxLen || budget < 1 || budget > kMaxLen)
        return QUARTZ_ERR_INVALID_ARG;
    if (!stride_ok(table_stride, 1) || !stride_ok(new_table_stride, 1) ||
        (weights && (!stride_ok(weights_stride_seq, 1) || !stride_ok(weights_stride_head, 1))))
        return QUARTZ_ERR_INVALID_ARG;
    if (seqs == 0 || max_len == 0) return QUARTZ_OK;
    if (!block_table || !seq_lens || !kept) return QUARTZ_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(block_table) | reinterpret_cast<uintptr_t>(new_table) |
         reinterpret_cast<uintptr_t>(seq_lens) | reinterpret_cast<uintptr_t>(kept) | reinterpret_cast<uintptr_t>(weights)) & 3)
        return QUARTZ_ERR_ALIGNMENT;
    if (weights && (repeats(weights_stride_seq, seqs) || repeats(weights_stride_head, cache->heads))) return QUARTZ_ERR_INVALID_ARG;
    if (const int32_t written = check_written(cache); written != QUARTZ_OK) return written;
    CompactCall a{seqs, block_table, new_table, table_stride, new_table_stride, seq_lens, kept, max_len, budget, weights,
                  weights_stride_seq, weights_stride_head, device_error_word()};
    if (!a.dev_err) return QUARTZ_ERR_CUDA;
    return map_cuda(launch_cache_compact(cache, a, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
