// Host side of the C ABI for several new tokens per sequence (include/quartz.h):
// argument validation and launches.  As in api.cu, nothing here allocates or
// synchronises.
#include <cmath>

#include "quartz_internal.h"

using namespace quartz;

namespace {

bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

int32_t map_cuda(cudaError_t e) { return e == cudaSuccess ? QUARTZ_OK : QUARTZ_ERR_CUDA; }

constexpr int64_t kMaxTokens = int64_t(1) << 30;
constexpr int64_t kMaxRowStride = int64_t(1) << 40;  // products with tokens and heads stay below 2^63 (2^30, 2^16)
constexpr int kMaxDim = 256, kMaxAxes = 16;

bool stride_ok(int64_t s) { return s >= 0 && s <= kMaxRowStride; }

// A stride that puts several written elements in one place.
bool repeats(int64_t stride, int64_t n) { return stride == 0 && n > 1; }

bool type_ok(int32_t t) { return t == QUARTZ_OUT_F16 || t == QUARTZ_OUT_BF16 || t == QUARTZ_OUT_F32; }

uintptr_t size_of(int32_t type) { return type == QUARTZ_OUT_F32 ? 4 : 2; }

int32_t check_rope(const quartz_rope_axes_t *r, int32_t dim)
{
    if (!r->positions || !r->freqs) return QUARTZ_ERR_INVALID_ARG;
    if (r->axes < 1 || r->axes > kMaxAxes || (r->axes > 1 && !r->pair_axis) || !stride_ok(r->axis_stride))
        return QUARTZ_ERR_INVALID_ARG;
    if (r->rotary < 2 || r->rotary % 2 || r->rotary > dim) return QUARTZ_ERR_INVALID_ARG;
    if ((r->interleaved & ~1) || (r->backward & ~1) || !std::isfinite(r->scale)) return QUARTZ_ERR_INVALID_ARG;
    if (!aligned(r->positions, 8) || !aligned(r->freqs, 8) || !aligned(r->pair_axis, 4)) return QUARTZ_ERR_ALIGNMENT;
    return QUARTZ_OK;
}

int32_t check_dim(int32_t dim)
{
    if (dim < 2) return QUARTZ_ERR_INVALID_ARG;
    return dim > kMaxDim ? QUARTZ_ERR_UNSUPPORTED : QUARTZ_OK;
}

int32_t check_side(const quartz_norm_side_t *s, int32_t type, int32_t w_type, int64_t tokens, bool backward)
{
    if (s->heads < 0 || s->heads > 65535) return QUARTZ_ERR_INVALID_ARG;
    if (backward && !aligned(s->dw, size_of(w_type))) return QUARTZ_ERR_ALIGNMENT;
    if (s->heads == 0) return QUARTZ_OK;
    if (!stride_ok(s->x_stride_token) || !stride_ok(s->x_stride_head) || !stride_ok(s->y_stride_token) ||
        !stride_ok(s->y_stride_head) || (backward && (!stride_ok(s->dy_stride_token) || !stride_ok(s->dy_stride_head))))
        return QUARTZ_ERR_INVALID_ARG;
    if (!aligned(s->w, size_of(w_type))) return QUARTZ_ERR_ALIGNMENT;
    if (tokens == 0) return QUARTZ_OK;
    if (!s->x || !s->y || (backward && !s->dy)) return QUARTZ_ERR_INVALID_ARG;
    if (!aligned(s->x, size_of(type)) || !aligned(s->y, size_of(type)) || (backward && !aligned(s->dy, size_of(type))))
        return QUARTZ_ERR_ALIGNMENT;
    if (repeats(s->y_stride_token, tokens) || repeats(s->y_stride_head, s->heads)) return QUARTZ_ERR_INVALID_ARG;
    return QUARTZ_OK;
}

HeadNormSide side_of(const quartz_norm_side_t &s)
{
    return {s.x, s.dy, s.y, s.x_stride_token, s.x_stride_head, s.dy_stride_token, s.dy_stride_head, s.y_stride_token,
            s.y_stride_head, s.w, s.dw, s.heads};
}

void set_rope(HeadNormArgs &a, const quartz_rope_axes_t *r)
{
    a.scale = 1.f;
    if (!r) return;
    a.positions = r->positions, a.axis_stride = r->axis_stride, a.freqs = r->freqs, a.pair_axis = r->pair_axis;
    a.axes = r->axes, a.rotary = r->rotary, a.interleaved = r->interleaved, a.backward = r->backward, a.scale = r->scale;
}

// Checks of a norm's call; `a` is filled.  Nothing is left to do where both
// sides have no heads.
int32_t norm_args(const quartz_norm_side_t *q, const quartz_norm_side_t *k, int32_t type, int32_t w_type, int64_t tokens,
                  int32_t dim, float eps, const quartz_rope_axes_t *rope, bool backward, HeadNormArgs &a)
{
    if (!q || !k || !type_ok(type) || !type_ok(w_type) || tokens < 0 || tokens > kMaxTokens) return QUARTZ_ERR_INVALID_ARG;
    if (!std::isfinite(eps) || eps < 0.f) return QUARTZ_ERR_INVALID_ARG;
    int32_t rc = check_dim(dim);
    if (rc == QUARTZ_OK && rope) rc = rope->backward ? QUARTZ_ERR_INVALID_ARG : check_rope(rope, dim);
    if (rc == QUARTZ_OK) rc = check_side(q, type, w_type, tokens, backward);
    if (rc == QUARTZ_OK) rc = check_side(k, type, w_type, tokens, backward);
    if (rc != QUARTZ_OK) return rc;
    a.side[0] = side_of(*q), a.side[1] = side_of(*k);
    for (HeadNormSide &s : a.side)
        if (!s.heads) {
            void *dw = s.dw;  // 0
            s = {};
            s.dw = dw;
        }
    a.tokens = tokens, a.type = type, a.w_type = w_type, a.dim = dim, a.eps = eps, a.inv_dim = 1.f / static_cast<float>(dim);
    set_rope(a, rope);
    return QUARTZ_OK;
}

int32_t check_tokens(const quartz_paged_cache_t *c, int64_t tokens, int64_t seqs, int32_t q_heads, int64_t max_len,
                     int64_t max_new)
{
    const int32_t rc = check_paged_cache(c);
    if (rc != QUARTZ_OK) return rc;
    if (seqs < 0 || seqs > 65535 || q_heads < 1 || q_heads > 65536 || q_heads % c->heads) return QUARTZ_ERR_INVALID_ARG;
    if (tokens < 0 || tokens > kMaxTokens || max_len < 0 || max_len > kMaxTokens || max_new < 0 ||
        max_new > kMaxTokens / (q_heads / c->heads))
        return QUARTZ_ERR_INVALID_ARG;
    return paged_tokens_countable(c, tokens, seqs, q_heads, max_len, max_new) ? QUARTZ_OK : QUARTZ_ERR_UNSUPPORTED;
}

}  // namespace

extern "C" {

int32_t quartz_rope_axes(const void *x, int64_t x_stride_token, int64_t x_stride_head, void *y, int64_t y_stride_token,
                         int64_t y_stride_head, int32_t type, int64_t tokens, int32_t heads, int32_t dim,
                         const quartz_rope_axes_t *rope, void *stream)
{
    if (!rope || !type_ok(type) || tokens < 0 || tokens > kMaxTokens) return QUARTZ_ERR_INVALID_ARG;
    int32_t rc = check_dim(dim);
    if (rc == QUARTZ_OK) rc = check_rope(rope, dim);
    if (rc != QUARTZ_OK) return rc;
    const quartz_norm_side_t s{x, x_stride_token, x_stride_head, nullptr, 0, 0, y, y_stride_token, y_stride_head, nullptr,
                               nullptr, heads};
    rc = check_side(&s, type, type, tokens, false);
    if (rc != QUARTZ_OK || tokens == 0 || heads == 0) return rc;
    HeadNormArgs a{};
    a.side[0] = side_of(s);
    a.tokens = tokens, a.type = type, a.w_type = type, a.dim = dim;
    set_rope(a, rope);
    a.dev_err = device_error_word();
    if (!a.dev_err) return QUARTZ_ERR_CUDA;
    return map_cuda(launch_rope_axes(a, static_cast<cudaStream_t>(stream)));
}

int32_t quartz_qk_norm_rope(const quartz_norm_side_t *q, const quartz_norm_side_t *k, int32_t type, int32_t w_type,
                            int64_t tokens, int32_t dim, float eps, const quartz_rope_axes_t *rope, void *stream)
{
    HeadNormArgs a{};
    const int32_t rc = norm_args(q, k, type, w_type, tokens, dim, eps, rope, false, a);
    if (rc != QUARTZ_OK || tokens == 0 || q->heads + k->heads == 0) return rc;
    a.dev_err = device_error_word();
    if (!a.dev_err) return QUARTZ_ERR_CUDA;
    return map_cuda(launch_head_norm(a, static_cast<cudaStream_t>(stream)));
}

size_t quartz_qk_norm_rope_workspace_size(int32_t dim)
{
    return check_dim(dim) == QUARTZ_OK ? head_norm_workspace_bytes(dim) : 0;
}

int32_t quartz_qk_norm_rope_backward(const quartz_norm_side_t *q, const quartz_norm_side_t *k, int32_t type,
                                     int32_t w_type, int64_t tokens, int32_t dim, float eps,
                                     const quartz_rope_axes_t *rope, void *workspace, size_t workspace_bytes,
                                     void *stream)
{
    HeadNormArgs a{};
    const int32_t rc = norm_args(q, k, type, w_type, tokens, dim, eps, rope, true, a);
    if (rc != QUARTZ_OK) return rc;
    const bool sums = a.side[0].dw || a.side[1].dw;
    if (sums) {
        if (!workspace || workspace_bytes < head_norm_workspace_bytes(dim)) return QUARTZ_ERR_WORKSPACE;
        if (!aligned(workspace, 16)) return QUARTZ_ERR_ALIGNMENT;
        a.part = static_cast<float *>(workspace);
    } else if (tokens == 0 || q->heads + k->heads == 0) {
        return QUARTZ_OK;
    }
    a.dev_err = device_error_word();
    if (!a.dev_err) return QUARTZ_ERR_CUDA;
    return map_cuda(launch_head_norm_backward(a, static_cast<cudaStream_t>(stream)));
}

size_t quartz_paged_attention_tokens_workspace_size(const quartz_paged_cache_t *cache, int64_t tokens, int64_t seqs,
                                                    int32_t q_heads, int64_t max_len, int64_t max_new)
{
    if (check_tokens(cache, tokens, seqs, q_heads, max_len, max_new) != QUARTZ_OK) return 0;
    return paged_tokens_workspace_bytes(cache, tokens, seqs, q_heads, max_len, max_new);
}

int32_t quartz_paged_attention_tokens(const void *q, int64_t q_stride_token, int64_t q_stride_head, int64_t tokens,
                                      int32_t q_heads, const quartz_paged_cache_t *cache, const int32_t *block_table,
                                      int64_t table_stride, const int32_t *seq_lens, const int32_t *starts,
                                      int64_t seqs, int64_t max_len, int64_t max_new,
                                      const quartz_tokens_mask_t *mask, float scale, void *o, int32_t o_type,
                                      void *workspace, size_t workspace_bytes, void *stream)
{
    const int32_t rc = check_tokens(cache, tokens, seqs, q_heads, max_len, max_new);
    if (rc != QUARTZ_OK) return rc;
    const quartz_tokens_mask_t m = mask ? *mask : quartz_tokens_mask_t{};
    constexpr float kLog2e = 1.4426950408889634f;  // the kernels work in the log2 domain
    if (!type_ok(o_type) || !std::isfinite(scale * kLog2e) || m.window < 0 || !std::isfinite(m.cap * kLog2e) || m.cap < 0.f ||
        (m.cap > 0.f && !std::isfinite(scale / m.cap)) || (m.tree && max_new > 64))
        return QUARTZ_ERR_INVALID_ARG;
    if (!stride_ok(q_stride_token) || !stride_ok(q_stride_head) || !stride_ok(table_stride)) return QUARTZ_ERR_INVALID_ARG;
    if (q_stride_token % 8 || q_stride_head % 8) return QUARTZ_ERR_ALIGNMENT;
    if (!aligned(m.tree, 8) || !aligned(m.prefix_lens, 4) || !aligned(m.slopes, 4)) return QUARTZ_ERR_ALIGNMENT;
    if (seqs == 0 || tokens == 0 || max_new == 0) return QUARTZ_OK;
    if (!q || !o || !seq_lens || !starts || (max_len > 0 && !block_table)) return QUARTZ_ERR_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(o, 16) || !aligned(block_table, 4) || !aligned(seq_lens, 4) || !aligned(starts, 4))
        return QUARTZ_ERR_ALIGNMENT;
    if (!workspace || workspace_bytes < paged_tokens_workspace_bytes(cache, tokens, seqs, q_heads, max_len, max_new))
        return QUARTZ_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return QUARTZ_ERR_ALIGNMENT;
    PagedTokensCall a{q, q_stride_token, q_stride_head, tokens, q_heads, block_table, table_stride, seq_lens, starts, seqs,
                      max_len, max_new, m, scale, o, o_type, workspace, device_error_word()};
    if (!a.dev_err) return QUARTZ_ERR_CUDA;
    return map_cuda(launch_paged_tokens(cache, a, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
