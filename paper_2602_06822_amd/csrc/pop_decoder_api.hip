// C ABI of the calls around the FFN (cache, attention, beams, norms, rotary positions): argument checks; the kernels stand in the files named below.
#include <limits.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>
#include <chrono>

#include "pop_block.h"  // pop_block.hip
#include "pop_cache.h"  // pop_cache.hip, pop_cache_attention.hip, pop_beam.hip

using namespace pop;

namespace {

#define POP_HIP(call)                                      \
    do {                                                   \
        hipError_t e__ = (call);                           \
        if (e__ != hipSuccess) return hip_fail(e__, #call); \
    } while (0)

inline hipStream_t as_stream(void *s) { return reinterpret_cast<hipStream_t>(s); }
inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool is_dtype(int t) { return t == POP_F32 || t == POP_BF16; }

// An axis of a grid counts its threads in 32 bits: workgroups of 256.
constexpr int kMostWorkgroups = (1 << 24) - 1;

inline bool aligned_to(const void *p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }
inline int size_of(pop_dtype_t t) { return t == POP_BF16 ? 2 : 4; }
// A workgroup of up to 1024 threads for each token.
constexpr int kMostTokenRows = 1 << 22;

int log_of_page(int page)
{
    for (int l = 4; l <= 8; ++l)
        if (page == 1 << l) return l;
    return -1;
}

int cache_shape(int n_kv, int d, int page, int n_pages, CacheShape *c)
{
    if (n_kv < 1 || d < 1 || page < 1 || n_pages < 1) return POP_ESHAPE;
    const int l = log_of_page(page);
    if (l < 0 || (d != 64 && d != 128 && d != 256) || n_kv > 65535 || (long long)n_pages * page > INT_MAX) return POP_EUNSUPPORTED;
    c->n_kv = n_kv, c->d = d, c->page = page, c->log_page = l, c->n_pages = n_pages;
    return POP_OK;
}

}  // namespace

unsigned long long pop::launch_tag()
{
    // odd multiples of one number below 2^48, from a place that differs from process to process: what an earlier program left in a
    // workspace is no tag of this one's
    static std::atomic<unsigned long long> n{(unsigned long long)std::chrono::steady_clock::now().time_since_epoch().count() * 2};
    const unsigned long long t = (n.fetch_add(2, std::memory_order_relaxed) | 1) * 0x9e3779b97f4b15ull;
    return t << 16;
}

extern "C" {

int pop_cache_bytes(int n_kv, int d, int page, int n_pages, size_t *bytes)
{
    if (!bytes) return POP_EINVAL;
    CacheShape c;
    const int rc = cache_shape(n_kv, d, page, n_pages, &c);
    if (rc != POP_OK) return rc;
    *bytes = cache_page_bytes(c) * n_pages;
    return POP_OK;
}

int pop_cache_plan(const int *cached_len, const int *new_len, int n_seq, int page, int *block_table, int table_stride, const int *ring,
                   int n_pages, const int *pool, int *pool_out, int max_tokens, int *context_len, int *q_start, int *slots,
                   int *positions, int *status, void *stream)
{
    if (n_seq < 0 || page < 1 || table_stride < 1 || n_pages < 1 || max_tokens < 0) return POP_ESHAPE;
    if (!q_start || !ring || !pool || !pool_out || !status || (max_tokens && !slots)) return POP_EINVAL;
    if (n_seq && (!cached_len || !new_len || !block_table || !context_len)) return POP_EINVAL;
    if (pool_out == pool || (n_seq && (context_len == cached_len || context_len == new_len))) return POP_EINVAL;
    const int l = log_of_page(page);
    if (l < 0 || (long long)n_pages * page > INT_MAX || (long long)table_stride * page > 1 << 30) return POP_EUNSUPPORTED;
    PlanArgs a = {cached_len, new_len, n_seq, l, block_table, table_stride, ring, pool, n_pages, pool_out, max_tokens, context_len,
                  q_start, slots, positions, status};
    POP_HIP(launch_cache_plan(a, as_stream(stream)));
    return POP_OK;
}

int pop_cache_write(void *cache, int n_kv, int d, int page, int n_pages, const void *k, const void *v, pop_dtype_t dtype,
                    long long k_stride, long long v_stride, const int *slots, int n_tokens, void *stream)
{
    CacheShape c;
    const int rc = cache_shape(n_kv, d, page, n_pages, &c);
    if (rc != POP_OK) return rc;
    if (!is_dtype(dtype)) return POP_EINVAL;
    const int unit = dtype == POP_BF16 ? 8 : 4;
    if (n_tokens < 0 || k_stride < (long long)n_kv * d || v_stride < (long long)n_kv * d || k_stride % unit || v_stride % unit) return POP_ESHAPE;
    if (n_tokens == 0) return POP_OK;
    if (!cache || !k || !v || !slots || !aligned16(cache) || !aligned16(k) || !aligned16(v)) return POP_EINVAL;
    if ((long long)n_tokens * n_kv > INT_MAX / (d / 8)) return POP_EUNSUPPORTED;
    POP_HIP(launch_cache_write(cache, c, k, v, dtype == POP_BF16, k_stride, v_stride, slots, n_tokens, as_stream(stream)));
    return POP_OK;
}

int pop_cache_read(const void *cache, int n_kv, int d, int page, int n_pages, const int *slots, int n_tokens, void *k, void *v,
                   pop_dtype_t dtype, void *stream)
{
    CacheShape c;
    const int rc = cache_shape(n_kv, d, page, n_pages, &c);
    if (rc != POP_OK) return rc;
    if (!is_dtype(dtype)) return POP_EINVAL;
    if (n_tokens < 0) return POP_ESHAPE;
    if (n_tokens == 0) return POP_OK;
    if (!cache || !k || !v || !slots || !aligned16(cache) || !aligned16(k) || !aligned16(v)) return POP_EINVAL;
    if ((long long)n_tokens * n_kv > INT_MAX / (d / 8)) return POP_EUNSUPPORTED;
    POP_HIP(launch_cache_read(cache, c, slots, n_tokens, k, v, dtype == POP_BF16, as_stream(stream)));
    return POP_OK;
}

static int attention_sizes(int n_tokens, int n_seq, int n_heads, int n_kv, int d, int max_new, int max_context)
{
    if (n_tokens < 0 || n_seq < 0 || n_heads < 1 || n_kv < 1 || n_heads % n_kv || max_new < 1 || max_context < 1) return POP_ESHAPE;
    if (d != 64 && d != 128 && d != 256) return POP_EUNSUPPORTED;
    if ((long long)n_seq * n_kv > 65535 || (long long)n_tokens * n_heads > INT_MAX / 2) return POP_EUNSUPPORTED;
    return POP_OK;
}

int pop_cache_attention_workspace(int n_tokens, int n_seq, int n_heads, int n_kv, int d, int max_new, int max_context, size_t *bytes)
{
    if (!bytes) return POP_EINVAL;
    const int rc = attention_sizes(n_tokens, n_seq, n_heads, n_kv, d, max_new, max_context);
    if (rc != POP_OK) return rc;
    *bytes = n_seq ? cache_attention_ws(n_tokens, n_seq, n_heads, n_kv, d, max_new, max_context) : 0;
    return POP_OK;
}

int pop_cache_attention_sinks_kind(pop_dtype_t dtype, pop_dtype_t ydtype, int n_tokens, int n_seq, int n_heads, int n_kv, int d, int max_new,
                                   int max_context, int window, int sinks, int *parts)
{
    const int rc = attention_sizes(n_tokens, n_seq, n_heads, n_kv, d, max_new, max_context);
    if (rc != POP_OK) return rc;
    if (window < 0 || sinks < 0) return POP_ESHAPE;
    if (!is_dtype(dtype) || !is_dtype(ydtype)) return POP_EINVAL;
    const bool none = n_seq == 0 || n_tokens == 0;
    const int of_blocks =
        none ? 0 : cache_attention_parts(n_tokens, n_seq, n_heads, n_kv, d, max_new, max_context, window, sinks, dtype == POP_BF16 && ydtype == POP_BF16);
    if (parts) *parts = of_blocks;
    return none ? 0 : of_blocks > 0 ? 2 : 1;
}

int pop_cache_attention_kind(pop_dtype_t dtype, pop_dtype_t ydtype, int n_tokens, int n_seq, int n_heads, int n_kv, int d, int max_new,
                             int max_context, int window, int *parts)
{
    return pop_cache_attention_sinks_kind(dtype, ydtype, n_tokens, n_seq, n_heads, n_kv, d, max_new, max_context, window, 0, parts);
}

int pop_cache_attention_sinks(const void *q, pop_dtype_t dtype, int n_tokens, const void *cache, int n_kv, int d, int page, int n_pages,
                              const int *block_table, int table_stride, const int *q_start, const int *context_len, int n_seq, int n_heads,
                              int max_new, int max_context, float scale, int window, int sinks, void *y, pop_dtype_t ydtype, void *workspace,
                              size_t workspace_bytes, void *stream)
{
    CacheShape c;
    int rc = cache_shape(n_kv, d, page, n_pages, &c);
    if (rc == POP_OK) rc = attention_sizes(n_tokens, n_seq, n_heads, n_kv, d, max_new, max_context);
    if (rc != POP_OK) return rc;
    if (table_stride < 1 || window < 0 || sinks < 0) return POP_ESHAPE;
    if ((long long)table_stride * page > 1 << 30) return POP_EUNSUPPORTED;
    if (!is_dtype(dtype) || !is_dtype(ydtype) || !isfinite(scale)) return POP_EINVAL;
    // rounds of 128 tokens are counted in 32 bits
    if (((long long)n_tokens * (n_heads / n_kv) / 16 + n_seq) * n_kv * ((long long)table_stride * page / 128 + 1) > INT_MAX) return POP_EUNSUPPORTED;
    if (n_seq == 0 || n_tokens == 0) return POP_OK;
    if (!q || !cache || !block_table || !q_start || !context_len || !y) return POP_EINVAL;
    if (!aligned16(q) || !aligned16(cache) || !aligned16(y) || !aligned16(workspace)) return POP_EINVAL;
    const size_t need = cache_attention_ws(n_tokens, n_seq, n_heads, n_kv, d, max_new, max_context);
    if (need && !workspace) return POP_EINVAL;
    if (workspace_bytes < need) return POP_ESHAPE;
    AttentionArgs a = {q, dtype == POP_BF16, n_tokens, static_cast<const unsigned char *>(cache), c, block_table, table_stride, q_start,
                       context_len, n_seq, n_heads, max_new, max_context, scale, window, y, ydtype == POP_BF16,
                       static_cast<float *>(workspace), sinks};
    POP_HIP(launch_cache_attention(a, as_stream(stream)));
    return POP_OK;
}

int pop_cache_attention(const void *q, pop_dtype_t dtype, int n_tokens, const void *cache, int n_kv, int d, int page, int n_pages,
                        const int *block_table, int table_stride, const int *q_start, const int *context_len, int n_seq, int n_heads,
                        int max_new, int max_context, float scale, int window, void *y, pop_dtype_t ydtype, void *workspace,
                        size_t workspace_bytes, void *stream)
{
    return pop_cache_attention_sinks(q, dtype, n_tokens, cache, n_kv, d, page, n_pages, block_table, table_stride, q_start, context_len, n_seq, n_heads,
                                     max_new, max_context, scale, window, 0, y, ydtype, workspace, workspace_bytes, stream);
}

static int shared_sizes(int n_tokens, int n_seq, int group, int n_heads, int n_kv, int d, int max_new, int max_context)
{
    const int rc = attention_sizes(n_tokens, n_seq, n_heads, n_kv, d, max_new, max_context);
    if (rc != POP_OK) return rc;
    return group < 1 || n_seq % group ? POP_ESHAPE : POP_OK;
}

int pop_cache_attention_shared_workspace(int n_tokens, int n_seq, int group, int n_heads, int n_kv, int d, int max_new, int max_context, size_t *bytes)
{
    if (!bytes) return POP_EINVAL;
    const int rc = shared_sizes(n_tokens, n_seq, group, n_heads, n_kv, d, max_new, max_context);
    if (rc != POP_OK) return rc;
    *bytes = n_seq ? cache_attention_shared_ws(n_tokens, n_seq, group, n_heads, n_kv, d, max_new, max_context) : 0;
    return POP_OK;
}

int pop_cache_attention_shared_used(pop_dtype_t dtype, pop_dtype_t ydtype, int n_tokens, int n_seq, int group, int n_heads, int n_kv, int d, int max_new,
                                    int max_context, size_t *bytes)
{
    if (!bytes) return POP_EINVAL;
    const int rc = shared_sizes(n_tokens, n_seq, group, n_heads, n_kv, d, max_new, max_context);
    if (rc != POP_OK) return rc;
    if (!is_dtype(dtype) || !is_dtype(ydtype)) return POP_EINVAL;
    *bytes = cache_attention_shared_used(n_tokens, n_seq, group, n_heads, n_kv, d, max_new, max_context, dtype == POP_BF16 && ydtype == POP_BF16);
    return POP_OK;
}

int pop_cache_attention_shared_kind(pop_dtype_t dtype, pop_dtype_t ydtype, int n_tokens, int n_seq, int group, int n_heads, int n_kv, int d, int max_new,
                                    int max_context)
{
    const int rc = shared_sizes(n_tokens, n_seq, group, n_heads, n_kv, d, max_new, max_context);
    if (rc != POP_OK) return rc;
    if (!is_dtype(dtype) || !is_dtype(ydtype)) return POP_EINVAL;
    return cache_attention_shared_kind(n_tokens, n_seq, group, n_heads, n_kv, d, max_new, max_context, dtype == POP_BF16 && ydtype == POP_BF16);
}

int pop_cache_attention_shared(const void *q, pop_dtype_t dtype, int n_tokens, const void *cache, int n_kv, int d, int page, int n_pages,
                               const int *block_table, int table_stride, const int *q_start, const int *context_len, int n_seq, int group,
                               const int *prefix_len, int n_heads, int max_new, int max_context, float scale, void *y, pop_dtype_t ydtype,
                               void *workspace, size_t workspace_bytes, void *stream)
{
    CacheShape c;
    int rc = cache_shape(n_kv, d, page, n_pages, &c);
    if (rc == POP_OK) rc = shared_sizes(n_tokens, n_seq, group, n_heads, n_kv, d, max_new, max_context);
    if (rc != POP_OK) return rc;
    if (table_stride < 1) return POP_ESHAPE;
    if ((long long)table_stride * page > 1 << 30) return POP_EUNSUPPORTED;
    if (!is_dtype(dtype) || !is_dtype(ydtype) || !isfinite(scale)) return POP_EINVAL;
    // rounds of 128 tokens, of prefixes and of what stands behind them, are counted in 32 bits
    if (((long long)n_tokens * (n_heads / n_kv) / 16 + n_seq) * n_kv * ((long long)table_stride * page / 128 + 1) > INT_MAX / 2) return POP_EUNSUPPORTED;
    if (n_seq == 0 || n_tokens == 0) return POP_OK;
    if (!q || !cache || !block_table || !q_start || !context_len || !prefix_len || !y) return POP_EINVAL;
    if (!aligned16(q) || !aligned16(cache) || !aligned16(y) || !aligned16(workspace)) return POP_EINVAL;
    const size_t need = cache_attention_shared_ws(n_tokens, n_seq, group, n_heads, n_kv, d, max_new, max_context);
    if (need && !workspace) return POP_EINVAL;
    if (workspace_bytes < need) return POP_ESHAPE;
    SharedArgs h = {{q, dtype == POP_BF16, n_tokens, static_cast<const unsigned char *>(cache), c, block_table, table_stride, q_start, context_len, n_seq,
                     n_heads, max_new, max_context, scale, 0, y, ydtype == POP_BF16, static_cast<float *>(workspace), 0},
                    Divisor(n_heads / n_kv), Divisor(n_kv), Divisor(group), group, prefix_len, workspace_bytes, nullptr, nullptr, nullptr, 0, 0, 0, 0};
    POP_HIP(launch_cache_attention_shared(h, as_stream(stream)));
    return POP_OK;
}

static int beam_sizes(int n_requests, int n_beams, int vocab, int k)
{
    if (n_requests < 0 || n_beams < 1 || vocab < 1 || k < 1 || (long long)n_beams * vocab < k) return POP_ESHAPE;
    if (n_beams > POP_MAX_BEAMS || k > 64 || vocab > 1 << 24 || n_requests > kMostWorkgroups / n_beams) return POP_EUNSUPPORTED;
    return POP_OK;
}

int pop_beam_workspace(int n_requests, int n_beams, int vocab, int k, size_t *bytes)
{
    if (!bytes) return POP_EINVAL;
    const int rc = beam_sizes(n_requests, n_beams, vocab, k);
    if (rc != POP_OK) return rc;
    *bytes = beam_ws(n_requests, n_beams, vocab, k);
    return POP_OK;
}

int pop_beam_select(const void *logits, pop_dtype_t dtype, const float *scores, const unsigned char *done, int n_requests, int n_beams,
                    int vocab, int k, int pad_token, float *out_scores, int *out_tokens, int *out_parents, void *workspace,
                    size_t workspace_bytes, void *stream)
{
    const int rc = beam_sizes(n_requests, n_beams, vocab, k);
    if (rc != POP_OK) return rc;
    if (!is_dtype(dtype)) return POP_EINVAL;
    if (pad_token < 0 || pad_token >= vocab) return POP_ESHAPE;
    if (n_requests == 0) return POP_OK;
    if (!logits || !scores || !out_scores || !out_tokens || !out_parents || !workspace) return POP_EINVAL;
    if (!aligned16(logits) || !aligned16(workspace) || out_scores == scores) return POP_EINVAL;
    if (workspace_bytes < beam_ws(n_requests, n_beams, vocab, k)) return POP_ESHAPE;
    BeamArgs a = {logits, dtype == POP_BF16, scores, done, n_requests, n_beams, vocab, k, pad_token, out_scores, out_tokens, out_parents, workspace};
    POP_HIP(launch_beam_select(a, as_stream(stream)));
    return POP_OK;
}

static int reorder_sizes(int n_seq, int n_beams, int table_stride)
{
    if (n_seq < 1 || n_beams < 1 || n_seq % n_beams || table_stride < 1) return POP_ESHAPE;
    if (n_beams > POP_MAX_BEAMS || n_seq / n_beams > kMostWorkgroups) return POP_EUNSUPPORTED;
    return POP_OK;
}

int pop_cache_reorder_workspace(int n_seq, int n_beams, int table_stride, size_t *bytes)
{
    if (!bytes) return POP_EINVAL;
    const int rc = reorder_sizes(n_seq, n_beams, table_stride);
    if (rc != POP_OK) return rc;
    *bytes = reorder_counts(n_seq, n_beams, table_stride) * sizeof(int);
    return POP_OK;
}

int pop_cache_reorder(const int *block_table, const int *len, const int *parents, int n_seq, int n_beams, int page, int table_stride,
                      int *new_table, int *new_len, int *copies, int *ring, int n_pages, const int *pool, int *pool_out, void *workspace,
                      size_t workspace_bytes, int *status, void *stream)
{
    const int rc = reorder_sizes(n_seq, n_beams, table_stride);
    if (rc != POP_OK) return rc;
    if (page < 1 || n_pages < 1) return POP_ESHAPE;
    const int l = log_of_page(page);
    if (l < 0 || (long long)n_pages * page > INT_MAX || (long long)table_stride * page > 1 << 30) return POP_EUNSUPPORTED;
    if (!ring || !pool || !pool_out || !status || pool_out == pool) return POP_EINVAL;
    if (!block_table || !len || !parents || !new_table || !new_len || !copies || new_table == block_table || new_len == len || !workspace)
        return POP_EINVAL;
    if (workspace_bytes < reorder_counts(n_seq, n_beams, table_stride) * sizeof(int)) return POP_ESHAPE;
    ReorderArgs a = {block_table, len, parents, n_seq, n_beams, l, table_stride, new_table, new_len, copies, ring, n_pages, pool, pool_out,
                     static_cast<int *>(workspace), status};
    POP_HIP(launch_cache_reorder(a, as_stream(stream)));
    return POP_OK;
}

int pop_cache_copy_pages(void *cache, int n_kv, int d, int page, int n_pages, const int *copies, int n_copies, void *stream)
{
    CacheShape c;
    const int rc = cache_shape(n_kv, d, page, n_pages, &c);
    if (rc != POP_OK) return rc;
    if (n_copies < 0) return POP_ESHAPE;
    if (n_copies > kMostWorkgroups) return POP_EUNSUPPORTED;
    if (n_copies == 0) return POP_OK;
    if (!cache || !copies || !aligned16(cache)) return POP_EINVAL;
    POP_HIP(launch_cache_copy_pages(cache, c, copies, n_copies, as_stream(stream)));
    return POP_OK;
}

int pop_block_norm(const void *x, pop_dtype_t xdtype, long long x_stride, const void *u, pop_dtype_t dtype, long long u_stride, const void *gate,
                   int gate_rows, long long gate_stride, int n_tokens, int d, const void *w_post, const void *w_pre, int post_norm,
                   float weight_offset, float eps, float x_scale, float u_scale, void *x_out, long long x_out_stride, void *z,
                   long long z_stride, void *stream)
{
    if (n_tokens < 0 || d < 1) return POP_ESHAPE;
    if (d > kMostNormWidth || n_tokens >= kMostTokenRows) return POP_EUNSUPPORTED;
    if (!is_dtype(xdtype) || !is_dtype(dtype)) return POP_EINVAL;
    if (!(eps > 0.0f) || !isfinite(eps) || !isfinite(weight_offset) || !isfinite(x_scale) || !isfinite(u_scale)) return POP_EINVAL;
    if (x_stride < d || (u && u_stride < d) || (x_out && x_out_stride < d) || (z && z_stride < d)) return POP_ESHAPE;
    if (gate ? (gate_rows != 1 && gate_rows != n_tokens) || (gate_rows > 1 && gate_stride < d) : gate_rows != 0) return POP_ESHAPE;
    if (n_tokens == 0) return POP_OK;
    if (!x || (!x_out && !z) || (!u && (gate || post_norm))) return POP_EINVAL;
    const int xs = size_of(xdtype), us = size_of(dtype);
    if (!aligned_to(x, xs) || !aligned_to(x_out, xs) || !aligned_to(u, us) || !aligned_to(gate, us) || !aligned_to(w_post, us) ||
        !aligned_to(w_pre, us) || !aligned_to(z, us))
        return POP_EINVAL;
    // a thread reads the channels that it writes before it writes them: an output may take an input's place, channel by channel
    const auto takes = [](const void *out, int os, long long of, const void *in, int is, long long from) { return out && out == in && (os != is || of != from); };
    if (takes(x_out, xs, x_out_stride, x, xs, x_stride) || takes(x_out, xs, x_out_stride, u, us, u_stride) || takes(z, us, z_stride, x, xs, x_stride) ||
        takes(z, us, z_stride, u, us, u_stride))
        return POP_EINVAL;
    if ((x_out && x_out == z) || (gate && (gate == x_out || gate == z)) || (w_pre && (w_pre == x_out || w_pre == z)) || (w_post && (w_post == x_out || w_post == z)))
        return POP_EINVAL;
    BlockNormArgs a = {x, xdtype == POP_BF16, x_stride, u, dtype == POP_BF16, u ? u_stride : 0, gate, gate && gate_rows > 1 ? gate_stride : 0, w_post, w_pre,
                       n_tokens, d, post_norm != 0, weight_offset, eps, x_scale, u_scale, x_out, x_out ? x_out_stride : 0, z, z ? z_stride : 0};
    POP_HIP(launch_block_norm(a, as_stream(stream)));
    return POP_OK;
}

int pop_rotary_frequencies(int rotary_dim, double base, int scaling, double factor, double context, double low, double high, double *turns,
                           float *amplitude)
{
    if (!turns || scaling < POP_ROTARY_PLAIN || scaling > POP_ROTARY_RAMP) return POP_EINVAL;
    if (rotary_dim < (scaling == POP_ROTARY_BASE ? 4 : 2) || rotary_dim % 2 || rotary_dim > kMostRotary) return POP_ESHAPE;
    if (!(base > 1.0) || !isfinite(base)) return POP_EINVAL;
    if (scaling != POP_ROTARY_PLAIN && (!(factor >= 1.0) || !isfinite(factor))) return POP_EINVAL;
    const bool banded = scaling >= POP_ROTARY_BANDS;
    if (banded && (!(context > 0.0) || !isfinite(context) || !(low > 0.0) || !(high > low) || !isfinite(high))) return POP_EINVAL;
    const double r = rotary_dim, whole = 2.0 * M_PI;
    if (scaling == POP_ROTARY_BASE) base *= pow(factor, r / (r - 2.0));
    if (!isfinite(base)) return POP_EINVAL;
    // the place i (no whole number) of the frequency that makes so many rotations over the context
    const auto place = [&](double rotations) { return r * log(context / (whole * rotations)) / (2.0 * log(base)); };
    double begin = 0.0, end = 0.0;
    if (scaling == POP_ROTARY_RAMP) {
        begin = fmin(fmax(floor(place(high)), 0.0), r - 1.0), end = fmin(fmax(ceil(place(low)), 0.0), r - 1.0);
        if (end == begin) end += 1e-3;
    }
    for (int i = 0; i < rotary_dim / 2; ++i) {
        const double f = pow(base, -2.0 * i / r) / whole;
        double kept = 1.0;  // how much of the frequency is not divided
        if (scaling == POP_ROTARY_LINEAR) kept = 0.0;
        if (scaling == POP_ROTARY_BANDS) kept = (context * f - low) / (high - low);
        if (scaling == POP_ROTARY_RAMP) kept = 1.0 - (i - begin) / (end - begin);
        kept = fmin(fmax(kept, 0.0), 1.0);
        turns[i] = kept == 1.0 ? f : (1.0 - kept) * f / factor + kept * f;
    }
    if (amplitude) *amplitude = scaling == POP_ROTARY_RAMP ? (float)(1.0 + 0.1 * log(factor)) : 1.0f;
    return POP_OK;
}

int pop_rotary(const void *q, const void *k, pop_dtype_t dtype, int n_tokens, int n_heads, int n_kv, int d, int rotary_dim, int layout,
               long long q_stride, long long k_stride, const int *positions, const double *turns, float amplitude, void *q_out, void *k_out,
               long long q_out_stride, long long k_out_stride, void *stream)
{
    if (n_tokens < 0 || n_heads < 1 || (k && n_kv < 1) || d < 1 || rotary_dim < 2 || rotary_dim % 2 || rotary_dim > d) return POP_ESHAPE;
    const int of_k = k ? n_kv : 0;
    if (rotary_dim > kMostRotary || ((long long)n_heads + of_k) * d >= 1 << 26 || n_tokens >= kMostTokenRows) return POP_EUNSUPPORTED;
    if (!is_dtype(dtype) || (layout != POP_ROTARY_HALVES && layout != POP_ROTARY_PAIRS) || !isfinite(amplitude)) return POP_EINVAL;
    if (q_stride < (long long)n_heads * d || q_out_stride < (long long)n_heads * d) return POP_ESHAPE;
    if (k && (k_stride < (long long)n_kv * d || k_out_stride < (long long)n_kv * d)) return POP_ESHAPE;
    if (n_tokens == 0) return POP_OK;
    if (!q || !q_out || !k != !k_out || !positions || !turns) return POP_EINVAL;
    const int size = size_of(dtype);
    if (!aligned_to(q, size) || !aligned_to(k, size) || !aligned_to(q_out, size) || !aligned_to(k_out, size) || !aligned_to(positions, 4) ||
        !aligned_to(turns, 8))
        return POP_EINVAL;
    if ((q_out == q && q_out_stride != q_stride) || (k && k_out == k && k_out_stride != k_stride) || q_out == k || q_out == k_out || k_out == q)
        return POP_EINVAL;
    RotaryArgs a = {q, k, dtype == POP_BF16, n_tokens, n_heads, of_k, d, rotary_dim, layout == POP_ROTARY_PAIRS, q_stride, k ? k_stride : 0, positions, turns,
                    amplitude, q_out, k_out, q_out_stride, k ? k_out_stride : 0};
    POP_HIP(launch_rotary(a, as_stream(stream)));
    return POP_OK;
}

}  // extern "C"
