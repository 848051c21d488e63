// C ABI of the calls around the FFN (cache, attention, beams): argument checks; the kernels stand in the files named below.
#include <limits.h>
#include <math.h>
#include <stdint.h>

#include <atomic>
#include <chrono>

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

int pop_cache_attention_kind(pop_dtype_t dtype, pop_dtype_t ydtype, int n_tokens, int n_seq, int n_heads, int n_kv, int d, int max_new,
                             int max_context, int window, int *parts)
{
    const int rc = attention_sizes(n_tokens, n_seq, n_heads, n_kv, d, max_new, max_context);
    if (rc != POP_OK) return rc;
    if (window < 0) return POP_ESHAPE;
    if (!is_dtype(dtype) || !is_dtype(ydtype)) return POP_EINVAL;
    const bool none = n_seq == 0 || n_tokens == 0;
    const int of_blocks =
        none ? 0 : cache_attention_parts(n_tokens, n_seq, n_heads, n_kv, d, max_new, max_context, window, dtype == POP_BF16 && ydtype == POP_BF16);
    if (parts) *parts = of_blocks;
    return none ? 0 : of_blocks > 0 ? 2 : 1;
}

int pop_cache_attention(const void *q, pop_dtype_t dtype, int n_tokens, const void *cache, int n_kv, int d, int page, int n_pages,
                        const int *block_table, int table_stride, const int *q_start, const int *context_len, int n_seq, int n_heads,
                        int max_new, int max_context, float scale, int window, void *y, pop_dtype_t ydtype, void *workspace,
                        size_t workspace_bytes, void *stream)
{
    CacheShape c;
    int rc = cache_shape(n_kv, d, page, n_pages, &c);
    if (rc == POP_OK) rc = attention_sizes(n_tokens, n_seq, n_heads, n_kv, d, max_new, max_context);
    if (rc != POP_OK) return rc;
    if (table_stride < 1 || window < 0) return POP_ESHAPE;
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
                       static_cast<float *>(workspace)};
    POP_HIP(launch_cache_attention(a, as_stream(stream)));
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

}  // extern "C"
