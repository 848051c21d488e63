// Format of the 4-bit cache of keys and values, shared by the kernels that write, read, move and attend over it.
//
// Values are e2m1 codes (sign, two bits of exponent, one of significand: 0 .5 1 1.5 2 3 4 6) with one scale byte for 32
// channels, 2^(byte - 127) (the OCP microscaling format MXFP4, which gfx950 converts to bf16 exactly, scale and all, two
// values an instruction).  A *tile* is 16 tokens of one kv head, contiguous:
//     K codes [16 tokens][D/2] | V codes [4 groups of 4 tokens][16][4 tokens][D/32] | K scales [16][D/32] | V scales [4][D/32][4]
// 16 (D + D/16) bytes, 17 lines of 128 bytes for D = 128.  The order is that of the matrix products' operands: a lane that
// holds a quarter of a token's channels of K reads one run of D/8 bytes; a lane that holds D/16 channels of V (all of one
// scale) and four tokens reads one run of D/8 bytes and one word of scales.  A token's own bytes stay whole (K: one run, V:
// runs of D/32 bytes), so a single token is written without reading others.  A page is [n_kv][page/16] tiles.
#pragma once
#include "pop_internal.h"

namespace pop {

struct CacheShape {
    int n_kv, d, page, log_page, n_pages;
};

__host__ __device__ constexpr int cache_tile_bytes(int d) { return 16 * (d + d / 16); }
__host__ __device__ inline size_t cache_page_bytes(const CacheShape &c)
{
    return (size_t)c.n_kv * (c.page / 16) * cache_tile_bytes(c.d);
}

// Byte offset of the tile that holds token `at` of a page, for one kv head (64-bit: a long cache passes 32 bits).
__device__ __forceinline__ size_t cache_tile_offset(int page, int head, int at, int n_kv, int log_page, int tile_bytes)
{
    return ((((size_t)page * n_kv + head) << (log_page - 4)) + (at >> 4)) * tile_bytes;
}

// Scale byte for a block whose largest magnitude has the float32 bits `top` (finite): its exponent less two, so that it lies
// in [4, 8) of the codes' range, and one more from a significand of 1.75 on (7 and above would be cut to 6, an error of over one
// step).  1 .. 252: a stored pattern never decodes to an infinity or a NaN, so what a mask hides cannot leak through a product.
__device__ __forceinline__ int cache_scale_byte(uint32_t top)
{
    const int byte = (int)((top + 0x200000u) >> 23) - 2;
    return min(max(byte, 1), 252);
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// The two values of byte B of `codes`, as packed bf16 (exact).
template <int B>
__device__ __forceinline__ uint32_t cache_pair(uint32_t codes, float scale)
{
    const bf16x2 v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, B);
    return __builtin_bit_cast(uint32_t, v);
}
// The same for a byte number that is a constant once loops are unrolled.
__device__ __forceinline__ uint32_t cache_pair_at(uint32_t codes, float scale, int byte)
{
    switch (byte) {
        case 0: return cache_pair<0>(codes, scale);
        case 1: return cache_pair<1>(codes, scale);
        case 2: return cache_pair<2>(codes, scale);
        default: return cache_pair<3>(codes, scale);
    }
}

__device__ __forceinline__ float cache_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Workgroups of one launch that hand their results to the last of them count themselves in a word {tag, number}.  The tag (48 bits)
// is the launch's own: a word with any other content counts as none, and the last one to arrive leaves it 0, so nothing has to be
// cleared before a launch, and a captured launch can be replayed.  Nobody waits.  A word that has the tag is added to; exchanges, which
// cost 0.6 us each where many arrive together (64 of them: 40 us), are left to whoever finds it without.
//
// Called by one thread once the workgroup's results are on their way past the caches and acknowledged; true for the last of
// `expected` (2 .. 65535).
__device__ __forceinline__ bool arrive_last(unsigned long long *word, unsigned long long tag, int expected)
{
    unsigned long long seen = __hip_atomic_fetch_add(word, 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if ((seen & ~0xffffull) != tag) {  // not there yet: that addition does not count, whatever it was added to
        for (seen += 1; (seen & ~0xffffull) != tag;)
            if (__hip_atomic_compare_exchange_strong(word, &seen, tag | 1, __ATOMIC_RELAXED, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) return false;
        seen = __hip_atomic_fetch_add(word, 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if ((int)(seen & 0xffffull) + 1 != expected) return false;
    __hip_atomic_store(word, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return true;
}
// Puts the tag there ahead of time, so that those who arrive add: `seen` is what coherent_load(word) gave.
__device__ __forceinline__ void announce(unsigned long long *word, unsigned long long seen, unsigned long long tag)
{
    if ((seen & ~0xffffull) != tag)
        __hip_atomic_compare_exchange_strong(word, &seen, tag, __ATOMIC_RELAXED, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
unsigned long long launch_tag();  // host: another one for every launch, never 0

// Launchers.  Arguments have been checked; each returns the launch's status.
struct PlanArgs {
    const int *cached, *fresh;  // [n_seq] tokens in the cache, new tokens
    int n_seq, log_page;
    int *table;                 // [n_seq][stride]
    int stride;
    const int *ring, *pool;
    int n_pages;
    int *pool_out;
    int max_tokens;
    int *context, *start, *slots, *positions, *status;
};
hipError_t launch_cache_plan(const PlanArgs &a, hipStream_t s);

struct ReorderArgs {
    const int *table, *length, *parents;
    int n_seq, group, log_page, stride;
    int *new_table, *new_length, *copies;
    int *ring;
    int n_pages;
    const int *pool;
    int *pool_out, *counts, *status;
};
size_t reorder_counts(int n_seq, int group, int stride);  // ints of scratch
hipError_t launch_cache_reorder(const ReorderArgs &a, hipStream_t s);
hipError_t launch_cache_copy_pages(void *cache, const CacheShape &c, const int *copies, int n, hipStream_t s);
hipError_t launch_cache_write(void *cache, const CacheShape &c, const void *k, const void *v, int is_bf16, long long k_stride,
                              long long v_stride, const int *slots, int n_tokens, hipStream_t s);
hipError_t launch_cache_read(const void *cache, const CacheShape &c, const int *slots, int n_tokens, void *k, void *v,
                             int is_bf16, hipStream_t s);

struct AttentionArgs {
    const void *q;
    int q_bf16, n_tokens;
    const unsigned char *cache;
    CacheShape c;
    const int *table;
    int stride;
    const int *start, *context;
    int n_seq, n_heads, max_new, max_context;
    float scale;
    int window;
    void *y;
    int y_bf16;
    float *ws;
    int sinks;  // first tokens that stay visible next to a window
};
// What a call runs: blocks of 128 columns and the parts of their tokens, or (no blocks) so many workgroups of the general kernel, which load
// codes past the caches or not.
struct AttentionLaunch {
    int blocks, splits, workgroups;
    bool past;
};
hipError_t launch_attention_sinks(const AttentionArgs &a, const AttentionLaunch &l, hipStream_t s);  // (pop_cache_attention_sinks.hip)
size_t cache_attention_ws(int n_tokens, int n_seq, int n_heads, int n_kv, int d, int max_new, int max_context);
// Parts that the prompt kernel splits the tokens of a block of 128 columns into, 0 where the general kernel takes the call.
int cache_attention_parts(int n_tokens, int n_seq, int n_heads, int n_kv, int d, int max_new, int max_context, int window, int sinks, int all_bf16);
hipError_t launch_cache_attention(const AttentionArgs &a, hipStream_t s);

// Division of numbers below 2^31 by one that the host knows: ceil(2^(31 + l) / d) with 2^l >= d is off by less than 2^l / d parts of a quotient.
struct Divisor {
    unsigned factor, shift;
    explicit Divisor(int d) : shift(31)
    {
        while (1ull << (shift - 31) < (unsigned)d) ++shift;
        factor = (unsigned)(((1ull << shift) + d - 1) / d);
    }
    __device__ __forceinline__ int of(int x) const { return (int)(((unsigned long long)(unsigned)x * factor) >> shift); }
};

struct SharedArgs {
    AttentionArgs a;
    Divisor by_share, by_kv, by_group;  // query heads to a kv head, kv heads, sequences of a group
    int group;          // sequences of a group
    const int *prefix;  // [n_seq / group] tokens that a group's sequences share
    size_t ws_bytes;    // of the caller's workspace
    // set by the launcher
    float *prefix_pieces, *own_pieces, *states;
    int prefix_columns, own_columns, prefix_places, own_places;
};
// 0: nothing to do, 1: each sequence for itself (launch_cache_attention), 2: the prefix by blocks of 16 or 32 columns of a group, 3: by blocks of 128.
int cache_attention_shared_kind(int n_tokens, int n_seq, int group, int n_heads, int n_kv, int d, int max_new, int max_context, int all_bf16);
// Bytes for calls of these sizes, or smaller n_tokens, n_seq, max_new and max_context, of any types.
size_t cache_attention_shared_ws(int n_tokens, int n_seq, int group, int n_heads, int n_kv, int d, int max_new, int max_context);
// Bytes that a call of these types and sizes lays out in its workspace.
size_t cache_attention_shared_used(int n_tokens, int n_seq, int group, int n_heads, int n_kv, int d, int max_new, int max_context, int all_bf16);
hipError_t launch_cache_attention_shared(SharedArgs h, hipStream_t s);  // (pop_cache_attention_shared.hip)

struct BeamArgs {
    const void *logits;
    int is_bf16;
    const float *scores;
    const unsigned char *done;
    int requests, beams, vocab, k, pad;
    float *out_scores;
    int *out_tokens, *out_parents;
    void *ws;
};
size_t beam_ws(int requests, int beams, int vocab, int k);
hipError_t launch_beam_select(const BeamArgs &a, hipStream_t s);

}  // namespace pop
