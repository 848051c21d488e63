// The 4-bit cache of keys and values and the block tables that address it: writing and reading tokens, the plan of a
// step (pages and slots from request lengths), the reordering of rows after a beam search's selection, page copies.
#include <limits.h>

#include "pop_cache.h"

namespace pop {

namespace {

// ---------------------------------------------------------------- tokens into the cache and out of it

// Eight channels of a row as float32, and whether one of them is no finite number.
template <bool BF16>
__device__ __forceinline__ void load8(const void *p, long long at, float (&x)[8])
{
    if constexpr (BF16) {
        const uint4 r = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p) + at);
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) x[2 * i] = bf16_lo(w[i]), x[2 * i + 1] = bf16_hi(w[i]);
    } else {
        const float4 *f = reinterpret_cast<const float4 *>(static_cast<const float *>(p) + at);
        const float4 a = f[0], b = f[1];
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    }
}

// The codes of eight channels and their block's scale byte; four neighbouring lanes hold a block.
__device__ __forceinline__ uint32_t quantise8(float (&x)[8], int *byte)
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    if (top >= 0x7f800000u) {  // an infinity becomes the largest number, a NaN zero: the format has neither
        top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = x[i] == x[i] ? fminf(fmaxf(x[i], -3.40282347e38f), 3.40282347e38f) : 0.0f;
            top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
        }
    }
    top = max(top, (uint32_t)__shfl_xor((int)top, 1, kWave));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2, kWave));
    *byte = cache_scale_byte(top);
    const float scale = cache_scale(*byte);
    // to the nearest code, halves to the even one, cut at 6
    uint32_t codes = 0;
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[0], x[1], scale, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[2], x[3], scale, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[4], x[5], scale, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[6], x[7], scale, 3);
    return codes;
}

// One thread: eight channels of K and of V of one token and head.  A workgroup has one head and as many tokens in a row as it holds (16
// for D = 128): what it stores is whole lines of one or two tiles, put together in one L2.  8191 tokens of 32 heads, 128 channels, bf16:
// 40.6 us, bound by memory (170 MB, 4.2 TB/s, where a copy has 4.8); with all heads of two tokens to a workgroup, whose lines come together
// from several L2s, 49.1.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void cache_write_kernel(unsigned char *__restrict__ cache, CacheShape c, const void *__restrict__ k,
                                                          const void *__restrict__ v, long long k_stride, long long v_stride,
                                                          const int *__restrict__ slots, int n_tokens)
{
    constexpr int kPer = D / 8, W = D / 32, kTokens = 256 / kPer;
    const int head = blockIdx.x % (unsigned)c.n_kv, token = (int)(blockIdx.x / (unsigned)c.n_kv) * kTokens + threadIdx.x / kPer;
    const int ch = threadIdx.x % kPer * 8;
    if (token >= n_tokens) return;  // (four lanes of a block leave together: kPer is a multiple of four)
    float xk[8], xv[8];
    load8<BF16>(k, token * k_stride + head * D + ch, xk);
    load8<BF16>(v, token * v_stride + head * D + ch, xv);
    const int slot = slots[token];  // (asked for together with the values)
    const int page = slot >> c.log_page;
    int bk, bv;
    const uint32_t ck = quantise8(xk, &bk), cv = quantise8(xv, &bv);
    if (slot < 0 || page >= c.n_pages) return;
    const int t = slot & 15;
    unsigned char *tile = cache + cache_tile_offset(page, head, slot & (c.page - 1), c.n_kv, c.log_page, cache_tile_bytes(D));
    *reinterpret_cast<uint32_t *>(tile + t * (D / 2) + ch / 2) = ck;
    unsigned char *tv = tile + 8 * D + (t >> 2) * (2 * D) + (t & 3) * W;  // lane n's bytes of this token: + n * 4 W
    if constexpr (W == 2) {
        *reinterpret_cast<uint16_t *>(tv + (ch / 4) * 8) = (uint16_t)cv;
        *reinterpret_cast<uint16_t *>(tv + (ch / 4 + 1) * 8) = (uint16_t)(cv >> 16);
    } else {
        *reinterpret_cast<uint32_t *>(tv + (ch / (D / 16)) * (4 * W) + (ch % (D / 16)) / 2) = cv;
    }
    if (ch % 32 == 0) {
        tile[16 * D + t * W + ch / 32] = (unsigned char)bk;
        tile[16 * D + 16 * W + (t >> 2) * (4 * W) + (ch / 32) * 4 + (t & 3)] = (unsigned char)bv;
    }
}

template <bool BF16>
__device__ __forceinline__ void store8(void *p, long long at, uint32_t codes, float scale)
{
    const uint4 r = {cache_pair<0>(codes, scale), cache_pair<1>(codes, scale), cache_pair<2>(codes, scale), cache_pair<3>(codes, scale)};
    if constexpr (BF16) {
        *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(p) + at) = r;
    } else {
        float4 *f = reinterpret_cast<float4 *>(static_cast<float *>(p) + at);
        f[0] = {bf16_lo(r.x), bf16_hi(r.x), bf16_lo(r.y), bf16_hi(r.y)};
        f[1] = {bf16_lo(r.z), bf16_hi(r.z), bf16_lo(r.w), bf16_hi(r.w)};
    }
}

// Dealt as the writer's threads are, so that a line of the cache comes into one L2 only: the same tokens 26.3 us (170 MB, 6.4 TB/s); with the
// heads of a token side by side, where the cache was fetched three times over, 35.9.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void cache_read_kernel(const unsigned char *__restrict__ cache, CacheShape c,
                                                         const int *__restrict__ slots, int n_tokens, void *__restrict__ k,
                                                         void *__restrict__ v)
{
    constexpr int kPer = D / 8, W = D / 32, kTokens = 256 / kPer;
    const int head = blockIdx.x % (unsigned)c.n_kv, token = (int)(blockIdx.x / (unsigned)c.n_kv) * kTokens + threadIdx.x / kPer;
    const int ch = threadIdx.x % kPer * 8;
    if (token >= n_tokens) return;
    const int slot = slots[token];
    const int page = slot >> c.log_page;
    const long long out = ((long long)token * c.n_kv + head) * D + ch;
    uint32_t ck = 0, cv = 0, bk = 1, bv = 1;
    if (slot >= 0 && page < c.n_pages) {
        const int t = slot & 15;
        const unsigned char *tile = cache + cache_tile_offset(page, head, slot & (c.page - 1), c.n_kv, c.log_page, cache_tile_bytes(D));
        ck = *reinterpret_cast<const uint32_t *>(tile + t * (D / 2) + ch / 2);
        const unsigned char *tv = tile + 8 * D + (t >> 2) * (2 * D) + (t & 3) * W;
        if constexpr (W == 2) {
            cv = *reinterpret_cast<const uint16_t *>(tv + (ch / 4) * 8) |
                 (uint32_t)*reinterpret_cast<const uint16_t *>(tv + (ch / 4 + 1) * 8) << 16;
        } else {
            cv = *reinterpret_cast<const uint32_t *>(tv + (ch / (D / 16)) * (4 * W) + (ch % (D / 16)) / 2);
        }
        bk = tile[16 * D + t * W + ch / 32];
        bv = tile[16 * D + 16 * W + (t >> 2) * (4 * W) + (ch / 32) * 4 + (t & 3)];
    }
    store8<BF16>(k, out, ck, cache_scale(bk));
    store8<BF16>(v, out, cv, cache_scale(bv));
}

// ---------------------------------------------------------------- page copies

// Bound by memory; a launch for few copies by its latency (2.3 us).  4 KB to a workgroup, one trip: a page of 34 KB has nine.
__global__ __launch_bounds__(256) void cache_copy_kernel(unsigned char *__restrict__ cache, size_t page_bytes, int n_pages,
                                                         const int *__restrict__ copies)
{
    const int src = copies[2 * blockIdx.x], dst = copies[2 * blockIdx.x + 1];
    if (src < 0 || dst < 0 || src >= n_pages || dst >= n_pages || src == dst) return;
    const size_t at = ((size_t)blockIdx.y * 256 + threadIdx.x) * 16;
    if (at < page_bytes)
        *reinterpret_cast<uint4 *>(cache + (size_t)dst * page_bytes + at) =
            *reinterpret_cast<const uint4 *>(cache + (size_t)src * page_bytes + at);
}

// ---------------------------------------------------------------- the plan of a step

__device__ __forceinline__ long long ceil_pages(long long tokens, int log_page)
{
    return (tokens + (1ll << log_page) - 1) >> log_page;
}

// Inclusive sums over the workgroup's 256 threads of three counts at once, and their totals.
struct Sums {
    long long tokens, pages;
    int seqs;
};
__device__ __forceinline__ Sums block_scan(Sums v, Sums *wave_totals, Sums *total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const long long t = __shfl_up(v.tokens, off, kWave), p = __shfl_up(v.pages, off, kWave);
        const int q = __shfl_up(v.seqs, off, kWave);
        if (lane >= off) v.tokens += t, v.pages += p, v.seqs += q;
    }
    if (lane == 63) wave_totals[wave] = v;
    __syncthreads();
    Sums before = {0, 0, 0}, all = {0, 0, 0};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (w < wave) before.tokens += wave_totals[w].tokens, before.pages += wave_totals[w].pages, before.seqs += wave_totals[w].seqs;
        all.tokens += wave_totals[w].tokens, all.pages += wave_totals[w].pages, all.seqs += wave_totals[w].seqs;
    }
    __syncthreads();
    v.tokens += before.tokens, v.pages += before.pages, v.seqs += before.seqs;
    *total = all;
    return v;
}

constexpr int kPlanTokens = 1024;  // slots a workgroup writes

// Latency-bound integer work.  Every workgroup sums all sequences' lengths for itself (a few kilobytes, from the L2 for all
// but the first), keeps the sequences whose new tokens meet its own 1024 slots, and writes those; nothing is handed from
// one workgroup to another, so one launch does it.  A fresh block is entered into the table by its first token's thread.  8 sequences of
// one token 3.3 us, 256 prompts of up to 2048 tokens 7.0.
__global__ __launch_bounds__(256) void cache_plan_kernel(PlanArgs a)
{
    __shared__ Sums wave_totals[4];
    __shared__ int s_start[kPlanTokens], s_seq[kPlanTokens];
    __shared__ long long s_first[kPlanTokens];  // pages taken before this sequence's
    __shared__ int s_lo, s_hi, s_wrong;
    const int tid = threadIdx.x;
    const long long t0 = (long long)blockIdx.x * kPlanTokens, t1 = t0 + kPlanTokens;
    if (tid == 0) s_lo = INT_MAX, s_hi = -1, s_wrong = 0;
    const int head = a.pool[0], count = a.pool[1];
    __syncthreads();
    Sums run = {0, 0, 0};
    int wrong = head < 0 || head >= a.n_pages || count < 0 || count > a.n_pages;
    for (int base = 0; base < a.n_seq; base += 256) {
        const int s = base + tid;
        Sums own = {0, 0, 0};
        int c = 0;
        if (s < a.n_seq) {
            c = a.cached[s];
            const int n = a.fresh[s];
            const long long have = ceil_pages(c, a.log_page), need = ceil_pages((long long)c + n, a.log_page);
            if (c < 0 || n < 0 || need > a.stride) wrong = 1;
            else own = {n, need - have, n > 0};
        }
        Sums total;
        const Sums upto = block_scan(own, wave_totals, &total);
        const long long begin = run.tokens + upto.tokens - own.tokens, end = begin + own.tokens;
        if (own.tokens > 0 && begin < t1 && end > t0) {
            // at most 1024 sequences in a row meet 1024 slots: their numbers among those with new tokens do not collide
            const int number = run.seqs + upto.seqs - 1, at = number & (kPlanTokens - 1);
            s_start[at] = (int)begin, s_seq[at] = s, s_first[at] = run.pages + upto.pages - own.pages;
            atomicMin(&s_lo, number);
            atomicMax(&s_hi, number);
        }
        if (blockIdx.x == 0 && s < a.n_seq) {
            a.start[s + 1] = (int)min(end, (long long)INT_MAX);
            a.context[s] = (int)((long long)c + own.tokens);
        }
        run.tokens += total.tokens, run.pages += total.pages, run.seqs += total.seqs;
    }
    if (wrong) s_wrong = 1;
    __syncthreads();
    const int status = (run.pages > count ? 1 : 0) | (run.tokens > a.max_tokens ? 2 : 0) | (s_wrong ? 4 : 0);
    if (blockIdx.x == 0) {
        if (tid == 0) {
            long long next = (long long)head + run.pages;
            if (next >= a.n_pages) next -= a.n_pages;
            a.start[0] = 0;
            *a.status = status;
            a.pool_out[0] = status ? head : (int)next;
            a.pool_out[1] = status ? count : count - (int)run.pages;
        }
        if (status) {  // nothing is taken: every sequence stays as it is
            for (int s = tid; s < a.n_seq; s += 256) a.start[s + 1] = 0, a.context[s] = a.cached[s];
        }
    }
    const long long n_slots = min(t1, (long long)a.max_tokens);
    for (long long t = t0 + tid; t < n_slots; t += 256) {
        int slot = -1, pos = -1;
        if (!status && t < run.tokens) {
            int lo = s_lo, hi = s_hi;  // the last of them that starts at or before t
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (s_start[mid & (kPlanTokens - 1)] <= (int)t) lo = mid;
                else hi = mid - 1;
            }
            const int at = lo & (kPlanTokens - 1), s = s_seq[at], c = a.cached[s];
            pos = c + (int)t - s_start[at];
            const int block = pos >> a.log_page, have = (int)ceil_pages(c, a.log_page);
            int *entry = a.table + (size_t)s * a.stride + block;
            int page;
            if (block >= have) {
                long long r = head + s_first[at] + (block - have);
                if (r >= a.n_pages) r -= a.n_pages;
                page = a.ring[r];
                if ((pos & ((1 << a.log_page) - 1)) == 0) *entry = page;
            } else {
                page = *entry;
            }
            if (page >= 0 && page < a.n_pages) slot = (page << a.log_page) + (pos & ((1 << a.log_page) - 1));
        }
        a.slots[t] = slot;
        if (a.positions) a.positions[t] = pos;
    }
}

// ---------------------------------------------------------------- reordering of rows

constexpr int kReorderBlocks = 256;  // blocks of a request that a workgroup sees to

// A request's rows, in LDS.
struct ReorderRows {
    int parent[POP_MAX_BEAMS], length[POP_MAX_BEAMS], blocks[POP_MAX_BEAMS], copy[POP_MAX_BEAMS];
    int last[POP_MAX_BEAMS];  // of a row that takes a copy: the page that is copied
    unsigned parented;  // rows that go on, by bit
    int wrong;          // some row has a negative length, or one that its table row has no room for
};

// What the request's rows are and which of them take a copy of their parent's last page: where it is partly filled and an earlier row
// goes on in it, and is a page.  All threads call it; the rows can be read when it returns.
__device__ __forceinline__ void reorder_rows(const ReorderArgs &a, int g, ReorderRows &r)
{
    const int c = threadIdx.x, row = g * a.group + c;
    if (c < a.group) {
        const int p = a.parents[row], len = a.length[row];
        r.parent[c] = p >= 0 && p < a.group ? p : -1;
        r.length[c] = len;
        r.blocks[c] = (int)min(ceil_pages(max(len, 0), a.log_page), (long long)a.stride);
    }
    if (c == 0) r.parented = 0, r.wrong = 0;
    __syncthreads();
    if (c < a.group) {
        const int p = r.parent[c];
        int copy = 0;
        if (r.length[c] < 0 || ceil_pages(r.length[c], a.log_page) > a.stride) r.wrong = 1;
        if (p >= 0) {
            const int len = r.length[p];
            if (len > 0 && (len & ((1 << a.log_page) - 1)))
                for (int b = 0; b < c; ++b) copy |= r.parent[b] == p;
            if (copy) {
                const int last = a.table[(size_t)(g * a.group + p) * a.stride + r.blocks[p] - 1];
                copy = last >= 0 && last < a.n_pages;
                r.last[c] = last;
            }
            atomicOr(&r.parented, 1u << p);
        }
        r.copy[c] = copy;
    }
    __syncthreads();
}

// Block j's entries of the rows: asked for before it is known how many blocks a row has.
template <int W>
__device__ __forceinline__ void load_entries(const ReorderArgs &a, int g, int j, int (&page)[W])
{
    const int *at = a.table + (size_t)g * a.group * a.stride + j;
#pragma unroll
    for (int r = 0; r < W; ++r) page[r] = r < a.group && j < a.stride ? at[(size_t)r * a.stride] : -1;
}

// Makes them the pages of block j of the rows, -1 for none, and gives by bit the rows whose page no row keeps: a page counts at the first row that has
// it.  A page that rows hold together stands at the same block of each (they share it since they were one row).
template <int W>
__device__ __forceinline__ unsigned freed_rows(const ReorderArgs &a, const ReorderRows &rows, int j, int (&page)[W])
{
#pragma unroll
    for (int r = 0; r < W; ++r)
        if (r >= a.group || j >= rows.blocks[r]) page[r] = -1;
    unsigned freed = 0;
#pragma unroll
    for (int r = 0; r < W; ++r) {
        bool lost = page[r] >= 0 && page[r] < a.n_pages && !(rows.parented >> r & 1);  // (rows beyond the group have no page)
#pragma unroll
        for (int q = 0; q < W; ++q)
            if (q != r && page[q] == page[r] && (q < r || (rows.parented >> q & 1))) lost = false;
        freed |= (unsigned)lost << r;
    }
    return freed;
}

// Sum over the workgroup, and over the threads in front of this one.
__device__ __forceinline__ int block_sum(int v, int *s_wave, int *before)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int incl = v;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int t = __shfl_up(incl, off, kWave);
        if (lane >= off) incl += t;
    }
    if (lane == 63) s_wave[wave] = incl;
    __syncthreads();
    int total = 0, ahead = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (w < wave) ahead += s_wave[w];
        total += s_wave[w];
    }
    __syncthreads();
    *before = ahead + incl - v;
    return total;
}

// Latency-bound integer work in two launches (one where a single workgroup sees to everything): what each part of the requests gives
// back and takes has to be known before the first page finds its place in the ring.  W: rows of a request at most.  counts: pages given back,
// by request and part, then copies by request, -1 where a length is wrong.  One request of four rows 4.5 us; 64 of eight rows of 250 blocks
// 4.4 + 9.0.
template <int W>
__global__ __launch_bounds__(kReorderBlocks) void reorder_count_kernel(ReorderArgs a)
{
    __shared__ ReorderRows s_rows;
    __shared__ int s_wave[4];
    const int g = blockIdx.x, j = blockIdx.y * kReorderBlocks + threadIdx.x;
    int page[W], before;
    load_entries(a, g, j, page);
    reorder_rows(a, g, s_rows);
    const int total = block_sum(__popc(freed_rows(a, s_rows, j, page)), s_wave, &before);
    if (threadIdx.x == 0) {
        a.counts[g * gridDim.y + blockIdx.y] = total;
        if (blockIdx.y == 0) {
            int n = 0;
            for (int c = 0; c < a.group; ++c) n += s_rows.copy[c];
            a.counts[gridDim.x * gridDim.y + g] = s_rows.wrong ? -1 : n;
        }
    }
}

template <int W>
__global__ __launch_bounds__(kReorderBlocks) void reorder_rows_kernel(ReorderArgs a, int alone)
{
    __shared__ ReorderRows s_rows;
    __shared__ int s_fresh[POP_MAX_BEAMS], s_wave[4], s_sums[4][5];
    const int g = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n_groups = gridDim.x, chunks = gridDim.y;
    const int part = g * chunks + blockIdx.y, n_parts = n_groups * chunks, j = blockIdx.y * kReorderBlocks + tid, first = g * a.group;
    const int head = a.pool[0], count = a.pool[1];
    int page[W], at;
    load_entries(a, g, j, page);
    // of the parts and requests in front of this one, and of all: pages given back, copies
    int freed_before = 0, freed_all = 0, copies_before = 0, copies_all = 0, wrong = 0;
    if (!alone) {
        for (int i = tid; i < n_parts; i += kReorderBlocks) {
            const int n = a.counts[i];
            freed_all += n, freed_before += i < part ? n : 0;
        }
        for (int i = tid; i < n_groups; i += kReorderBlocks) {
            const int n = a.counts[n_parts + i];
            copies_all += n, copies_before += i < g ? n : 0, wrong |= n < 0;
        }
        freed_before = wave_sum(freed_before), freed_all = wave_sum(freed_all);
        copies_before = wave_sum(copies_before), copies_all = wave_sum(copies_all);
        wrong = __any(wrong);
        if (lane == 0)
            s_sums[wave][0] = freed_before, s_sums[wave][1] = freed_all, s_sums[wave][2] = copies_before, s_sums[wave][3] = copies_all, s_sums[wave][4] = wrong;
    }
    reorder_rows(a, g, s_rows);  // (its barriers stand behind the sums)
    const unsigned freed = freed_rows(a, s_rows, j, page);
    const int mine = block_sum(__popc(freed), s_wave, &at);
    if (alone) {
        freed_all = mine, wrong = s_rows.wrong;
        for (int c = 0; c < a.group; ++c) copies_all += s_rows.copy[c];
    } else {
        freed_before = freed_all = copies_before = copies_all = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w)
            freed_before += s_sums[w][0], freed_all += s_sums[w][1], copies_before += s_sums[w][2], copies_all += s_sums[w][3], wrong |= s_sums[w][4];
    }
    // (where a length is wrong, only that is said: the copies were not counted)
    int status = wrong ? POP_PLAN_INVALID : copies_all > count ? POP_PLAN_PAGES : 0;
    if (head < 0 || head >= a.n_pages || count < 0 || count > a.n_pages ||
        (long long)count + freed_all > a.n_pages)
        status |= POP_PLAN_INVALID;  // no ring of this many pages: one stands in it and in a row as well, or in rows of two requests
    if (part == 0 && tid == 0) {
        long long next = (long long)head + copies_all;
        if (next >= a.n_pages) next -= a.n_pages;
        *a.status = status;
        a.pool_out[0] = status ? head : (int)next;
        a.pool_out[1] = status ? count : count - copies_all + freed_all;
    }
    // the copies of this request
    const auto copied = [&](int c) { return !status && s_rows.copy[c]; };
    if (tid < a.group) {
        int fresh = -1;
        if (copied(tid)) {
            long long r = (long long)head + copies_before;
            for (int c = 0; c < tid; ++c) r += s_rows.copy[c];
            if (r >= a.n_pages) r -= a.n_pages;
            fresh = a.ring[r];
        }
        s_fresh[tid] = fresh;
        if (blockIdx.y == 0) {
            const int row = first + tid, p = s_rows.parent[tid];
            a.copies[2 * row] = copied(tid) ? s_rows.last[tid] : -1;
            a.copies[2 * row + 1] = fresh;
            a.new_length[row] = status ? a.length[row] : p < 0 ? 0 : s_rows.length[p];
        }
    }
    __syncthreads();
    if (j < a.stride) {
        for (int c = 0; c < a.group; ++c) {
            const int p = status ? c : s_rows.parent[c];
            int entry = -1;
            if (p >= 0) {
#pragma unroll
                for (int r = 0; r < W; ++r) entry = r == p ? page[r] : entry;  // (-1 behind a row's last block)
                if (copied(c) && j == s_rows.blocks[p] - 1) entry = s_fresh[c];  // (whatever the ring holds)
            }
            a.new_table[(size_t)(first + c) * a.stride + j] = entry;
        }
        if (!status) {
            long long to = (long long)head + count + freed_before + at;
#pragma unroll
            for (int r = 0; r < W; ++r)
                if (freed >> r & 1) {
                    while (to >= a.n_pages) to -= a.n_pages;
                    a.ring[to++] = page[r];
                }
        }
    }
}

}  // namespace

hipError_t launch_cache_write(void *cache, const CacheShape &c, const void *k, const void *v, int is_bf16, long long k_stride,
                              long long v_stride, const int *slots, int n_tokens, hipStream_t s)
{
    const int tokens = 2048 / c.d;  // of a workgroup
    const unsigned grid = (unsigned)((n_tokens + tokens - 1) / tokens) * c.n_kv;
    unsigned char *to = static_cast<unsigned char *>(cache);
#define POP_WRITE(D)                                                                                                         \
    (is_bf16 ? cache_write_kernel<D, true><<<grid, 256, 0, s>>>(to, c, k, v, k_stride, v_stride, slots, n_tokens)            \
             : cache_write_kernel<D, false><<<grid, 256, 0, s>>>(to, c, k, v, k_stride, v_stride, slots, n_tokens))
    if (c.d == 64) POP_WRITE(64);
    else if (c.d == 128) POP_WRITE(128);
    else POP_WRITE(256);
#undef POP_WRITE
    return hipGetLastError();
}

hipError_t launch_cache_read(const void *cache, const CacheShape &c, const int *slots, int n_tokens, void *k, void *v, int is_bf16,
                             hipStream_t s)
{
    const int tokens = 2048 / c.d;  // of a workgroup
    const unsigned grid = (unsigned)((n_tokens + tokens - 1) / tokens) * c.n_kv;
    const unsigned char *from = static_cast<const unsigned char *>(cache);
#define POP_READ(D)                                                                              \
    (is_bf16 ? cache_read_kernel<D, true><<<grid, 256, 0, s>>>(from, c, slots, n_tokens, k, v)      \
             : cache_read_kernel<D, false><<<grid, 256, 0, s>>>(from, c, slots, n_tokens, k, v))
    if (c.d == 64) POP_READ(64);
    else if (c.d == 128) POP_READ(128);
    else POP_READ(256);
#undef POP_READ
    return hipGetLastError();
}

hipError_t launch_cache_copy_pages(void *cache, const CacheShape &c, const int *copies, int n, hipStream_t s)
{
    const size_t bytes = cache_page_bytes(c);
    cache_copy_kernel<<<dim3((unsigned)n, (unsigned)((bytes + 4095) / 4096)), 256, 0, s>>>(static_cast<unsigned char *>(cache), bytes,
                                                                                          c.n_pages, copies);
    return hipGetLastError();
}

hipError_t launch_cache_plan(const PlanArgs &a, hipStream_t s)
{
    const int grid = a.max_tokens > kPlanTokens ? (int)(((long long)a.max_tokens + kPlanTokens - 1) / kPlanTokens) : 1;
    cache_plan_kernel<<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

size_t reorder_counts(int n_seq, int group, int stride)
{
    return (size_t)(n_seq / group) * ((stride + kReorderBlocks - 1) / kReorderBlocks + 1);
}

template <int W>
static hipError_t launch_reorder(const ReorderArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)(a.n_seq / a.group), (unsigned)((a.stride + kReorderBlocks - 1) / kReorderBlocks));
    const int alone = grid.x * grid.y == 1;
    if (!alone) {
        reorder_count_kernel<W><<<grid, kReorderBlocks, 0, s>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    reorder_rows_kernel<W><<<grid, kReorderBlocks, 0, s>>>(a, alone);
    return hipGetLastError();
}

hipError_t launch_cache_reorder(const ReorderArgs &a, hipStream_t s)
{
    if (a.group == 1) return launch_reorder<1>(a, s);
    if (a.group <= 4) return launch_reorder<4>(a, s);
    if (a.group <= 8) return launch_reorder<8>(a, s);
    return launch_reorder<POP_MAX_BEAMS>(a, s);
}

}  // namespace pop
