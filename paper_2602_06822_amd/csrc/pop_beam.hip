// Beam search's selection: of all (beam, token) of a request the k best by  score of the beam + logit - logsumexp(logits).
//
// One pass over the logits, bound by memory where there are many rows and by latency where there are few.  A wave goes over its part of
// a row a tile at a time, the next tile's loads under way: each lane sums exponentials against a maximum of its own and keeps the
// maximum of each of its *segments* (its 16 values of a tile).  Then every wave ranks its lanes' maxima: the k-th largest is a lower
// bound of the row's k-th largest value, and the largest of the workgroup's four bounds leaves about k segments that can hold one of
// its k best.  Only those are read again, what reaches the bound is listed in LDS, and the lists are ranked.  So a value costs
// seven operations in the pass.  The last workgroup of a request to finish joins the sums and ranks what the others found.
//
// 32 requests of 8 rows of 131071 float32, 16 best: 30.3 us, of which the pass is 18 (134 MB, 7 TB/s) and what follows a chain of a
// dozen latencies: bound 2.1, reading again 1.6, ranking 1.0, handing over 0.9, the last workgroup's join 3.4.  One request of 4 rows of 32000
// bf16: 11.3 us, the same chain.  (The first tile asked for before the beams' states, which then return behind it: 32.7.)
#include <math.h>

#include <algorithm>

#include "pop_cache.h"

namespace pop {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int kListed = 768;   // words of a wave's list
constexpr int kRoom = 512;     // of which these are free when a round of eight values a lane begins
constexpr int kMostK = 64;

// Largest first, equal ones by place: a 64-bit word of an ordered value and the place's complement.  0 is "nothing".
__device__ __forceinline__ unsigned long long rank_word(float v, uint32_t place)
{
    return (unsigned long long)score_key(v) << 32 | (uint32_t)~place;
}
__device__ __forceinline__ float ranked_value(unsigned long long w)
{
    const uint32_t key = (uint32_t)(w >> 32);
    return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}
__device__ __forceinline__ float finite_or_zero(float x) { return x > -INFINITY ? x : 0.0f; }
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// The leading BITS bits of the k-th largest of the 64 lanes' values, k <= 64, bit by bit: k lanes at least are not below the result.
template <int BITS>
__device__ __forceinline__ uint32_t kth_of_lanes(uint32_t v, int k)
{
    uint32_t found = 0;
#pragma unroll 4
    for (int bit = 31; bit >= 32 - BITS; --bit) {
        const uint32_t next = found | 1u << bit;
        found = __popcll(__ballot(v >= next)) >= k ? next : found;
    }
    return found;
}

// A wave's list, of n words, all different: what cannot be among its k largest is dropped, and at most kListed - kRoom words are left.
// The list is gone over 64 words at a time, in place; such code runs once or twice in a launch, and most of what it costs is to fetch it.
__device__ __attribute__((noinline)) int thin_out(unsigned long long *list, int n, int k, int lane)
{
    const auto word = [&](int i) { return i + lane < n ? list[i + lane] : 0; };
    const auto keep = [&](unsigned long long bound) {
        int left = 0;
#pragma unroll 1
        for (int i = 0; i < n; i += 64) {
            const unsigned long long w = word(i), m = __ballot(w != 0 && w >= bound);
            if (w != 0 && w >= bound) list[left + __popcll(m & ((1ull << lane) - 1))] = w;
            left += __popcll(m);
        }
        n = left;
    };
    const auto largest = [&] {  // (its upper half)
        uint32_t most = 0;
#pragma unroll 1
        for (int i = 0; i < n; i += 64) most = max(most, (uint32_t)(word(i) >> 32));
        return most;
    };
    keep((unsigned long long)kth_of_lanes<20>(largest(), k) << 32);
    if (n <= kListed - kRoom) return n;
    // a crowd of equal values: k lanes have the k-th largest value or more, and among words with just this value a place of `place` or more
    const uint32_t value = kth_of_lanes<32>(largest(), k);
    uint32_t place = 0;
#pragma unroll 1
    for (int i = 0; i < n; i += 64) {
        const unsigned long long w = word(i);
        const uint32_t v = (uint32_t)(w >> 32);
        place = v >= value ? max(place, v > value ? ~0u : (uint32_t)w) : place;
    }
    keep((unsigned long long)value << 32 | kth_of_lanes<32>(place, k));
    if (n <= kListed - kRoom) return n;
    // (only where k is near 64) the k largest are counted out
    constexpr int P = kListed / 64;
    unsigned long long w[P];
#pragma unroll
    for (int i = 0; i < P; ++i) w[i] = word(i * 64);
    int rank[P] = {};
    for (int e = 0; e < n; ++e) {
        const unsigned long long other = list[e];
#pragma unroll
        for (int i = 0; i < P; ++i) rank[i] += other > w[i];
    }
#pragma unroll
    for (int i = 0; i < P; ++i)
        if (w[i] != 0 && rank[i] < k) list[rank[i]] = w[i];
    return min(n, k);
}

constexpr int kWaveTiles = 17;  // of a wave

struct BeamShared {
    unsigned long long list[4][kListed];
    unsigned long long found[kMostK];
    float most[4][kWaveTiles][64];
    uint16_t segment[4][kWaveTiles * 64];
    uint32_t bound[4];
    int n[4];
    float ref[4], sum[4], top[POP_MAX_BEAMS], log[POP_MAX_BEAMS], was[POP_MAX_BEAMS];
    int closed[POP_MAX_BEAMS], last;
};

// Appends a lane's word, if it has one, to its wave's list of n, which has room for it.
__device__ __forceinline__ void append(unsigned long long *list, int &n, bool lists, unsigned long long word, int lane)
{
    const unsigned long long m = __ballot(lists);
    if (lists) list[n + __popcll(m & ((1ull << lane) - 1))] = word;
    n += __popcll(m);
}

// The k largest words of the four waves' lists, in order to put(rank, word).  All threads; n[] has been written.  Each wave counts, for
// all words, those of its own list that come in front of them: two words a lane, eight reads under way; then the four counts are added
// up.  (One thread to a word over all four lists: 2.1 us where this takes 1.0, of 16 words out of about 80.)
template <class Put>
__device__ __forceinline__ void select_listed(BeamShared &s, int k, Put put)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n0 = s.n[0], n1 = n0 + s.n[1], n2 = n1 + s.n[2], n = n2 + s.n[3], own = s.n[wave];  // n <= 4 (kListed - kRoom)
    const auto word = [&](int e) { return e < n0 ? s.list[0][e] : e < n1 ? s.list[1][e - n0] : e < n2 ? s.list[2][e - n1] : s.list[3][e - n2]; };
    const auto counts = [&](int w) { return reinterpret_cast<int *>(s.most[w]); };  // (the maxima have been used)
    if (lane < 8) s.list[wave][own + lane] = 0;  // (a list's end, so that eight can be read)
#pragma unroll 1
    for (int e = lane; e < n; e += 128) {
        const unsigned long long a = word(e), b = e + 64 < n ? word(e + 64) : ~0ull;
        int of_a = 0, of_b = 0;
#pragma unroll 1
        for (int i = 0; i < own; i += 8) {
            unsigned long long other[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) other[j] = s.list[wave][i + j];
#pragma unroll
            for (int j = 0; j < 8; ++j) of_a += other[j] > a, of_b += other[j] > b;
        }
        counts(wave)[e] = of_a;
        if (e + 64 < n) counts(wave)[e + 64] = of_b;
    }
    __syncthreads();
#pragma unroll 1
    for (int e = threadIdx.x; e < n; e += 256) {
        const int rank = counts(0)[e] + counts(1)[e] + counts(2)[e] + counts(3)[e];
        if (rank < k) put(rank, word(e));
    }
}

// A beam that proposes nothing by its logits: it has ended, or it is not alive.
__device__ __forceinline__ bool closed(const BeamArgs &a, int row)
{
    const int done = a.done ? a.done[row] : 0;
    return (a.scores[row] == -INFINITY) | (done != 0);  // (both loads under way together)
}

// ws: per row and stretch {reference, sum of exponentials relative to it}, then per row and stretch k words, then a counter for each request.
__device__ __forceinline__ unsigned long long *stats_of(const BeamArgs &a) { return static_cast<unsigned long long *>(a.ws); }
__device__ __forceinline__ unsigned long long *words_of(const BeamArgs &a, int stretches)
{
    return stats_of(a) + (size_t)a.requests * a.beams * stretches;
}
__device__ __forceinline__ void hand_over(unsigned long long *p, unsigned long long v)
{
    __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Sums of a request's beams and the k best of what their stretches found: 16 lanes to a beam for the sums, then every wave lists what is
// among the best of its candidates.
__device__ __forceinline__ void join_request(const BeamArgs &a, BeamShared &s, int request, int stretches, unsigned long long is_open)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row0 = request * a.beams;
    constexpr int E = 4;
    const unsigned long long *words = words_of(a, stretches) + (size_t)row0 * stretches * a.k;
    const int per = stretches * a.k, total = a.beams * per;
    const float by_per = __builtin_amdgcn_rcpf((float)per);
    unsigned long long w[E];
    const auto load = [&](int tile) {
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const int c = tile + i * 256 + threadIdx.x;
            w[i] = c < total ? coherent_load(words + c) : 0;
        }
    };
    load(0);  // (under way with the sums)
    {
        const int b = threadIdx.x / 16, i0 = threadIdx.x % 16;
        float ref = -INFINITY, sum = 0.0f;
        const bool open = b < a.beams && (is_open >> b & 1);
        const float was = b < a.beams ? a.scores[row0 + b] : 0.0f;
        if (open) {
            const unsigned long long *st = stats_of(a) + (size_t)(row0 + b) * stretches;
            for (int i = i0; i < stretches; i += 16) {
                const unsigned long long w = coherent_load(st + i);
                const float next = fmaxf(ref, __uint_as_float((uint32_t)w)), shift = finite_or_zero(next);
                sum = sum * exp_of(ref - shift) + __uint_as_float((uint32_t)(w >> 32)) * exp_of(__uint_as_float((uint32_t)w) - shift);
                ref = next;
            }
        }
        float most = ref;
#pragma unroll
        for (int off = 8; off > 0; off >>= 1) most = fmaxf(most, __shfl_xor(most, off, kWave));
        const float shift = finite_or_zero(most);
        sum *= exp_of(ref - shift);
#pragma unroll
        for (int off = 8; off > 0; off >>= 1) sum += __shfl_xor(sum, off, kWave);
        if (b < a.beams && i0 == 0) {
            s.was[b] = was;
            s.closed[b] = !open;
            s.top[b] = shift, s.log[b] = __builtin_amdgcn_logf(sum) * kLn2;
        }
    }
    __syncthreads();
    int n = 0;
    for (int tile = 0; tile < total; tile += 256 * E) {
        if (tile > 0) load(tile);
        if (n > kListed - kRoom) n = thin_out(s.list[wave], n, a.k, lane);
#pragma unroll
        for (int i = 0; i < E; ++i) {
            if (tile + i * 256 >= total) break;
            // (total < 2^20, per < 2^16: half a word is far more than what the product is rounded by)
            const int c = tile + i * 256 + threadIdx.x, b = (int)(((float)c + 0.5f) * by_per), left = c - b * per;
            uint32_t token = 0xffffffffu;
            float score = -INFINITY;
            if (c < total && !s.closed[b]) {
                if (w[i]) {
                    token = ~(uint32_t)w[i];
                    const float x = ranked_value(w[i]);
                    if (x > -INFINITY) score = s.was[b] + ((x - s.top[b]) - s.log[b]);
                }
            } else if (c < total && left < a.k) {  // an ended beam goes on by the padding token; else its tokens are the last resort, in their order
                const bool ended = a.done && a.done[row0 + b];
                token = ended ? (left == 0 ? a.pad : left - 1 < a.pad ? left - 1 : left) : left;
                if (ended && left == 0) score = s.was[b];
            }
            w[i] = token < (uint32_t)a.vocab ? rank_word(score, (uint32_t)b * (uint32_t)a.vocab + token) : 0;
            append(s.list[wave], n, w[i] != 0, w[i], lane);
        }
    }
    if (n > 32) n = thin_out(s.list[wave], n, a.k, lane);
    if (lane == 0) s.n[wave] = n;
    if (threadIdx.x < kMostK) s.found[threadIdx.x] = 0;
    __syncthreads();
    select_listed(s, a.k, [&](int rank, unsigned long long word) { s.found[rank] = word; });
    __syncthreads();
    if ((int)threadIdx.x < a.k) {
        const unsigned long long word = s.found[threadIdx.x];
        const uint32_t place = ~(uint32_t)word;
        const int at = request * a.k + threadIdx.x;
        a.out_scores[at] = word ? ranked_value(word) : -INFINITY;
        a.out_tokens[at] = word ? (int)(place % (uint32_t)a.vocab) : -1;
        a.out_parents[at] = word ? (int)(place / (uint32_t)a.vocab) : -1;
    }
}

// Grid: (rows, stretches); `tiles` tiles of NV vectors a lane to a stretch, taken by the waves in turn.  Rows begin where they begin: a
// stretch starts at a 16-byte boundary of memory, and the vectors that a row's ends cut are read value by value.
template <bool BF16, int NV>
__global__ __launch_bounds__(256, 3) void beam_select_kernel(BeamArgs a, int stretches, int tiles, unsigned long long tag)
{
    constexpr int V = BF16 ? 8 : 4, E = NV * V;
    __shared__ BeamShared s;
    const int row = blockIdx.x, stretch = blockIdx.y, request = row / a.beams, row0 = request * a.beams;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // the request's open beams: their workgroups are counted; without any, that of the first stretch of its first row joins
    const unsigned long long is_open = __ballot(lane < a.beams && !closed(a, row0 + min(lane, a.beams - 1)));
    const int open = __popcll(is_open);
    const bool reads = is_open >> (row - row0) & 1;
    if (!reads && !(open == 0 && row == row0 && stretch == 0)) return;
    const int expected = open * stretches;
    unsigned long long *const counter = words_of(a, stretches) + (size_t)a.requests * a.beams * stretches * a.k + request;
    if (reads) {
        unsigned long long counted = 0;
        const bool announces = expected > 1 && threadIdx.x == 0;
        if (announces) counted = coherent_load(counter);
        const size_t row_at = (size_t)row * a.vocab;
        const int skew = (int)(row_at % V);  // (the row itself need not start at a 16-byte boundary)
        const int n_tiles = (a.vocab + skew + 64 * E - 1) / (64 * E), tile_end = min((stretch + 1) * tiles, n_tiles);
        // from that boundary to the end of the tensor, in whole words: what lies behind it is not read
        const size_t size = BF16 ? 2 : 4, left = ((size_t)a.requests * a.beams * a.vocab - (row_at - skew)) * size;
        const __amdgpu_buffer_rsrc_t rows = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<char *>(static_cast<const char *>(a.logits)) + (row_at - skew) * size, 0, (int)min(left & ~(size_t)3, (size_t)0x7ffffffc), 0x00020000);
        auto load = [&](u32x4 (&r)[NV], int tile) {
#pragma unroll
            for (int i = 0; i < NV; ++i) r[i] = __builtin_amdgcn_raw_buffer_load_b128(rows, ((tile * NV + i) * 64 + lane) * 16, 0, 0);
        };
        const auto values = [&](float *x, const u32x4 &r) {
#pragma unroll
            for (int j = 0; j < V; ++j) x[j] = BF16 ? (j % 2 ? bf16_hi(r[j / 2]) : bf16_lo(r[j / 2])) : __uint_as_float(r[j]);
        };
        // the tensor's last value, where it has half a word of its own
        float odd_value = 0.0f;
        const bool odd = BF16 && (left & 2) && row == a.requests * a.beams - 1;
        if (odd) odd_value = __uint_as_float((uint32_t)static_cast<const uint16_t *>(a.logits)[row_at + a.vocab - 1] << 16);
        // sum: of e^(x - top).  The difference comes before the factor log2 e: it is exact where the weight is large, while x log2 e is
        // rounded by more than an exponential can hold from 2^31 on, and passes float32's range where masks of its lowest value stand.
        float top = -INFINITY, sum = 0.0f;
        const int first = stretch * tiles + wave;
        u32x4 now[NV], next[NV];
        load(now, first);
        if (announces) announce(counter, counted, tag);
        int mine = 0;  // tiles of this wave
        for (int tile = first; tile < tile_end; tile += 4, ++mine) {
            load(next, tile + 4);
            float x[E];
#pragma unroll
            for (int i = 0; i < NV; ++i) values(&x[i * V], now[i]);
            if (tile == 0 || tile == n_tiles - 1) {  // the row's ends
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const int at = ((tile * NV + i / V) * 64 + lane) * V - skew + i % V;
                    if (odd && at == a.vocab - 1) x[i] = odd_value;
                    if (at < 0 || at >= a.vocab) x[i] = -INFINITY;
                }
            }
            float most = -INFINITY;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                x[i] = fmaxf(x[i], -INFINITY);  // a NaN is no proposal
                most = fmaxf(most, x[i]);
            }
            s.most[wave][mine][lane] = most;
            if (most > top) {
                sum *= exp_of(top - most);
                top = most;
            }
            const float shift = finite_or_zero(top);
#pragma unroll
            for (int i = 0; i < E; ++i) sum += exp_of(x[i] - shift);
#pragma unroll
            for (int i = 0; i < NV; ++i) now[i] = next[i];
        }
        const uint32_t k_th = kth_of_lanes<20>(score_key(top), a.k);
        if (lane == 0) s.bound[wave] = k_th;
        __syncthreads();
        constexpr uint32_t kMinusInfinity = 0x007fffffu;  // as an ordered key
        const float limit = ranked_value((unsigned long long)max(max(max(s.bound[0], s.bound[1]), max(s.bound[2], s.bound[3])), kMinusInfinity) << 32);
        // segments with a value that reaches the limit, and those values; minus infinities are no such value
        int n_segments = 0, n = 0;
#pragma unroll 1
        for (int t = 0; t < mine; t += 4) {
            float most[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) most[j] = t + j < mine ? s.most[wave][t + j][lane] : -INFINITY;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool is = most[j] >= limit && most[j] > -INFINITY;
                const unsigned long long m = __ballot(is);
                if (is) s.segment[wave][n_segments + __popcll(m & ((1ull << lane) - 1))] = (uint16_t)((t + j) * 64 + lane);
                n_segments += __popcll(m);
            }
        }
        constexpr int kRound = 64 / NV;  // segments that a load takes
        int segment[2], vector[2];
        u32x4 again[2];
        const auto fetch = [&](int base) {  // two rounds
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int i = base + u * kRound + lane / NV;
                segment[u] = i < n_segments ? s.segment[wave][i] : -1;
                vector[u] = ((first + 4 * (segment[u] >> 6)) * NV + lane % NV) * 64 + (segment[u] & 63);
                again[u] = __builtin_amdgcn_raw_buffer_load_b128(rows, segment[u] >= 0 ? vector[u] * 16 : 0x7ffffff0, 0, 0);
            }
        };
        fetch(0);
        // meanwhile the wave's sums
        float most = top;
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) most = fmaxf(most, __shfl_xor(most, off, kWave));
        sum = wave_sum(sum * exp_of(top - finite_or_zero(most)));
        if (lane == 0) s.ref[wave] = most, s.sum[wave] = sum;
        if (threadIdx.x < kMostK) s.found[threadIdx.x] = 0;
#pragma unroll 1
        for (int base = 0; base < n_segments; base += 2 * kRound) {
            if (base > 0) fetch(base);
#pragma unroll 1
            for (int u = 0; u < 2; ++u) {
                if (base + u * kRound >= n_segments) break;
                if (n > kListed - kRoom) n = thin_out(s.list[wave], n, a.k, lane);
                float x[V];
                values(x, u == 0 ? again[0] : again[1]);
                const int at0 = (u == 0 ? vector[0] : vector[1]) * V - skew;
                const bool there = (u == 0 ? segment[0] : segment[1]) >= 0;
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const int at = at0 + j;
                    if (odd && at == a.vocab - 1) x[j] = odd_value;
                    append(s.list[wave], n, there && at >= 0 && at < a.vocab && x[j] >= limit && x[j] > -INFINITY, rank_word(x[j], (uint32_t)at), lane);
                }
            }
        }
        if (n > 32) n = thin_out(s.list[wave], n, a.k, lane);
        if (lane == 0) s.n[wave] = n;
        __syncthreads();
        if (s.n[0] + s.n[1] + s.n[2] + s.n[3] < a.k) {
            // fewer than k: tokens at minus infinity, the first of them, which stand among the stretch's first 2 k tokens
            __syncthreads();
            const int at = stretch * tiles * 64 * E - skew + (int)threadIdx.x + (stretch == 0 ? skew : 0);
            bool lists = (int)threadIdx.x < 2 * a.k && at < a.vocab && at < tile_end * 64 * E - skew;
            float v = 0.0f;
            if (lists) v = BF16 ? __uint_as_float((uint32_t)static_cast<const uint16_t *>(a.logits)[row_at + at] << 16) : static_cast<const float *>(a.logits)[row_at + at];
            lists = lists && !(v > -INFINITY);
            append(s.list[wave], n, lists, rank_word(-INFINITY, (uint32_t)at), lane);
            if (lane == 0) s.n[wave] = n;
        }
        __syncthreads();
        // the workgroup's sums and its k largest
        select_listed(s, a.k, [&](int rank, unsigned long long word) { s.found[rank] = word; });
        const float all = fmaxf(fmaxf(s.ref[0], s.ref[1]), fmaxf(s.ref[2], s.ref[3]));
        float total = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) total += s.sum[w] * exp_of(s.ref[w] - finite_or_zero(all));
        __syncthreads();
        const size_t part = (size_t)row * stretches + stretch;
        if ((int)threadIdx.x < a.k) hand_over(words_of(a, stretches) + part * a.k + threadIdx.x, s.found[threadIdx.x]);
        if (threadIdx.x == 0) hand_over(stats_of(a) + part, (unsigned long long)__float_as_uint(total) << 32 | __float_as_uint(all));
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's stores are acknowledged
        __syncthreads();
        if (threadIdx.x == 0) s.last = expected == 1 || arrive_last(counter, tag, expected);
        __syncthreads();
        if (!s.last) return;
    }
    join_request(a, s, request, stretches, is_open);
}

// Tiles of 16 values a lane (32: 256 rows of 131071 float32 3.6 us more).  A stretch has a tile for each wave at least, a
// sixteenth of the row (a request of 8 rows of 131071: 33 stretches a row 7.6 us more than 17), and what leaves about 512
// workgroups: more of them have more ends, where the best values are found (256 rows: 768 workgroups 6 us more, 1024 19 more).
constexpr int kLaneValues = 16;
struct Stretches {
    int tiles, n;
};
Stretches beam_stretches(int requests, int beams, int vocab, int is_bf16)
{
    const long long rows = (long long)requests * beams, tile = 64 * kLaneValues, n_tiles = (vocab + (is_bf16 ? 7 : 3) + tile - 1) / tile;
    const long long of_row = std::min(std::max(512 / rows, 1ll), 16ll);
    const long long tiles = std::min(std::max((n_tiles + of_row - 1) / of_row, 4ll), 4ll * kWaveTiles);
    Stretches s;
    s.n = (int)((n_tiles + tiles - 1) / tiles);
    s.tiles = (int)((n_tiles + s.n - 1) / s.n);  // (all alike)
    return s;
}

}  // namespace

size_t beam_ws(int requests, int beams, int vocab, int k)
{
    const int n = std::max(beam_stretches(requests, beams, vocab, 0).n, beam_stretches(requests, beams, vocab, 1).n);
    return (size_t)requests * (beams * (size_t)n * (k + 1) + 1) * 8;
}

hipError_t launch_beam_select(const BeamArgs &a, hipStream_t s)
{
    const Stretches st = beam_stretches(a.requests, a.beams, a.vocab, a.is_bf16);
    const dim3 grid((unsigned)(a.requests * a.beams), (unsigned)st.n);
    const unsigned long long tag = launch_tag();
    if (a.is_bf16) beam_select_kernel<true, kLaneValues / 8><<<grid, 256, 0, s>>>(a, st.n, st.tiles, tag);
    else beam_select_kernel<false, kLaneValues / 4><<<grid, 256, 0, s>>>(a, st.n, st.tiles, tag);
    return hipGetLastError();
}

}  // namespace pop
