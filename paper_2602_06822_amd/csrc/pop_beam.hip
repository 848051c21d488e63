// Beam search's selection: of all (beam, token) of a request the k best by  score of the beam + logit - logsumexp(logits).
//
// One pass over the logits: a workgroup holds a stretch of a row in registers, sums its exponentials and finds its k largest
// logits; a workgroup per request then joins the stretches' sums and ranks what they found.  The k largest of a set: every wave
// ranks its lanes' maxima, the k-th of which no more than k - 1 lanes exceed, so it bounds the set's k-th from below; what
// reaches the bound (k and a few more, as a rule) goes into a list in LDS, where each entry counts the ones before it.
#include <math.h>

#include "pop_cache.h"

namespace pop {

namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int kListed = 1024;

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

struct SelectShared {
    unsigned long long list[kListed], best[4];
    uint32_t bound[4];
    int n;
};

// The k (<= 64) largest of the workgroup's words, E to a thread and all different (0: none), in order to put(rank, word); ranks that
// no word has are not put.  256 threads.
template <int E, class Put>
__device__ __forceinline__ void select_largest(const unsigned long long (&w)[E], int k, SelectShared &s, Put put)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) most = max(most, (uint32_t)(w[i] >> 32));
    int before = 0;
#pragma unroll
    for (int i = 0; i < 64; ++i) {
        const uint32_t other = (uint32_t)__builtin_amdgcn_readlane((int)most, i);
        before += other > most || (other == most && i < lane);
    }
    if (threadIdx.x == 0) s.n = 0;
    if (before == k - 1) s.bound[wave] = most;
    __syncthreads();
    const uint32_t bound = max(max(s.bound[0], s.bound[1]), max(s.bound[2], s.bound[3]));
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (w[i] && (uint32_t)(w[i] >> 32) >= bound) {
            const int at = atomicAdd(&s.n, 1);
            if (at < kListed) s.list[at] = w[i];
        }
    __syncthreads();
    const int n = s.n;
    if (n <= kListed) {
        for (int e = threadIdx.x; e < n; e += 256) {
            const unsigned long long mine = s.list[e];
            int rank = 0;
            for (int i = 0; i < n; ++i) rank += s.list[i] > mine;
            if (rank < k) put(rank, mine);
        }
    } else {  // a crowd of equal values at the bound: the largest after the last one found, k times
        unsigned long long last = ~0ull;
        for (int r = 0; r < k; ++r) {
            unsigned long long best = 0;
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (w[i] < last && w[i] > best) best = w[i];
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) {
                const unsigned long long o = __shfl_xor(best, off, kWave);
                best = o > best ? o : best;
            }
            __syncthreads();
            if (lane == 0) s.best[wave] = best;
            __syncthreads();
            last = max(max(s.best[0], s.best[1]), max(s.best[2], s.best[3]));
            if (last == 0) break;
            if (threadIdx.x == 0) put(r, last);
        }
    }
    __syncthreads();
}

// A beam that proposes nothing by its logits: it has ended, or it is not alive.
__device__ __forceinline__ bool closed(const BeamArgs &a, int row)
{
    return (a.done && a.done[row]) || a.scores[row] == -INFINITY;
}

// ws: per row and stretch {maximum, sum of exponentials}, then per row and stretch k words.
__device__ __forceinline__ float2 *stats_of(const BeamArgs &a) { return static_cast<float2 *>(a.ws); }
__device__ __forceinline__ unsigned long long *words_of(const BeamArgs &a, int stretches)
{
    return static_cast<unsigned long long *>(a.ws) + (size_t)a.requests * a.beams * stretches;
}

// Grid: (rows, stretches); E logits to a thread.  Rows begin where they begin: a stretch starts at a 16-byte boundary of memory, and the
// vectors that a row's ends cut are read value by value.
template <bool BF16, int E>
__global__ __launch_bounds__(256) void beam_rows_kernel(BeamArgs a, int stretches)
{
    constexpr int V = BF16 ? 8 : 4;
    __shared__ SelectShared s;
    __shared__ float s_max[4], s_sum[4];
    const int row = blockIdx.x;
    if (closed(a, row)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const size_t row_at = (size_t)row * a.vocab;
    const int skew = (int)(row_at % V);
    const size_t base = row_at - skew;  // a multiple of V values: a 16-byte boundary
    float x[E];
    unsigned long long w[E];
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < E / V; ++i) {
        const int at = (blockIdx.y * (E / V) + i) * 256 * V + threadIdx.x * V - skew;  // token of the vector's first value
        if (at >= 0 && at + V <= a.vocab) {
            if constexpr (BF16) {
                const uint4 r = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(a.logits) + base + skew + at);
                const uint32_t u[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) x[i * V + 2 * j] = bf16_lo(u[j]), x[i * V + 2 * j + 1] = bf16_hi(u[j]);
            } else {
                const float4 r = *reinterpret_cast<const float4 *>(static_cast<const float *>(a.logits) + base + skew + at);
                x[i * V] = r.x, x[i * V + 1] = r.y, x[i * V + 2] = r.z, x[i * V + 3] = r.w;
            }
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                x[i * V + j] = -INFINITY;
                if (at + j >= 0 && at + j < a.vocab)
                    x[i * V + j] = BF16 ? __uint_as_float((uint32_t)static_cast<const uint16_t *>(a.logits)[row_at + at + j] << 16)
                                        : static_cast<const float *>(a.logits)[row_at + at + j];
            }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float &v = x[i * V + j];
            v = v == v ? v : -INFINITY;  // a NaN is no proposal
            top = fmaxf(top, v);
            w[i * V + j] = at + j >= 0 && at + j < a.vocab ? rank_word(v, (uint32_t)(at + j)) : 0;
        }
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, kWave));
    if (lane == 0) s_max[wave] = top;
    __syncthreads();
    top = fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3]));
    const float shift = top > -INFINITY ? top : 0.0f;
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < E; ++i) sum += __builtin_amdgcn_exp2f((x[i] - shift) * kLog2e);
    sum = wave_sum(sum);
    if (lane == 0) s_sum[wave] = sum;
    unsigned long long *words = words_of(a, stretches) + ((size_t)row * stretches + blockIdx.y) * a.k;
    for (int i = threadIdx.x; i < a.k; i += 256) words[i] = 0;
    __syncthreads();
    if (threadIdx.x == 0) stats_of(a)[(size_t)row * stretches + blockIdx.y] = {top, s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3]};
    select_largest<E>(w, a.k, s, [&](int rank, unsigned long long word) { words[rank] = word; });
}

// One workgroup per request.  256 threads: 16 lanes to a beam for the sums, then tiles of 2048 candidates.
__global__ __launch_bounds__(256) void beam_join_kernel(BeamArgs a, int stretches)
{
    constexpr int E = 8;
    __shared__ SelectShared s;
    __shared__ float s_lse[POP_MAX_BEAMS], s_was[POP_MAX_BEAMS];
    __shared__ int s_closed[POP_MAX_BEAMS];
    __shared__ unsigned long long s_found[64];
    const int request = blockIdx.x, row0 = request * a.beams;
    {
        const int b = threadIdx.x / 16, i0 = threadIdx.x % 16;
        float top = -INFINITY, sum = 0.0f;
        if (b < a.beams && !closed(a, row0 + b)) {
            const float2 *st = stats_of(a) + (size_t)(row0 + b) * stretches;
            for (int i = i0; i < stretches; i += 16) top = fmaxf(top, st[i].x);
#pragma unroll
            for (int off = 8; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, kWave));
            const float shift = top > -INFINITY ? top : 0.0f;
            for (int i = i0; i < stretches; i += 16) sum += st[i].y * __builtin_amdgcn_exp2f((st[i].x - shift) * kLog2e);
#pragma unroll
            for (int off = 8; off > 0; off >>= 1) sum += __shfl_xor(sum, off, kWave);
            top = shift;
        }
        if (b < a.beams && i0 == 0) {
            s_was[b] = a.scores[row0 + b];
            s_closed[b] = closed(a, row0 + b);
            s_lse[b] = top + __builtin_amdgcn_logf(sum) * kLn2;
        }
    }
    if (threadIdx.x < 64) s_found[threadIdx.x] = 0;
    __syncthreads();
    const unsigned long long *words = words_of(a, stretches) + (size_t)row0 * stretches * a.k;
    const int per = stretches * a.k, total = a.beams * per;
    for (int tile = 0; tile < total; tile += 256 * (E - 1)) {
        unsigned long long w[E];
#pragma unroll
        for (int i = 0; i < E - 1; ++i) {
            const int c = tile + i * 256 + threadIdx.x, b = c / per, left = c - b * per;
            w[i] = 0;
            if (c >= total) continue;
            uint32_t token = 0xffffffffu;
            float score = -INFINITY;
            if (!s_closed[b]) {
                const unsigned long long word = words[c];
                if (word) {
                    token = ~(uint32_t)word;
                    const float x = ranked_value(word);
                    if (x > -INFINITY) score = s_was[b] + (x - s_lse[b]);
                }
            } else if (left < a.k) {  // an ended beam goes on by the padding token; else its tokens are the last resort, in their order
                const bool ended = a.done && a.done[row0 + b];
                token = ended ? (left == 0 ? a.pad : left - 1 < a.pad ? left - 1 : left) : left;
                if (ended && left == 0) score = s_was[b];
            }
            if (token < (uint32_t)a.vocab) w[i] = rank_word(score, (uint32_t)b * (uint32_t)a.vocab + token);
        }
        w[E - 1] = threadIdx.x < a.k ? s_found[threadIdx.x] : 0;  // what the tiles before left
        __syncthreads();
        select_largest<E>(w, a.k, s, [&](int rank, unsigned long long word) { s_found[rank] = word; });
    }
    if ((int)threadIdx.x < a.k) {
        const unsigned long long word = s_found[threadIdx.x];
        const uint32_t place = ~(uint32_t)word;
        const int at = request * a.k + threadIdx.x;
        a.out_scores[at] = word ? ranked_value(word) : -INFINITY;
        a.out_tokens[at] = word ? (int)(place % (uint32_t)a.vocab) : -1;
        a.out_parents[at] = word ? (int)(place / (uint32_t)a.vocab) : -1;
    }
}

// Values to a thread: 8 where that leaves fewer than four workgroups to a compute unit, else 32.
struct Stretches {
    int e, n;
};
Stretches beam_stretches(int requests, int beams, int vocab, int is_bf16)
{
    const int lead = is_bf16 ? 7 : 3;
    Stretches s;
    s.e = (long long)requests * beams * ((vocab + lead + 2047) / 2048) <= 1024 ? 8 : 32;
    s.n = (vocab + lead + 256 * s.e - 1) / (256 * s.e);
    return s;
}

}  // namespace

size_t beam_ws(int requests, int beams, int vocab, int k)
{
    const int n = max(beam_stretches(requests, beams, vocab, 0).n, beam_stretches(requests, beams, vocab, 1).n);
    return (size_t)requests * beams * n * (k + 1) * 8;
}

hipError_t launch_beam_select(const BeamArgs &a, hipStream_t s)
{
    const Stretches st = beam_stretches(a.requests, a.beams, a.vocab, a.is_bf16);
    const dim3 grid((unsigned)(a.requests * a.beams), (unsigned)st.n);
    if (a.is_bf16) {
        if (st.e == 8) beam_rows_kernel<true, 8><<<grid, 256, 0, s>>>(a, st.n);
        else beam_rows_kernel<true, 32><<<grid, 256, 0, s>>>(a, st.n);
    } else {
        if (st.e == 8) beam_rows_kernel<false, 8><<<grid, 256, 0, s>>>(a, st.n);
        else beam_rows_kernel<false, 32><<<grid, 256, 0, s>>>(a, st.n);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    beam_join_kernel<<<(unsigned)a.requests, 256, 0, s>>>(a, st.n);
    return hipGetLastError();
}

}  // namespace pop
