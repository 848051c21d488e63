// Attention over the 4-bit paged cache: y = softmax(scale q k^T + mask) v for every query row of every sequence.
//
// A query column is one (new token, query head) of a kv head's group; columns of one kv head share its keys and values.
// A step of a wave is 32 tokens: S^T = K q^T as two 16 x 16 tiles of matrix products (rows are tokens, columns are query
// columns), the running maximum and sum of a softmax per column, O^T += V^T P^T.  Transposed like this, S^T leaves the
// products in the layout in which P^T enters them (a lane has the same column and the same tokens), and the statistics of a
// column are one register of a lane.  The tokens of a step are in the order tile, group of four, token, which is the order
// of the cache's bytes: a lane's K and V codes are loads of D/8 bytes each, a wave's loads are contiguous kilobytes.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "pop_cache.h"

namespace pop {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef const __attribute__((address_space(4))) int *scalar_ints;  // read by scalar loads

constexpr float kLog2e = 1.44269504088896340736f;
// A column's maximum starts here: below every score times log2 e down to a score of -2.3e38, and a difference with it is no NaN.
constexpr float kLowest = -3.40282347e38f;
// A new maximum is taken only where it exceeds the old one by this many powers of two: until then the weights are at most
// 2^8, which 32 bits hold as exactly, and O is not rescaled.
constexpr float kSlack = 8.0f;
// Weights are 2^(s scale - m), relative to a maximum m that is a rounded product itself: what the rounding takes off stays in all weights of the
// column and cancels, but from 2^32 on it is more than an exponential can hold.  Beyond kFar a column goes by the power of two below the
// scale instead, with which the product of its maximum is exact: scores of that size that differ at all (float32 has 24 bits) differ by 2^6
// or more there, so weights are 1 or nothing by either factor.  (A factor to a lane instead of one for all: four chunks of 955 to 2048 tokens
// over 2867 to 6144 358 -> 361 us, single tokens as before; rounding the products of such steps alone, in a branch, 368 to 372.)
constexpr float kFar = 1073741824.0f;

// The column's factor and its maximum in that unit, where the maximum has just become `raw` (a score without the scale) or stays as it is.
__device__ __forceinline__ void choose_unit(float &by, float &m, float raw, float scale)
{
    const float size = fabsf(m * (scale / by));  // (by the scale, whichever unit it is in: a power of two goes in and out without rounding)
    const float next = m != kLowest && size > kFar ? __uint_as_float(__float_as_uint(scale) & 0x7f800000u) : scale;
    if (next != by) by = next, m = raw * next;
}
// A maximum by the scale, to be compared with those of others.
__device__ __forceinline__ float by_scale(float m, float by, float scale) { return by == scale ? m : m * (scale / by); }

__device__ __forceinline__ bf16x8 as_bf16x8(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    const u32x4 v = {a, b, c, d};
    return __builtin_bit_cast(bf16x8, v);
}

// Two float32 values rounded to bf16 (to nearest even), packed.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    const bf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
}

// The lower and the upper halves of two words.
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// One lane's part of a tile: a quarter of a token's channels of K (D/8 bytes and their scale bytes), D/16 channels of four tokens
// of V (D/8 bytes and four scale bytes).
template <int D>
struct TileRegs {
    uint32_t k[D / 32], v[D / 32], ks, vs;
};

// Loads of a lane go through a descriptor of the tile: its address is in scalar registers, a lane's offsets within a tile stay the
// same for all tiles, and a descriptor of no bytes stands for a tile that is not there: its loads give zeros and fetch nothing, so
// that a wave always has the same number of loads in flight.
template <int D>
struct TileOffsets {
    int k, v, ks, vs;
    __device__ __forceinline__ TileOffsets(int n, int g)
    {
        constexpr int W = D / 32;
        k = n * (D / 2) + g * (D / 8);
        v = 8 * D + (g * 16 + n) * (4 * W);
        ks = 16 * D + n * W + g * D / 128;
        vs = 16 * D + 16 * W + (g * W + n * (D / 16) / 32) * 4;
    }
};

template <int D, bool PAST>
__device__ __forceinline__ void load_tile(TileRegs<D> &r, const unsigned char *tile, bool there, const TileOffsets<D> &o)
{
    constexpr int kAux = PAST ? 2 : 0;  // non-temporal
    const __amdgpu_buffer_rsrc_t d = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(tile), 0, there ? cache_tile_bytes(D) : 0, 0x00020000);
    if constexpr (D == 64) {
        const u32x2 a = __builtin_amdgcn_raw_buffer_load_b64(d, o.k, 0, kAux), b = __builtin_amdgcn_raw_buffer_load_b64(d, o.v, 0, kAux);
        r.k[0] = a[0], r.k[1] = a[1], r.v[0] = b[0], r.v[1] = b[1];
    } else {
#pragma unroll
        for (int i = 0; i < D / 128; ++i) {
            const u32x4 a = __builtin_amdgcn_raw_buffer_load_b128(d, o.k + 16 * i, 0, kAux), b = __builtin_amdgcn_raw_buffer_load_b128(d, o.v + 16 * i, 0, kAux);
#pragma unroll
            for (int j = 0; j < 4; ++j) r.k[4 * i + j] = a[j], r.v[4 * i + j] = b[j];
        }
    }
    if constexpr (D == 256) r.ks = __builtin_amdgcn_raw_buffer_load_b16(d, o.ks, 0, kAux);
    else r.ks = __builtin_amdgcn_raw_buffer_load_b8(d, o.ks, 0, kAux);
    r.vs = __builtin_amdgcn_raw_buffer_load_b32(d, o.vs, 0, kAux);
}

// Operand of the s-th 32 channels: 8 of the lane's D/4, in the order of their bytes.
template <int D>
__device__ __forceinline__ bf16x8 k_operand(const TileRegs<D> &r, int s)
{
    const float scale = cache_scale(D == 256 ? (r.ks >> (8 * (s / 4))) & 255u : r.ks);
    const uint32_t c = r.k[s];
    return as_bf16x8(cache_pair<0>(c, scale), cache_pair<1>(c, scale), cache_pair<2>(c, scale), cache_pair<3>(c, scale));
}

// What one kv head's columns of one sequence see: columns are numbered token by token, head by head.
struct Columns {
    int first_pos;  // position of the sequence's first new token
    int n;          // columns in all
    int share;      // query heads to a kv head
    int length;     // tokens in the cache
    int window;     // INT_MAX for none
};

template <int TERMS>
__device__ __forceinline__ void split_terms(const float (&x)[8], bf16x8 (&t)[TERMS])
{
    float r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = x[i];
#pragma unroll
    for (int j = 0; j < TERMS; ++j) {
        const uint32_t a = pack_bf16(r[0], r[1]), b = pack_bf16(r[2], r[3]), c = pack_bf16(r[4], r[5]), d = pack_bf16(r[6], r[7]);
        t[j] = as_bf16x8(a, b, c, d);
        if (j + 1 < TERMS) {
            r[0] -= bf16_lo(a), r[1] -= bf16_hi(a), r[2] -= bf16_lo(b), r[3] -= bf16_hi(b);
            r[4] -= bf16_lo(c), r[5] -= bf16_hi(c), r[6] -= bf16_lo(d), r[7] -= bf16_hi(d);
        }
    }
}

__device__ __forceinline__ void store_y2(const AttentionArgs &a, size_t at, float x, float y)
{
    if (a.y_bf16) *reinterpret_cast<uint32_t *>(static_cast<uint16_t *>(a.y) + at) = pack_bf16(x, y);
    else *reinterpret_cast<float2 *>(static_cast<float *>(a.y) + at) = {x, y};
}

// Sum over the lanes up to this one, of numbers that are not negative, no more than INT_MAX; or the largest of them.
template <bool MOST, int CTRL, int ROWS>
__device__ __forceinline__ int dpp_step(int v)
{
    const int from = __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
    return MOST ? max(v, from) : __builtin_elementwise_add_sat(v, from);
}
template <bool MOST = false>
__device__ __forceinline__ int wave_scan(int v)
{
    v = dpp_step<MOST, 0x111, 0xf>(v), v = dpp_step<MOST, 0x112, 0xf>(v);  // rows of 16
    v = dpp_step<MOST, 0x114, 0xf>(v), v = dpp_step<MOST, 0x118, 0xf>(v);
    v = dpp_step<MOST, 0x142, 0xa>(v);  // pairs of rows
    return dpp_step<MOST, 0x143, 0xc>(v);
}

constexpr int kNoWindow = 0x7fffffff, kMostTokens = 1 << 30;  // (a sequence's table holds no more: checked by the caller)

// Sequences' rows of q and y: rows outside the tensors are not touched.
__device__ __forceinline__ bool sequence_columns(const AttentionArgs &a, int start, int next, int context, int share, Columns *c)
{
    const bool there = start >= 0 && next > start && next <= a.n_tokens;
    const int fresh = there ? next - start : 0;
    context = min(max(context, 0), kMostTokens);
    c->length = min(context, a.stride << a.c.log_page);
    c->first_pos = context - fresh;
    c->share = share;
    c->n = fresh * share;
    c->window = a.window > 0 ? min(a.window, kMostTokens) : kNoWindow;
    return there;
}

// Tokens [lo, hi) that some of the columns [begin, end) see, lo a multiple of 32, and the first and the last of the columns' positions.
struct SeenTokens {
    int lo, hi, first_pos, last_pos;
};
__device__ __forceinline__ SeenTokens seen_tokens(const Columns &c, int begin, int end)
{
    SeenTokens s;
    s.first_pos = c.first_pos + begin / c.share, s.last_pos = c.first_pos + (end - 1) / c.share;
    s.hi = max(min(s.last_pos + 1, c.length), 0);
    s.lo = c.window == kNoWindow ? 0 : min(max(s.first_pos - c.window + 1, 0) & ~31, s.hi);
    return s;
}

// One step of a wave: 32 tokens of one kv head against 16 columns.
template <int D, int QT, int PT>
struct WaveSums {
    bf16x8 q[D / 32][QT];  // the lane's part of q: channels [g D/4, (g + 1) D/4) of column n
    f32x4 o[D / 16];       // O^T: channel (4 g + i) D/16 + j of column n in o[j][i]
    float m, l;            // maximum that the weights are relative to; the lane's part of their sum
    float by;              // the factor of the column's scores: the scale, or see choose_unit

    // limit[u]: tokens of tile u from this position on are not there; masked: some of the 32 are not seen by some column.
    __device__ __forceinline__ void step(const TileRegs<D> (&r)[2], const int (&limit)[2], bool masked, int t0, int pos, int window, int g,
                                         float scale)
    {
        f32x4 s[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            s[u] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                const bf16x8 k = k_operand<D>(r[u], c);
#pragma unroll
                for (int t = QT - 1; t >= 0; --t) s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[c][t], s[u], 0, 0, 0);
            }
        }
        uint32_t vs[2] = {r[0].vs, r[1].vs};
        if (masked) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int t = t0 + 16 * u + 4 * g;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (!(t + i < limit[u] && t + i <= pos && pos - (t + i) < window)) s[u][i] = -INFINITY;
                // scale bytes of tokens that are not there become 2^-127, so that whatever stands in their place is finite
                const int left = limit[u] - t;
                vs[u] = left >= 4 ? vs[u] : left <= 0 ? 0u : vs[u] & ((1u << (8 * left)) - 1);
            }
        }
        float top = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
        if (__any(top * by > m + kSlack)) {  // (by > 0)
            top = fmaxf(top, __shfl_xor(top, 16, kWave));
            top = fmaxf(top, __shfl_xor(top, 32, kWave));
            const float next = fmaxf(m, top * by), factor = __builtin_amdgcn_exp2f(m - next);
            m = next;
            choose_unit(by, m, top, scale);
            l *= factor;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) o[j] *= factor;
        }
        float p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            p[i] = __builtin_amdgcn_exp2f(fmaf(s[i / 4][i % 4], by, -m));
            l += p[i];
        }
        bf16x8 w[PT];
        split_terms<PT>(p, w);
        float sv[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) sv[i] = cache_scale((vs[i / 4] >> (8 * (i % 4))) & 255u);
        constexpr int W = D / 32;  // bytes of a token: channels 2 b and 2 b + 1 of the lane's D/16 in byte b
#pragma unroll
        for (int b = 0; b < W; ++b) {
            uint32_t c[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int at = (i % 4) * W + b;
                c[i] = cache_pair_at(r[i / 4].v[at / 4], sv[i], at % 4);
            }
            const bf16x8 even = as_bf16x8(low_halves(c[0], c[1]), low_halves(c[2], c[3]), low_halves(c[4], c[5]), low_halves(c[6], c[7]));
            const bf16x8 odd = as_bf16x8(high_halves(c[0], c[1]), high_halves(c[2], c[3]), high_halves(c[4], c[5]), high_halves(c[6], c[7]));
#pragma unroll
            for (int t = PT - 1; t >= 0; --t) {
                o[2 * b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(even, w[t], o[2 * b], 0, 0, 0);
                o[2 * b + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(odd, w[t], o[2 * b + 1], 0, 0, 0);
            }
        }
    }
};

constexpr int kBuffers = 2;   // steps that a wave has in registers: the one it uses and the next
constexpr int kRound = 128;   // tokens of a round: a step of each of the four waves
constexpr int kWorkgroups = 512;

// How the work is dealt.  A unit is one kv head's block of 16 columns of one sequence: a number of rounds over the tokens that the
// sequence's columns see.  All units stand in one row (sequence, block, head), and every workgroup takes the same number of rounds of
// it, wherever units begin and end: ragged batches and single long sequences of single tokens load all compute units alike.  (Chunks less so: a
// unit has the rounds of its whole sequence's columns, of which its own block may see few, under a window or where little is cached;
// rounds behind what a block sees cost nothing, those in front of it, under a window, are gone over masked.)  A piece of a unit
// is what one workgroup has of it.  Where that gains less than pieces cost, workgroups take units.
struct SequenceWork {
    int rounds;  // of a unit
    int blocks;
    Columns cols;
    SeenTokens seen;
    int row0;
};
__device__ __forceinline__ SequenceWork sequence_work(const AttentionArgs &a, int start, int next, int context, int share)
{
    SequenceWork w;
    w.rounds = 0, w.blocks = 0, w.row0 = start;
    if (!sequence_columns(a, start, next, context, share, &w.cols)) return w;
    w.blocks = (w.cols.n + 15) / 16;
    w.seen = seen_tokens(w.cols, 0, w.cols.n);
    w.rounds = max((w.seen.hi - w.seen.lo + kRound - 1) / kRound, 1);
    return w;
}

// Whether whole units are dealt: pieces cost as much as about 7 rounds of a compute unit (4 where nobody has more than one round), so the
// compute unit with the longest unit may have that many more than the even share.  Microseconds, pieces / units, D 128, 4 query heads to
// a kv head: 64 sequences x 8 kv heads x 500 tokens 15.5 / 9.3, x 1000 19.6 / 12.5, x 4000 38.3 / 35.5; 8 x 32 x 500 13.4 / 7.1, x 2000 17.7 / 14.3, x
// 4000 23.9 / 23.2; 8 x 8 x 1000 11.3 / 8.9, x 2000 12.1 / 13.2; 1 x 8 x 500 8.0 / 7.9, x 1000 8.1 / 9.0, x 4000 8.9 / 21.3.
__device__ __forceinline__ bool deal_units(int units, int rounds, int longest)
{
    const float all = (float)rounds, on_average = all * __builtin_amdgcn_rcpf((float)max(units, 1));
    return (float)((units - 1) >> 8) * on_average + (float)longest <= all * (1.0f / 256) + (rounds <= 256 ? 4.5f : 7.75f);
}

// What workgroups hand to each other goes past the caches (scope of the device), 16 bytes a lane at a time: the descriptor is a wave's.
__device__ __forceinline__ void store_past(f32x4 *wave_base, int vector, int lane, f32x4 v)
{
    const __amdgpu_buffer_rsrc_t d = __builtin_amdgcn_make_buffer_rsrc(wave_base, 0, 0x7fffffff, 0x00020000);
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), d, (vector * 64 + lane) * 16, 0, 16);
}
__device__ __forceinline__ f32x4 load_past(const void *wave_base, int bytes)
{
    const __amdgpu_buffer_rsrc_t d = __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(wave_base), 0, 0x7fffffff, 0x00020000);
    return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(d, bytes, 0, 16));
}

// Partial results: two places for each workgroup, its first piece if the unit began in front of it and its last if the unit goes on
// behind it; then the counters of the units' pieces, by the workgroup that has the first.
template <int D>
__device__ __forceinline__ float *partial_of(const AttentionArgs &a, int place)
{
    return a.ws + (size_t)place * 16 * (D + 4);
}

__device__ __forceinline__ void store_pair(float *p, float x, float y)
{
    const unsigned long long v = (unsigned long long)__float_as_uint(y) << 32 | __float_as_uint(x);
    __hip_atomic_store(reinterpret_cast<unsigned long long *>(p), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 load_pair(const float *p)
{
    const unsigned long long v = coherent_load(reinterpret_cast<const unsigned long long *>(p));
    return {__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32))};
}

// Workgroup: 4 waves.  In a round wave w takes tokens 32 w .. 32 w + 31 and asks for the next round's codes before it uses this one's.
// Units that end and begin with a workgroup are written to y; the pieces of others are joined by the last workgroup that finishes
// one, in the order of the tokens.  QT, PT: bf16 terms that q and the softmax weights are split into: q one if it is bf16 (exact),
// else three (24 bits); the weights one if q and the output are bf16 (rounded to 8 significant bits, as the output is, which adds about as
// much error again: 2.2e-3 of the result where the output's own rounding makes 1.65e-3), else three.  K and V
// are exact in bf16.
//
// Bound by memory on long contexts (two of up to 131072 tokens, 32 heads over 8, D 128: 43 us, 224 MB at 5.2 TB/s; the instructions of the
// conversion take 45 % of the time, waits 27), by its chain of latencies on short ones (eight of up to 4096, 32 heads: 22.3 us, of which
// the codes' 87 MB take 11.5; lengths 1.6, q and table 1.1 a unit, the waves' sums 0.8, pieces stored and counted 1.0, joined 1.5).
// Counting all pieces at the workgroup's end (24.2) and asking for the next unit before the last one's sums (22.7, long contexts 45) cost
// more than they hide, as do three or four steps in registers (23.9, 25.2).  A chunk in float32 is bound by its three
// products (two of 1024 tokens over 4096, 32 heads over 8: 262 us, 0.9 PFLOP/s).
template <int D, int QT, int PT, bool PAST>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void cache_attention_kernel(AttentionArgs a, unsigned long long tag)
{
    constexpr int kTile = cache_tile_bytes(D);
    constexpr int kPass = D > 128 ? 128 : D;  // channels of a pass of the join through LDS
    __shared__ float s_o[4][16][kPass + 4];
    __shared__ float s_m[4][16], s_l[4][16];
    __shared__ int s_last;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
    const int share = a.n_heads / a.c.n_kv, n_kv = a.c.n_kv;
    // a positive scale: the sign, or all of it where it is zero, goes into q (a masked score stays -inf)
    const float scale = a.scale != 0.0f ? fabsf(a.scale) * kLog2e : 1.0f;
    const TileOffsets<D> offsets(n, g);

    // what there is: every wave sums all sequences' work for itself, a lane that of a run of sequences
    const int per_lane = (a.n_seq + 63) / 64;
    int my_rounds = 0, my_units = 0, my_longest = 0, my_start = 0, my_next = 0, my_context = 0;
    for (int i = 0; i < per_lane; ++i) {
        const int s = lane * per_lane + i;
        if (s < a.n_seq) {
            my_start = a.start[s], my_next = a.start[s + 1], my_context = a.context[s];
            const SequenceWork w = sequence_work(a, my_start, my_next, my_context, share);
            my_rounds = __builtin_elementwise_add_sat(my_rounds, w.rounds * w.blocks * n_kv);
            my_units = __builtin_elementwise_add_sat(my_units, w.blocks * n_kv);
            my_longest = max(my_longest, w.rounds);
        }
    }
    const int rounds_upto = wave_scan(my_rounds), units_upto = wave_scan(my_units);
    const int all_rounds = __builtin_amdgcn_readlane(rounds_upto, 63), all_units = __builtin_amdgcn_readlane(units_upto, 63);
    const bool by_units =
        __builtin_amdgcn_readfirstlane(deal_units(all_units, all_rounds, __builtin_amdgcn_readlane(wave_scan<true>(my_longest), 63)));
    // this workgroup's share of them, and the sequence that it begins with
    const int upto = by_units ? units_upto : rounds_upto;
    const unsigned total = by_units ? all_units : all_rounds, n_wg = min(gridDim.x, total);
    if (blockIdx.x >= n_wg) return;
    // the first `longer` workgroups have one more than the others
    const unsigned fewest = total / n_wg, longer = total - fewest * n_wg;
    const auto workgroup_of = [&](unsigned round) {
        const unsigned of_longer = longer * (fewest + 1);
        return (int)(round < of_longer ? round / (fewest + 1) : longer + (round - of_longer) / fewest);
    };
    const int first_of_all = blockIdx.x * fewest + min(blockIdx.x, longer), end = first_of_all + (int)fewest + (blockIdx.x < longer);
    int at = first_of_all;
    const int owner = __ffsll((unsigned long long)__ballot(upto > at)) - 1;
    int seq = owner * per_lane, seq_at = owner > 0 ? __builtin_amdgcn_readlane(upto, owner - 1) : 0;  // where the sequence begins
    unsigned long long *const counters = reinterpret_cast<unsigned long long *>(partial_of<D>(a, 2 * (int)gridDim.x));
    const size_t page_bytes = cache_page_bytes(a.c);

    while (at < end) {
        int start, next, context;
        if (per_lane == 1) {  // (a lane has them)
            start = __builtin_amdgcn_readlane(my_start, seq), next = __builtin_amdgcn_readlane(my_next, seq);
            context = __builtin_amdgcn_readlane(my_context, seq);
        } else {
            start = a.start[seq], next = a.start[seq + 1], context = a.context[seq];
        }
        const SequenceWork w = sequence_work(a, start, next, context, share);
        const int dealt = by_units ? 1 : w.rounds, of_seq = dealt * w.blocks * n_kv;  // (of a unit, of the sequence's)
        if ((unsigned)at >= (unsigned)seq_at + (unsigned)of_seq) {
            seq_at += of_seq, ++seq;
            continue;
        }
        const int unit = (int)((unsigned)(at - seq_at) / (unsigned)dealt), block = (int)((unsigned)unit / (unsigned)n_kv), head = unit - block * n_kv;
        const int unit_at = seq_at + unit * dealt, begin = at - unit_at, stop = by_units ? w.rounds : min(w.rounds, end - unit_at);
        const Columns &cols = w.cols;
        const SeenTokens seen = seen_tokens(cols, block * 16, min(block * 16 + 16, cols.n));
        const scalar_ints table = (scalar_ints)(uintptr_t)(a.table + (size_t)seq * a.stride);
        const int col = block * 16 + n, token = col / share, qh = head * share + col % share;
        const bool live = col < cols.n;
        const int pos = live ? cols.first_pos + token : -1;  // a column that is not there sees nothing
        WaveSums<D, QT, PT> sums;
        {
            const int t1 = min(seen.hi, w.seen.lo + stop * kRound), first = w.seen.lo + begin * kRound + wave * 32;
            const unsigned char *const cache = a.cache + (size_t)(head * (a.c.page >> 4)) * kTile;
            TileRegs<D> r[kBuffers][2];
            int limit[kBuffers][2], page[2];
            // the pages of a step's tiles; past the last step that of the last token again, of which nothing is loaded
            auto look_up = [&](int t0) {
                if (a.c.page == 16) {
#pragma unroll
                    for (int u = 0; u < 2; ++u) page[u] = table[min(t0 + 16 * u, t1 - 1) >> 4];
                } else {  // one page holds both
                    page[0] = page[1] = table[min(t0, t1 - 1) >> a.c.log_page];
                }
            };
            auto load = [&](TileRegs<D> (&to)[2], int (&lim)[2], int t0) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int t = t0 + 16 * u;
                    lim[u] = (unsigned)page[u] < (unsigned)a.c.n_pages ? t1 : 0;
                    const unsigned char *tile = cache + (size_t)(lim[u] ? (unsigned)page[u] : 0u) * page_bytes + ((t & (a.c.page - 1)) >> 4) * kTile;
                    load_tile<D, PAST>(to[u], tile, t < lim[u], offsets);
                }
            };
            if (first < t1) look_up(first);
            else page[0] = page[1] = -1;
            // the lane's q, and for the first unit the counter of the one that goes on behind this workgroup: all under way together
            constexpr int kQ = QT == 1 ? D / 32 : D / 16;
            u32x4 q[kQ];
            const size_t q_at = ((size_t)(w.row0 + token) * a.n_heads + qh) * D + g * (D / 4);
            const u32x4 *q_from = QT == 1 ? reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(a.q) + q_at)
                                          : reinterpret_cast<const u32x4 *>(static_cast<const float *>(a.q) + q_at);
#pragma unroll
            for (int i = 0; i < kQ; ++i) {
                q[i] = u32x4{0, 0, 0, 0};
                if (live) q[i] = q_from[i];
            }
            unsigned long long counted = 0;
            const bool first_unit = at == first_of_all && !by_units && threadIdx.x == 0;
            if (first_unit) counted = coherent_load(counters + blockIdx.x);
#pragma unroll
            for (int i = 0; i < kBuffers - 1; ++i) {
                load(r[i], limit[i], first + kRound * i);
                if (first < t1) look_up(first + kRound * (i + 1));
            }
            if (first_unit) announce(counters + blockIdx.x, counted, tag);
            const uint32_t sign = a.scale < 0.0f ? (QT == 1 ? 0x80008000u : 0x80000000u) : 0u, keep = a.scale != 0.0f ? ~0u : 0u;
#pragma unroll
            for (int i = 0; i < kQ; ++i) q[i] = (q[i] ^ sign) & keep;
#pragma unroll
            for (int s = 0; s < D / 32; ++s) {
                if constexpr (QT == 1) {
                    sums.q[s][0] = __builtin_bit_cast(bf16x8, q[s]);
                } else {
                    float x[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(q[2 * s + i / 4][i % 4]);
                    split_terms<QT>(x, sums.q[s]);
                }
            }
#pragma unroll
            for (int j = 0; j < D / 16; ++j) sums.o[j] = f32x4{0, 0, 0, 0};
            sums.m = kLowest, sums.l = 0.0f, sums.by = scale;
            for (int t0 = first; t0 < t1;) {
#pragma unroll
                for (int i = 0; i < kBuffers; ++i) {
                    constexpr int kAhead = kBuffers - 1;
                    load(r[(i + kAhead) % kBuffers], limit[(i + kAhead) % kBuffers], t0 + kRound * kAhead);
                    look_up(t0 + kRound * kBuffers);
                    const bool all = t0 + 32 <= min(limit[i][0], limit[i][1]) && t0 + 31 <= seen.first_pos && seen.last_pos - t0 < cols.window;
                    if (t0 < t1) sums.step(r[i], limit[i], !all, t0, pos, cols.window, g, scale);
                    t0 += kRound;
                }
            }
        }
        sums.l += __shfl_xor(sums.l, 16, kWave);
        sums.l += __shfl_xor(sums.l, 32, kWave);

        // the four waves' sums, joined in their order: into y, or for the workgroup that joins the unit's pieces
        const int n_live = min(16, cols.n - block * 16);
        const bool whole = begin == 0 && stop == w.rounds;
        // what the four waves left in s_m, s_l and s_o, each relative to its own maximum
        const auto merge = [&](int pass, bool to_y, float *part) {
            for (int e = threadIdx.x; e < n_live * (kPass / 2); e += 256) {
                const int c = e / (kPass / 2), ch = e % (kPass / 2) * 2, gc = block * 16 + c;
                float most = kLowest, sum = 0.0f, x = 0.0f, y = 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) most = fmaxf(most, s_m[i][c]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float f = __builtin_amdgcn_exp2f(s_m[i][c] - most);
                    sum += f * s_l[i][c], x += f * s_o[i][c][ch], y += f * s_o[i][c][ch + 1];
                }
                if (to_y) {
                    const size_t row = (size_t)(w.row0 + gc / share) * a.n_heads + head * share + gc % share;
                    const float by = sum > 0.0f ? 1.0f / sum : 0.0f;
                    store_y2(a, row * D + pass * kPass + ch, x * by, y * by);
                } else {
                    store_pair(part + c * (D + 4) + pass * kPass + ch, x, y);
                    if (ch == 0 && pass == 0) store_pair(part + c * (D + 4) + D, most, sum);
                }
            }
        };
        if (g == 0) s_m[wave][n] = by_scale(sums.m, sums.by, scale), s_l[wave][n] = sums.l;
        float *const part = partial_of<D>(a, 2 * blockIdx.x + (begin == 0));
#pragma unroll
        for (int pass = 0; pass < D / kPass; ++pass) {
            // a lane has channels [g D/4, (g + 1) D/4) of column n, D/16 at a time; a pass takes those of some of the groups
            constexpr int kPer = kPass / (D / 4);
            if (live && g / kPer == pass) {
                float *to = &s_o[wave][n][(g % kPer) * (D / 4)];
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < D / 16; j += 4)
                        *reinterpret_cast<float4 *>(to + i * (D / 16) + j) = {sums.o[j][i], sums.o[j + 1][i], sums.o[j + 2][i], sums.o[j + 3][i]};
            }
            __syncthreads();
            merge(pass, whole, part);
            __syncthreads();
        }
        if (!whole) {
            // pieces of the unit: one for each of the workgroups that its first and its last round fall to and those between them
            const int wg0 = workgroup_of(unit_at), pieces = workgroup_of(unit_at + w.rounds - 1) - wg0 + 1;
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's stores are acknowledged
            __syncthreads();
            if (threadIdx.x == 0)
                s_last = arrive_last(counters + wg0, tag, pieces);
            __syncthreads();
            if (s_last) {
                // wave w takes pieces w, w + 4, ..; four channels to a lane, so several columns to a load; G such groups of columns
                // and P pieces under way together
                constexpr int kLanes = kPass / 4, kColumns = 64 / kLanes;
                const auto join = [&](auto groups, auto at_once, int pass) {
                    constexpr int G = decltype(groups)::value, P = decltype(at_once)::value;
#pragma unroll 1
                    for (int c0 = 0; c0 < n_live; c0 += G * kColumns) {
                        f32x4 acc[G];
                        float most[G], sum[G];
#pragma unroll
                        for (int i = 0; i < G; ++i) acc[i] = f32x4{0, 0, 0, 0}, most[i] = kLowest, sum[i] = 0.0f;
#pragma unroll 1
                        for (int i0 = wave; i0 < pieces; i0 += 4 * P) {
                            f32x4 v[G][P];
                            float2 ml[G][P];
#pragma unroll
                            for (int i = 0; i < G; ++i)
#pragma unroll
                                for (int k = 0; k < P; ++k) {
                                    const int c = c0 + i * kColumns + lane / kLanes, from = i0 + 4 * k;
                                    v[i][k] = f32x4{0, 0, 0, 0}, ml[i][k] = {kLowest, 0.0f};
                                    if (c < n_live && from < pieces) {
                                        const float *p = partial_of<D>(a, from == 0 ? 2 * wg0 + 1 : 2 * (wg0 + from)) + c * (D + 4);
                                        ml[i][k] = load_pair(p + D);
                                        v[i][k] = load_past(a.ws, (int)(p - a.ws) * 4 + pass * kPass * 4 + lane % kLanes * 16);
                                    }
                                }
#pragma unroll
                            for (int i = 0; i < G; ++i)
#pragma unroll
                                for (int k = 0; k < P; ++k) {
                                    const float next = fmaxf(most[i], ml[i][k].x);
                                    const float f = __builtin_amdgcn_exp2f(most[i] - next), e = __builtin_amdgcn_exp2f(ml[i][k].x - next);
                                    most[i] = next, sum[i] = f * sum[i] + e * ml[i][k].y, acc[i] = f * acc[i] + e * v[i][k];
                                }
                        }
#pragma unroll
                        for (int i = 0; i < G; ++i) {
                            const int c = c0 + i * kColumns + lane / kLanes;
                            if (c < n_live) {
                                *reinterpret_cast<f32x4 *>(&s_o[wave][c][lane % kLanes * 4]) = acc[i];
                                if (lane % kLanes == 0) s_m[wave][c] = most[i], s_l[wave][c] = sum[i];
                            }
                        }
                    }
                };
#pragma unroll 1
                for (int pass = 0; pass < D / kPass; ++pass) {
                    if (pieces <= 8) join(std::integral_constant<int, 8>(), std::integral_constant<int, 2>(), pass);
                    else join(std::integral_constant<int, 2>(), std::integral_constant<int, 8>(), pass);
                    __syncthreads();
                    merge(pass, true, nullptr);
                    __syncthreads();
                }
            }
        }
        at = unit_at + (by_units ? 1 : stop);
    }
}

// ---------------------------------------------------------------- prompts

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kPromptTile = 64;  // tokens that the workgroup has in LDS at a time: a tile of the cache for each wave

// Where a tile's keys and values stand in LDS, as operands of 32 x 32 x 16 products.  K: 16-byte runs of 8 channels, [D/8][64 tokens].
// V: for 16 tokens and each half of a wave, 16-byte runs of that half's 8 tokens, [4 x 2][D]; a lane that converts four tokens of channels
// n D/16 + c writes its halves of the runs at place c 16 + n, so that neighbouring lanes write neighbouring runs.  O^T's rows are in
// the order of those places.  The second half of a wave has its two fours of tokens in the other order, in V as in S^T's rows: the lanes that
// write at the same time then meet in no bank (D 64, two chunks of 1024 tokens over 4096, 32 heads over 8: 86 -> 77 us; D 128 is not bound by LDS).
// Keys are read in the half of an iteration in front of its barrier, values behind it too: two and three tiles of them, and one
// barrier a tile.  80 KB for D = 128: two workgroups to a compute unit; D = 256 has one.
template <int D>
struct PromptTiles {
    uint32_t k[2][D / 8 * kPromptTile * 4], v[3][8 * D * 4];
};

// One wave's tile of the cache, converted into LDS.
template <int D>
__device__ __forceinline__ void convert_tile(uint32_t *to_k, uint32_t *to_v, const TileRegs<D> &r, int j, int left, int n, int g)
{
    constexpr int W = D / 32;
#pragma unroll
    for (int q = 0; q < W; ++q)
        *reinterpret_cast<bf16x8 *>(&to_k[((g * W + q) * kPromptTile + 16 * j + n) * 4]) = k_operand<D>(r, q);
    // scale bytes of tokens that are not there become 2^-127, so that whatever stands in their place is finite
    left -= 4 * g;
    const uint32_t vs = left >= 4 ? r.vs : left <= 0 ? 0u : r.vs & ((1u << (8 * left)) - 1);
    float sv[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) sv[i] = cache_scale((vs >> (8 * i)) & 255u);
#pragma unroll
    for (int b = 0; b < W; ++b) {
        uint32_t c[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = i * W + b;
            c[i] = cache_pair_at(r.v[at / 4], sv[i], at % 4);
        }
        uint32_t *run = &to_v[((2 * j + (g & 1)) * D + 2 * b * 16 + n) * 4 + ((g >> 1) ^ (g & 1)) * 2];
        *reinterpret_cast<u32x2 *>(run) = u32x2{low_halves(c[0], c[1]), low_halves(c[2], c[3])};
        *reinterpret_cast<u32x2 *>(run + 16 * 4) = u32x2{high_halves(c[0], c[1]), high_halves(c[2], c[3])};
    }
}

// The q-th longest of all sequences' blocks of 128 columns, by the position that its last column reaches (equal ones by sequence, then the
// later block first): found by bisection over positions, a lane for a run of sequences.  False if there are not that many.
__device__ __forceinline__ bool nth_longest_block(const AttentionArgs &a, int q, int share, int lane, int *seq, int *block)
{
    const int per_lane = (a.n_seq + 63) / 64;
    // blocks of a sequence that reach no further than t >= 0
    const auto up_to = [&](const Columns &c, int t) {
        const long long reach = ((long long)t - c.first_pos + 1) * c.share;
        return reach >= c.n ? (c.n + 127) / 128 : reach <= 0 ? 0 : (int)(reach / 128);
    };
    const auto columns = [&](int s, Columns *c) {
        c->n = 0, c->first_pos = 0, c->share = share;
        if (s < a.n_seq && !sequence_columns(a, a.start[s], a.start[s + 1], a.context[s], share, c)) c->n = 0;
    };
    Columns own;  // (the lane's sequence where it has one only)
    columns(lane * per_lane, &own);
    const auto count = [&](int t) {  // of the lane's sequences: blocks up to t
        int n = 0;
        for (int i = 0; i < per_lane; ++i) {
            Columns c = own;
            if (per_lane > 1) columns(lane * per_lane + i, &c);
            n = __builtin_elementwise_add_sat(n, up_to(c, t));
        }
        return n;
    };
    const auto total = [](int n) { return __builtin_amdgcn_readlane(wave_scan(n), 63); };
    int top = 0;
    for (int i = 0; i < per_lane; ++i) {
        Columns c = own;
        if (per_lane > 1) columns(lane * per_lane + i, &c);
        if (c.n > 0) top = max(top, c.first_pos + (c.n - 1) / share);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = max(top, __shfl_xor(top, off, kWave));
    top = __builtin_amdgcn_readfirstlane(top);
    const int all = total(count(top));
    if (q >= all) return false;
    int lo = 0, hi = top;  // the least position that no more than q blocks pass
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (all - total(count(mid)) <= q) hi = mid;
        else lo = mid + 1;
    }
    // blocks that reach just this position, by sequence; those at negative positions count with 0
    int mine = count(lo), below = lo > 0 ? count(lo - 1) : 0;
    const int left = q - (all - total(mine)), upto = wave_scan(mine - below);
    const int owner = __ffsll((unsigned long long)__ballot(upto > left)) - 1;
    if (owner < 0) return false;  // (more blocks than 32 bits count: starts that do not ascend)
    int rest = left - __builtin_amdgcn_readlane(upto - (mine - below), owner), s = owner * per_lane;
    for (; s < a.n_seq; ++s) {
        Columns c;
        columns(s, &c);
        const int last = up_to(c, lo), n = last - (lo > 0 ? up_to(c, lo - 1) : 0);
        if (rest < n) {
            *seq = __builtin_amdgcn_readfirstlane(s), *block = __builtin_amdgcn_readfirstlane(last - 1 - rest);
            return true;
        }
        rest -= n;
    }
    return false;
}

// Matrix-bound.  Workgroup: 4 waves, 32 columns each, of one kv head and sequence; 64 tokens at a time are converted to bf16 in LDS, a
// tile of the cache by each wave, while the tokens before them are used.  A step is 32 tokens: S^T = K q^T (32 tokens x 32 columns),
// softmax, O^T += V^T P^T; S^T of a step is asked for before the softmax of the one before, so that the matrix pipe has work
// meanwhile.  The longest units come first, since workgroups start in order (four chunks of 955 to 2048 tokens over 2867 to 6144: 372 us,
// block by block from the sequences' ends 385).  That is 0.87 PFLOP/s, where a large product of a library has 1.18: the matrix pipe is busy
// 40 % of the time, vector instructions (exponentials, conversions, maxima) 50, a wave waits 31, and two waves to a pipe do not interleave
// better: products in groups with vector instructions between them (412), priorities (382), 8 waves to a workgroup (395), 64
// columns to a wave (616), 32 tokens a barrier (414) and operands asked for earlier (368) gave no more.  Grid: (units, splits): where units are few the
// tokens of each are split, and the last workgroup to finish a unit joins its pieces, which stand in memory as they stood in the
// registers of each wave, in the order of the tokens.
template <int D>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void cache_prompt_kernel(AttentionArgs a, int units, int splits, unsigned long long tag)
{
    constexpr int kTile = cache_tile_bytes(D), kCols = 32, kBlock = 4 * kCols;
    extern __shared__ __align__(16) unsigned char s_raw[];
    PromptTiles<D> &s_tiles = *reinterpret_cast<PromptTiles<D> *>(s_raw);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
    const int lc = lane & 31, h = lane >> 5, row = lc ^ (lc & 4) << 1;  // (row: the token of S^T's row lc)
    const int share = a.n_heads / a.c.n_kv, n_kv = a.c.n_kv;
    const int head = blockIdx.x % n_kv;
    const float scale = a.scale != 0.0f ? fabsf(a.scale) * kLog2e : 1.0f;
    const TileOffsets<D> offsets(n, g);
    const size_t page_bytes = cache_page_bytes(a.c);
    const unsigned char *const cache = a.cache + (size_t)(head * (a.c.page >> 4)) * kTile;

    // a unit's pieces, and behind all of them the units' counters
    constexpr int kVectors = D / 8 + 1;  // of four floats a lane and piece: O^T, and the maxima and sums
    f32x4 *const pieces = reinterpret_cast<f32x4 *>(a.ws) + ((size_t)blockIdx.x * splits * 4 + wave) * kVectors * 64;
    unsigned long long *const counter =
        reinterpret_cast<unsigned long long *>(reinterpret_cast<f32x4 *>(a.ws) + (size_t)gridDim.x * splits * 4 * kVectors * 64) + blockIdx.x;
    bool announced = true;  // (units that the caller did not announce have no room for pieces: one workgroup sees to each)

    for (int rank = blockIdx.x / n_kv;; rank += units, announced = false) {
        int seq, block;
        if (!nth_longest_block(a, rank, share, lane, &seq, &block)) break;
        Columns cols;
        const int row0 = a.start[seq];
        sequence_columns(a, row0, a.start[seq + 1], a.context[seq], share, &cols);
        const scalar_ints table = (scalar_ints)(uintptr_t)(a.table + (size_t)seq * a.stride);
        const SeenTokens seen = seen_tokens(cols, block * kBlock, min((block + 1) * kBlock, cols.n));
        const int col0 = block * kBlock + wave * kCols;
        // positions of the wave's columns (of columns that are not there: none)
        const int wave_first = cols.first_pos + col0 / share;
        const int wave_last = col0 < cols.n ? cols.first_pos + (min(col0 + kCols, cols.n) - 1) / share : -1;
        bf16x8 q[D / 16];
        const uint32_t sign = a.scale < 0.0f ? 0x80008000u : 0u, keep = a.scale != 0.0f ? ~0u : 0u;
        const int col = col0 + lc;
        const bool live = col < cols.n;
        const int pos = live ? cols.first_pos + col / share : -1;
        const u32x4 *from = reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(a.q) +
                                                            ((size_t)(row0 + col / share) * a.n_heads + head * share + col % share) * D);
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            u32x4 x = {0, 0, 0, 0};
            if (live) x = from[2 * s + h];
            q[s] = __builtin_bit_cast(bf16x8, (x ^ sign) & keep);
        }
        f32x16 o[D / 32], s0, s1;
        float m = kLowest, l = 0.0f;
        float by = scale;  // (see choose_unit)
#pragma unroll
        for (int j = 0; j < D / 32; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[j][i] = 0.0f;
        // tokens in front of this one are all there: 0 if some page is none
        int full = seen.hi;
        for (int i = (seen.lo >> a.c.log_page) + lane; i << a.c.log_page < seen.hi; i += 64)
            if ((unsigned)table[i] >= (unsigned)a.c.n_pages) full = 0;
        full = __any(full == 0) ? 0 : full;
        const int first = seen.lo, all_tiles = (seen.hi - seen.lo + kPromptTile - 1) / kPromptTile;
        const int parts = announced ? max(min(splits, all_tiles), 1) : 1, part = blockIdx.y;
        if (part >= parts) continue;
        const int tile0 = (int)((long long)all_tiles * part / parts), n_tiles = (int)((long long)all_tiles * (part + 1) / parts);  // [tile0, n_tiles)
        unsigned long long counted = 0;
        if (parts > 1 && threadIdx.x == 0) counted = coherent_load(counter);

        TileRegs<D> regs;
        int limit = 0;
        auto load = [&](int tile) {  // this wave's 16 tokens
            const int t = first + tile * kPromptTile + 16 * wave;
            const int page = t < seen.hi ? table[t >> a.c.log_page] : -1;
            limit = (unsigned)page < (unsigned)a.c.n_pages ? seen.hi : 0;
            load_tile<D, false>(regs, cache + (size_t)(limit ? (unsigned)page : 0u) * page_bytes + ((t & (a.c.page - 1)) >> 4) * kTile, t < limit, offsets);
        };
        auto convert = [&](int tile) {
            convert_tile<D>(s_tiles.k[tile % 2], s_tiles.v[tile % 3], regs, wave, limit - (first + tile * kPromptTile + 16 * wave), n, g);
        };
        auto scores = [&](f32x16 &s, int tile, int half) {
            const uint32_t *const from = s_tiles.k[tile % 2];
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = 0.0f;
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                const bf16x8 x = *reinterpret_cast<const bf16x8 *>(&from[((2 * k + h) * kPromptTile + 32 * half + row) * 4]);
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, q[k], s, 0, 0, 0);
            }
        };
        auto weights = [&](f32x16 &s, bf16x8 (&p)[2], int tile, int half) {
            const int t0 = first + tile * kPromptTile + 32 * half;
            if (!(t0 + 32 <= full && t0 + 31 <= wave_first && wave_last - t0 < cols.window)) {
                int lim0 = seen.hi, lim1 = seen.hi;
                if (full == 0) {
                    if (t0 < seen.hi && (unsigned)table[t0 >> a.c.log_page] >= (unsigned)a.c.n_pages) lim0 = 0;
                    if (t0 + 16 < seen.hi && (unsigned)table[(t0 + 16) >> a.c.log_page] >= (unsigned)a.c.n_pages) lim1 = 0;
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int t = t0 + (8 * (i / 4) ^ 8 * h) + 4 * h + i % 4;
                    if (!(t < (i < 8 ? lim0 : lim1) && t <= pos && pos - t < cols.window)) s[i] = -INFINITY;
                }
            }
            float top = s[0];
#pragma unroll
            for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
            if (__any(top * by > m + kSlack)) {
                top = fmaxf(top, __shfl_xor(top, 32, kWave));
                const float next = fmaxf(m, top * by), factor = __builtin_amdgcn_exp2f(m - next);
                m = next;
                choose_unit(by, m, top, scale);
                l *= factor;
#pragma unroll
                for (int j = 0; j < D / 32; ++j) o[j] *= factor;
            }
            float x[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                x[i] = __builtin_amdgcn_exp2f(fmaf(s[i], by, -m));
                l += x[i];
            }
#pragma unroll
            for (int j = 0; j < 2; ++j)
                p[j] = as_bf16x8(pack_bf16(x[8 * j], x[8 * j + 1]), pack_bf16(x[8 * j + 2], x[8 * j + 3]), pack_bf16(x[8 * j + 4], x[8 * j + 5]),
                                 pack_bf16(x[8 * j + 6], x[8 * j + 7]));
        };
        auto values = [&](bf16x8 (&p)[2], int tile, int half) {
            const uint32_t *const from = s_tiles.v[tile % 3];
#pragma unroll
            for (int j = 0; j < D / 32; ++j)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const bf16x8 x = *reinterpret_cast<const bf16x8 *>(&from[((2 * (2 * half + k) + h) * D + 32 * j + lc) * 4]);
                    o[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, p[k], o[j], 0, 0, 0);
                }
        };

        bf16x8 p[2];
        if (n_tiles > tile0) {
            load(tile0);
            if (parts > 1 && threadIdx.x == 0) announce(counter, counted, tag);
            convert(tile0);
            if (n_tiles > tile0 + 1) load(tile0 + 1);
            __syncthreads();
            scores(s0, tile0, 0);
            for (int tile = tile0; tile < n_tiles; ++tile) {
                const int t0 = first + tile * kPromptTile;
                const bool more = tile + 1 < n_tiles, active = t0 <= wave_last;  // (uniform)
                if (active) {
                    scores(s1, tile, 1);
                    weights(s0, p, tile, 0);
                    values(p, tile, 0);
                }
                if (more) {
                    convert(tile + 1);
                    if (tile + 2 < n_tiles) load(tile + 2);
                }
                __syncthreads();
                if (active) {
                    if (more) scores(s0, tile + 1, 0);
                    weights(s1, p, tile, 1);
                    values(p, tile, 1);
                }
            }
        }
        if (parts > 1) {
            f32x4 *const mine = pieces + (size_t)part * 4 * kVectors * 64;
#pragma unroll
            for (int j = 0; j < D / 32; ++j)
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    store_past(mine, 4 * j + b, lane, f32x4{o[j][4 * b], o[j][4 * b + 1], o[j][4 * b + 2], o[j][4 * b + 3]});
            store_past(mine, kVectors - 1, lane, f32x4{by_scale(m, by, scale), l, 0.0f, 0.0f});
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's stores are acknowledged
            __syncthreads();
            int *const s_last = reinterpret_cast<int *>(s_raw);
            if (threadIdx.x == 0) *s_last = arrive_last(counter, tag, parts);
            __syncthreads();
            const bool last = *s_last;
            __syncthreads();  // (the next unit's tiles take its place)
            if (!last) continue;
            m = kLowest, l = 0.0f;
#pragma unroll
            for (int j = 0; j < D / 32; ++j)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[j][i] = 0.0f;
#pragma unroll 1
            for (int i = 0; i < parts; ++i) {
                const f32x4 *from = pieces + (size_t)i * 4 * kVectors * 64;
                f32x4 x[kVectors];
#pragma unroll
                for (int v = 0; v < kVectors; ++v) x[v] = load_past(from, (v * 64 + lane) * 16);
                const float top = fmaxf(m, x[kVectors - 1][0]);
                const float f = __builtin_amdgcn_exp2f(m - top), e = __builtin_amdgcn_exp2f(x[kVectors - 1][0] - top);
                m = top, l = f * l + e * x[kVectors - 1][1];
#pragma unroll
                for (int j = 0; j < D / 32; ++j)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[j][r] = f * o[j][r] + e * x[4 * j + r / 4][r % 4];
            }
        }
        const float sum = l + __shfl_xor(l, 32, kWave), per = sum > 0.0f ? 1.0f / sum : 0.0f;
        if (live) {
            uint16_t *y = static_cast<uint16_t *>(a.y) + ((size_t)(row0 + col / share) * a.n_heads + head * share + col % share) * D;
            // channels r D/16 .. of the lane's eight r: the places c 16 + r of all c
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    constexpr int C = D / 16;
                    uint32_t w[C / 2];
#pragma unroll
                    for (int e = 0; e < C; e += 2) w[e / 2] = pack_bf16(o[e / 2][4 * b + i] * per, o[e / 2][8 + 4 * b + i] * per);
                    uint32_t *to = reinterpret_cast<uint32_t *>(y + (8 * b + 4 * h + i) * C);
                    if constexpr (C == 4) *reinterpret_cast<u32x2 *>(to) = u32x2{w[0], w[1]};
                    else
#pragma unroll
                        for (int e = 0; e < C / 2; e += 4) *reinterpret_cast<u32x4 *>(to + e) = u32x4{w[e], w[e + 1], w[e + 2], w[e + 3]};
                }
        }
        __syncthreads();  // (the next block's tiles take these buffers)
    }
}

// Two workgroups to a compute unit hide each other's beginnings and ends, but cost the last of a unit's workgroups more pieces to join:
// two where there are 128 units, else one, and at most twice the square root of a unit's rounds (32 at least) for its pieces.  (Microseconds
// with 512 / 256 workgroups, D 128: 8 sequences x 40 heads x 4096 tokens 25.8 / 30.6, 64 x 8 x 1000, by pieces, 21.2 / 31.0; 2 x 8 x 131072 47.5 / 43,
// 1 x 8 x 131072 33.6 / 27.9, 1 x 32 x 4096 10.8 / 9.7.  With 16, 32, 48, 64, 96 pieces: 1 x 1 x 131072 46.9, 29.2, 26.6, 23.7, 25.1; 2 x 2 x
// 60000 23.8, 19.0, 17.2, 17.7, 17.7; 1 x 1 x 16000 14.5, 13.0, 15.5, 15.8, 19.5.)  D = 256 has registers for one.
int attention_workgroups(int n_seq, int n_heads, int n_kv, int d, int max_new, long long max_context)
{
    const long long blocks = ((long long)max_new * (n_heads / n_kv) + 15) / 16, rounds = (max_context + kRound - 1) / kRound;
    const long long units = std::max((long long)n_seq * n_kv * blocks, 1ll);
    const long long pieces = std::max(32ll, (long long)(2.0 * sqrt((double)rounds)));  // of a unit
    return (int)std::min(units * std::min(rounds, pieces), units >= 128 && d < 256 ? (long long)kWorkgroups : kWorkgroups / 2ll);
}

// From this many bytes of cache on (at the longest length) codes are loaded past the caches: what one layer's attention reads, other
// layers and the FFN's weights have displaced from the 256 MB last-level cache by the next step.  Microseconds, ordinary / past: caches
// of 62 MB, three in turn 21.1 / 21.4, eight 24.1 / 21.7; of 83 MB, three 22.2 / 22.8, six 25.2 / 23.0; of 136 MB, three 32.8 / 29.6; of 22 MB,
// three 14.1 / 14.6, twelve 14.9 / 14.7.
constexpr long long kPastBytes = 48ll << 20;

// Blocks of 128 columns that the sequences can have (each no more than the longest chunk, all no more than the rows hold), and the parts
// that the tokens of each are split into.  Another part costs its unit's last workgroup, which joins them one by one, about half of
// what 64 tokens cost; so sqrt(2 x tiles of 64) of them, and either one workgroup to a compute unit or all that fit.  (Microseconds, D 128, 512
// columns over 4 kv heads, 16000 tokens: 8 parts 65.6, 16 48.5, 22 54.5; 60000 tokens: 8 195, 16 115, 32 102; 1024 columns over 8 kv heads, 6000
// tokens: 8 37.0, 13 40.2; 16000: 8 66.2, 16 61.6.)
struct PromptGrid {
    int blocks, splits, most_splits;
    // (for these sizes and all smaller ones, which may be split into more parts)
    long long bytes(int n_kv, int d) const
    {
        const long long units = std::min<long long>((long long)blocks * n_kv, kWorkgroups);
        return most_splits == 1 ? 0 : std::min<long long>(units * most_splits, kWorkgroups) * 4 * (d / 8 + 1) * 64 * 16 + units * 8;
    }
};
PromptGrid prompt_grid(int n_tokens, int n_seq, int n_heads, int n_kv, int max_new, long long max_context)
{
    PromptGrid g;
    const long long share = n_heads / n_kv, tiles = (max_context + kPromptTile - 1) / kPromptTile;
    g.blocks = (int)std::min((max_new * share + 127) / 128 * n_seq, n_tokens * share / 128 + n_seq);
    g.most_splits = (int)std::max(1ll, std::min(32ll, (long long)sqrt(2.0 * tiles)));
    const long long fit = kWorkgroups / ((long long)g.blocks * n_kv);
    g.splits = (int)std::max(1ll, g.most_splits >= fit ? fit : std::min<long long>(g.most_splits, fit / 2));
    return g;
}

// Whether the prompt kernel takes a call: its blocks of 128 columns need half the time for each column, but it begins 11 us later, and 19 where
// units are few and their parts have to be joined.  A round of 128 tokens for all compute units: 0.57 us for a unit of 16 columns each, 2.4 for a
// block each.  Microseconds, general / prompt kernel, D 128, 4 query heads to each of 8 kv heads: 4 sequences x 512 new tokens 36.3 / 24.8, over 3000
// cached ones 126 / 94; 1 x 512 17.5 / 21.3, over 1000 32.7 / 31.2, over 3000 61 / 49; 1 x 128 over 700 10.0 / 20.0, over 16000 78 / 62; 32 heads
// of their own, 32 new tokens over 60000 91 / 121.  D = 256 has registers and LDS for one workgroup to a compute unit, so it takes whole blocks, and
// units for all compute units (two chunks of 1024 over 4096: 433 / 290).  (Every unit is counted with the longest context's rounds, and D = 64
// like D = 128: near the border, and for windows, which leave the prompt kernel's blocks less than that, either kernel may be the faster.)
constexpr int kPromptColumns = 65;  // with fewer it never does
bool takes_prompt(const PromptGrid &g, int n_tokens, int n_seq, int n_heads, int n_kv, int d, int max_new, long long max_context)
{
    const long long share = n_heads / n_kv, columns = max_new * share, blocks = (long long)g.blocks * n_kv;
    if (columns < kPromptColumns || (d == 256 && (columns < 128 || blocks < 256))) return false;
    const double units = (double)n_kv * std::min((columns + 15) / 16 * n_seq, n_tokens * share / 16 + n_seq), rounds = (double)((max_context + kRound - 1) / kRound);
    return rounds * (0.57 * units - 2.4 * (double)blocks) > 256.0 * (blocks < 256 ? 19.0 : 11.0);
}

// Positions that a row can see, at most, as far as the caller says.
long long longest_seen(int max_new, int max_context, int window)
{
    return window > 0 ? std::min((long long)max_context, (long long)window + max_new + 31) : max_context;
}

// The prompt kernel's grid for a call that it takes, else one without blocks.
PromptGrid prompt_of(int n_tokens, int n_seq, int n_heads, int n_kv, int d, int max_new, long long seen, bool all_bf16)
{
    PromptGrid none = {0, 1, 1};
    if (!all_bf16) return none;
    PromptGrid g = prompt_grid(n_tokens, n_seq, n_heads, n_kv, max_new, seen);
    if (d == 256) g.splits = 1;
    return takes_prompt(g, n_tokens, n_seq, n_heads, n_kv, d, max_new, seen) ? g : none;
}

template <int D>
hipError_t launch_prompt(const AttentionArgs &a, const PromptGrid &g, hipStream_t s)
{
    constexpr int kBytes = (int)sizeof(PromptTiles<D>);
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(cache_prompt_kernel<D>), hipFuncAttributeMaxDynamicSharedMemorySize, kBytes);
    if (e != hipSuccess) return e;
    cache_prompt_kernel<D><<<dim3((unsigned)(g.blocks * a.c.n_kv), (unsigned)g.splits), 256, kBytes, s>>>(a, g.blocks, g.splits, launch_tag());
    return hipGetLastError();
}

template <int D>
hipError_t launch_d(const AttentionArgs &a, hipStream_t s)
{
    const long long seen = longest_seen(a.max_new, a.max_context, a.window);
    const PromptGrid g = prompt_of(a.n_tokens, a.n_seq, a.n_heads, a.c.n_kv, D, a.max_new, seen, a.q_bf16 && a.y_bf16);
    if (g.blocks > 0) return launch_prompt<D>(a, g, s);
    const unsigned grid = (unsigned)attention_workgroups(a.n_seq, a.n_heads, a.c.n_kv, D, a.max_new, seen);
    const unsigned long long tag = launch_tag();
    if (!a.q_bf16) cache_attention_kernel<D, 3, 3, false><<<grid, 256, 0, s>>>(a, tag);
    else if (!a.y_bf16) cache_attention_kernel<D, 1, 3, false><<<grid, 256, 0, s>>>(a, tag);
    else if (a.n_seq * seen * a.c.n_kv * (D + D / 16) < kPastBytes) cache_attention_kernel<D, 1, 1, false><<<grid, 256, 0, s>>>(a, tag);
    else cache_attention_kernel<D, 1, 1, true><<<grid, 256, 0, s>>>(a, tag);
    return hipGetLastError();
}

}  // namespace

size_t cache_attention_ws(int n_tokens, int n_seq, int n_heads, int n_kv, int d, int max_new, int max_context)
{
    const bool chunks = d < 256 && (long long)max_new * (n_heads / n_kv) >= kPromptColumns;
    const long long prompt = chunks ? prompt_grid(n_tokens, n_seq, n_heads, n_kv, max_new, max_context).bytes(n_kv, d) : 0;
    return std::max((size_t)prompt, (size_t)attention_workgroups(n_seq, n_heads, n_kv, d, max_new, max_context) * (2 * 16 * (d + 4) * sizeof(float) + 8));
}

int cache_attention_parts(int n_tokens, int n_seq, int n_heads, int n_kv, int d, int max_new, int max_context, int window, int all_bf16)
{
    const PromptGrid g = prompt_of(n_tokens, n_seq, n_heads, n_kv, d, max_new, longest_seen(max_new, max_context, window), all_bf16 != 0);
    return g.blocks > 0 ? g.splits : 0;
}

hipError_t launch_cache_attention(const AttentionArgs &a, hipStream_t s)
{
    if (a.c.d == 64) return launch_d<64>(a, s);
    if (a.c.d == 128) return launch_d<128>(a, s);
    return launch_d<256>(a, s);
}

}  // namespace pop
