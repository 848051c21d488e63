// Device code that the attention kernels over the 4-bit cache share: operands from a tile's codes, the running softmax of a wave's columns, what
// workgroups hand to each other.
//
// A query column is one (new token, query head) of a kv head's group; columns of one kv head share its keys and values.
// A step of a wave is 32 tokens: S^T = K q^T as two 16 x 16 tiles of matrix products (rows are tokens, columns are query
// columns), the running maximum and sum of a softmax per column, O^T += V^T P^T.  Transposed like this, S^T leaves the
// products in the layout in which P^T enters them (a lane has the same column and the same tokens), and the statistics of a
// column are one register of a lane.  The tokens of a step are in the order tile, group of four, token, which is the order
// of the cache's bytes: a lane's K and V codes are loads of D/8 bytes each, a wave's loads are contiguous kilobytes.
#pragma once
#include "pop_cache.h"

namespace pop {

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

// Tokens [lo, hi) that some of the columns [begin, end) see, lo a multiple of 32, and the first and the last of the columns' positions.  Where first
// tokens stay visible (SINKS) and lie apart from those, steps for them stand in front of lo, from `begin` on; else begin is lo.
struct SeenTokens {
    int lo, hi, first_pos, last_pos, begin;
    // The token of place t of [begin, hi).
    template <bool SINKS>
    __device__ __forceinline__ int token(int t) const
    {
        return SINKS && t < lo ? t - begin : t;
    }
};
template <bool SINKS>
__device__ __forceinline__ SeenTokens seen_tokens(const Columns &c, int begin, int end, int sinks)
{
    SeenTokens s;
    s.first_pos = c.first_pos + begin / c.share, s.last_pos = c.first_pos + (end - 1) / c.share;
    s.hi = max(min(s.last_pos + 1, c.length), 0);
    s.lo = c.window == kNoWindow ? 0 : min(max(s.first_pos - c.window + 1, 0) & ~31, s.hi);
    s.begin = s.lo;
    if (SINKS) {
        const int kept = (min(sinks, kMostTokens) + 31) & ~31;
        if (s.lo <= kept) s.lo = s.begin = 0;
        else s.begin = s.lo - kept;
    }
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
    template <bool SINKS>
    __device__ __forceinline__ void step(const TileRegs<D> (&r)[2], const int (&limit)[2], bool masked, int t0, int pos, int window, int sinks, int g,
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
                    if (!(t + i < limit[u] && t + i <= pos && (pos - (t + i) < window || (SINKS && t + i < sinks)))) s[u][i] = -INFINITY;
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

// ---- blocks of 128 columns

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

// ---- joining

// The pieces of a unit's columns (channels [pass kPass, (pass + 1) kPass) of them), joined into four sums that the waves leave in LDS: wave w takes
// pieces w, w + 4, ..; four channels to a lane, so several columns to a load; G such groups of columns and P pieces under way together.
// place(i): piece i, n_live rows of D channels, the column's maximum and sum, and two floats more.
template <int D, int kPass, int G, int P, class Place>
__device__ __forceinline__ void join_pieces(const float *ws, Place place, int pieces, int n_live, int wave, int lane, int pass, float (&s_o)[4][16][kPass + 4],
                                            float (&s_m)[4][16], float (&s_l)[4][16])
{
    constexpr int kLanes = kPass / 4, kColumns = 64 / kLanes;
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
                        const float *p = place(from) + c * (D + 4);
                        ml[i][k] = load_pair(p + D);
                        v[i][k] = load_past(ws, (int)(p - ws) * 4 + pass * kPass * 4 + lane % kLanes * 16);
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
}

}  // namespace pop
