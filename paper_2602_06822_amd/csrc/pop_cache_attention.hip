// Attention over the 4-bit paged cache: y = softmax(scale q k^T + mask) v for every query row of every sequence.
//
// A query column is one (new token, query head) of a kv head's group; columns of one kv head share its keys and values.
// A step of a wave is 32 tokens: S^T = K q^T as two 16 x 16 tiles of matrix products (rows are tokens, columns are query
// columns), the running maximum and sum of a softmax per column, O^T += V^T P^T.  Transposed like this, S^T leaves the
// products in the layout in which P^T enters them (a lane has the same column and the same tokens), and the statistics of a
// column are one register of a lane.  The tokens of a step are in the order tile, group of four, token, which is the order
// of the cache's bytes: a lane's K and V codes are loads of D/8 bytes each, a wave's loads are contiguous kilobytes.
#include <math.h>

#include "pop_cache.h"

namespace pop {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896340736f;
// A column's maximum starts here: below every finite score, and a difference with it is no NaN.
constexpr float kLowest = -1.0e37f;
// A new maximum is taken only where it exceeds the old one by this many powers of two: until then the weights are at most
// 2^8, which 32 bits hold as exactly, and O is not rescaled.
constexpr float kSlack = 8.0f;

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

template <int D>
__device__ __forceinline__ void load_tile(TileRegs<D> &r, const unsigned char *tile, int n, int g)
{
    constexpr int W = D / 32;
    const unsigned char *k = tile + n * (D / 2) + g * (D / 8), *v = tile + 8 * D + (g * 16 + n) * (4 * W);
    if constexpr (D == 64) {
        const uint2 a = *reinterpret_cast<const uint2 *>(k), b = *reinterpret_cast<const uint2 *>(v);
        r.k[0] = a.x, r.k[1] = a.y, r.v[0] = b.x, r.v[1] = b.y;
    } else {
#pragma unroll
        for (int i = 0; i < D / 128; ++i) {
            const uint4 a = reinterpret_cast<const uint4 *>(k)[i], b = reinterpret_cast<const uint4 *>(v)[i];
            r.k[4 * i] = a.x, r.k[4 * i + 1] = a.y, r.k[4 * i + 2] = a.z, r.k[4 * i + 3] = a.w;
            r.v[4 * i] = b.x, r.v[4 * i + 1] = b.y, r.v[4 * i + 2] = b.z, r.v[4 * i + 3] = b.w;
        }
    }
    const unsigned char *ks = tile + 16 * D + n * W + g * D / 128;
    if constexpr (D == 256) r.ks = *reinterpret_cast<const uint16_t *>(ks);
    else r.ks = *ks;
    r.vs = *reinterpret_cast<const uint32_t *>(tile + 16 * D + 16 * W + (g * W + n * (D / 16) / 32) * 4);
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

// The general kernel.  Workgroup: 4 waves; grid: (splits, column blocks, kv heads x sequences).  Wave w takes steps w, w + 4, .. of
// the split's tokens.  QT, PT: bf16 terms that q and the softmax weights are split into: q one if it is bf16 (exact), else three (24
// bits); the weights one if the output is bf16 (rounded to 8 significant bits, as the output is), else three.  K and V are exact in bf16.
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

__device__ __forceinline__ void store_y(const AttentionArgs &a, size_t at, float y)
{
    if (a.y_bf16) static_cast<uint16_t *>(a.y)[at] = (uint16_t)pack_bf16(y, 0.0f);
    else static_cast<float *>(a.y)[at] = y;
}

// Sequences' rows of q and y: rows outside the tensors are not touched.
__device__ __forceinline__ bool sequence_columns(const AttentionArgs &a, int seq, int share, int *first_row, Columns *c)
{
    const int start = a.start[seq], fresh = a.start[seq + 1] - start;
    c->length = min(max(a.context[seq], 0), (int)min((long long)a.stride << a.c.log_page, (long long)0x7fffffff));
    c->first_pos = a.context[seq] - fresh;
    c->share = share;
    c->n = fresh * share;
    c->window = a.window > 0 ? a.window : 0x7fffffff;
    *first_row = start;
    return start >= 0 && fresh > 0 && fresh <= a.n_tokens - start;
}

template <int D, int QT, int PT>
__global__ __launch_bounds__(256) void cache_attention_kernel(AttentionArgs a, int splits)
{
    constexpr int kTile = cache_tile_bytes(D);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
    const int share = a.n_heads / a.c.n_kv;
    const int head = blockIdx.z % a.c.n_kv, seq = blockIdx.z / a.c.n_kv;
    Columns cols;
    int row0;
    if (!sequence_columns(a, seq, share, &row0, &cols)) return;
    const int *table = a.table + (size_t)seq * a.stride;

    __shared__ float s_o[16][D + 1];
    __shared__ float s_m[4][16], s_l[4][16];

    for (int block = blockIdx.y; block * 16 < cols.n; block += gridDim.y) {
        const int col = block * 16 + n, token = col / share, qh = head * share + col % share;
        const bool live = col < cols.n;
        const int pos = live ? cols.first_pos + token : -1;  // a column that is not there sees nothing
        // the lane's part of q: channels [g D/4, (g + 1) D/4)
        bf16x8 q[D / 32][QT];
#pragma unroll
        for (int s = 0; s < D / 32; ++s) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = 0.0f;
            if (live) {
                const size_t at = ((size_t)(row0 + token) * a.n_heads + qh) * D + g * (D / 4) + 8 * s;
                if (QT == 1) {
                    const uint4 w = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(a.q) + at);
                    x[0] = bf16_lo(w.x), x[1] = bf16_hi(w.x), x[2] = bf16_lo(w.y), x[3] = bf16_hi(w.y);
                    x[4] = bf16_lo(w.z), x[5] = bf16_hi(w.z), x[6] = bf16_lo(w.w), x[7] = bf16_hi(w.w);
                } else {
                    const float4 *f = reinterpret_cast<const float4 *>(static_cast<const float *>(a.q) + at);
                    const float4 u = f[0], w = f[1];
                    x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w, x[4] = w.x, x[5] = w.y, x[6] = w.z, x[7] = w.w;
                }
            }
            split_terms<QT>(x, q[s]);
        }
        // tokens that some column of the block sees
        const int last_col = min(block * 16 + 15, cols.n - 1);
        const int lo_pos = cols.first_pos + block * 16 / share, hi_pos = cols.first_pos + last_col / share;
        const int hi = min(hi_pos + 1, cols.length);
        const int lo = (int)max((long long)lo_pos - cols.window + 1, 0ll) & ~31;
        // a split's share of them, in whole rounds of the four waves
        const long long steps = hi > lo ? (hi - lo + 31) / 32 : 0, per = (steps + splits * 4 - 1) / (splits * 4) * 4;
        const long long begin = blockIdx.x * per, end = min(steps, begin + per);

        f32x4 o[D / 16];
#pragma unroll
        for (int j = 0; j < D / 16; ++j) o[j] = f32x4{0, 0, 0, 0};
        float m = kLowest, l = 0.0f;
        const float scale = a.scale * kLog2e;

        for (long long step = begin + wave; step < end; step += 4) {
            const int t0 = lo + (int)step * 32;
            TileRegs<D> r[2];
            int there[2];  // tokens of each tile that the cache holds
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int t = t0 + 16 * u;
                int page = t < hi ? table[t >> a.c.log_page] : -1;
                there[u] = page >= 0 && page < a.c.n_pages ? min(hi - t, 16) : 0;
                if (there[u] == 0) page = 0;
                load_tile<D>(r[u], a.cache + cache_tile_offset(page, head, t & (a.c.page - 1), a.c.n_kv, a.c.log_page, kTile), n, g);
            }
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
            float p[8];
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int u = i / 4, at = 4 * g + i % 4, t = t0 + 16 * u + at;
                const bool sees = at < there[u] && t <= pos && pos - t < cols.window;
                p[i] = sees ? s[u][i % 4] * scale : -INFINITY;
                top = fmaxf(top, p[i]);
            }
            if (__any(top > m + kSlack)) {
                top = fmaxf(top, __shfl_xor(top, 16, kWave));
                top = fmaxf(top, __shfl_xor(top, 32, kWave));
                const float next = fmaxf(m, top), factor = exp2f(m - next);
                m = next;
                l *= factor;
#pragma unroll
                for (int j = 0; j < D / 16; ++j) o[j] *= factor;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                p[i] = __builtin_amdgcn_exp2f(p[i] - m);
                l += p[i];
            }
            bf16x8 w[PT];
            split_terms<PT>(p, w);
            // V: four tokens a tile, D/16 channels; scale bytes of tokens that are not there become 2^-127, so that whatever
            // stands in their place is finite
            float sv[8];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int left = there[u] - 4 * g;
                const uint32_t vs = left >= 4 ? r[u].vs : left <= 0 ? 0u : r[u].vs & ((1u << (8 * left)) - 1);
#pragma unroll
                for (int i = 0; i < 4; ++i) sv[4 * u + i] = cache_scale((vs >> (8 * i)) & 255u);
            }
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
        // the four waves' sums, joined in their order; a lane has channels [g D/4, (g + 1) D/4) of column n
        l += __shfl_xor(l, 16, kWave);
        l += __shfl_xor(l, 32, kWave);
        __syncthreads();
        if (g == 0) s_m[wave][n] = m, s_l[wave][n] = l;
        __syncthreads();
        const float top = fmaxf(fmaxf(s_m[0][n], s_m[1][n]), fmaxf(s_m[2][n], s_m[3][n]));
        const float factor = exp2f(m - top);
        for (int w = 0; w < 4; ++w) {
            if (wave == w) {
#pragma unroll
                for (int j = 0; j < D / 16; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float *at = &s_o[n][(4 * g + i) * (D / 16) + j];
                        *at = (w ? *at : 0.0f) + factor * o[j][i];
                    }
            }
            __syncthreads();
        }
        for (int e = threadIdx.x; e < 16 * D; e += 256) {
            const int c = e / D, ch = e % D, gc = block * 16 + c;
            if (gc >= cols.n) continue;
            float most = kLowest, sum = 0.0f;
#pragma unroll
            for (int w = 0; w < 4; ++w) most = fmaxf(most, s_m[w][c]);
#pragma unroll
            for (int w = 0; w < 4; ++w) sum += exp2f(s_m[w][c] - most) * s_l[w][c];
            const float acc = s_o[c][ch];
            const size_t row = (size_t)(row0 + gc / share) * a.n_heads + head * share + gc % share;
            if (splits == 1) {
                store_y(a, row * D + ch, sum > 0.0f ? acc / sum : 0.0f);
            } else {
                float *part = a.ws + (row * splits + blockIdx.x) * (D + 2);
                part[ch] = acc;
                if (ch == 0) part[D] = most, part[D + 1] = sum;
            }
        }
        __syncthreads();
    }
}

// Joins the splits of each row, in their order.
template <int D>
__global__ __launch_bounds__(256) void cache_join_kernel(AttentionArgs a, int splits)
{
    const int per = 256 / D;
    const long long row = (long long)blockIdx.x * per + threadIdx.x / D;
    const int ch = threadIdx.x % D;
    const int token = (int)(row / a.n_heads);
    if (token >= a.n_tokens || token < a.start[0] || token >= a.start[a.n_seq]) return;
    const float *part = a.ws + row * splits * (D + 2);
    float top = kLowest, sum = 0.0f, acc = 0.0f;
    for (int i = 0; i < splits; ++i) top = fmaxf(top, part[i * (D + 2) + D]);
    for (int i = 0; i < splits; ++i) {
        const float f = exp2f(part[i * (D + 2) + D] - top);
        sum += f * part[i * (D + 2) + D + 1];
        acc += f * part[i * (D + 2) + ch];
    }
    store_y(a, row * D + ch, sum > 0.0f ? acc / sum : 0.0f);
}

// Column blocks of 16, and how many ways the tokens of each are split: enough workgroups for every compute unit to hold four,
// splits of 256 tokens at least.
struct AttentionGrid {
    int blocks, splits;
};
AttentionGrid attention_grid(int n_seq, int n_heads, int n_kv, int max_new, int max_context)
{
    AttentionGrid g;
    g.blocks = (int)min(((long long)max_new * (n_heads / n_kv) + 15) / 16, 65535ll);
    const long long units = (long long)n_seq * n_kv * g.blocks;
    const long long want = (1024 + units - 1) / units, most = ((long long)max_context + 255) / 256;
    g.splits = (int)max(1ll, min(want, most));
    return g;
}

template <int D>
hipError_t launch_d(const AttentionArgs &a, hipStream_t s)
{
    const AttentionGrid g = attention_grid(a.n_seq, a.n_heads, a.c.n_kv, a.max_new, a.max_context);
    const dim3 grid((unsigned)g.splits, (unsigned)g.blocks, (unsigned)(a.n_seq * a.c.n_kv));
    if (!a.q_bf16) cache_attention_kernel<D, 3, 3><<<grid, 256, 0, s>>>(a, g.splits);
    else if (!a.y_bf16) cache_attention_kernel<D, 1, 3><<<grid, 256, 0, s>>>(a, g.splits);
    else cache_attention_kernel<D, 1, 1><<<grid, 256, 0, s>>>(a, g.splits);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || g.splits == 1) return e;
    const long long rows = (long long)a.n_tokens * a.n_heads;
    cache_join_kernel<D><<<(unsigned)((rows + 256 / D - 1) / (256 / D)), 256, 0, s>>>(a, g.splits);
    return hipGetLastError();
}

}  // namespace

size_t cache_attention_ws(int n_tokens, int n_seq, int n_heads, int n_kv, int d, int max_new, int max_context)
{
    const AttentionGrid g = attention_grid(n_seq, n_heads, n_kv, max_new, max_context);
    return g.splits == 1 ? 0 : (size_t)n_tokens * n_heads * g.splits * (d + 2) * sizeof(float);
}

hipError_t launch_cache_attention(const AttentionArgs &a, hipStream_t s)
{
    if (a.c.d == 64) return launch_d<64>(a, s);
    if (a.c.d == 128) return launch_d<128>(a, s);
    return launch_d<256>(a, s);
}

}  // namespace pop
