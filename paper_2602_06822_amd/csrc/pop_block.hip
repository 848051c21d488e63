// What stands between a decoder layer's blocks: residual sums with the norms around a block, rotary positions.
#include <algorithm>
#include <type_traits>

#include "pop_block.h"

namespace pop {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    const bf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
}

// Eight channels of a row from `at` on: 16-byte loads.
template <bool BF16>
struct Eight {
    u32x4 raw[BF16 ? 1 : 2];
    __device__ __forceinline__ void load(const void *p, long long at)
    {
        const u32x4 *from = reinterpret_cast<const u32x4 *>(static_cast<const char *>(p) + at * (BF16 ? 2 : 4));
#pragma unroll
        for (int i = 0; i < (BF16 ? 1 : 2); ++i) raw[i] = from[i];
    }
    __device__ __forceinline__ float operator[](int i) const
    {
        if constexpr (BF16) return i % 2 ? bf16_hi(raw[0][i / 2]) : bf16_lo(raw[0][i / 2]);
        else return __uint_as_float(raw[i / 4][i % 4]);
    }
};

template <bool BF16>
__device__ __forceinline__ void store_eight(void *p, long long at, const float (&x)[8])
{
    u32x4 *to = reinterpret_cast<u32x4 *>(static_cast<char *>(p) + at * (BF16 ? 2 : 4));
    if constexpr (BF16) {
        to[0] = u32x4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
    } else {
        const f32x4 a = {x[0], x[1], x[2], x[3]}, b = {x[4], x[5], x[6], x[7]};
        to[0] = __builtin_bit_cast(u32x4, a), to[1] = __builtin_bit_cast(u32x4, b);
    }
}

template <bool BF16>
__device__ __forceinline__ float load_one(const void *p, long long at)
{
    if constexpr (BF16) return __uint_as_float((uint32_t)static_cast<const uint16_t *>(p)[at] << 16);
    else return static_cast<const float *>(p)[at];
}
template <bool BF16>
__device__ __forceinline__ void store_one(void *p, long long at, float x)
{
    if constexpr (BF16) static_cast<__bf16 *>(p)[at] = (__bf16)x;
    else static_cast<float *>(p)[at] = x;
}

// ---------------------------------------------------------------- residual sums and norms

// Sum over a row's threads, the same in all of them: L lanes, or (0) the workgroup.
template <int L>
__device__ __forceinline__ float row_sum(float v, float *s_sums)
{
#pragma unroll
    for (int off = (L ? L : kWave) / 2; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
    const int waves = blockDim.x / kWave;
    if (L || waves == 1) return v;
    if (threadIdx.x % kWave == 0) s_sums[threadIdx.x / kWave] = v;
    __syncthreads();
    v = 0.0f;
    for (int i = 0; i < waves; ++i) v += s_sums[i];
    return v;
}

// Eight of a row's channels: those from `at` on (V8), or every `apart`-th one.
template <bool BF16, bool V8>
__device__ __forceinline__ void row_load(const void *p, long long row, int at, int apart, int d, float (&x)[8])
{
    if constexpr (V8) {
        Eight<BF16> e;
        e.load(p, row + at);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = e[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = at + i * apart;
            x[i] = c < d ? load_one<BF16>(p, row + c) : 0.0f;
        }
    }
}
template <bool BF16, bool V8>
__device__ __forceinline__ void row_store(void *p, long long row, int at, int apart, int d, const float (&x)[8])
{
    if constexpr (V8) {
        store_eight<BF16>(p, row + at, x);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = at + i * apart;
            if (c < d) store_one<BF16>(p, row + c, x[i]);
        }
    }
}

// A row has a workgroup (L = 0) or L lanes, a thread N eights of its channels in registers: everything is read once and written once.  The sums of
// squares are float32: a thread's up to 8 N terms one by one, the rest a tree.
//
// Bound by memory: 4096 rows of 5120, float32 stream, bf16 block and gate, both norms 59 us (294 MB at 5.0 TB/s, where a copy has 4.8); 2047 rows
// of 4096 in bf16 12.4 us (67 MB at 5.4).  A step's few rows: 2.8 us on the device, less than the call.  Narrow rows (heads' norms) by lanes, several to a wave:
// 65536 rows of 128 in bf16 12.3 us, with a wave to each 21.7; 58205 of 160 15.4, with both norms and a gate 17.8, the stream in float32 23.5.  Channel by channel, every lane's next to
// the other's: 2047 rows of 4099 in bf16 24.0 us (2.8 TB/s), of 4100 in float32 23.1 (5.8).
template <bool XBF16, bool BF16, bool V8, int N, int L>
__global__ __launch_bounds__(L ? 256 : 1024) void block_norm_kernel(BlockNormArgs a)
{
    __shared__ float s_sums[2][16];
    const int lanes = L ? L : (int)blockDim.x, lane = L ? threadIdx.x % L : threadIdx.x;
    const long long row = L ? (long long)blockIdx.x * (256 / (L ? L : 1)) + threadIdx.x / (L ? L : 1) : blockIdx.x;
    if (L && row >= a.n) return;  // (a row's lanes leave together, and nobody waits for them)
    const int step = lanes * 8, first = V8 ? lane * 8 : lane;
    float v[N][8];
#pragma unroll
    for (int j = 0; j < N; ++j) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[j][i] = 0.0f;
        if (a.u && first + j * step < a.d) row_load<BF16, V8>(a.u, row * a.u_stride, first + j * step, lanes, a.d, v[j]);
    }
    if (a.post) {
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(v[j][i], v[j][i], sum);
        const float by = 1.0f / sqrtf(row_sum<L>(sum, s_sums[0]) / (float)a.d + a.eps);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if (first + j * step >= a.d) continue;
            float w[8] = {1, 1, 1, 1, 1, 1, 1, 1};
            if (a.w_post) row_load<BF16, V8>(a.w_post, 0, first + j * step, lanes, a.d, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[j][i] = v[j][i] * by * (a.w_post ? w[i] + a.offset : 1.0f);
        }
    }
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        if (first + j * step >= a.d) continue;
        float x[8];
        row_load<XBF16, V8>(a.x, row * a.x_stride, first + j * step, lanes, a.d, x);
        if (a.gate) {
            float g[8];
            row_load<BF16, V8>(a.gate, row * a.gate_stride, first + j * step, lanes, a.d, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[j][i] *= g[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[j][i] = a.u ? fmaf(a.x_scale, x[i], a.u_scale * v[j][i]) : a.x_scale * x[i];
            sum = fmaf(v[j][i], v[j][i], sum);
        }
        if (a.x_out) row_store<XBF16, V8>(a.x_out, row * a.x_out_stride, first + j * step, lanes, a.d, v[j]);
    }
    if (!a.z) return;
    const float by = 1.0f / sqrtf(row_sum<L>(sum, s_sums[1]) / (float)a.d + a.eps);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        if (first + j * step >= a.d) continue;
        float w[8] = {1, 1, 1, 1, 1, 1, 1, 1};
        if (a.w_pre) row_load<BF16, V8>(a.w_pre, 0, first + j * step, lanes, a.d, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[j][i] = v[j][i] * by * (a.w_pre ? w[i] + a.offset : 1.0f);
        row_store<BF16, V8>(a.z, row * a.z_stride, first + j * step, lanes, a.d, v[j]);
    }
}

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

template <bool XBF16, bool BF16, bool V8>
hipError_t launch_norm(const BlockNormArgs &a, hipStream_t s)
{
    const int eights = (a.d + 7) / 8;
    const auto rows_in = [&](int lanes) { return (unsigned)((a.n + 256 / lanes - 1) / (256 / lanes)); };
    if (eights <= 8) block_norm_kernel<XBF16, BF16, V8, 1, 8><<<rows_in(8), 256, 0, s>>>(a);
    else if (eights <= 16) block_norm_kernel<XBF16, BF16, V8, 1, 16><<<rows_in(16), 256, 0, s>>>(a);
    else if (eights <= 32) block_norm_kernel<XBF16, BF16, V8, 1, 32><<<rows_in(32), 256, 0, s>>>(a);
    else {
        const int n = eights <= 1024 ? 1 : eights <= 2048 ? 2 : eights <= 4096 ? 4 : 8;
        const unsigned threads = (unsigned)(((eights + n - 1) / n + 63) / 64 * 64);
        switch (n) {
            case 1: block_norm_kernel<XBF16, BF16, V8, 1, 0><<<a.n, threads, 0, s>>>(a); break;
            case 2: block_norm_kernel<XBF16, BF16, V8, 2, 0><<<a.n, threads, 0, s>>>(a); break;
            case 4: block_norm_kernel<XBF16, BF16, V8, 4, 0><<<a.n, threads, 0, s>>>(a); break;
            default: block_norm_kernel<XBF16, BF16, V8, 8, 0><<<a.n, threads, 0, s>>>(a); break;
        }
    }
    return hipGetLastError();
}

// ---------------------------------------------------------------- rotary positions

// A token's sines and cosines: angles are products of 64 bits in revolutions, of which the whole ones are taken off before they are rounded
// to 32.  Times the amplitude.
__device__ __forceinline__ float2 turn_of(int position, double per_token, float amplitude)
{
    const double t = (double)position * per_token;
    float sn, cs;
    sincospif(2.0f * (float)(t - rint(t)), &sn, &cs);
    return {amplitude * cs, amplitude * sn};
}

// A workgroup has a run of tokens (`tokens`) and of each the same part of its heads' eights of channels; sines and cosines stand in LDS, a thread
// computes some and all heads use them.  kHalves: an eight and the one it is turned with together; kPairs: an eight by itself; kStaged: halves that are
// no whole eights, where the other channels come out of LDS; eights behind the turned part are copied.  A thread asks for kTogether of them before
// it waits, the first ones before the angles are computed (kStaged: all of them).
//
// Bound by memory: 8191 tokens of 32 + 32 heads of 128 in bf16, out of a projection's rows, 55 us (268 MB at 4.9 TB/s, where a copy has 4.8); channel by
// channel, as in the kernel below, 80.  4000 tokens of 32 + 8 heads, 46 of 128 channels turned: 25 us staged, channel by channel 41.  A step's eight tokens: 3.5 us
// on the device, less than the call.
enum { kHalves = 0, kPairs = 1, kStaged = 2 };
constexpr int kTogether = 4, kMostTurns = 1024;
template <bool BF16, int FORM>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a, int tokens, int part)
{
    constexpr bool PAIRS = FORM == kPairs;
    typedef typename std::conditional<BF16, uint16_t, float>::type Stored;
    __shared__ float2 s_turn[kMostTurns + 4];
    __shared__ int s_position[64];
    __shared__ __align__(16) Stored s_eights[FORM == kStaged ? 256 * kTogether * 8 : 8];
    const int token0 = blockIdx.x * tokens, here = min(tokens, a.n - token0), half = a.r / 2;
    const int turned = FORM == kHalves ? a.r / 16 : (a.r + 7) / 8, per_head = FORM == kHalves ? turned + (a.d - a.r) / 8 : a.d / 8, per_token = (a.n_heads + a.n_kv) * per_head;
    const int first = blockIdx.y * part, mine = min(part, per_token - first), total = here * mine;
    struct Place {
        const void *from;
        void *to;
        long long in, out;
        int token, chunk;
    };
    const auto place = [&](int e) {
        Place p;
        p.token = e / mine;
        const int i = first + e - p.token * mine, head = i / per_head;
        p.chunk = i - head * per_head;
        const bool of_k = head >= a.n_heads;
        const long long row = token0 + p.token, h = of_k ? head - a.n_heads : head;
        const int ch = FORM != kHalves || p.chunk < turned ? 8 * p.chunk : a.r + 8 * (p.chunk - turned);
        p.from = of_k ? a.k : a.q, p.to = of_k ? a.k_out : a.q_out;
        p.in = row * (of_k ? a.k_stride : a.q_stride) + h * a.d + ch;
        p.out = row * (of_k ? a.k_out_stride : a.q_out_stride) + h * a.d + ch;
        return p;
    };
    Eight<BF16> x[kTogether], y[kTogether];
    const auto ask = [&](int e0) {
#pragma unroll
        for (int u = 0; u < kTogether; ++u) {
            const int e = e0 + 256 * u;
            if (e < total) {
                const Place p = place(e);
                x[u].load(p.from, p.in);
                if (FORM == kHalves && p.chunk < turned) y[u].load(p.from, p.in + half);
            }
        }
    };
    ask(threadIdx.x);
    for (int i = threadIdx.x; i < here * half; i += 256) {
        const int token = i / half;
        s_turn[i] = turn_of(a.positions[token0 + token], a.turns[i - token * half], a.amplitude);
    }
    if (threadIdx.x < here) s_position[threadIdx.x] = a.positions[token0 + threadIdx.x];
    if constexpr (FORM == kStaged) {  // (whole heads, no more than a thread's kTogether: checked by the launcher)
#pragma unroll
        for (int u = 0; u < kTogether; ++u) {
            const int e = threadIdx.x + 256 * u;
#pragma unroll
            for (int i = 0; i < (BF16 ? 1 : 2); ++i)
                if (e < total) reinterpret_cast<u32x4 *>(s_eights)[(BF16 ? 1 : 2) * e + i] = x[u].raw[i];
        }
    }
    __syncthreads();
    for (int e0 = threadIdx.x; e0 < total; e0 += 256 * kTogether) {
#pragma unroll
        for (int u = 0; u < kTogether; ++u) {
            const int e = e0 + 256 * u;
            if (e >= total) break;
            const Place p = place(e);
            if (s_position[p.token] < 0) continue;
            if (p.chunk >= turned) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = x[u][i];
                store_eight<BF16>(p.to, p.out, v);
            } else if constexpr (PAIRS) {
                const float2 *const t = s_turn + p.token * half + 4 * p.chunk;
                float v[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool turns = 8 * p.chunk + 2 * i < a.r;
                    v[2 * i] = turns ? x[u][2 * i] * t[i].x - x[u][2 * i + 1] * t[i].y : x[u][2 * i];
                    v[2 * i + 1] = turns ? x[u][2 * i] * t[i].y + x[u][2 * i + 1] * t[i].x : x[u][2 * i + 1];
                }
                store_eight<BF16>(p.to, p.out, v);
            } else if constexpr (FORM == kStaged) {
                const float2 *const t = s_turn + p.token * half;
                const Stored *const of_head = s_eights + (e - p.chunk) * 8;
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int c = 8 * p.chunk + i;
                    v[i] = x[u][i];
                    if (c < half) v[i] = v[i] * t[c].x - load_one<BF16>(of_head, c + half) * t[c].y;
                    else if (c < a.r) v[i] = load_one<BF16>(of_head, c - half) * t[c - half].y + v[i] * t[c - half].x;
                }
                store_eight<BF16>(p.to, p.out, v);
            } else {
                const float2 *const t = s_turn + p.token * half + 8 * p.chunk;
                float v[8], w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    v[i] = x[u][i] * t[i].x - y[u][i] * t[i].y;
                    w[i] = x[u][i] * t[i].y + y[u][i] * t[i].x;
                }
                store_eight<BF16>(p.to, p.out, v);
                store_eight<BF16>(p.to, p.out + half, w);
            }
        }
        ask(e0 + 256 * kTogether);
    }
}

// Rows and heads of any alignment: channels one by one, a token to a workgroup.  4000 tokens of 32 + 8 heads of 126 in bf16, 46 channels turned: 39.8 us (2.0 TB/s); all of them 23.0 (3.5).
template <bool BF16>
__global__ __launch_bounds__(256) void rotary_any_kernel(RotaryArgs a)
{
    __shared__ float2 s_turn[kMostRotary / 2];
    const int token = blockIdx.x, position = a.positions[token], half = a.r / 2;
    if (position < 0) return;
    for (int i = threadIdx.x; i < half; i += 256) s_turn[i] = turn_of(position, a.turns[i], a.amplitude);
    __syncthreads();
    const int per = half + (a.d - a.r), heads = a.n_heads + a.n_kv;
    for (int e = threadIdx.x; e < heads * per; e += 256) {
        const int head = e / per, i = e % per;
        const bool of_k = head >= a.n_heads;
        const void *from = of_k ? a.k : a.q;
        void *to = of_k ? a.k_out : a.q_out;
        const int h = of_k ? head - a.n_heads : head;
        const long long in = token * (of_k ? a.k_stride : a.q_stride) + (long long)h * a.d;
        const long long out = token * (of_k ? a.k_out_stride : a.q_out_stride) + (long long)h * a.d;
        if (i < half) {
            const int c0 = a.pairs ? 2 * i : i, c1 = a.pairs ? 2 * i + 1 : i + half;
            const float x = load_one<BF16>(from, in + c0), y = load_one<BF16>(from, in + c1);
            const float2 t = s_turn[i];
            store_one<BF16>(to, out + c0, x * t.x - y * t.y);
            store_one<BF16>(to, out + c1, x * t.y + y * t.x);
        } else {
            const int c = a.r + i - half;
            store_one<BF16>(to, out + c, load_one<BF16>(from, in + c));
        }
    }
}

template <bool BF16>
hipError_t launch_rotary_as(const RotaryArgs &a, hipStream_t s)
{
    const bool v8 = a.d % 8 == 0 && (a.q_stride | a.k_stride | a.q_out_stride | a.k_out_stride) % 8 == 0 && aligned16(a.q) && aligned16(a.k) &&
                    aligned16(a.q_out) && aligned16(a.k_out);
    const int form = a.pairs ? kPairs : a.r % 16 == 0 ? kHalves : kStaged, most = 256 * kTogether;
    const int per_head = form == kHalves ? a.r / 16 + (a.d - a.r) / 8 : a.d / 8, per_token = (a.n_heads + a.n_kv) * per_head;
    if (!v8 || (form == kStaged && per_head > most)) {
        rotary_any_kernel<BF16><<<a.n, 256, 0, s>>>(a);
        return hipGetLastError();
    }
    // full threads where there is work for all compute units, else as many workgroups as there are eights for
    const int at_once = (long long)a.n * per_token >= 512ll * most || (form == kStaged && per_head > 256) ? most : 256;
    const int tokens = std::max(1, std::min({at_once / per_token, kMostTurns / (a.r / 2), 64}));
    const int part = std::min(per_token, form == kStaged ? at_once / per_head * per_head : at_once);
    const dim3 grid((unsigned)((a.n + tokens - 1) / tokens), (unsigned)((per_token + part - 1) / part));
    if (form == kPairs) rotary_kernel<BF16, kPairs><<<grid, 256, 0, s>>>(a, tokens, part);
    else if (form == kHalves) rotary_kernel<BF16, kHalves><<<grid, 256, 0, s>>>(a, tokens, part);
    else rotary_kernel<BF16, kStaged><<<grid, 256, 0, s>>>(a, tokens, part);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_block_norm(const BlockNormArgs &a, hipStream_t s)
{
    const bool v8 = a.d % 8 == 0 && (a.x_stride | a.u_stride | a.gate_stride | a.x_out_stride | a.z_stride) % 8 == 0 && aligned16(a.x) && aligned16(a.u) &&
                    aligned16(a.gate) && aligned16(a.w_post) && aligned16(a.w_pre) && aligned16(a.x_out) && aligned16(a.z);
    if (a.x_bf16) {
        if (a.bf16) return v8 ? launch_norm<true, true, true>(a, s) : launch_norm<true, true, false>(a, s);
        return v8 ? launch_norm<true, false, true>(a, s) : launch_norm<true, false, false>(a, s);
    }
    if (a.bf16) return v8 ? launch_norm<false, true, true>(a, s) : launch_norm<false, true, false>(a, s);
    return v8 ? launch_norm<false, false, true>(a, s) : launch_norm<false, false, false>(a, s);
}

hipError_t launch_rotary(const RotaryArgs &a, hipStream_t s) { return a.bf16 ? launch_rotary_as<true>(a, s) : launch_rotary_as<false>(a, s); }

}  // namespace pop
