// The kernels of attention over the 4-bit paged cache: y = softmax(scale q k^T + mask) v for every query row of every sequence.
// SINKS: with a window, the first `sinks` tokens stay visible as well: steps for them stand in front of the window's, so that both are one run of places, and the rest of the
// context is neither looked up nor read.  32 sequences of up to 131072 tokens, window 4096, 4 first tokens, 32 heads over 8, D 128: 27.2 us, 143 MB at 5.3 TB/s, bound by
// memory; 4 chunks of up to 2048 over 16384, window 1001, 17 first tokens, 32 heads: 187 us, matrix-bound as chunks without a window are, with 1.17 times the pairs that are
// seen in their blocks (0.59 PFLOP/s of those).  Passing over what lies in front of each wave's own window took 205 (registers), not looking at what lies behind it 198.
#pragma once
#include <math.h>

#include "pop_cache_attention_dev.h"

namespace pop {

namespace {

constexpr int kBuffers = 2;   // steps that a wave has in registers: the one it uses and the next
constexpr int kRound = 128;   // tokens of a round: a step of each of the four waves

// How the work is dealt.  A unit is one kv head's block of 16 columns of one sequence: a number of rounds over the tokens that the
// sequence's columns see.  All units stand in one row (sequence, block, head), and every workgroup takes the same number of rounds of
// it, wherever units begin and end: ragged batches and single long sequences of single tokens load all compute units alike.  (Chunks less so: a
// unit has the rounds of its whole sequence's columns, of which its own block may see few, under a window or where little is cached;
// rounds behind what a block sees cost nothing, those in front of it, under a window, are gone over masked; with first tokens a unit has its own.)  A piece of a unit
// is what one workgroup has of it.  Where that gains less than pieces cost, workgroups take units.
struct SequenceWork {
    int rounds;  // of a unit
    int blocks;
    Columns cols;
    SeenTokens seen;
    int row0;
};
template <bool SINKS>
__device__ __forceinline__ SequenceWork sequence_work(const AttentionArgs &a, int start, int next, int context, int share)
{
    SequenceWork w;
    w.rounds = 0, w.blocks = 0, w.row0 = start;
    if (!sequence_columns(a, start, next, context, share, &w.cols)) return w;
    w.blocks = (w.cols.n + 15) / 16;
    w.seen = seen_tokens<SINKS>(w.cols, 0, w.cols.n, a.sinks);
    int places = w.seen.hi - w.seen.begin;
    if (SINKS) {  // of no block are there more than this; each goes over its own
        const int kept = (min(a.sinks, kMostTokens) + 31) & ~31;
        places = min(places, __builtin_elementwise_add_sat(__builtin_elementwise_add_sat(w.cols.window, kept), 15 / share + 1 + 31));
    }
    w.rounds = max((places + kRound - 1) / kRound, 1);
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

// Partial results: two places for each workgroup, its first piece if the unit began in front of it and its last if the unit goes on
// behind it; then the counters of the units' pieces, by the workgroup that has the first.
template <int D>
__device__ __forceinline__ float *partial_of(const AttentionArgs &a, int place)
{
    return a.ws + (size_t)place * 16 * (D + 4);
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
template <int D, int QT, int PT, bool PAST, bool SINKS>
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
            const SequenceWork w = sequence_work<SINKS>(a, my_start, my_next, my_context, share);
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
        const SequenceWork w = sequence_work<SINKS>(a, start, next, context, share);
        const int dealt = by_units ? 1 : w.rounds, of_seq = dealt * w.blocks * n_kv;  // (of a unit, of the sequence's)
        if ((unsigned)at >= (unsigned)seq_at + (unsigned)of_seq) {
            seq_at += of_seq, ++seq;
            continue;
        }
        const int unit = (int)((unsigned)(at - seq_at) / (unsigned)dealt), block = (int)((unsigned)unit / (unsigned)n_kv), head = unit - block * n_kv;
        const int unit_at = seq_at + unit * dealt, begin = at - unit_at, stop = by_units ? w.rounds : min(w.rounds, end - unit_at);
        const Columns &cols = w.cols;
        const SeenTokens seen = seen_tokens<SINKS>(cols, block * 16, min(block * 16 + 16, cols.n), a.sinks);
        const scalar_ints table = (scalar_ints)(uintptr_t)(a.table + (size_t)seq * a.stride);
        const int col = block * 16 + n, token = col / share, qh = head * share + col % share;
        const bool live = col < cols.n;
        const int pos = live ? cols.first_pos + token : -1;  // a column that is not there sees nothing
        WaveSums<D, QT, PT> sums;
        {
            // (the places that the unit's rounds are of)
            const SeenTokens &of = SINKS ? seen : w.seen;
            const int t1 = min(seen.hi, of.begin + stop * kRound), first = of.begin + begin * kRound + wave * 32;
            const unsigned char *const cache = a.cache + (size_t)(head * (a.c.page >> 4)) * kTile;
            TileRegs<D> r[kBuffers][2];
            int limit[kBuffers][2], page[2];
            // the pages of a step's tiles; past the last step that of the last token again, of which nothing is loaded
            auto look_up = [&](int t0) {
                if (a.c.page == 16) {
#pragma unroll
                    for (int u = 0; u < 2; ++u) page[u] = table[of.template token<SINKS>(min(t0 + 16 * u, t1 - 1)) >> 4];
                } else {  // one page holds both
                    page[0] = page[1] = table[of.template token<SINKS>(min(t0, t1 - 1)) >> a.c.log_page];
                }
            };
            auto load = [&](TileRegs<D> (&to)[2], int (&lim)[2], int t0) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int t = of.template token<SINKS>(t0 + 16 * u);
                    lim[u] = (unsigned)page[u] < (unsigned)a.c.n_pages ? t1 - (t0 + 16 * u - t) : 0;
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
                    const int t = of.template token<SINKS>(t0);
                    const bool all = t + 32 <= min(limit[i][0], limit[i][1]) && t + 31 <= seen.first_pos &&
                                     (seen.last_pos - t < cols.window || (SINKS && t + 32 <= a.sinks));
                    if (t0 < t1) sums.template step<SINKS>(r[i], limit[i], !all, t, pos, cols.window, a.sinks, g, scale);
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
                const auto place = [&](int piece) { return partial_of<D>(a, piece == 0 ? 2 * wg0 + 1 : 2 * (wg0 + piece)); };
#pragma unroll 1
                for (int pass = 0; pass < D / kPass; ++pass) {
                    if (pieces <= 8) join_pieces<D, kPass, 8, 2>(a.ws, place, pieces, n_live, wave, lane, pass, s_o, s_m, s_l);
                    else join_pieces<D, kPass, 2, 8>(a.ws, place, pieces, n_live, wave, lane, pass, s_o, s_m, s_l);
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

// The q-th of all sequences' blocks of 128 columns, by sequence, the later block first: under a window that most blocks fill, all are about as long.
__device__ __forceinline__ bool nth_block(const AttentionArgs &a, int q, int share, int lane, int *seq, int *block)
{
    const int per_lane = (a.n_seq + 63) / 64;
    const auto blocks = [&](int s) {
        Columns c;
        if (s >= a.n_seq || !sequence_columns(a, a.start[s], a.start[s + 1], a.context[s], share, &c)) return 0;
        return (c.n + 127) / 128;
    };
    int n = 0;
    for (int i = 0; i < per_lane; ++i) n = __builtin_elementwise_add_sat(n, blocks(lane * per_lane + i));
    const int upto = wave_scan(n), owner = __ffsll((unsigned long long)__ballot(upto > q)) - 1;
    if (owner < 0) return false;
    int rest = q - __builtin_amdgcn_readlane(upto - n, owner), s = owner * per_lane;
    for (; s < a.n_seq; ++s) {
        const int of = blocks(s);
        if (rest < of) {
            *seq = __builtin_amdgcn_readfirstlane(s), *block = __builtin_amdgcn_readfirstlane(of - 1 - rest);
            return true;
        }
        rest -= of;
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
template <int D, bool SINKS>
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
        if (!(SINKS ? nth_block(a, rank, share, lane, &seq, &block) : nth_longest_block(a, rank, share, lane, &seq, &block))) break;
        Columns cols;
        const int row0 = a.start[seq];
        sequence_columns(a, row0, a.start[seq + 1], a.context[seq], share, &cols);
        const scalar_ints table = (scalar_ints)(uintptr_t)(a.table + (size_t)seq * a.stride);
        const SeenTokens seen = seen_tokens<SINKS>(cols, block * kBlock, min((block + 1) * kBlock, cols.n), a.sinks);
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
        // tokens in front of this one that are seen are all there: 0 if some page of theirs is none (pages that no column sees may be: steps that
        // reach into one are masked by the window; four chunks of up to 2048 over 16384, window 4096, 4 first tokens, pages of 16 that are given back, with those
        // next to what is seen counted too 890 us, so 521)
        int full = seen.hi;
        const int window0 = cols.window == kNoWindow ? 0 : max(seen.first_pos - cols.window + 1, 0);
        for (int i = (max(seen.lo, window0) >> a.c.log_page) + lane; i << a.c.log_page < seen.hi; i += 64)
            if ((unsigned)table[i] >= (unsigned)a.c.n_pages) full = 0;
        if (SINKS)
            for (int i = lane; i << a.c.log_page < min(a.sinks, seen.hi); i += 64)
                if ((unsigned)table[i] >= (unsigned)a.c.n_pages) full = 0;
        full = __any(full == 0) ? 0 : full;
        const int first = seen.begin, all_tiles = (seen.hi - seen.begin + kPromptTile - 1) / kPromptTile;
        const int parts = announced ? max(min(splits, all_tiles), 1) : 1, part = blockIdx.y;
        if (part >= parts) continue;
        const int tile0 = (int)((long long)all_tiles * part / parts), n_tiles = (int)((long long)all_tiles * (part + 1) / parts);  // [tile0, n_tiles)
        unsigned long long counted = 0;
        if (parts > 1 && threadIdx.x == 0) counted = coherent_load(counter);

        TileRegs<D> regs;
        int limit = 0;
        auto load = [&](int tile) {  // this wave's 16 tokens
            const int t = seen.template token<SINKS>(first + tile * kPromptTile + 16 * wave);
            const int page = t < seen.hi ? table[t >> a.c.log_page] : -1;
            limit = (unsigned)page < (unsigned)a.c.n_pages ? seen.hi : 0;
            load_tile<D, false>(regs, cache + (size_t)(limit ? (unsigned)page : 0u) * page_bytes + ((t & (a.c.page - 1)) >> 4) * kTile, t < limit, offsets);
        };
        auto convert = [&](int tile) {
            convert_tile<D>(s_tiles.k[tile % 2], s_tiles.v[tile % 3], regs, wave, limit - seen.template token<SINKS>(first + tile * kPromptTile + 16 * wave), n, g);
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
            const int t0 = seen.template token<SINKS>(first + tile * kPromptTile + 32 * half);
            if (!(t0 + 32 <= full && t0 + 31 <= wave_first && (wave_last - t0 < cols.window || (SINKS && t0 + 32 <= a.sinks)))) {
                int lim0 = seen.hi, lim1 = seen.hi;
                if (full == 0) {
                    if (t0 < seen.hi && (unsigned)table[t0 >> a.c.log_page] >= (unsigned)a.c.n_pages) lim0 = 0;
                    if (t0 + 16 < seen.hi && (unsigned)table[(t0 + 16) >> a.c.log_page] >= (unsigned)a.c.n_pages) lim1 = 0;
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int t = t0 + (8 * (i / 4) ^ 8 * h) + 4 * h + i % 4;
                    if (!(t < (i < 8 ? lim0 : lim1) && t <= pos && (pos - t < cols.window || (SINKS && t < a.sinks)))) s[i] = -INFINITY;
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
                const int t0 = seen.template token<SINKS>(first + tile * kPromptTile);
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

template <int D, bool SINKS>
hipError_t launch_attention_d(const AttentionArgs &a, const AttentionLaunch &l, hipStream_t s)
{
    const unsigned long long tag = launch_tag();
    if (l.blocks > 0) {
        constexpr int kBytes = (int)sizeof(PromptTiles<D>);
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(cache_prompt_kernel<D, SINKS>), hipFuncAttributeMaxDynamicSharedMemorySize, kBytes);
        if (e != hipSuccess) return e;
        cache_prompt_kernel<D, SINKS><<<dim3((unsigned)(l.blocks * a.c.n_kv), (unsigned)l.splits), 256, kBytes, s>>>(a, l.blocks, l.splits, tag);
        return hipGetLastError();
    }
    const unsigned grid = (unsigned)l.workgroups;
    if (!a.q_bf16) cache_attention_kernel<D, 3, 3, false, SINKS><<<grid, 256, 0, s>>>(a, tag);
    else if (!a.y_bf16) cache_attention_kernel<D, 1, 3, false, SINKS><<<grid, 256, 0, s>>>(a, tag);
    else if (!l.past) cache_attention_kernel<D, 1, 1, false, SINKS><<<grid, 256, 0, s>>>(a, tag);
    else cache_attention_kernel<D, 1, 1, true, SINKS><<<grid, 256, 0, s>>>(a, tag);
    return hipGetLastError();
}

template <bool SINKS>
hipError_t launch_attention_as(const AttentionArgs &a, const AttentionLaunch &l, hipStream_t s)
{
    if (a.c.d == 64) return launch_attention_d<64, SINKS>(a, l, s);
    if (a.c.d == 128) return launch_attention_d<128, SINKS>(a, l, s);
    return launch_attention_d<256, SINKS>(a, l, s);
}

}  // namespace

}  // namespace pop
