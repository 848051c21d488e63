// Attention over the 4-bit paged cache for groups of sequences that share a prefix: y = softmax(scale q k^T + mask) v, the prefix's keys and
// values read and converted once for a block of the columns of all sequences of a group.
//
// With m, l and O the maximum, the sum of weights and the weighted sum of values over a set of tokens, two sets join as
//     m = max(m1, m2),  l = 2^(m1 - m) l1 + 2^(m2 - m) l2,  O = 2^(m1 - m) O1 + 2^(m2 - m) O2,   y = O / l.
// The first kernel leaves m, l and O of runs of tokens of the prefix and of the tokens behind it, the second joins them for every column.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "pop_cache_attention_dev.h"

namespace pop {

namespace {

constexpr int kRound = 128;  // tokens of a round: a step of each of the four waves
constexpr int kWorkgroups = 512;
// What a unit costs its workgroup beside its rounds (its columns, q and table, the waves' sums), in rounds.
constexpr int kUnitCost = 4;
// A prefix shorter than this is read by each sequence for itself, also in a call that could share longer ones: units of its own and joining cost more. (Microseconds,
// shared / not: 8 sequences x 32 heads 512 tokens 13.7 / 13.6, 1024 14.9 / 15.9; 16 x 32 over 8 512 tokens 12.9 / 12.7, 1024 15.5 / 14.5; 4 groups of 4 x 32
// 512 tokens 14.4 / 14.4, 1024 18.6 / 16.7, 1500 17.1 / 18.3.)
constexpr int kLeastPrefix = 1024;

// One step of a wave: 32 tokens of one kv head against NC blocks of 16 columns, whose keys and values are converted once.
template <int D, int QT, int PT, int NC>
struct WideSums {
    bf16x8 q[NC][D / 32][QT];
    f32x4 o[NC][D / 16];
    float m[NC], l[NC], by[NC];  // (as in WaveSums, by block)

    // LIVE: blocks that have columns.
    template <int LIVE>
    __device__ __forceinline__ void step(const TileRegs<D> (&r)[2], const int (&limit)[2], bool masked, int t0, const int (&pos)[NC], int g, float scale)
    {
        f32x4 s[2][LIVE];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int x = 0; x < LIVE; ++x) s[u][x] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                const bf16x8 k = k_operand<D>(r[u], c);
#pragma unroll
                for (int t = QT - 1; t >= 0; --t)
#pragma unroll
                    for (int x = 0; x < LIVE; ++x) s[u][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[x][c][t], s[u][x], 0, 0, 0);
            }
        }
        uint32_t vs[2] = {r[0].vs, r[1].vs};
        if (masked) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int t = t0 + 16 * u + 4 * g;
#pragma unroll
                for (int x = 0; x < LIVE; ++x)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!(t + i < limit[u] && t + i <= pos[x])) s[u][x][i] = -INFINITY;
                // scale bytes of tokens that are not there become 2^-127, so that whatever stands in their place is finite
                const int left = limit[u] - t;
                vs[u] = left >= 4 ? vs[u] : left <= 0 ? 0u : vs[u] & ((1u << (8 * left)) - 1);
            }
        }
        bf16x8 w[LIVE][PT];
#pragma unroll
        for (int x = 0; x < LIVE; ++x) {
            const f32x4 &a = s[0][x], &b = s[1][x];
            float top = fmaxf(fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3])), fmaxf(fmaxf(b[0], b[1]), fmaxf(b[2], b[3])));
            if (__any(top * by[x] > m[x] + kSlack)) {  // (by > 0)
                top = fmaxf(top, __shfl_xor(top, 16, kWave));
                top = fmaxf(top, __shfl_xor(top, 32, kWave));
                const float next = fmaxf(m[x], top * by[x]), factor = __builtin_amdgcn_exp2f(m[x] - next);
                m[x] = next;
                choose_unit(by[x], m[x], top, scale);
                l[x] *= factor;
#pragma unroll
                for (int j = 0; j < D / 16; ++j) o[x][j] *= factor;
            }
            float p[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                p[i] = __builtin_amdgcn_exp2f(fmaf(i < 4 ? a[i % 4] : b[i % 4], by[x], -m[x]));
                l[x] += p[i];
            }
            split_terms<PT>(p, w[x]);
        }
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
            for (int t = PT - 1; t >= 0; --t)
#pragma unroll
                for (int x = 0; x < LIVE; ++x) {
                    o[x][2 * b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(even, w[x][t], o[x][2 * b], 0, 0, 0);
                    o[x][2 * b + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(odd, w[x][t], o[x][2 * b + 1], 0, 0, 0);
                }
        }
    }
};

// The least and the largest of a row of 16 lanes, in all of them.
template <int ROR>
__device__ __forceinline__ int turned_row(int v) { return __builtin_amdgcn_update_dpp(0, v, 0x120 + ROR, 0xf, 0xf, false); }
__device__ __forceinline__ int row_min(int v)
{
    v = min(v, turned_row<8>(v)), v = min(v, turned_row<4>(v)), v = min(v, turned_row<2>(v));
    return min(v, turned_row<1>(v));
}
__device__ __forceinline__ int row_max(int v)
{
    v = max(v, turned_row<8>(v)), v = max(v, turned_row<4>(v)), v = max(v, turned_row<2>(v));
    return max(v, turned_row<1>(v));
}

// v of lane `from` (modulo 64).
__device__ __forceinline__ int lane_value(int v, int from) { return __builtin_amdgcn_ds_bpermute(from * 4, v); }

// Sequences in packs: a group, or 64 sequences of a larger one (and what is left of it).  A wave looks at as many whole packs at a time as 64
// lanes hold, a lane for a sequence.
struct Packs {
    int group, per_group, at_once;  // sequences of a group, parts of one; sequences that a wave looks at where a group is a pack
    __device__ __forceinline__ explicit Packs(const SharedArgs &h) : group(h.group), per_group((h.group + 63) / 64), at_once(h.group >= 64 ? 64 : h.by_group.of(64) * h.group) {}
    __device__ __forceinline__ int looks(int n_seq) const { return per_group > 1 ? n_seq / group * per_group : (n_seq + at_once - 1) / at_once; }
    // The look's first sequence and how many there are.
    __device__ __forceinline__ int first(int look) const { return per_group > 1 ? look / per_group * group + look % per_group * 64 : look * at_once; }
    __device__ __forceinline__ int count(int look, int n_seq) const
    {
        return per_group > 1 ? min(64, group - look % per_group * 64) : min(at_once, n_seq - look * at_once);
    }
};

// What a lane knows of its sequence, and of its pack.  Units of a sequence: if it is its pack's first, those of the prefix (blocks of the columns of all
// its sequences); then its own (blocks of its columns over the tokens behind the prefix).
struct Sequence {
    int start, fresh, context;  // rows, new tokens (0: left out), tokens in the cache
    int fresh_upto;             // new tokens of the look's sequences up to this one
    int pack0, pack_n;          // lanes of the pack
    int prefix;                 // shared tokens that are read once: a multiple of 32, 0 for none
    int prefix_rounds, prefix_blocks, rounds, blocks;

    // Row and position of a token: of the pack's sequences one after another, which begin behind `before` tokens of the look, or of lane `owner`'s.
    __device__ __forceinline__ void column(bool of_pack, int owner, int before, int token, int lane, int *row, int *pos) const
    {
        const int pack0_of = __builtin_amdgcn_readlane(pack0, owner);
        const bool lane_outside = lane < pack0_of || lane >= pack0_of + pack_n;
        int of = owner, local = token;
        if (of_pack) {
            if (__all(fresh == 1 || lane_outside)) {  // a token each
                of = pack0_of + token, local = 0;
            } else {
                int lo = 0;  // sequences whose tokens all stand in front of this one
#pragma unroll
                for (int half = 32; half > 0; half >>= 1)
                    if (lane_value(fresh_upto, lo + half - 1) <= before + token) lo += half;
                of = lo;
                local = before + token - (lane_value(fresh_upto, max(lo - 1, 0)) & (lo > 0 ? -1 : 0));
            }
        }
        // (within the sequence's rows whatever sums that have saturated say)
        const int rows = lane_value(fresh, of), at = max(min(local, rows - 1), 0);
        *row = lane_value(start, of) + at;
        *pos = lane_value(context, of) - rows + at;
    }
    // The lane of the longest of the pack's sequences, whose row of the table the prefix is read from.
    __device__ __forceinline__ int source(int pack0, int pack_n, int lane) const
    {
        const bool member = lane >= pack0 && lane < pack0 + pack_n && fresh > 0;
        const int most = __builtin_amdgcn_readlane(wave_scan<true>(member ? context : 0), 63);
        return __ffsll((unsigned long long)__ballot(member && context == most)) - 1;
    }
};

// (sequences whose rows overlap may have more than 32 bits count: they stop there)
__device__ __forceinline__ int columns_of(int tokens, int share) { return (int)min((long long)tokens * share, 0x7fff0000ll); }
__device__ __forceinline__ int saturated(long long v) { return (int)min(v, 0x7fffffffll); }

// UNITS: both kinds, or one of them.
enum { kBoth = 0, kOfPrefix = 1, kOwn = 2 };
template <int COLUMNS, int UNITS>
__device__ __forceinline__ Sequence look_at(const SharedArgs &h, const Packs &packs, int look, int lane)
{
    const AttentionArgs &a = h.a;
    const int first = packs.first(look), count = packs.count(look, a.n_seq), share = a.n_heads / a.c.n_kv, s = first + lane;
    Sequence q;
    q.start = 0, q.fresh = 0, q.context = 0;
    int prefix = 0;
    if (lane < count) {
        const int next = a.start[s + 1];
        q.start = a.start[s], q.context = min(max(a.context[s], 0), kMostTokens);
        prefix = h.prefix[h.by_group.of(s)];
        if (q.start >= 0 && next > q.start && next <= a.n_tokens) q.fresh = next - q.start;
    }
    q.fresh_upto = wave_scan(q.fresh);
    q.pack0 = packs.per_group > 1 ? 0 : h.by_group.of(lane) * packs.group;
    q.pack_n = packs.per_group > 1 ? count : packs.group;  // (the same for all lanes)
    // the longest of the pack's sequences, whose row of the table the prefix is read from; one alone shares nothing
    const unsigned long long live = __ballot(q.fresh > 0);
    const unsigned long long members = (q.pack_n >= 64 ? ~0ull : (1ull << q.pack_n) - 1) << q.pack0;
    int longest = q.fresh > 0 ? q.context : 0;
    if (q.pack_n >= count) {  // (one pack)
        longest = __builtin_amdgcn_readlane(wave_scan<true>(longest), 63);
    } else {
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int other = lane_value(longest, lane + off);
            if (lane + off < q.pack0 + q.pack_n) longest = max(longest, other);
        }
        longest = lane_value(longest, q.pack0);
    }
    const int table = a.stride << a.c.log_page;
    prefix = min(min(prefix, longest), table) & ~31;
    q.prefix = prefix >= kLeastPrefix && __popcll(live & members) > 1 ? prefix : 0;
    const int in_front = lane_value(q.fresh_upto, max(q.pack0 - 1, 0));
    const int in_pack = lane_value(q.fresh_upto, min(q.pack0 + q.pack_n, 64) - 1) - (q.pack0 > 0 ? in_front : 0);
    const bool heads_pack = lane == q.pack0 && q.prefix > 0;
    q.prefix_rounds = heads_pack ? (q.prefix + kRound - 1) / kRound : 0;
    q.prefix_blocks = heads_pack && UNITS != kOwn ? (columns_of(in_pack, share) + COLUMNS - 1) / COLUMNS : 0;
    q.blocks = UNITS == kOfPrefix ? 0 : (columns_of(q.fresh, share) + COLUMNS - 1) / COLUMNS;
    q.rounds = q.fresh > 0 ? max((min(q.context, table) - q.prefix + kRound - 1) / kRound, 1) : 0;
    return q;
}

__device__ __forceinline__ int times(int a, int b) { return saturated((long long)a * b); }

// How the work is dealt.  A unit is one kv head's block of columns over the prefix (of a pack) or over its own tokens (of a sequence), so many rounds; with what
// it costs beside them all units make up `all`, and a unit is split into as many parts as it has of that, in workgroups, but at least one.  A part is an item; items
// of prefixes, which are long, and own ones are dealt each by themselves, in turn to all workgroups: most have one.  (Both in one row: where a group's items are a whole
// part of the workgroups, the prefixes of all groups fall to the same few.  Microseconds, in one row / each by themselves / each sequence for itself, 32 heads over 8: 16 groups of 14
// rows, D 64, 30229 tokens 893 / 186 / 534, D 128, 8000 tokens 338 / 91 / 228; 4 groups of 8, D 128, 8000 tokens 25.5 / 25.2 / 43.5, one of 64 32.7 / 29.5 / 65.)  (What had parts of
// several units a workgroup, in equal numbers of rounds: 8 sequences x 32 heads, 4000 tokens and 200 of their own, 11.6 us; 64 sequences x 8 heads, 700 of their own, 13.6.)  Parts of units that have several have a place for their results each; there
// are no more of those than workgroups.
// A unit has no more parts than kPartsOfRoot roots of its rounds: each costs its columns' joining about a thirtieth of a microsecond. (3, 5, 8: 2 kv heads x 32 columns
// over 32768 tokens 19.1, 18.9, 20.4 us, 8 chunks of 5 over 8000 31.4, 31.2, 34.3.)
constexpr float kPartsOfRoot = 4.0f;
struct Dealing {
    int all;
    float per_round;  // parts
    __device__ __forceinline__ explicit Dealing(int all_) : all(max(all_, 1)), per_round((float)gridDim.x / (float)max(all_, 1)) {}
    __device__ __forceinline__ int parts(int rounds) const
    {
        // the whole number in rounds gridDim.x / all, so that all units' together are no more than gridDim.x (sums that have saturated: one each)
        const long long share = (long long)rounds * gridDim.x;
        int n = all == 0x7fffffff ? 0 : (int)((float)rounds * per_round);
        if ((long long)(n + 1) * all <= share) ++n;
        if ((long long)n * all > share) --n;
        n = min(n, (int)(kPartsOfRoot * __builtin_amdgcn_sqrtf((float)rounds)));
        return min(max(n, 1), max(rounds, 1));
    }
};

// A workgroup's items of a row of them: one of every gridDim.x, in each run of those 40 / 512 of the workgroups further on, so that items which are longer than others at regular
// distances (the first row of every group, every eighth prefix) do not all fall to the same workgroups; 40 of them are five on every XCD, which so keeps its kv heads.  (Microseconds,
// without that / with it / each sequence for itself, D 128: 64 groups of 8 rows, 32 heads over 8, 1024 tokens, 8000 of the first rows' own 548 / 190 / 207 (37 of 512: 234); 64 groups of 4 x
// 16 heads, 1024 tokens, of every eighth group 8192, 169 / 122 / 188; 64 rows x 32 heads, 2000 tokens, up to 700 of their own 44.5 / 49.1 / 86.)
struct Turns {
    unsigned slot, row, items;  // the place in the run, the run's first item, items of the run
    __device__ __forceinline__ explicit Turns(unsigned first) : slot(first), row(0), items(gridDim.x) {}
    __device__ __forceinline__ unsigned item() const { return row + slot; }
    __device__ __forceinline__ void next()
    {
        row += items;
        if (items == gridDim.x) slot += gridDim.x * 40u >> 9, slot -= slot >= gridDim.x ? gridDim.x : 0u;
        items = gridDim.x;
    }
};

// Item `at` of units of so many rounds: its unit, and which part of it, rounds [begin, stop).
struct PartOf {
    int unit, part, begin, stop;
};
__device__ __forceinline__ PartOf part_of(int at, int rounds, int parts)
{
    PartOf p = {at, 0, 0, rounds};
    if (parts > 1) {
        p.unit = (int)((unsigned)at / (unsigned)parts), p.part = at - p.unit * parts;
        const int each = (int)((unsigned)rounds / (unsigned)parts), more = rounds - each * parts;
        p.begin = p.part * each + min(p.part, more), p.stop = p.begin + each + (p.part < more);
    }
    return p;
}

// The workspace: places for results of parts, a row for each of a unit's columns; and results of every (token, head) over the prefix and over its own
// tokens.  A row is O, m and l (D + 2 floats) and two more; in the latter's last four stand
//     m, l, kWhole, 0         of a unit that is one part,
//     first, n, kPieces, c    where it is n: row c of the n places from `first` on (integers),
//     -, -, kDone, -          of own tokens without a prefix in one part: y is there.
// The last of the four, of own tokens, has its sign set where there is no prefix.
enum { kDone = 0, kWhole = 1, kPieces = 2 };
template <int D>
__device__ __forceinline__ float *piece_of(float *pieces, int columns, int place)
{
    return pieces + (size_t)place * columns * (D + 4);
}
template <int D>
__device__ __forceinline__ float *state_of(const SharedArgs &h, int own, size_t row)
{
    return h.states + ((size_t)own * h.a.n_tokens * h.a.n_heads + row) * (D + 4);
}

// Workgroup: 4 waves; in a round of 128 tokens each has 32.
//
// Bound by its chain of latencies: 8 sequences x 32 heads, D 128, a prefix of 4000 tokens and up to 200 of their own, 11.1 us (21 MB, which memory gives in
// 3.3): the launch 0.5, lengths and dealing 1.7, the item and its columns 1.0, table, codes and q 1.2, up to six rounds 4, the waves' sums 1.1. Codes are asked
// for ahead of all that the columns need (12.2 behind it); three workgroups to a compute unit instead of two 11.1.
template <int D, int QT, int PT, int NC, int UNITS>
__global__ __launch_bounds__(256, D == 256 || (D == 128 && NC == 2 && QT == 3) ? 1 : 2) void shared_attention_kernel(SharedArgs h)
{
    constexpr int kTile = cache_tile_bytes(D), kColumns = 16 * NC;
    constexpr int kPass = D > 128 ? 128 : D;
    __shared__ float s_o[4][16][kPass + 4];
    __shared__ float s_m[4][16], s_l[4][16];
    __shared__ int s_row[kColumns];
    const AttentionArgs &a = h.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
    const int share = a.n_heads / a.c.n_kv, n_kv = a.c.n_kv;
    const float scale = a.scale != 0.0f ? fabsf(a.scale) * kLog2e : 1.0f;
    const TileOffsets<D> offsets(n, g);
    const Packs packs(h);
    const int looks = packs.looks(a.n_seq);

    Sequence own;
    int all = 0;
    for (int look = 0; look < looks; ++look) {
        own = look_at<kColumns, UNITS>(h, packs, look, lane);
        const int cost = __builtin_elementwise_add_sat(times(times(own.prefix_rounds + kUnitCost, own.prefix_blocks), n_kv),
                                                       times(times(own.rounds + kUnitCost, own.blocks), n_kv));
        all = __builtin_elementwise_add_sat(all, __builtin_amdgcn_readlane(wave_scan(cost), 63));
    }
    const Dealing dealing(all);
    int upto1 = 0, upto2 = 0, places_upto = 0;  // items (of prefixes, own) and places of the look's sequences up to the lane's
    int look = 0, before1 = 0, before2 = 0, places_before = 0;  // the look that `own` is of, and items and places in front of it
    int parts1 = 1, parts2 = 1;  // parts of a unit of the prefix and of an own one
    const auto deal = [&]() {
        parts1 = dealing.parts(own.prefix_rounds), parts2 = dealing.parts(own.rounds);
        const int items1 = times(times(own.prefix_blocks, n_kv), parts1);
        const int items2 = times(times(own.blocks, n_kv), parts2);
        upto1 = wave_scan(items1), upto2 = wave_scan(items2);
        places_upto = wave_scan((parts1 > 1 ? items1 : 0) + (parts2 > 1 ? items2 : 0));
    };
    if (looks > 1) own = look_at<kColumns, UNITS>(h, packs, 0, lane);
    deal();
    const size_t page_bytes = cache_page_bytes(a.c);

    // the workgroup's next items.  Own ones go on where those of prefixes end, and there again after the last workgroup: who has one more of a prefix has two fewer own ones
    // (4 groups of 4 x 32 heads, 1500 tokens: with one fewer 20.9, so 17.1).  Of several looks that place is not known yet: they begin with the last workgroup.
    const unsigned longer = (unsigned)__builtin_amdgcn_readlane(upto1, 63) % gridDim.x, others = gridDim.x - longer;
    Turns of_prefixes(blockIdx.x), of_own(gridDim.x - 1 - blockIdx.x);
    if (looks == 1) {
        if (blockIdx.x < longer) of_own = Turns(others + blockIdx.x), of_own.row = others;
        else of_own = Turns(blockIdx.x - longer), of_own.items = others;
    }
    for (;;) {
        const int of_look1 = __builtin_amdgcn_readlane(upto1, 63), of_look2 = __builtin_amdgcn_readlane(upto2, 63);
        const bool shared = of_prefixes.item() < (unsigned)before1 + (unsigned)of_look1;
        if (!shared && of_own.item() >= (unsigned)before2 + (unsigned)of_look2) {
            if (++look >= looks) break;
            before1 += of_look1, before2 += of_look2, places_before += __builtin_amdgcn_readlane(places_upto, 63);
            own = look_at<kColumns, UNITS>(h, packs, look, lane);
            deal();
            continue;
        }
        const int of_item = (int)(shared ? of_prefixes.item() - (unsigned)before1 : of_own.item() - (unsigned)before2), upto = shared ? upto1 : upto2;
        const int owner = __ffsll((unsigned long long)__ballot(upto > of_item)) - 1;
        const int prefix = __builtin_amdgcn_readlane(own.prefix, owner);
        const int rounds = __builtin_amdgcn_readlane(shared ? own.prefix_rounds : own.rounds, owner), parts = __builtin_amdgcn_readlane(shared ? parts1 : parts2, owner);
        const auto in_front = [&](int v) { return owner > 0 ? __builtin_amdgcn_readlane(v, owner - 1) : 0; };  // (of sums up to the lane's sequence)
        const int at = of_item - in_front(upto);
        int place0 = places_before + in_front(places_upto);
        // (a sequence's places of the prefix come first)
        if (!shared && __builtin_amdgcn_readlane(parts1, owner) > 1) place0 += __builtin_amdgcn_readlane(upto1, owner) - in_front(upto1);
        if (shared) of_prefixes.next();
        else of_own.next();
        const PartOf of = part_of(at, rounds, parts);
        const int unit = of.unit, part = of.part, begin = of.begin, stop = of.stop;
        const int block = h.by_kv.of(unit), head = unit - block * n_kv;
        place0 += unit * parts;  // (of parts that have places)

        // tokens, and the row of the table that names their pages: for the prefix that of the longest sequence
        const int pack0 = __builtin_amdgcn_readlane(own.pack0, owner), pack_n = __builtin_amdgcn_readlane(own.pack_n, owner);
        const int context = __builtin_amdgcn_readlane(own.context, owner);
        int source = owner, lo = prefix, hi = max(min(context, a.stride << a.c.log_page), prefix);
        if (shared) {
            source = own.source(pack0, pack_n, lane);
            lo = 0, hi = prefix;
        }
        const int seq = packs.first(look) + source;
        const scalar_ints table = (scalar_ints)(uintptr_t)(a.table + (size_t)seq * a.stride);
        const int first = lo + begin * kRound + wave * 32;
        int t1 = min(hi, lo + stop * kRound);

        WideSums<D, QT, PT, NC> sums;
        const unsigned char *const cache = a.cache + (size_t)(head * (a.c.page >> 4)) * kTile;
        TileRegs<D> r[2][2];
        int limit[2][2], page[2];
        // the pages of a step's tiles; past the last step that of the last token again, of which nothing is loaded
        const auto look_up = [&](int t0) {
            if (a.c.page == 16) {
#pragma unroll
                for (int u = 0; u < 2; ++u) page[u] = table[min(t0 + 16 * u, t1 - 1) >> 4];
            } else {  // one page holds both
                page[0] = page[1] = table[min(t0, t1 - 1) >> a.c.log_page];
            }
        };
        const auto load = [&](TileRegs<D> (&to)[2], int (&lim)[2], int t0) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int t = t0 + 16 * u;
                lim[u] = (unsigned)page[u] < (unsigned)a.c.n_pages ? t1 : 0;
                const unsigned char *tile = cache + (size_t)(lim[u] ? (unsigned)page[u] : 0u) * page_bytes + ((t & (a.c.page - 1)) >> 4) * kTile;
                load_tile<D, false>(to[u], tile, t < lim[u], offsets);
            }
        };
        if (first < t1) look_up(first);  // (asked for ahead of all that the columns need)
        else page[0] = page[1] = -1;

        // columns: of the pack's sequences one after another, or of this one
        const int before = shared ? (pack0 > 0 ? __builtin_amdgcn_readlane(own.fresh_upto, pack0 - 1) : 0) : 0;
        const int tokens = shared ? __builtin_amdgcn_readlane(own.fresh_upto, pack0 + pack_n - 1) - before : __builtin_amdgcn_readlane(own.fresh, owner);
        const int n_columns = columns_of(tokens, share), n_live = min(kColumns, n_columns - block * kColumns);
        int row[NC], pos[NC], qh[NC];
        int lowest = kMostTokens, highest = -1;  // of the live columns' positions
#pragma unroll
        for (int x = 0; x < NC; ++x) {
            const int col = block * kColumns + 16 * x + n, there = min(col, n_columns - 1), token = h.by_share.of(there);
            qh[x] = head * share + there - token * share;
            own.column(shared, owner, before, token, lane, &row[x], &pos[x]);
            if (col < n_columns) lowest = min(lowest, pos[x]), highest = max(highest, pos[x]);
            else pos[x] = -1, row[x] = -1;  // a column that is not there sees nothing
            if (wave == 0 && g == 0) s_row[16 * x + n] = row[x] * a.n_heads + qh[x];
        }
        lowest = __builtin_amdgcn_readfirstlane(row_min(lowest)), highest = __builtin_amdgcn_readfirstlane(row_max(highest));
        const int tiles = (n_live + 15) / 16;
        load(r[0], limit[0], first);
        t1 = min(t1, highest + 1);  // (behind that nothing is seen)
        {
            if (first < t1) look_up(first + kRound);
            const uint32_t sign = a.scale < 0.0f ? (QT == 1 ? 0x80008000u : 0x80000000u) : 0u, keep = a.scale != 0.0f ? ~0u : 0u;
#pragma unroll
            for (int x = 0; x < NC; ++x) {
                constexpr int kQ = QT == 1 ? D / 32 : D / 16;
                const size_t q_at = ((size_t)max(row[x], 0) * a.n_heads + qh[x]) * D + g * (D / 4);
                const u32x4 *q_from = QT == 1 ? reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(a.q) + q_at)
                                              : reinterpret_cast<const u32x4 *>(static_cast<const float *>(a.q) + q_at);
                u32x4 q[kQ];
#pragma unroll
                for (int i = 0; i < kQ; ++i) {
                    q[i] = u32x4{0, 0, 0, 0};
                    if (row[x] >= 0) q[i] = q_from[i];
                    q[i] = (q[i] ^ sign) & keep;
                }
#pragma unroll
                for (int s = 0; s < D / 32; ++s) {
                    if constexpr (QT == 1) {
                        sums.q[x][s][0] = __builtin_bit_cast(bf16x8, q[s]);
                    } else {
                        float v[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(q[2 * s + i / 4][i % 4]);
                        split_terms<QT>(v, sums.q[x][s]);
                    }
                }
#pragma unroll
                for (int j = 0; j < D / 16; ++j) sums.o[x][j] = f32x4{0, 0, 0, 0};
                sums.m[x] = kLowest, sums.l[x] = 0.0f, sums.by[x] = scale;
            }
            const auto all_steps = [&](auto live) {
                for (int t0 = first; t0 < t1;) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        load(r[1 - i], limit[1 - i], t0 + kRound);
                        look_up(t0 + 2 * kRound);
                        const bool whole = t0 + 32 <= min(limit[i][0], limit[i][1]) && t0 + 31 <= lowest;
                        if (t0 < t1) sums.template step<decltype(live)::value>(r[i], limit[i], !whole, t0, pos, g, scale);
                        t0 += kRound;
                    }
                }
            };
            if (NC > 1 && tiles == 1) all_steps(std::integral_constant<int, 1>());
            else all_steps(std::integral_constant<int, NC>());
        }

        const bool whole = parts == 1;
        // what the four waves left in LDS of 16 columns, each relative to its own maximum: a piece, or all there is of the unit's tokens
        const auto merge = [&](int x, int live, int pass) {
            for (int e = threadIdx.x; e < live * (kPass / 2); e += 256) {
                const int c = e / (kPass / 2), ch = e % (kPass / 2) * 2;
                float most = kLowest, sum = 0.0f, u = 0.0f, v = 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) most = fmaxf(most, s_m[i][c]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float f = __builtin_amdgcn_exp2f(s_m[i][c] - most);
                    sum += f * s_l[i][c], u += f * s_o[i][c][ch], v += f * s_o[i][c][ch + 1];
                }
                const size_t of = s_row[16 * x + c];
                float *const state = state_of<D>(h, !shared, of), *const to = whole ? state : piece_of<D>(h.own_pieces, kColumns, place0 + part) + (16 * x + c) * (D + 4);
                const bool done = whole && !shared && prefix == 0;
                if (done) {
                    const float by = sum > 0.0f ? 1.0f / sum : 0.0f;
                    store_y2(a, of * D + pass * kPass + ch, u * by, v * by);
                } else {
                    *reinterpret_cast<float2 *>(to + pass * kPass + ch) = {u, v};
                }
                if (ch == 0 && pass == 0) {
                    if (!whole) *reinterpret_cast<float2 *>(to + D) = {most, sum};
                    if (whole) *reinterpret_cast<float4 *>(state + D) = {most, sum, __int_as_float(done ? kDone : kWhole), 0.0f};
                    else if (part == 0) *reinterpret_cast<int4 *>(state + D) = {place0, parts, kPieces, (16 * x + c) | (!shared && prefix == 0 ? (int)0x80000000 : 0)};
                }
            }
        };
#pragma unroll
        for (int x = 0; x < NC; ++x) {
            if (x >= tiles) break;
            sums.l[x] += __shfl_xor(sums.l[x], 16, kWave);
            sums.l[x] += __shfl_xor(sums.l[x], 32, kWave);
            if (g == 0) s_m[wave][n] = by_scale(sums.m[x], sums.by[x], scale), s_l[wave][n] = sums.l[x];
#pragma unroll
            for (int pass = 0; pass < D / kPass; ++pass) {
                // a lane has channels [g D/4, (g + 1) D/4) of column n, D/16 at a time; a pass takes those of some of the groups
                constexpr int kPer = kPass / (D / 4);
                if (g / kPer == pass) {
                    float *to = &s_o[wave][n][(g % kPer) * (D / 4)];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int j = 0; j < D / 16; j += 4)
                            *reinterpret_cast<float4 *>(to + i * (D / 16) + j) = {sums.o[x][j][i], sums.o[x][j + 1][i], sums.o[x][j + 2][i], sums.o[x][j + 3][i]};
                }
                __syncthreads();
                merge(x, min(16, n_live - 16 * x), pass);
                __syncthreads();
            }
        }
    }
}

// The prefix where a pack has many columns: matrix-bound, in blocks of 128 columns (as cache_prompt_kernel).  Workgroup: 4 waves, 32 columns each; 64
// tokens at a time are converted to bf16 in LDS, a tile of the cache by each wave, while the tokens before them are used. A
// workgroup has two such sets of waves, each with half of the part's tiles, and joins their sums in LDS: half as many results in memory as with a workgroup for each
// (64 sequences of 32768 tokens, 256 columns over 8 kv heads: 76.9 -> 71.4 us in all three launches). Products 0.87 PFLOP/s in the loop (39.5 of its 52 us); the
// sequences' lengths, columns and first tiles take 6.4 in front of it, the results behind it 5 (17 MB at 4.2 TB/s; halves that write half of the channels each: the same).
// Registers decide here: a wave that sees nothing of a part has a loop of its own, and what can be computed of the lane's number ahead of the loop is kept from being
// so (76 registers in scratch memory and 104 us with both as the compiler had them).
constexpr int kBlockColumns = 128;
constexpr int kHalves = 2;
template <int D>
__global__ __launch_bounds__(256 * kHalves, kHalves) void shared_blocks_kernel(SharedArgs h)
{
    constexpr int kTile = cache_tile_bytes(D), kCols = 32;
    extern __shared__ __align__(16) unsigned char s_raw[];
    const AttentionArgs &a = h.a;
    const int lane_of_block = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) & 3, half = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8), n = lane_of_block & 15, g = lane_of_block >> 4;
    const int lc = lane_of_block & 31, half_of = lane_of_block >> 5, token_row = lc ^ (lc & 4) << 1;  // (token_row: the token of S^T's row lc)
    PromptTiles<D> &s_tiles = reinterpret_cast<PromptTiles<D> *>(s_raw)[half];
    const int share = a.n_heads / a.c.n_kv, n_kv = a.c.n_kv;
    const float scale = a.scale != 0.0f ? fabsf(a.scale) * kLog2e : 1.0f;
    const TileOffsets<D> offsets(n, g);
    const size_t page_bytes = cache_page_bytes(a.c);
    const Packs packs(h);
    const int looks = packs.looks(a.n_seq);

    const auto tiles_of = [&](int prefix) { return (prefix + kPromptTile - 1) / kPromptTile; };
    const auto look_up = [&](int look, int lane) { return look_at<kBlockColumns, kOfPrefix>(h, packs, look, lane); };
    Dealing dealing(0);
    bool dealt = false;
    // (what the lanes know of the sequences is looked up anew for every item: it does not fit next to a block's registers, and nor does what
    // could be computed of the lane's number ahead of the loop)
    for (Turns turns(blockIdx.x);; turns.next()) {
        const unsigned item = turns.item();
        int lane = lane_of_block;
        asm volatile("" : "+v"(lane));
        int look = 0, items_before = 0, place0 = 0;  // the look that `own` is of, and items and places in front of it
        Sequence own = look_up(0, lane);
        if (!dealt) {
            int all = 0;
            for (int i = 0; i < looks; ++i) {
                const Sequence q = i == 0 ? own : look_up(i, lane);
                all = __builtin_elementwise_add_sat(all, __builtin_amdgcn_readlane(wave_scan(times(times(tiles_of(q.prefix), q.prefix_blocks), n_kv)), 63));
            }
            dealing = Dealing(all), dealt = true;
        }
        int items, upto, places_upto;
        const auto deal = [&]() {
            const int parts = dealing.parts(tiles_of(own.prefix));
            items = times(times(own.prefix_blocks, n_kv), parts);
            upto = wave_scan(items), places_upto = wave_scan(parts > 1 ? items : 0);
        };
        deal();
        while (item >= (unsigned)items_before + (unsigned)__builtin_amdgcn_readlane(upto, 63)) {
            if (++look >= looks) return;
            items_before += __builtin_amdgcn_readlane(upto, 63), place0 += __builtin_amdgcn_readlane(places_upto, 63);
            own = look_up(look, lane);
            deal();
        }
        const int of_item = (int)(item - (unsigned)items_before), owner = __ffsll((unsigned long long)__ballot(upto > of_item)) - 1;
        const int prefix = __builtin_amdgcn_readlane(own.prefix, owner), tiles = tiles_of(prefix), parts = dealing.parts(tiles);
        const PartOf of = part_of(of_item - (owner > 0 ? __builtin_amdgcn_readlane(upto, owner - 1) : 0), tiles, parts);
        // (the first half of the waves has the first half of the tiles)
        const int part = of.part, most = (of.stop - of.begin + kHalves - 1) / kHalves, tile0 = of.begin + half * most, stop = min(tile0 + most, of.stop), block = h.by_kv.of(of.unit), head = of.unit - block * n_kv;
        place0 += (owner > 0 ? __builtin_amdgcn_readlane(places_upto, owner - 1) : 0) + of.unit * parts;

        const int pack0 = __builtin_amdgcn_readlane(own.pack0, owner), pack_n = __builtin_amdgcn_readlane(own.pack_n, owner);
        const int before = pack0 > 0 ? __builtin_amdgcn_readlane(own.fresh_upto, pack0 - 1) : 0;
        const int n_columns = columns_of(__builtin_amdgcn_readlane(own.fresh_upto, pack0 + pack_n - 1) - before, share);
        const int seq = packs.first(look) + own.source(pack0, pack_n, lane);
        const scalar_ints table = (scalar_ints)(uintptr_t)(a.table + (size_t)seq * a.stride);
        const unsigned char *const cache = a.cache + (size_t)(head * (a.c.page >> 4)) * kTile;
        const int col = block * kBlockColumns + wave * kCols + lc;
        const bool live = col < n_columns;
        int row, pos;
        const int there = min(col, n_columns - 1), token = h.by_share.of(there);
        own.column(true, owner, before, token, lane, &row, &pos);
        if (!live) pos = -1;  // a column that is not there sees nothing
        // positions of the wave's columns (of columns that are not there: none)
        int lowest = live ? pos : kMostTokens, highest = pos;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1)
            lowest = min(lowest, __shfl_xor(lowest, off, kWave)), highest = max(highest, __shfl_xor(highest, off, kWave));
        lowest = __builtin_amdgcn_readfirstlane(lowest), highest = __builtin_amdgcn_readfirstlane(highest);
        const int y_row = row * a.n_heads + head * share + there - token * share;
        bf16x8 q[D / 16];
        const uint32_t sign = a.scale < 0.0f ? 0x80008000u : 0u, keep = a.scale != 0.0f ? ~0u : 0u;
        const u32x4 *from = reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(a.q) + (size_t)y_row * D);
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            u32x4 x = {0, 0, 0, 0};
            if (live) x = from[2 * s + half_of];
            q[s] = __builtin_bit_cast(bf16x8, (x ^ sign) & keep);
        }
        f32x16 o[D / 32], s0, s1;
        float m = kLowest, l = 0.0f;
        float by = scale;  // (see choose_unit)
#pragma unroll
        for (int j = 0; j < D / 32; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[j][i] = 0.0f;
        const int lo = tile0 * kPromptTile, hi = min(prefix, stop * kPromptTile);
        // tokens in front of this one are all there: 0 if some page is none
        int full = hi;
        for (int i = (lo >> a.c.log_page) + lane; i << a.c.log_page < hi; i += 64)
            if ((unsigned)table[i] >= (unsigned)a.c.n_pages) full = 0;
        full = __any(full == 0) ? 0 : full;

        TileRegs<D> regs;
        int limit = 0;
        auto load = [&](int tile) {  // this wave's 16 tokens
            const int t = tile * kPromptTile + 16 * wave;
            const int page = t < hi ? table[t >> a.c.log_page] : -1;
            limit = (unsigned)page < (unsigned)a.c.n_pages ? hi : 0;
            load_tile<D, false>(regs, cache + (size_t)(limit ? (unsigned)page : 0u) * page_bytes + ((t & (a.c.page - 1)) >> 4) * kTile, t < limit, offsets);
        };
        auto convert = [&](int tile) {
            convert_tile<D>(s_tiles.k[tile % 2], s_tiles.v[tile % 3], regs, wave, limit - (tile * kPromptTile + 16 * wave), n, g);
        };
        auto scores = [&](f32x16 &s, int tile, int half) {
            const uint32_t *const k_from = s_tiles.k[tile % 2];
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = 0.0f;
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                const bf16x8 x = *reinterpret_cast<const bf16x8 *>(&k_from[((2 * k + half_of) * kPromptTile + 32 * half + token_row) * 4]);
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, q[k], s, 0, 0, 0);
            }
        };
        auto weights = [&](f32x16 &s, bf16x8 (&p)[2], int tile, int half) {
            const int t0 = tile * kPromptTile + 32 * half;
            if (!(t0 + 32 <= full && t0 + 31 <= lowest)) {
                int lim0 = hi, lim1 = hi;
                if (full == 0) {
                    if (t0 < hi && (unsigned)table[t0 >> a.c.log_page] >= (unsigned)a.c.n_pages) lim0 = 0;
                    if (t0 + 16 < hi && (unsigned)table[(t0 + 16) >> a.c.log_page] >= (unsigned)a.c.n_pages) lim1 = 0;
                }
                int of_half = half_of;  // (opaque: else the sixteen places within a step are computed ahead of the loop, and stay in registers)
                asm volatile("" : "+v"(of_half));
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int t = t0 + (8 * (i / 4) ^ 8 * of_half) + 4 * of_half + i % 4;
                    if (!(t < (i < 8 ? lim0 : lim1) && t <= pos)) s[i] = -INFINITY;
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
            const uint32_t *const v_from = s_tiles.v[tile % 3];
#pragma unroll
            for (int j = 0; j < D / 32; ++j)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const bf16x8 x = *reinterpret_cast<const bf16x8 *>(&v_from[((2 * (2 * half + k) + half_of) * D + 32 * j + lc) * 4]);
                    o[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, p[k], o[j], 0, 0, 0);
                }
        };
        bf16x8 p[2];
        if (tile0 < stop) {
            load(tile0);
            convert(tile0);
            if (tile0 + 1 < stop) load(tile0 + 1);
        }
        __syncthreads();
        // (a wave whose columns see none of the piece only converts: with that as a branch within the loop registers do not suffice)
        if (highest < lo || tile0 >= stop) {
            for (int tile = tile0; tile < stop; ++tile) {
                if (tile + 1 < stop) {
                    convert(tile + 1);
                    if (tile + 2 < stop) load(tile + 2);
                }
                __syncthreads();
            }
        } else {
            scores(s0, tile0, 0);
            for (int tile = tile0; tile < stop; ++tile) {
                const bool more = tile + 1 < stop;
                scores(s1, tile, 1);
                weights(s0, p, tile, 0);
                values(p, tile, 0);
                if (more) {
                    convert(tile + 1);
                    if (tile + 2 < stop) load(tile + 2);
                }
                __syncthreads();
                if (more) scores(s0, tile + 1, 0);
                weights(s1, p, tile, 1);
                values(p, tile, 1);
            }
        }
        for (int i = max(stop - tile0, 0); i < most; ++i) __syncthreads();  // (a half with a tile less)
        l += __shfl_xor(l, 32, kWave);
        m = by_scale(m, by, scale);
        {
            // the halves' sums, joined by the first one
            __syncthreads();
            f32x4 *const s_o = reinterpret_cast<f32x4 *>(s_raw) + wave * (D / 8 + 1) * 64 + lc + 32 * half_of;
            if (half == 1) {
#pragma unroll
                for (int j = 0; j < D / 32; ++j)
#pragma unroll
                    for (int b = 0; b < 4; ++b) s_o[(4 * j + b) * 64] = f32x4{o[j][4 * b], o[j][4 * b + 1], o[j][4 * b + 2], o[j][4 * b + 3]};
                s_o[D / 8 * 64] = f32x4{m, l, 0.0f, 0.0f};
            }
            __syncthreads();
            if (half == 0) {
                const f32x4 ml = s_o[D / 8 * 64];
                const float top = fmaxf(m, ml[0]), f = __builtin_amdgcn_exp2f(m - top), e = __builtin_amdgcn_exp2f(ml[0] - top);
                m = top, l = f * l + e * ml[1];
#pragma unroll
                for (int j = 0; j < D / 32; ++j)
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        const f32x4 x = s_o[(4 * j + b) * 64];
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[j][4 * b + i] = f * o[j][4 * b + i] + e * x[i];
                    }
            }
        }
        const bool whole = parts == 1;
        if (live && half == 0) {
            float *const state = state_of<D>(h, 0, y_row);
            float *const to = whole ? state : piece_of<D>(h.prefix_pieces, kBlockColumns, place0 + part) + (wave * kCols + lc) * (D + 4);
            // channels r D/16 .. of the lane's eight r: the places c 16 + r of all c
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    constexpr int C = D / 16;
#pragma unroll
                    for (int e = 0; e < C; e += 4)
                        *reinterpret_cast<f32x4 *>(to + (8 * b + 4 * half_of + i) * C + e) =
                            f32x4{o[e / 2][4 * b + i], o[e / 2][8 + 4 * b + i], o[e / 2 + 1][4 * b + i], o[e / 2 + 1][8 + 4 * b + i]};
                }
            if (half_of == 0) {
                if (whole) *reinterpret_cast<float4 *>(state + D) = {m, l, __int_as_float(kWhole), 0.0f};
                else *reinterpret_cast<float2 *>(to + D) = {m, l};
                if (!whole && part == 0) *reinterpret_cast<int4 *>(state + D) = {place0, parts, kPieces, wave * kCols + lc};
            }
        }
        __syncthreads();  // (the next unit's tiles take these buffers)
    }
}

// y of the columns whose results stand in the workspace.  Workgroup: one (token, head); a group of D/4 lanes for a row of results, four channels to
// a lane, rows in the order of the tokens. A launch of its own costs 3 to 4 us (8 x 32 rows; 2048 rows of 17 parts 7.8); the first kernel's workgroups, counting
// themselves and joining what they are the last of, took 10 us longer (25.4 -> 14.5 in all).
template <int D>
__global__ __launch_bounds__(256) void shared_join_kernel(SharedArgs h)
{
    constexpr int kLanes = D / 4, kGroups = 256 / kLanes, kTogether = 4;
    __shared__ f32x4 s_o[kGroups][kLanes];
    __shared__ float s_m[kGroups], s_l[kGroups];
    const AttentionArgs &a = h.a;
    const int group = threadIdx.x / kLanes, ch = threadIdx.x % kLanes * 4;
    const size_t rows = (size_t)a.n_tokens * a.n_heads;
    for (size_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const float *const of_own = state_of<D>(h, 1, row), *const of_prefix = state_of<D>(h, 0, row);
        int4 own = *reinterpret_cast<const int4 *>(of_own + D), prefix = *reinterpret_cast<const int4 *>(of_prefix + D);
        // is it some sequence's row? (of one that is not, the workspace says nothing)
        const int token = (int)(row / a.n_heads);
        bool found = false;
        for (int i = threadIdx.x; i < a.n_seq; i += 256) {
            const int start = a.start[i], next = a.start[i + 1];
            found |= start >= 0 && start <= token && token < next && next <= a.n_tokens;
        }
        if (!__syncthreads_or(found) || own.z == kDone) continue;
        // (sequences whose rows overlap may have left out some: what stands there then names no places beyond those that there are)
        const auto within = [](int4 &e, int places, int columns) {
            if (e.z == kPieces && ((unsigned)e.x > (unsigned)places || (unsigned)e.y > (unsigned)(places - e.x) || (e.w & 255) >= columns)) e.y = 0;
        };
        within(own, h.own_places, h.own_columns), within(prefix, h.prefix_places, h.prefix_columns);
        // (a sequence with a prefix leaves kWhole or kPieces of its own tokens, and so does one whose own unit several workgroups have)
        const bool shares = own.w >= 0;
        const int n1 = !shares ? 0 : prefix.z == kPieces ? prefix.y : 1, n = n1 + (own.z == kPieces ? own.y : 1);
        f32x4 o = {0, 0, 0, 0};
        float m = kLowest, l = 0.0f;
        for (int i0 = group; i0 < n; i0 += kGroups * kTogether) {
            f32x4 v[kTogether];
            float2 ml[kTogether];
#pragma unroll
            for (int k = 0; k < kTogether; ++k) {
                const int i = i0 + kGroups * k;
                v[k] = f32x4{0, 0, 0, 0}, ml[k] = {kLowest, 0.0f};
                if (i < n) {
                    const int4 e = i < n1 ? prefix : own;
                    const float *p = i < n1 ? of_prefix : of_own;
                    if (e.z == kPieces)
                        p = (i < n1 ? piece_of<D>(h.prefix_pieces, h.prefix_columns, e.x + i) : piece_of<D>(h.own_pieces, h.own_columns, e.x + i - n1)) +
                            (e.w & 255) * (D + 4);
                    ml[k] = *reinterpret_cast<const float2 *>(p + D);
                    v[k] = *reinterpret_cast<const f32x4 *>(p + ch);
                }
            }
#pragma unroll
            for (int k = 0; k < kTogether; ++k) {
                const float top = fmaxf(m, ml[k].x), f = __builtin_amdgcn_exp2f(m - top), e = __builtin_amdgcn_exp2f(ml[k].x - top);
                m = top, l = f * l + e * ml[k].y, o = f * o + e * v[k];
            }
        }
        s_o[group][ch / 4] = o;
        if (ch == 0) s_m[group] = m, s_l[group] = l;
        __syncthreads();
        if (threadIdx.x < D / 2) {
            const int c = threadIdx.x * 2;
            float most = kLowest, sum = 0.0f, x = 0.0f, y = 0.0f;
#pragma unroll
            for (int i = 0; i < kGroups; ++i) most = fmaxf(most, s_m[i]);
#pragma unroll
            for (int i = 0; i < kGroups; ++i) {
                const float f = __builtin_amdgcn_exp2f(s_m[i] - most);
                sum += f * s_l[i], x += f * s_o[i][c / 4][c % 4], y += f * s_o[i][c / 4][c % 4 + 1];
            }
            const float by = sum > 0.0f ? 1.0f / sum : 0.0f;
            store_y2(a, row * D + c, x * by, y * by);
        }
        __syncthreads();
    }
}

// How a call is launched: all units by the first kernel, or prefixes by the one for blocks of 128 columns, where a pack's columns (new tokens x query heads to a kv
// head) and the prefix are long enough, and own tokens by the first.
struct SharedGrid {
    int prefix_wg, own_wg;  // workgroups of the kernel for blocks of 128 (0: the other one has all units), and of the other one
    int nc;
    size_t row, states;  // bytes of a row of the workspace, and of all results of (token, head)
    size_t prefix_pieces() const { return (size_t)prefix_wg * kBlockColumns * row; }
    size_t own_pieces() const { return (size_t)own_wg * 16 * nc * row; }
    size_t bytes() const { return prefix_pieces() + own_pieces() + states; }
};
long long columns_of_pack(int n_tokens, int group, int n_heads, int n_kv, int max_new)
{
    return std::min<long long>(n_tokens, (long long)std::min(group, 64) * max_new) * (n_heads / n_kv);
}
// Microseconds that a round takes a block of 32 and one of 128 columns, and what a third launch and larger results cost (measured: see shared_grid).
struct BlockCosts {
    double narrow, wide, launch;
    explicit BlockCosts(int d) : narrow(d == 64 ? 0.0022 : 0.0027), wide(d == 64 ? 0.0056 : 0.0069), launch(d == 64 ? 8.0 : 11.0) {}
    double saved_a_round(long long columns) const { return narrow * (double)((columns + 31) / 32) - wide * (double)((columns + 127) / 128); }
};
// The most that a call of these sizes and any types, or of smaller ones, has: its workspace.  shared_grid takes its grids from this one, so that what a call lays out is
// never more.  (A pack has room for blocks of 128 if any number of its columns, or fewer, may take them: the first block decides.)
SharedGrid most_grid(int n_tokens, int group, int n_heads, int n_kv, int d, int max_new)
{
    const BlockCosts costs(d);
    const long long of_pack = std::min(columns_of_pack(n_tokens, group, n_heads, n_kv, max_new), (long long)kBlockColumns);
    SharedGrid g = {0, d < 256 ? kWorkgroups : kWorkgroups / 2, d < 256 ? 2 : 1, (d + 4) * sizeof(float), 0};
    if (d < 256 && costs.saved_a_round(of_pack) > 0.0) g.prefix_wg = kWorkgroups / 2;
    g.states = 2 * (size_t)n_tokens * n_heads * g.row;
    return g;
}
// Microseconds that a round of 128 tokens takes all compute units together, for 16 columns: measured for D = 128, the others in proportion.
double round_cost(int d, bool all_bf16) { return (d == 64 ? 0.0015 : d == 128 ? 0.0022 : 0.0054) * (all_bf16 ? 1.0 : 1.45); }

SharedGrid shared_grid(int n_tokens, int n_seq, int group, int n_heads, int n_kv, int d, int max_new, int max_context, bool all_bf16)
{
    const SharedGrid most = most_grid(n_tokens, group, n_heads, n_kv, d, max_new);
    const long long share = n_heads / n_kv, rounds = (max_context + (long long)kRound - 1) / kRound, packs = (long long)n_seq / group * ((group + 63) / 64);
    const long long of_pack = columns_of_pack(n_tokens, group, n_heads, n_kv, max_new), of_seq = std::min(n_tokens, max_new) * share;
    SharedGrid g = most;
    // Blocks of 128 columns take a round in 0.0069 us, blocks of 32 in 0.0027 each, but a third launch and larger results cost 11 (D = 64: 0.0056, 0.0022, 8).
    // Microseconds, blocks of 32 / of 128.  D 128, 32 heads over 8, prefixes of 8000 tokens: 64 columns 21.9 / 30.2, 128 26.3 / 35.9, 256 29.3 / 41.2; of 32000: 64
    // columns 29.1 / 39.7; of 32768: 256 columns 72.3 / 69.7; 20000 tokens, 32 heads over 2, 1024 columns 93.7 / 84.2.  D 64, one group over 8 kv heads: 96 columns, 40000
    // tokens 30.9 / 36.6, 128 columns, 57492 tokens 50.9 / 45.8, 256 columns, 8000 tokens 24.4 / 33.0, 16000 39.1 / 39.0; 33 to 64 columns: 32 kv heads, 65536 tokens, 33
    // columns 83.8 / 114.0, 64 columns 118.3 / 122.0, 12 groups of 16 rows, 8 kv heads, 37128 tokens, 64 columns 168 / 247, and so 59 of 60 calls of any sizes.
    // (Several groups' own tokens take longer behind the blocks than between them: 152 columns over 16 kv heads, 6 groups of 5877 tokens 115 / 148; 256 over 8, 4 of 28796 179 / 138.)
    // D 256, 80 columns over 4 kv heads, 8000 tokens 22.0 / 42.6: never.
    const BlockCosts costs(d);
    const bool in_blocks = all_bf16 && most.prefix_wg > 0 && (double)(packs * n_kv) * (double)rounds * costs.saved_a_round(of_pack) > costs.launch;
    g.prefix_wg = in_blocks ? (int)std::min<long long>(packs * n_kv * ((of_pack + kBlockColumns - 1) / kBlockColumns) * 2 * rounds, most.prefix_wg) : 0;
    g.nc = (in_blocks ? of_seq : of_pack) > 16 ? most.nc : 1;
    const long long columns = 16 * g.nc, units = n_kv * (n_seq * ((of_seq + columns - 1) / columns) + (in_blocks ? 0 : packs * ((of_pack + columns - 1) / columns)));
    const long long per_unit = std::min(rounds + kUnitCost, std::max(32ll, (long long)(2.0 * sqrt((double)rounds))));
    g.own_wg = (int)std::min<long long>(units * per_unit, most.own_wg);
    return g;
}

// Whether reading the prefix once can pay, were it all of the context.  Each row for itself takes a round's cost for every 16 columns of a sequence and 5.4 us (10
// where units are fewer than compute units, whose parts have to be joined); shared, as many rounds as a pack has blocks of columns, and 12.4 us in two launches (14.5
// with 32 columns to a block, or float32; 19.5 with both).  (Microseconds, each for itself / shared, D 128, own tokens up to 200.  8 sequences x 32 heads, prefix 1000 10.9 / 12.9, 2000 15.6 / 13.5,
// 4000 24.3 / 14.2; 2 x 32, 4000 15.3 / 14.4, 8000 20.1 / 16.0; 4 x 32, 1000 10.6 / 12.4, 2000 15.6 / 12.9; 8 x 32 over 8, 4000 15.8 / 16.1, 8000 20.0 / 17.4;
// float32, 8 x 32, 1000 14.2 / 15.1, 2000 20.9 / 15.0, 8 x 16 over 4, 8000 19.1 / 21.3; D 256, 8 x 8, 4000 24.5 / 16.1.)
bool pays(int n_tokens, int n_seq, int group, int n_heads, int n_kv, int d, int max_new, int max_context, bool all_bf16)
{
    const long long share = n_heads / n_kv, of_seq = std::min<long long>(n_tokens, max_new) * share;
    const long long of_pack = columns_of_pack(n_tokens, group, n_heads, n_kv, max_new), packs = (long long)n_seq / group * ((group + 63) / 64);
    const double cost = round_cost(d, all_bf16) * (double)((max_context + (long long)kRound - 1) / kRound);
    const double units = (double)n_seq * n_kv * (double)((of_seq + 15) / 16), of_prefix = (double)packs * n_kv * (of_pack > 16 && d < 256 ? 1.23 * (double)((of_pack + 31) / 32) : (double)((of_pack + 15) / 16));
    return cost * units + (units >= 256 ? 5.4 : 10.0) > cost * of_prefix + (of_pack > 16 && !all_bf16 ? 19.5 : of_pack > 16 || !all_bf16 ? 14.5 : 12.4);
}

template <int D, int QT, int PT, int NC>
hipError_t launch_units(const SharedArgs &h, const SharedGrid &g, hipStream_t s)
{
    if (g.prefix_wg == 0) {
        shared_attention_kernel<D, QT, PT, NC, kBoth><<<(unsigned)g.own_wg, 256, 0, s>>>(h);
    } else if constexpr (QT == 1 && PT == 1 && D < 256) {
        constexpr int kBytes = kHalves * (int)sizeof(PromptTiles<D>);
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(shared_blocks_kernel<D>), hipFuncAttributeMaxDynamicSharedMemorySize, kBytes);
        if (e != hipSuccess) return e;
        shared_blocks_kernel<D><<<(unsigned)g.prefix_wg, 256 * kHalves, kBytes, s>>>(h);
        shared_attention_kernel<D, QT, PT, NC, kOwn><<<(unsigned)g.own_wg, 256, 0, s>>>(h);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    shared_join_kernel<D><<<(unsigned)std::min((long long)h.a.n_tokens * h.a.n_heads, 1ll << 16), 256, 0, s>>>(h);
    return hipGetLastError();
}
template <int D, int QT, int PT>
hipError_t launch_types(const SharedArgs &h, const SharedGrid &g, hipStream_t s)
{
    if constexpr (D < 256) {
        if (g.nc == 2) return launch_units<D, QT, PT, 2>(h, g, s);
    }
    return launch_units<D, QT, PT, 1>(h, g, s);
}
template <int D>
hipError_t launch_shared_d(const SharedArgs &h, const SharedGrid &g, hipStream_t s)
{
    if (!h.a.q_bf16) return launch_types<D, 3, 3>(h, g, s);
    if (!h.a.y_bf16) return launch_types<D, 1, 3>(h, g, s);
    return launch_types<D, 1, 1>(h, g, s);
}

}  // namespace

int cache_attention_shared_kind(int n_tokens, int n_seq, int group, int n_heads, int n_kv, int d, int max_new, int max_context, int all_bf16)
{
    if (n_seq == 0 || n_tokens == 0) return 0;
    // chunks for which the kernel for blocks of 128 columns pays are bound by their products: they gain nothing from a prefix that is read once
    if (group == 1 || cache_attention_parts(n_tokens, n_seq, n_heads, n_kv, d, max_new, max_context, 0, 0, all_bf16) > 0) return 1;
    if (!pays(n_tokens, n_seq, group, n_heads, n_kv, d, max_new, max_context, all_bf16 != 0)) return 1;
    return shared_grid(n_tokens, n_seq, group, n_heads, n_kv, d, max_new, max_context, all_bf16 != 0).prefix_wg > 0 ? 3 : 2;
}

size_t cache_attention_shared_ws(int n_tokens, int n_seq, int group, int n_heads, int n_kv, int d, int max_new, int max_context)
{
    const size_t each = cache_attention_ws(n_tokens, n_seq, n_heads, n_kv, d, max_new, max_context);
    return group == 1 ? each : std::max(each, most_grid(n_tokens, group, n_heads, n_kv, d, max_new).bytes());
}

size_t cache_attention_shared_used(int n_tokens, int n_seq, int group, int n_heads, int n_kv, int d, int max_new, int max_context, int all_bf16)
{
    const int kind = cache_attention_shared_kind(n_tokens, n_seq, group, n_heads, n_kv, d, max_new, max_context, all_bf16);
    if (kind == 0) return 0;
    if (kind == 1) return cache_attention_ws(n_tokens, n_seq, n_heads, n_kv, d, max_new, max_context);
    return shared_grid(n_tokens, n_seq, group, n_heads, n_kv, d, max_new, max_context, all_bf16 != 0).bytes();
}

hipError_t launch_cache_attention_shared(SharedArgs h, hipStream_t s)
{
    const AttentionArgs &a = h.a;
    const bool all_bf16 = a.q_bf16 && a.y_bf16;
    if (cache_attention_shared_kind(a.n_tokens, a.n_seq, h.group, a.n_heads, a.c.n_kv, a.c.d, a.max_new, a.max_context, all_bf16) < 2)
        return launch_cache_attention(a, s);
    const SharedGrid g = shared_grid(a.n_tokens, a.n_seq, h.group, a.n_heads, a.c.n_kv, a.c.d, a.max_new, a.max_context, all_bf16);
    if (g.bytes() > h.ws_bytes) return hipErrorInvalidValue;  // (never: see most_grid)
    char *const ws = reinterpret_cast<char *>(a.ws);
    h.prefix_pieces = reinterpret_cast<float *>(ws), h.own_pieces = reinterpret_cast<float *>(ws + g.prefix_pieces());
    h.states = reinterpret_cast<float *>(ws + g.prefix_pieces() + g.own_pieces());
    h.own_columns = 16 * g.nc, h.prefix_columns = g.prefix_wg ? kBlockColumns : h.own_columns;
    h.own_places = g.own_wg, h.prefix_places = g.prefix_wg ? g.prefix_wg : g.own_wg;
    if (!g.prefix_wg) h.prefix_pieces = h.own_pieces;
    if (a.c.d == 64) return launch_shared_d<64>(h, g, s);
    if (a.c.d == 128) return launch_shared_d<128>(h, g, s);
    return launch_shared_d<256>(h, g, s);
}

}  // namespace pop
