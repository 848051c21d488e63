// Attention over the 4-bit paged cache: which kernel takes a call, and its grid and workspace.
#include <math.h>

#include <algorithm>

#include "pop_cache_attention_kernels.h"

namespace pop {

namespace {

constexpr int kWorkgroups = 512;

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
long long longest_seen(int max_new, int max_context, int window, int sinks)
{
    return window > 0 ? std::min((long long)max_context, (long long)window + max_new + 31 + (sinks + 31ll) / 32 * 32) : max_context;
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

}  // namespace

size_t cache_attention_ws(int n_tokens, int n_seq, int n_heads, int n_kv, int d, int max_new, int max_context)
{
    const bool chunks = d < 256 && (long long)max_new * (n_heads / n_kv) >= kPromptColumns;
    const long long prompt = chunks ? prompt_grid(n_tokens, n_seq, n_heads, n_kv, max_new, max_context).bytes(n_kv, d) : 0;
    return std::max((size_t)prompt, (size_t)attention_workgroups(n_seq, n_heads, n_kv, d, max_new, max_context) * (2 * 16 * (d + 4) * sizeof(float) + 8));
}

int cache_attention_parts(int n_tokens, int n_seq, int n_heads, int n_kv, int d, int max_new, int max_context, int window, int sinks, int all_bf16)
{
    const PromptGrid g = prompt_of(n_tokens, n_seq, n_heads, n_kv, d, max_new, longest_seen(max_new, max_context, window, sinks), all_bf16 != 0);
    return g.blocks > 0 ? g.splits : 0;
}

hipError_t launch_cache_attention(const AttentionArgs &a, hipStream_t s)
{
    const long long seen = longest_seen(a.max_new, a.max_context, a.window, a.sinks);
    const PromptGrid g = prompt_of(a.n_tokens, a.n_seq, a.n_heads, a.c.n_kv, a.c.d, a.max_new, seen, a.q_bf16 && a.y_bf16);
    AttentionLaunch l = {g.blocks, g.splits, 0, false};
    if (g.blocks == 0) {
        l.workgroups = attention_workgroups(a.n_seq, a.n_heads, a.c.n_kv, a.c.d, a.max_new, seen);
        l.past = a.n_seq * seen * a.c.n_kv * (a.c.d + a.c.d / 16) >= kPastBytes;
    }
    if (a.window > 0 && a.sinks > 0) return launch_attention_sinks(a, l, s);
    return launch_attention_as<false>(a, l, s);
}

}  // namespace pop
