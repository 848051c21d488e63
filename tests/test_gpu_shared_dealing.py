"""How attention of sequences that share a prefix deals its work: groups whose items are a whole part of the workgroups."""
import numpy as np
import pytest
import torch

from test_gpu_decoder import BF16, i32, pop  # noqa: F401  (pop: the fixture)

pytestmark = pytest.mark.gpu


def median_us(call, n=10):
    times = []
    for _ in range(5):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        for _ in range(n):
            call()
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b) / n * 1e3)
    return sorted(times)[2]


class Batch:
    """Groups of rows with a prefix and so many tokens of their own (`of_first`: more of each group's first row)."""

    def __init__(self, pop, groups, rows, heads, n_kv, prefix, of_first=0):  # noqa: F811
        d, page, n_seq = 128, 64, groups * rows
        lengths = prefix + 1 + np.arange(n_seq) % rows * 200 // rows
        lengths[::rows] += of_first
        blocks, shared = -(-int(lengths.max()) // page), prefix // page
        table = np.full((n_seq, blocks), -1)
        used = 0
        for s in range(n_seq):
            n, first = -(-int(lengths[s]) // page), s // rows * rows
            of_others = shared if s > first else 0
            table[s, :of_others] = table[first, :of_others]
            table[s, of_others:n] = used + np.arange(n - of_others)
            used += n - of_others
        # all codes and scales the same (6 x 2^-8), so that y is that value whatever q is
        cache = torch.full((pop.pop_cache_bytes(n_kv, d, page, used),), 0x77, dtype=torch.uint8, device="cuda")
        q = torch.randn(n_seq, heads, d, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
        self.y = torch.zeros_like(q)
        sizes = (n_seq, n_seq, rows, heads, n_kv, d, 1, int(lengths.max()))
        assert pop.pop_cache_attention_shared_kind(BF16, BF16, *sizes) == 2
        self.ws = torch.empty(pop.pop_cache_attention_shared_workspace(*sizes), dtype=torch.uint8, device="cuda")
        args = (q, BF16, n_seq, cache, n_kv, d, page, used, i32(table), blocks, i32(np.arange(n_seq + 1)), i32(lengths), n_seq)
        of_groups, rest = i32([prefix] * groups), (heads, 1, int(lengths.max()), d ** -0.5)
        self.once = lambda: pop.pop_cache_attention_shared(*args, rows, of_groups, *rest, self.y, BF16, self.ws)
        self.each = lambda: pop.pop_cache_attention(*args, *rest, 0, self.y, BF16, self.ws)

    def times(self):
        """(shared, each row for itself)"""
        for call in (self.each, self.once):
            self.y.zero_()
            call()
            torch.cuda.synchronize()
            # weights rounded to bf16 over a sum of unrounded ones, and the output's rounding
            assert bool(((self.y.float() - 6 * 2.0 ** -8).abs() <= 6 * 2.0 ** -8 * (2 * 2.0 ** -8 + 2.0 ** -12)).all())
        for _ in range(3):
            self.each(), self.once()
        torch.cuda.synchronize()
        return median_us(self.once), median_us(self.each)


@pytest.mark.parametrize("groups,rows,heads,n_kv,prefix", [(16, 14, 32, 8, 8000), (32, 7, 64, 16, 3000)])
def test_reading_prefixes_once_is_worth_it(pop, groups, rows, heads, n_kv, prefix):  # noqa: F811
    """Prefixes of all groups in turn to all workgroups: less than three quarters of what each row for itself takes (0.4 measured; 1.5 and 1.3 where
    they fall to the same few workgroups)."""
    shared_us, each_us = Batch(pop, groups, rows, heads, n_kv, prefix).times()
    assert shared_us < 0.75 * each_us, (shared_us, each_us)


@pytest.mark.parametrize("groups,rows,heads,n_kv,prefix", [(64, 8, 32, 8, 1024), (8, 8, 32, 32, 2048)])
def test_longer_rows_at_regular_distances(pop, groups, rows, heads, n_kv, prefix):  # noqa: F811
    """The first row of each group has 8000 tokens of its own, the others few: what is read twice without sharing is little, but the long rows do not all fall to the
    same workgroups (0.9 measured; 2.6 and 1.9 where they do)."""
    shared_us, each_us = Batch(pop, groups, rows, heads, n_kv, prefix, of_first=8000).times()
    assert shared_us < 1.3 * each_us, (shared_us, each_us)


@pytest.mark.parametrize("n_kv,heads,d", [(4, 160, 64), (5, 200, 128)])
def test_more_blocks_than_workgroups(pop, n_kv, heads, d):  # noqa: F811
    """Prefixes in blocks of 128 columns, more of them than workgroups, against the other kernel: both round weights (2^-8 of the values that they weigh) and y."""
    groups, rows, page = 70, 2, 16
    rng = np.random.default_rng(d)
    prefix = rng.integers(1030, 1200, groups)
    lengths = np.repeat(prefix, rows) + rng.integers(1, 40, groups * rows)
    n_seq, blocks = groups * rows, 80
    table = np.full((n_seq, blocks), -1)
    used = 0
    for s in range(n_seq):
        n, first = -(-int(lengths[s]) // page), s // rows * rows
        of_others = int(prefix[s // rows]) // page if s > first else 0
        table[s, :of_others] = table[first, :of_others]
        table[s, of_others:n] = used + np.arange(n - of_others)
        used += n - of_others
    tile = 16 * (d + d // 16)
    cache = torch.randint(0, 256, (used, n_kv, tile), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda", dtype=torch.int32).to(torch.uint8)
    cache[..., 16 * d:] = 125  # scales: 2^-2, values up to 1.5
    # the page that a prefix ends in holds the same tokens in all rows of a group (of which the others' own are a part)
    for s in range(n_seq):
        at = int(prefix[s // rows]) // page
        cache[table[s, at]] = cache[table[s // rows * rows, at]]
    assert cache.numel() == pop.pop_cache_bytes(n_kv, d, page, used)
    q = torch.randn(n_seq, heads, d, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    out = []
    for kind, longest in ((2, int(lengths.max())), (3, 1 << 22)):
        sizes = (n_seq, n_seq, rows, heads, n_kv, d, 1, longest)
        assert pop.pop_cache_attention_shared_kind(BF16, BF16, *sizes) in ((1, 2) if kind == 2 else (3,))
        y, ws = torch.zeros_like(q), torch.full((pop.pop_cache_attention_shared_workspace(*sizes),), 0xFF, dtype=torch.uint8, device="cuda")
        pop.pop_cache_attention_shared(q, BF16, n_seq, cache, n_kv, d, page, used, i32(table), blocks, i32(np.arange(n_seq + 1)), i32(lengths), n_seq, rows,
                                       i32(prefix), heads, 1, longest, d ** -0.5, y, BF16, ws)
        torch.cuda.synchronize()
        out.append(y.double())
    assert bool((out[0] - out[1]).abs().max() <= 2 * (2.0 ** -8 + 2.0 ** -8 + 2.0 ** -16) * 1.5) and bool(out[0].any())
