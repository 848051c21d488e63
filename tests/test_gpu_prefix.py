"""Attention over the 4-bit cache with first tokens that stay visible next to a window, and of sequences that share a prefix, on the GPU against the
64-bit oracle."""
import numpy as np
import pytest
import torch

from oracle import decoder_oracle as orc
from test_gpu_decoder import BF16, DT, F32, TYPES, Cached, f64, i32, pop  # noqa: F401  (pop: the fixture)
from test_gpu_decoder import _queries as queries

pytestmark = pytest.mark.gpu


def starts_of(new):
    return np.concatenate([[0], np.cumsum(new)])


def bound_of(want, sizes, d, length, ydtype):
    """Products and sums in 32 bits (the scores' error turns into a relative one of the weights), weights rounded to bf16 where the output is
    bf16, the output's own rounding."""
    weight, product = sizes
    scores = (d + 8) * 2.0 ** -24 * product
    bound = weight * (2 * scores + (length + 32) * 2.0 ** -24 + 2.0 ** -21) + 2.0 ** -23 * np.abs(want)
    return bound + (2.0 ** -8 * weight + 2.0 ** -8 * np.abs(want) if ydtype == BF16 else 0.0)


def check(c, y, q, start, ydtype, scale, window=0, sinks=0, there=None, context=None):
    y, qh = f64(y), f64(q)
    context = c.context if context is None else context
    for s, length in enumerate(context):
        a, b = start[s], start[s + 1]
        sizes = []
        seen = min(length, len(c.k[s]))  # (a table may be shorter than its context)
        want = orc.attention(qh[a:b], c.k[s][:seen], c.v[s][:seen], scale, length - (b - a), window, None if there is None else there[s][:seen], sizes, sinks)
        off = np.abs(y[a:b] - want) - bound_of(want, sizes, c.d, length, ydtype)
        assert (off <= 1e-30).all(), (s, float(off.max()), np.unravel_index(off.argmax(), off.shape))


def attend(pop, c, q, start, dtype, ydtype, heads, scale, window, sinks, max_new=None, max_context=None, table=None, context=None, stream=None, entry="sinks"):
    table = c.table if table is None else table
    context = c.context if context is None else context
    n, n_seq = q.shape[0], len(context)
    max_new = max(int(np.diff(start).max()), 1) if max_new is None else max_new
    max_context = max(max(context), 1) if max_context is None else max_context
    y = torch.full(q.shape, 7.0, dtype=DT[ydtype], device="cuda")
    ws = torch.full((pop.pop_cache_attention_workspace(n, n_seq, heads, c.n_kv, c.d, max_new, max_context),), 0xFF, dtype=torch.uint8, device="cuda")
    args = [q, dtype, n, c.cache, c.n_kv, c.d, c.page, c.n_pages, i32(table), table.shape[1], i32(start), i32(context), n_seq, heads, max_new,
            max_context, scale, window]
    torch.cuda.synchronize()
    if entry == "sinks":
        pop.pop_cache_attention_sinks(*args, sinks, y, ydtype, ws, stream=stream)
    else:
        pop.pop_cache_attention(*args, y, ydtype, ws, stream=stream)
    if stream is not None:
        torch.cuda.synchronize()
    return y


def given_back(c, start, window, sinks):
    """The table without the pages that no token sees, in whose place others stand that hold no numbers."""
    table = c.table.copy()
    for s, length in enumerate(c.context):
        lo = max(length - int(start[s + 1] - start[s]) - window + 1, 0)
        for b in range(table.shape[1]):
            if b * c.page >= sinks and (b + 1) * c.page <= lo:
                table[s, b] = -1
    return table


# ---------------------------------------------------------------- first tokens next to a window

@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype,ydtype", TYPES)
def test_sinks_single_tokens(pop, d, dtype, ydtype):  # noqa: F811
    """Lengths around the tile, the step and the page; windows and first tokens that meet, end inside a tile, lie far apart; an empty sequence."""
    rng = np.random.default_rng(d)
    for heads, n_kv, page in ((2, 2, 16), (6, 2, 32), (16, 1, 64), (20, 1, 16)):
        c = Cached(pop, rng, [1, 2, 15, 16, 17, 31, 33, 64, 65, 0, 129, 700], n_kv, d, page)
        start = starts_of([0 if x == 0 else 1 for x in c.context])
        q = queries(rng, start[-1], heads, d, dtype)
        for window, sinks in ((1, 1), (20, 4), (33, 33), (100, 32), (300, 500), (64, 31), (5, (1 << 31) - 1), ((1 << 31) - 1, 7)):
            y = attend(pop, c, q, start, dtype, ydtype, heads, d ** -0.5, window, sinks, table=given_back(c, start, window, sinks))
            check(c, y, q, start, ydtype, d ** -0.5, window, sinks)


CHUNKS = [(4, 4, 128, 16, [40, 7, 200, 90], [40, 3, 100, 1]), (6, 2, 64, 64, [130, 64, 33], [70, 64, 5]), (2, 1, 256, 16, [75], [75]),
          (5, 1, 128, 32, [700, 1], [150, 1]), (8, 1, 64, 16, [900, 1300], [17, 40])]


@pytest.mark.parametrize("dtype,ydtype", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("window,sinks", [(1, 3), (20, 4), (50, 64), (100, 33), (300, 1)])
def test_sinks_chunks(pop, dtype, ydtype, window, sinks):  # noqa: F811
    rng = np.random.default_rng(window)
    for heads, n_kv, d, page, context, new in CHUNKS:
        c = Cached(pop, rng, context, n_kv, d, page)
        start = starts_of(new)
        q = queries(rng, start[-1], heads, d, dtype)
        for sizes in ({}, dict(max_new=1, max_context=1)):
            y = attend(pop, c, q, start, dtype, ydtype, heads, 0.07, window, sinks, table=given_back(c, start, window, sinks), **sizes)
            check(c, y, q, start, ydtype, 0.07, window, sinks)


IN_BLOCKS = dict(max_new=1 << 19, max_context=1 << 19)  # sizes for which blocks of 128 columns are taken, whatever the chunks really have


def assert_in_blocks(pop, c, n, heads, window):  # noqa: F811
    """(First tokens only add to what a window sees, which makes blocks pay the more.)"""
    assert pop.pop_cache_attention_kind(BF16, BF16, n, len(c.context), heads, c.n_kv, c.d, 1 << 19, 1 << 19, window)[0] == 2


@pytest.mark.parametrize("window,sinks", [(60, 4), (1, 64), (33, 100), (400, 17)])
@pytest.mark.parametrize("heads,n_kv,d,page,context,new", [
    (4, 4, 128, 16, [240, 7, 400, 0], [200, 3, 380, 0]), (6, 2, 64, 64, [630, 64, 33], [70, 64, 5]), (5, 1, 128, 32, [300, 1], [150, 1]),
    (2, 1, 128, 64, [2900, 65], [130, 65]), (3, 3, 64, 32, [1500], [97]), (16, 1, 64, 16, [63, 64, 65, 1127, 129], [9, 8, 7, 33, 5])])
def test_sinks_in_blocks_of_128_columns(pop, window, sinks, heads, n_kv, d, page, context, new):  # noqa: F811
    rng = np.random.default_rng(d + window + len(context))
    c = Cached(pop, rng, context, n_kv, d, page)
    start = starts_of(new)
    q = queries(rng, start[-1], heads, d, BF16)
    assert_in_blocks(pop, c, len(q), heads, window)
    for scale in (0.07, -0.4, 0.0):
        y = attend(pop, c, q, start, BF16, BF16, heads, scale, window, sinks, table=given_back(c, start, window, sinks), **IN_BLOCKS)
        check(c, y, q, start, BF16, scale, window, sinks)
    # pages that are none among those that are seen
    table = c.table.copy()
    table[0, ::3] = -1
    there = [np.repeat((t >= 0) & (t < c.n_pages), page) for t in table]
    y = attend(pop, c, q, start, BF16, BF16, heads, 0.07, window, sinks, table=table, **IN_BLOCKS)
    check(c, y, q, start, BF16, 0.07, window, sinks, there=there)


@pytest.mark.parametrize("heads,n_kv,d,page,new,before,window,sinks", [(32, 32, 128, 64, 600, 1500, 501, 17), (16, 16, 64, 16, 1200, 900, 700, 70),
                                                                     (64, 64, 256, 32, 300, 900, 333, 4)])
def test_sinks_large_chunks(pop, heads, n_kv, d, page, new, before, window, sinks):  # noqa: F811
    """Chunks of a size that blocks of 128 columns are made for, and by the caller's sizes too; some tokens and heads are checked."""
    rng = np.random.default_rng(new)
    context, news = [before + new, before + new // 2], [new, new // 3]
    c = Cached(pop, rng, context, n_kv, d, page)
    start = starts_of(news)
    q = queries(rng, start[-1], heads, d, BF16)
    assert_in_blocks(pop, c, len(q), heads, window)
    qh, table = f64(q), given_back(c, start, window, sinks)
    for sizes in ({}, IN_BLOCKS):
        yh = f64(attend(pop, c, q, start, BF16, BF16, heads, d ** -0.5, window, sinks, table=table, **sizes))
        for s, length in enumerate(context):
            for i in range(0, news[s], 97):
                for h in range(0, heads, 7):
                    of, at = [], start[s] + i
                    first = length - news[s] + i
                    want = orc.attention(qh[at:at + 1, h:h + 1], c.k[s][:, h:h + 1], c.v[s][:, h:h + 1], d ** -0.5, first, window, None, of, sinks)
                    assert (np.abs(yh[at, h] - want[0]) <= bound_of(want, of, d, length, BF16)[0]).all(), (s, i, h)


@pytest.mark.parametrize("dtype,ydtype", [(BF16, BF16), (F32, F32)])
def test_sinks_long_sequences(pop, dtype, ydtype):  # noqa: F811
    """Units that are split, with pieces that begin and end in front of the window; many sequences; pages that the first tokens have not."""
    rng = np.random.default_rng(4)
    c = Cached(pop, rng, [20000, 300, 9000], 2, 128, 64)
    start = starts_of([1, 1, 3])
    q = queries(rng, start[-1], 4, 128, dtype)
    for window, sinks in ((9000, 1000), (100, 4), (5000, 2049)):
        table = given_back(c, start, window, sinks)
        y = attend(pop, c, q, start, dtype, ydtype, 4, 0.08, window, sinks, table=table)
        check(c, y, q, start, ydtype, 0.08, window, sinks)
        assert torch.equal(y, attend(pop, c, q, start, dtype, ydtype, 4, 0.08, window, sinks, table=table))
    table[:, 0] = -1
    there = [np.repeat((t >= 0) & (t < c.n_pages), 64) for t in table]
    check(c, attend(pop, c, q, start, dtype, ydtype, 4, 0.08, window, sinks, table=table), q, start, ydtype, 0.08, window, sinks, there=there)
    lengths = [int(x) for x in rng.integers(1, 400, 90)]
    c = Cached(pop, rng, lengths, 1, 64, 16)
    q = queries(rng, 90, 5, 64, dtype)
    y = attend(pop, c, q, np.arange(91), dtype, ydtype, 5, 0.1, 40, 6)
    check(c, y, q, np.arange(91), ydtype, 0.1, 40, 6)


@pytest.mark.parametrize("new", [1, 20])
def test_sinks_where_nothing_else_is_seen(pop, new):  # noqa: F811
    """A context beyond the table: the window has passed it, the first tokens are there; a context shorter than its new tokens."""
    rng = np.random.default_rng(6)
    for page, blocks in ((16, 5), (32, 4)):
        c = Cached(pop, rng, [blocks * page], 2, 64, page, spare=0)
        q = queries(rng, new, 4, 64, BF16)
        start = np.array([0, new])
        y = attend(pop, c, q, start, BF16, BF16, 4, 0.1, 30, 37, context=[blocks * page + 500])
        check(c, y, q, start, BF16, 0.1, 30, 37, context=[blocks * page + 500])
        y = attend(pop, c, q, start, BF16, BF16, 4, 0.1, 30, 37, context=[new // 2])
        check(c, y, q, start, BF16, 0.1, 30, 37, context=[new // 2])
        y = attend(pop, c, q, start, BF16, BF16, 4, 0.1, 30, 37, table=np.full((1, blocks), -1))
        assert (f64(y) == 0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_sinks_without_a_window_or_without_tokens_are_plain_attention(pop, dtype):  # noqa: F811
    rng = np.random.default_rng(8)
    c = Cached(pop, rng, [700, 90, 33], 2, 128, 16)
    for new in ([1, 1, 1], [300, 40, 33]):
        start = starts_of(new)
        q = queries(rng, start[-1], 8, 128, dtype)
        for window in (0, 60):
            plain = attend(pop, c, q, start, dtype, dtype, 8, 0.1, window, 0, entry="plain")
            assert torch.equal(plain, attend(pop, c, q, start, dtype, dtype, 8, 0.1, window, 0))
            if window == 0:
                assert torch.equal(plain, attend(pop, c, q, start, dtype, dtype, 8, 0.1, 0, 9))


def test_sinks_on_another_stream_and_in_a_replayed_graph(pop):  # noqa: F811
    rng = np.random.default_rng(10)
    c = Cached(pop, rng, [3000, 77], 2, 128, 16)
    q = queries(rng, 2, 4, 128, BF16)
    want = attend(pop, c, q, np.array([0, 1, 2]), BF16, BF16, 4, 0.09, 700, 20)
    assert torch.equal(want, attend(pop, c, q, np.array([0, 1, 2]), BF16, BF16, 4, 0.09, 700, 20, stream=torch.cuda.Stream()))
    y, table, start, context = torch.zeros_like(q), i32(c.table), i32([0, 1, 2]), i32([3000, 77])
    ws = torch.full((pop.pop_cache_attention_workspace(2, 2, 4, 2, 128, 1, 3000),), 0xFF, dtype=torch.uint8, device="cuda")

    def call():
        pop.pop_cache_attention_sinks(q, BF16, 2, c.cache, 2, 128, 16, c.n_pages, table, table.shape[1], start, context, 2, 4, 1, 3000, 0.09, 700, 20, y,
                                      BF16, ws)

    call()
    torch.cuda.synchronize()
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        context.copy_(i32([3000 - 611 * i, 77 - i]))
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        y.zero_()
        call()
        torch.cuda.synchronize()
        assert torch.equal(got, y) and bool(y.any())


@pytest.mark.parametrize("window,sinks", [(90, 20), (30, 70)])
@pytest.mark.parametrize("n_seq,heads,n_kv,d", [(65, 4, 1, 64), (150, 8, 2, 64), (129, 16, 4, 128)])
def test_sinks_many_sequences_in_blocks_of_128_columns(pop, n_seq, heads, n_kv, d, window, sinks):  # noqa: F811
    """Several sequences to a lane; empty ones, ones without new tokens."""
    rng = np.random.default_rng(n_seq + window)
    context = [int(x) for x in rng.integers(0, 300, n_seq)]
    new = [int(rng.integers(0, c + 1)) if i % 9 else 0 for i, c in enumerate(context)]
    c = Cached(pop, rng, context, n_kv, d, 16)
    start = starts_of(new)
    q = queries(rng, start[-1], heads, d, BF16)
    assert_in_blocks(pop, c, len(q), heads, window)
    y = attend(pop, c, q, start, BF16, BF16, heads, 0.1, window, sinks, table=given_back(c, start, window, sinks), **IN_BLOCKS)
    check(c, y, q, start, BF16, 0.1, window, sinks)


@pytest.mark.parametrize("dtype,blocks", [(F32, False), (BF16, False), (BF16, True)])
def test_sinks_starts_that_do_not_ascend(pop, dtype, blocks):  # noqa: F811
    """Sequences whose rows are none or leave the tensors are left out; the others' rows, wherever they stand, are right; rows of none stay."""
    rng = np.random.default_rng(15)
    c = Cached(pop, rng, [300, 200, 90, 64, 500, 7], 2, 64, 16)
    n = 150
    q = queries(rng, n, 8, 64, dtype)
    for starts, kept in (([100, 140, 20, 60, 5000, 7000, -3], [0, 2]), ([150, 80, 149, 90, 2 ** 31 - 1, -2 ** 31, 0], [1]), ([-5, -1, 140, 3, 3, 10, 9], [4])):
        h = f64(attend(pop, c, q, starts, dtype, dtype, 8, 0.1, 50, 40, **(IN_BLOCKS if blocks else dict(max_new=40, max_context=500))))
        written = np.zeros(n, bool)
        for s in kept:
            a, b = starts[s], starts[s + 1]
            written[a:b] = True
            sizes = []
            want = orc.attention(f64(q[a:b]), c.k[s], c.v[s], 0.1, c.context[s] - (b - a), 50, None, sizes, 40)
            assert (np.abs(h[a:b] - want) <= bound_of(want, sizes, 64, c.context[s], dtype) + 1e-30).all(), (starts, s)
        assert (h[~written] == 7.0).all()


# ---------------------------------------------------------------- a prefix that is shared

LIFT = 1024  # prefixes that are shorter are not shared


def lifted(groups):
    """Groups whose prefixes are all longer by that; rows that are not much shorter than their prefix with them."""
    return [(p + LIFT, [c + LIFT if c >= p - 50 and c else c for c in lengths]) if p > 0 else (p, lengths) for p, lengths in groups]


class Grouped:
    """Groups of sequences whose first tokens are the same: (prefix, [context ..]).  Full pages of the prefix are shared by all rows, the page that it ends in is
    copied; a row that is shorter than the prefix has what it reaches.  The cache's other bytes are all ones (a scale of all ones is no number)."""

    def __init__(self, pop, rng, groups, n_kv, d, page, spare=1):  # noqa: F811
        self.group, self.n_kv, self.d, self.page = len(groups[0][1]), n_kv, d, page
        self.context = [x for _, lengths in groups for x in lengths]
        self.prefix = [p for p, _ in groups]
        self.n_pages = sum(-(-x // page) for x in self.context) + 2
        order = rng.permutation(self.n_pages)
        self.table = np.full((len(self.context), max(-(-x // page) for x in self.context) + spare), -1)
        self.cache = torch.full((pop.pop_cache_bytes(n_kv, d, page, self.n_pages),), 0xFF, dtype=torch.uint8, device="cuda")
        self.k, self.v = [], []
        used = 0
        for g, (p, lengths) in enumerate(groups):
            common = {}
            first = [(rng.standard_normal((max(p, 0), n_kv, d)) * np.where(np.arange(d) % 29 == 3, 5.0, 1.0)).astype(np.float32),
                     (rng.standard_normal((max(p, 0), n_kv, d)) + 0.2).astype(np.float32)]
            for i, c in enumerate(lengths):
                row = self.table[g * self.group + i]
                for b in range(-(-c // page)):
                    if (b + 1) * page <= min(p, c) and b in common:
                        row[b] = common[b]
                    else:
                        row[b] = order[used]
                        used += 1
                        if (b + 1) * page <= min(p, c):
                            common[b] = row[b]
                kv = []
                for x in first:
                    own = rng.standard_normal((max(c - len(x), 0), n_kv, d)).astype(np.float32)
                    kv.append(np.concatenate([x[:c], own]))
                t = np.arange(c)
                if c:
                    pop.pop_cache_write(self.cache, n_kv, d, page, self.n_pages, *(torch.from_numpy(x).cuda() for x in kv), F32,
                                        i32(row[t // page] * page + t % page), c)
                self.k.append(orc.decode(*orc.encode(kv[0])))
                self.v.append(orc.decode(*orc.encode(kv[1])))
        torch.cuda.synchronize()


LONG = 1 << 22  # a context for which sharing pays, whatever the sequences really have


def attend_shared(pop, c, q, start, dtype, ydtype, heads, scale, prefix=None, max_new=None, max_context=LONG, table=None, context=None, stream=None, kinds=(2, 3)):
    table = c.table if table is None else table
    context = c.context if context is None else context
    n, n_seq = q.shape[0], len(context)
    max_new = max(int(np.diff(start).max()), 1) if max_new is None else max_new
    sizes = (n, n_seq, c.group, heads, c.n_kv, c.d, max_new, max_context)
    if 1 not in kinds and pop.pop_cache_attention_shared_kind(dtype, ydtype, *sizes) == 1:  # (a chunk that is bound by its products, by these sizes)
        sizes = (n, n_seq, c.group, heads, c.n_kv, c.d, 1, max_context)
    assert pop.pop_cache_attention_shared_kind(dtype, ydtype, *sizes) in kinds
    y = torch.full(q.shape, 7.0, dtype=DT[ydtype], device="cuda")
    ws = torch.full((pop.pop_cache_attention_shared_workspace(*sizes),), 0xFF, dtype=torch.uint8, device="cuda")
    args = (q, dtype, n, c.cache, c.n_kv, c.d, c.page, c.n_pages, i32(table), table.shape[1], i32(start), i32(context), n_seq, c.group,
            i32(c.prefix if prefix is None else prefix), heads, *sizes[6:], scale, y, ydtype, ws)
    torch.cuda.synchronize()
    pop.pop_cache_attention_shared(*args, stream=stream)
    if stream is not None:
        torch.cuda.synchronize()
    return y


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype,ydtype", TYPES)
def test_shared_single_tokens(pop, d, dtype, ydtype):  # noqa: F811
    """Prefixes of all kinds of lengths; columns that fill one, two and more blocks of 16; groups that share nothing, rows shorter than the prefix."""
    rng = np.random.default_rng(d)
    for heads, n_kv, page, groups in (
            (2, 2, 16, [(700, [701, 730, 900])]), (8, 1, 32, [(257, [300, 257, 258, 1000, 289, 290, 256, 400])]),
            (4, 2, 64, [(300, [333, 0, 350, 301]), (0, [40, 1, 17, 500]), (1000, [1001, 1064, 999, 200])]),
            (5, 1, 16, [(515, [516 + 7 * i for i in range(9)])]), (6, 2, 128, [(290, [300, 310]), (100, [130, 120]), (640, [700, 641])])):
        c = Grouped(pop, rng, lifted(groups), n_kv, d, page)
        start = starts_of([0 if x == 0 else 1 for x in c.context])
        q = queries(rng, start[-1], heads, d, dtype)
        y = attend_shared(pop, c, q, start, dtype, ydtype, heads, d ** -0.5)
        check(c, y, q, start, ydtype, d ** -0.5)
        assert torch.equal(y, attend_shared(pop, c, q, start, dtype, ydtype, heads, d ** -0.5))


@pytest.mark.parametrize("dtype,ydtype", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("heads,n_kv,d,page", [(4, 4, 128, 16), (6, 2, 64, 64), (3, 1, 256, 32)])
def test_shared_chunks(pop, dtype, ydtype, heads, n_kv, d, page):  # noqa: F811
    """Several new tokens to a sequence, some of them in the prefix, rows without any, a context shorter than its new tokens; sizes that the caller
    underestimates, and prefix lengths that say less, more and nothing."""
    rng = np.random.default_rng(d)
    c = Grouped(pop, rng, lifted([(400, [401, 420, 395, 500, 30]), (300, [330, 299, 0, 310, 700])]), n_kv, d, page)
    start = starts_of([1, 5, 4, 0, 17, 33, 9, 0, 2, 64])
    q = queries(rng, start[-1], heads, d, dtype)
    for scale in (0.07, -0.3, 0.0):
        check(c, attend_shared(pop, c, q, start, dtype, ydtype, heads, scale), q, start, ydtype, scale)
    for change in (dict(max_new=1, max_context=1, kinds=(1,)), dict(max_new=1), dict(prefix=[LIFT + 399, LIFT + 280]), dict(prefix=[0, -5]),
                   dict(prefix=[-(1 << 31), LIFT + 300]), dict(prefix=[LIFT + 400, LIFT + 1]), dict(prefix=[LIFT, LIFT - 1])):
        check(c, attend_shared(pop, c, q, start, dtype, ydtype, heads, 0.07, **change), q, start, ydtype, 0.07)
    short = list(c.context)
    short[5] = 12  # of 33 new tokens
    y = attend_shared(pop, c, q, start, dtype, ydtype, heads, 0.07, context=short)
    check(c, y, q, start, ydtype, 0.07, context=short)
    assert (f64(y)[start[5]:start[6] - 12] == 0).all()


@pytest.mark.parametrize("group,n_groups,heads,n_kv,d", [(64, 1, 2, 1, 64), (65, 1, 4, 2, 64), (130, 2, 2, 2, 128), (33, 5, 1, 1, 64), (2, 70, 3, 1, 64), (200, 1, 8, 1, 64)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_shared_many_sequences(pop, group, n_groups, heads, n_kv, d, dtype):  # noqa: F811
    """More sequences than lanes, groups of more than that, some rows empty."""
    rng = np.random.default_rng(group)
    groups = []
    for g in range(n_groups):
        p = int(rng.integers(250, 600))
        groups.append((p, [0 if rng.random() < 0.1 else p + int(rng.integers(-20, 60)) for _ in range(group)]))
    c = Grouped(pop, rng, lifted(groups), n_kv, d, 16)
    start = starts_of([0 if x == 0 else int(rng.integers(1, 3)) for x in c.context])
    q = queries(rng, start[-1], heads, d, dtype)
    y = attend_shared(pop, c, q, start, dtype, dtype, heads, 0.1)
    check(c, y, q, start, dtype, 0.1)


@pytest.mark.parametrize("dtype,ydtype", [(BF16, BF16), (F32, F32)])
@pytest.mark.parametrize("heads,n_kv,group", [(4, 2, 4), (8, 1, 8), (1, 1, 2)])
def test_shared_long_prefixes(pop, dtype, ydtype, heads, n_kv, group):  # noqa: F811
    """Units that many workgroups have; sizes as they are, and longer ones."""
    rng = np.random.default_rng(heads)
    c = Grouped(pop, rng, [(20001, [20002 + 611 * i for i in range(group)])], n_kv, 128, 64)
    q = queries(rng, group, heads, 128, dtype)
    for sizes in (dict(max_context=max(c.context), kinds=(1, 2)), {}):
        y = attend_shared(pop, c, q, np.arange(group + 1), dtype, ydtype, heads, 0.08, **sizes)
        check(c, y, q, np.arange(group + 1), ydtype, 0.08)
    assert torch.equal(y, attend_shared(pop, c, q, np.arange(group + 1), dtype, ydtype, heads, 0.08))


@pytest.mark.parametrize("heads,n_kv,d,page,group,prefix", [(8, 1, 128, 64, 40, 4000), (6, 1, 64, 16, 17, 2999), (16, 1, 128, 128, 9, 1700)])
def test_shared_prefixes_in_blocks_of_128_columns(pop, heads, n_kv, d, page, group, prefix):  # noqa: F811
    """Blocks that are full and nearly empty, prefixes that end inside a tile, rows that are shorter and empty; pages that are none."""
    rng = np.random.default_rng(d)
    lengths = [prefix + int(rng.integers(1, 300)) for _ in range(group)]
    lengths[3], lengths[5] = prefix // 2, 0
    c = Grouped(pop, rng, [(prefix, lengths)], n_kv, d, page)
    start = starts_of([0 if x == 0 else 1 for x in c.context])
    q = queries(rng, start[-1], heads, d, BF16)
    for scale in (d ** -0.5, -0.2):
        y = attend_shared(pop, c, q, start, BF16, BF16, heads, scale, kinds=(3,))
        check(c, y, q, start, BF16, scale)
    assert torch.equal(y, attend_shared(pop, c, q, start, BF16, BF16, heads, scale, kinds=(3,)))
    table = c.table.copy()
    table[:, 2:4] = -1  # (of all rows: they share them)
    there = [np.repeat((t >= 0) & (t < c.n_pages), page) for t in table]
    check(c, attend_shared(pop, c, q, start, BF16, BF16, heads, 0.1, table=table, kinds=(3,)), q, start, BF16, 0.1, there=there)


def test_shared_pages_that_are_none(pop):  # noqa: F811
    """Pages of the prefix that no row has, pages behind it that one has not, nothing at all: what is not there is not seen."""
    rng = np.random.default_rng(12)
    c = Grouped(pop, rng, [(1536, [1564, 1554, 1624])], 2, 128, 16)
    start = starts_of([2, 1, 1])
    q = queries(rng, 4, 4, 128, BF16)
    for blocks, of in (([3, 4, 20], [0, 1, 2]), ([96], [1]), (range(97, 102), [2])):
        table = c.table.copy()
        for s in of:
            table[s, list(blocks)] = -1 if s % 2 else c.n_pages
        there = [np.repeat((t >= 0) & (t < c.n_pages), 16) for t in table]
        y = attend_shared(pop, c, q, start, BF16, BF16, 4, 0.1, table=table)
        check(c, y, q, start, BF16, 0.1, there=there)
    y = attend_shared(pop, c, q, start, BF16, BF16, 4, 0.1, table=np.full_like(c.table, -1))
    assert (f64(y) == 0).all()
    # contexts beyond the table
    c = Grouped(pop, rng, [(1344, [1344, 1344])], 2, 64, 16, spare=0)
    q = queries(rng, 2, 4, 64, BF16)
    y = attend_shared(pop, c, q, np.arange(3), BF16, BF16, 4, 0.1, context=[1900, 1344], prefix=[1 << 30])
    check(c, y, q, np.arange(3), BF16, 0.1, context=[1900, 1344])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_shared_starts_that_do_not_ascend(pop, dtype):  # noqa: F811
    """Sequences whose rows are none or leave the tensors are left out; the others' rows, wherever they stand, are right; rows of none stay."""
    rng = np.random.default_rng(15)
    c = Grouped(pop, rng, lifted([(300, [310, 320, 330]), (400, [420, 500, 401])]), 2, 64, 16)
    n = 150
    q = queries(rng, n, 8, 64, dtype)
    for starts, kept in (([100, 140, 20, 60, 5000, 7000, -3], [0, 2]), ([150, 80, 149, 90, 2 ** 31 - 1, -2 ** 31, 0], [1]), ([-5, -1, 140, 3, 3, 10, 9], [4]),
                         ([0, 10, 20, 30, 40, 50, 60], [0, 1, 2, 3, 4, 5])):
        h = f64(attend_shared(pop, c, q, starts, dtype, dtype, 8, 0.1, max_new=40))
        written = np.zeros(n, bool)
        for s in kept:
            a, b = starts[s], starts[s + 1]
            written[a:b] = True
            sizes = []
            want = orc.attention(f64(q[a:b]), c.k[s], c.v[s], 0.1, c.context[s] - (b - a), 0, None, sizes)
            assert (np.abs(h[a:b] - want) <= bound_of(want, sizes, 64, c.context[s], dtype) + 1e-30).all(), (starts, s)
        assert (h[~written] == 7.0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_shared_scores_far_from_zero(pop, dtype):  # noqa: F811
    """Scores of 2^34 in the prefix or behind it: the part that holds the largest decides, and equal ones share."""
    rng = np.random.default_rng(16)
    c = Grouped(pop, rng, lifted([(300, [340, 310])]), 1, 64, 16)
    q = queries(rng, 2, 2, 64, dtype)
    for scale in (2.0 ** 28, -(2.0 ** 30), 2.0 ** 34):
        h = f64(attend_shared(pop, c, q, np.arange(3), dtype, dtype, 2, scale))
        plain = f64(attend(pop, c, q, np.arange(3), dtype, dtype, 2, scale, 0, 0))
        # one token, or tokens of the same score, have all of the weight: sums of a few of their values
        assert np.isfinite(h).all() and np.abs(h - plain).max() <= 2.0 ** -7 * np.abs(plain).max()


def test_shared_group_of_one_is_plain_attention(pop):  # noqa: F811
    rng = np.random.default_rng(17)
    c = Cached(pop, rng, [700, 90], 2, 128, 16)
    c.group = 1
    q = queries(rng, 2, 8, 128, BF16)
    y = attend_shared(pop, c, q, np.arange(3), BF16, BF16, 8, 0.1, prefix=[600, 50], kinds=(1,))
    assert torch.equal(y, attend(pop, c, q, np.arange(3), BF16, BF16, 8, 0.1, 0, 0))


@pytest.mark.parametrize("dtype", [BF16])
def test_shared_chunks_in_blocks_of_128_columns(pop, dtype):  # noqa: F811
    """Chunks that are bound by their products read each row's pages."""
    rng = np.random.default_rng(18)
    c = Grouped(pop, rng, [(300, [500, 450])], 2, 64, 16)
    start = starts_of([190, 150])
    q = queries(rng, start[-1], 4, 64, dtype)
    assert pop.pop_cache_attention_kind(BF16, BF16, len(q), 2, 4, 2, 64, 1 << 19, 1 << 19)[0] == 2
    y = attend_shared(pop, c, q, start, BF16, BF16, 4, 0.1, max_new=1 << 19, max_context=1 << 19, kinds=(1,))
    check(c, y, q, start, BF16, 0.1)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_shared_rows_of_several_sequences(pop, dtype):  # noqa: F811
    """Rows that two sequences say are theirs are undefined; the others' are right, and nothing beyond the rows is written."""
    rng = np.random.default_rng(21)
    c = Grouped(pop, rng, lifted([(300, [340, 330, 320]), (310, [340, 330, 320])]), 2, 64, 16)
    q = queries(rng, 40, 8, 64, dtype)
    starts = [0, 10, 5, 20, 3, 15, 32]  # sequences 0, 2, 4 and 5: rows 0-9, 5-19, 3-14, 15-31
    h = f64(attend_shared(pop, c, q, starts, dtype, dtype, 8, 0.1, max_new=20))
    for rows, s in ((range(0, 3), 0), (range(20, 32), 5)):
        a, b = starts[s], starts[s + 1]
        sizes = []
        want = orc.attention(f64(q[a:b]), c.k[s], c.v[s], 0.1, c.context[s] - (b - a), 0, None, sizes)
        bound = bound_of(want, sizes, 64, c.context[s], dtype)
        for r in rows:
            assert (np.abs(h[r] - want[r - a]) <= bound[r - a] + 1e-30).all(), (s, r)
    assert (h[32:] == 7.0).all()


@pytest.mark.parametrize("heads,n_kv", [(4, 2), (16, 1), (64, 1)])
def test_shared_on_another_stream_and_in_a_replayed_graph(pop, heads, n_kv):  # noqa: F811
    rng = np.random.default_rng(19)
    c = Grouped(pop, rng, [(3000, [3100, 3001, 3050])], n_kv, 128, 16)
    q = queries(rng, 3, heads, 128, BF16)
    want = attend_shared(pop, c, q, np.arange(4), BF16, BF16, heads, 0.09)
    assert torch.equal(want, attend_shared(pop, c, q, np.arange(4), BF16, BF16, heads, 0.09, stream=torch.cuda.Stream()))
    y, table, start, context, prefix = torch.zeros_like(q), i32(c.table), i32([0, 1, 2, 3]), i32(c.context), i32([3000])
    ws = torch.full((pop.pop_cache_attention_shared_workspace(3, 3, 3, heads, n_kv, 128, 1, LONG),), 0xFF, dtype=torch.uint8, device="cuda")

    def call():
        pop.pop_cache_attention_shared(q, BF16, 3, c.cache, n_kv, 128, 16, c.n_pages, table, table.shape[1], start, context, 3, 3, prefix, heads, 1, LONG, 0.09,
                                       y, BF16, ws)

    call()
    torch.cuda.synchronize()
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    other = torch.cuda.CUDAGraph()  # of another size, over the same workspace
    y2 = torch.zeros_like(q)
    with torch.cuda.graph(other):
        pop.pop_cache_attention_shared(q, BF16, 2, c.cache, n_kv, 128, 16, c.n_pages, table, table.shape[1], start, context, 2, 2, prefix, heads, 1, LONG, 0.09,
                                       y2, BF16, ws)
    for i in range(4):
        context.copy_(i32([3100 - i, 3001 - 7 * i, 3050 + i]))
        prefix.copy_(i32([3000 - 900 * i]))
        y.zero_()
        graph.replay()
        other.replay()
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        y.zero_()
        call()
        torch.cuda.synchronize()
        # (the third row is said to be longer than what was written: what stands there is no number, and comes out as none, the same every time)
        assert torch.equal(got.view(torch.int16), y.view(torch.int16)) and bool(y.any()) and bool(y2[:2].any())


def test_shared_calls_at_once(pop):  # noqa: F811
    """Calls on two streams, each with a workspace of its own, over one cache."""
    rng = np.random.default_rng(20)
    c = Grouped(pop, rng, [(2000, [2100, 2050, 2001, 2300])], 2, 128, 64)
    cases = []
    for heads in (4, 64):  # narrow blocks, blocks of 128
        q = queries(rng, 4, heads, 128, BF16)
        sizes = (4, 4, 4, heads, 2, 128, 1, LONG)
        ws = torch.full((pop.pop_cache_attention_shared_workspace(*sizes),), 0xFF, dtype=torch.uint8, device="cuda")
        cases.append((q, heads, ws, torch.zeros_like(q), torch.cuda.Stream(), attend_shared(pop, c, q, np.arange(5), BF16, BF16, heads, 0.1)))
    table, start, context, prefix = i32(c.table), i32(np.arange(5)), i32(c.context), i32(c.prefix)
    torch.cuda.synchronize()
    for _ in range(5):
        for q, heads, ws, y, stream, _ in cases:
            pop.pop_cache_attention_shared(q, BF16, 4, c.cache, 2, 128, 64, c.n_pages, table, table.shape[1], start, context, 4, 4, prefix, heads, 1, LONG, 0.1, y,
                                           BF16, ws, stream=stream)
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for _, _, _, y, _, want in cases)
