"""The calls around the FFN on the GPU against their 64-bit oracle: the 4-bit cache, plans, reordering, attention, beams."""
import numpy as np
import pytest
import torch

from oracle import decoder_oracle as orc

pytestmark = pytest.mark.gpu
F32, BF16 = 0, 1
DT = {F32: torch.float32, BF16: torch.bfloat16}


@pytest.fixture(scope="module")
def pop():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2602_06822_amd import binding
    return binding


def i32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()


def f64(t):
    torch.cuda.synchronize()
    return t.double().cpu().numpy()


def ints(t):
    torch.cuda.synchronize()
    return t.cpu().numpy()


# ---------------------------------------------------------------- writing and reading

def _hard_rows(rng, shape):
    """Rows with blocks of very different sizes, ties at every code, and numbers that are none."""
    x = rng.standard_normal(shape) * np.exp2(rng.integers(-100, 100, shape[:-1] + (shape[-1] // 32, 1)).repeat(32, -1).reshape(shape).astype(float))
    flat = x.reshape(-1, 32)
    ties = np.array([4.0, .25, .75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 6.5, 0, -.25, -.75, -5.0, -0.0, 1.0])
    flat[::5, :16] = ties * np.exp2(rng.integers(-40, 40, (len(flat[::5]), 1)))
    flat[::5, 16:] = 0
    flat[1::7] = 0
    flat[2::11, 3] = np.inf
    flat[3::11, 4] = -np.inf
    flat[4::11, 5] = np.nan
    flat[5::11] = 1e-44
    return x


@pytest.mark.parametrize("d,n_kv,page", [(64, 1, 16), (64, 3, 32), (128, 2, 16), (128, 5, 64), (256, 2, 128)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_write_and_read(pop, d, n_kv, page, dtype):
    rng = np.random.default_rng(d + page)
    n, n_pages = 37, 5
    wide = torch.from_numpy(_hard_rows(rng, (n, 3 * n_kv, d)).astype(np.float32)).cuda().to(DT[dtype]).view(n, -1)
    k, v = wide[:, n_kv * d:2 * n_kv * d], wide[:, 2 * n_kv * d:]
    slots = rng.permutation(n_pages * page)[:n].astype(np.int32)
    slots[5], slots[11], slots[12] = -1, n_pages * page, 2 ** 31 - 1
    bytes_ = pop.pop_cache_bytes(n_kv, d, page, n_pages)
    cache = torch.full((bytes_,), 0xA5, dtype=torch.uint8, device="cuda")
    want = np.full((n_pages, n_kv, page // 16, orc.tile_bytes(d)), 0xA5, dtype=np.uint8)
    assert want.size == bytes_
    pop.pop_cache_write(cache, n_kv, d, page, n_pages, k, v, dtype, i32(slots), n)
    kh, vh = (x.float().cpu().numpy().reshape(n, n_kv, d) for x in (k, v))
    kept = [t for t in range(n) if 0 <= slots[t] < n_pages * page]
    for t in kept:
        for h in range(n_kv):
            orc.store(want, page, d, slots[t], h, kh[t, h], vh[t, h])
    assert np.array_equal(ints(cache).reshape(want.shape), want)
    ko = torch.full((n, n_kv, d), 9.0, dtype=DT[dtype], device="cuda")
    vo = torch.full_like(ko, 9.0)
    pop.pop_cache_read(cache, n_kv, d, page, n_pages, i32(slots), n, ko, vo, dtype)
    wk, wv = np.zeros((n, n_kv, d)), np.zeros((n, n_kv, d))
    for t in kept:
        for h in range(n_kv):
            wk[t, h], wv[t, h] = orc.load(want, page, d, slots[t], h)
    assert np.array_equal(f64(ko), wk) and np.array_equal(f64(vo), wv)


# ---------------------------------------------------------------- plans

def _run_plan(pop, cached, new, page, table, ring, pool, max_tokens):
    n = len(cached)
    t, out = i32(table), [i32(np.full(m, 77)) for m in (n, n + 1, max_tokens, max_tokens, 2, 1)]
    ctx, start, slots, pos, pool_out, status = out
    pop.pop_cache_plan(i32(cached), i32(new), n, page, t, table.shape[1], i32(ring), len(ring), i32(pool), pool_out, max_tokens,
                       ctx, start, slots, pos, status)
    return ints(t), ints(ctx), ints(start), ints(slots), ints(pos), tuple(ints(pool_out)), int(ints(status)[0])


def _same(got, want):
    for i, (a, b) in enumerate(zip(got, want)):
        assert np.array_equal(np.asarray(a), np.asarray(b)), i


@pytest.mark.parametrize("n_seq,most_cached,most_new,page", [(1, 0, 1, 16), (1, 5000, 3000, 16), (3, 40, 40, 16), (8, 300, 1, 32),
                                                             (70, 50, 3, 16), (300, 100, 30, 64), (1030, 20, 2, 16), (5, 4000, 2500, 256)])
def test_plan(pop, n_seq, most_cached, most_new, page):
    for seed in range(4):
        rng = np.random.default_rng(seed * 100 + n_seq)
        cached, new = rng.integers(0, most_cached + 1, n_seq), rng.integers(0 if seed else 1, most_new + 1, n_seq)
        if seed == 3:
            new[:] = 0
        have = -(-cached // page)
        stride = int((-(-(cached + new) // page)).max()) + int(rng.integers(0, 3)) + (1 if seed == 3 else 0)
        need = int((-(-(cached + new) // page) - have).sum())
        n_pages = int(have.sum()) + need + int(rng.integers(0, 5)) + 1
        order = rng.permutation(n_pages)
        table, used = np.full((n_seq, max(stride, 1)), -1), 0
        for s in range(n_seq):
            table[s, :have[s]] = order[used:used + have[s]]
            used += have[s]
        free = order[used:]
        head = int(rng.integers(0, n_pages))
        ring = np.full(n_pages, -5)
        ring[(head + np.arange(len(free))) % n_pages] = free
        spare = int(rng.integers(0, 3))
        args = (cached, new, page, table, ring, (head, len(free)), int(new.sum()) + spare)
        got = _run_plan(pop, *args)
        assert got[-1] == 0
        _same(got, orc.plan(*args))
        if need > 0:  # one page short
            args = (cached, new, page, table, ring, (head, need - 1), int(new.sum()) + spare)
            _same(_run_plan(pop, *args), orc.plan(*args))
        if new.sum() > 0:  # one slot short
            args = (cached, new, page, table, ring, (head, len(free)), int(new.sum()) - 1)
            _same(_run_plan(pop, *args), orc.plan(*args))


@pytest.mark.parametrize("cached,new,pool", [([3, -1, 2], [1, 1, 1], (0, 6)), ([3, 0, 2], [1, -4, 1], (0, 6)), ([3, 33, 2], [1, 1, 1], (0, 6)),
                                             ([3, 2147483647, 2], [1, 2147483647, 1], (0, 6)), ([3, 0, 2], [1, 1, 1], (-1, 6)),
                                             ([3, 0, 2], [1, 1, 1], (8, 6)), ([3, 0, 2], [1, 1, 1], (0, 9)), ([3, 0, 2], [1, 1, 1], (0, -1))])
def test_plan_says_what_is_wrong(pop, cached, new, pool):
    args = (np.array(cached), np.array(new), 16, np.arange(6).reshape(3, 2), np.arange(8), pool, 5)
    got = _run_plan(pop, *args)
    assert got[-1] & 4
    _same(got[:-1], orc.plan(*args)[:-1])


def test_plan_passes_over_pages_that_are_none(pop):
    table, ring = np.array([[-1, 3], [99, -1]]), np.array([77, 2, 0, 0])
    args = (np.array([4, 16]), np.array([2, 3]), 16, table, ring, (0, 2), 6)
    got = _run_plan(pop, *args)
    assert got[3].tolist() == [-1] * 6 and got[4].tolist() == [4, 5, 16, 17, 18, -1]
    _same(got, orc.plan(*args))


# ---------------------------------------------------------------- reordering

def _run_reorder(pop, table, length, parents, n_beams, page, ring, pool):
    n, stride = table.shape
    new_table, new_len, copies = i32(np.full((n, stride), 55)), i32(np.full(n, 55)), i32(np.full((n, 2), 55))
    r, pool_out, status = i32(ring), i32([55, 55]), i32([55])
    ws = torch.full((max(pop.pop_cache_reorder_workspace(n, n_beams, stride), 16),), 0x5A, dtype=torch.uint8, device="cuda")
    pop.pop_cache_reorder(i32(table), i32(length), i32(parents), n, n_beams, page, stride, new_table, new_len, copies, r, len(ring),
                          i32(pool), pool_out, ws, status)
    return ints(new_table), ints(new_len), ints(copies), ints(r), tuple(ints(pool_out)), int(ints(status)[0])


@pytest.mark.parametrize("groups,n_beams,page,start,stride", [(1, 1, 16, 40, 9), (1, 4, 16, 30, 8), (3, 2, 32, 0, 5), (5, 5, 16, 100, 20),
                                                              (2, 16, 16, 16, 6), (3, 4, 16, 9000, 600), (300, 3, 16, 20, 6)])
def test_beams_grow_fork_and_end(pop, groups, n_beams, page, start, stride):
    """Steps of plan and reorder on the GPU, each against the oracle; no page is ever lost or held twice."""
    rng = np.random.default_rng(groups * 31 + n_beams)
    n = groups * n_beams
    n_pages = n * stride + 3
    table = np.full((n, stride), -1)
    order = rng.permutation(n_pages)
    ring, pool = order.copy(), (0, n_pages)
    length = np.zeros(n, int)
    first = np.zeros(n, int)
    first[::n_beams] = start
    for step in range(6):
        new = first if step == 0 else np.where(length > 0, rng.integers(0, 7, n), 0)
        new = np.where(length + new > stride * page, 0, new)
        args = (length, new, page, table, ring, pool, int(new.sum()) + 1)
        got = _run_plan(pop, *args)
        _same(got, orc.plan(*args))
        table, length, pool = got[0], got[1], tuple(int(x) for x in got[5])
        parents = np.zeros(n, int) if step == 0 else rng.integers(-1 if step > 2 else 0, n_beams + (step > 3), n)
        args = (table, length, parents, n_beams, page, ring, pool)
        got = _run_reorder(pop, *args)
        _same(got, orc.reorder(*args))
        assert got[-1] == 0
        table, length, ring, pool = got[0], got[1], got[3], tuple(int(x) for x in got[4])
        held = np.unique(table[table >= 0])
        free = ring[(pool[0] + np.arange(pool[1])) % n_pages]
        assert np.array_equal(np.sort(np.concatenate([held, free])), np.arange(n_pages))


def test_reorder_without_pages_changes_nothing(pop):
    table = np.array([[1, 2, -1], [1, 3, -1], [4, 5, 6], [4, 5, 7]])
    for pool, status in (((0, 1), 1), ((0, 0), 1), ((9, 2), 4), ((0, 10), 4), ((0, 9), 4)):
        args = (table, np.array([20, 20, 40, 40]), np.array([0, 0, 1, 1]), 2, 16, np.array([0, 8, 0, 0, 0, 0, 0, 0, 0]), pool)
        got = _run_reorder(pop, *args)
        assert got[-1] & status
        want = np.where(np.arange(3) < np.array([[2], [2], [3], [3]]), table, -1)
        assert np.array_equal(got[0], want) and got[1].tolist() == [20, 20, 40, 40]
        assert got[2].tolist() == [[-1, -1]] * 4 and np.array_equal(got[3], args[5]) and got[4] == pool


def test_copy_pages(pop):
    for n_kv, d, page, n_pages in ((3, 64, 16, 9), (2, 256, 64, 9), (32, 128, 16, 9)):
        size = pop.pop_cache_bytes(n_kv, d, page, n_pages)
        cache = torch.randint(0, 256, (n_pages, size // n_pages), dtype=torch.uint8, device="cuda")
        want = cache.cpu().numpy().copy()
        copies = np.array([[0, 5], [-1, -1], [1, 6], [2, 9], [9, 3], [0, 7], [4, 4], [-1, 2], [3, -1]])
        for a, b in ((0, 5), (1, 6), (0, 7)):
            want[b] = want[a]
        pop.pop_cache_copy_pages(cache, n_kv, d, page, n_pages, i32(copies), len(copies))
        assert np.array_equal(ints(cache), want)


# ---------------------------------------------------------------- attention

class Cached:
    """Sequences of given lengths in a cache whose other bytes are all ones (a scale of all ones is no number)."""

    def __init__(self, pop, rng, context, n_kv, d, page, spare=1):
        self.context, self.n_kv, self.d, self.page = list(context), n_kv, d, page
        blocks = [-(-c // page) for c in context]
        self.n_pages = sum(blocks) + 2
        order = rng.permutation(self.n_pages)
        self.table = np.full((len(context), max(blocks) + spare), -1)
        used = 0
        for s, b in enumerate(blocks):
            self.table[s, :b] = order[used:used + b]
            used += b
        self.cache = torch.full((pop.pop_cache_bytes(n_kv, d, page, self.n_pages),), 0xFF, dtype=torch.uint8, device="cuda")
        self.k, self.v = [], []
        for s, c in enumerate(context):
            k = rng.standard_normal((c, n_kv, d)) * np.where(np.arange(d) % 29 == 3, 5.0, 1.0)
            v = rng.standard_normal((c, n_kv, d)) + 0.2
            t = np.arange(c)
            slots = self.table[s, t // page] * page + t % page
            if c:
                kd, vd = (torch.from_numpy(x.astype(np.float32)).cuda() for x in (k, v))
                pop.pop_cache_write(self.cache, n_kv, d, page, self.n_pages, kd, vd, F32, i32(slots), c)
            self.k.append(orc.decode(*orc.encode(k.astype(np.float32))))
            self.v.append(orc.decode(*orc.encode(v.astype(np.float32))))


def _attend(pop, c, q, start, dtype, ydtype, heads, scale, window=0, max_new=None, max_context=None, table=None, context=None, stream=None):
    table = c.table if table is None else table
    context = c.context if context is None else context
    n_tokens, n_seq = q.shape[0], len(context)
    max_new = max(np.diff(start).max(), 1) if max_new is None else max_new
    max_context = max(max(context), 1) if max_context is None else max_context
    y = torch.full(q.shape, 7.0, dtype=DT[ydtype], device="cuda")
    ws = torch.full((pop.pop_cache_attention_workspace(n_tokens, n_seq, heads, c.n_kv, c.d, max_new, max_context) + 16,), 0xFF, dtype=torch.uint8,
                    device="cuda")
    args = (q, dtype, n_tokens, c.cache, c.n_kv, c.d, c.page, c.n_pages, i32(table), table.shape[1], i32(start), i32(context), n_seq,
            heads, max_new, max_context, scale, window, y, ydtype, ws)
    torch.cuda.synchronize()
    pop.pop_cache_attention(*args, stream=stream)
    if stream is not None:
        torch.cuda.synchronize()  # (the caller's own stream does not wait for this one)
    return y


def _check(c, y, q, start, dtype, ydtype, scale, window=0, there=None, context=None):
    """Bounds: products and sums in 32 bits (the scores' error turns into a relative one of the weights), weights rounded to
    bf16 where the output is bf16, the output's own rounding (bf16 keeps 8 significant bits: to nearest is up to 2^-8 of a number)."""
    y, qh = f64(y), f64(q)
    context = c.context if context is None else context
    for s, length in enumerate(context):
        a, b = start[s], start[s + 1]
        sizes = []
        k, v = c.k[s][:length], c.v[s][:length]
        want = orc.attention(qh[a:b], k, v, scale, length - (b - a), window, None if there is None else there[s][:length], sizes)
        weight, product = sizes
        scores = (c.d + 8) * 2.0 ** -24 * product
        bound = weight * (2 * scores + (length + 32) * 2.0 ** -24 + 2.0 ** -21) + 2.0 ** -23 * np.abs(want)
        if ydtype == BF16:
            bound = bound + 2.0 ** -8 * weight + 2.0 ** -8 * np.abs(want)
        off = np.abs(y[a:b] - want) - bound
        assert (off <= 1e-30).all(), (s, float(off.max()), np.unravel_index(off.argmax(), off.shape))


def _queries(rng, n, heads, d, dtype):
    return torch.from_numpy((1.5 * rng.standard_normal((n, heads, d))).astype(np.float32)).cuda().to(DT[dtype])


TYPES = [(BF16, BF16), (BF16, F32), (F32, F32), (F32, BF16)]


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype,ydtype", TYPES)
def test_single_tokens(pop, d, dtype, ydtype):
    """Lengths around the tile, the step and the page; an empty sequence; one that is split over workgroups."""
    rng = np.random.default_rng(d)
    for heads, n_kv, page in ((2, 2, 16), (6, 2, 32), (16, 1, 64), (20, 1, 16)):
        c = Cached(pop, rng, [1, 2, 15, 16, 17, 31, 33, 64, 65, 0, 129, 700], n_kv, d, page)
        start = np.concatenate([[0], np.cumsum([0 if x == 0 else 1 for x in c.context])])
        q = _queries(rng, start[-1], heads, d, dtype)
        y = _attend(pop, c, q, start, dtype, ydtype, heads, d ** -0.5)
        _check(c, y, q, start, dtype, ydtype, d ** -0.5)


@pytest.mark.parametrize("dtype,ydtype", [(BF16, BF16), (F32, F32)])
@pytest.mark.parametrize("window", [0, 1, 20, 100])
def test_chunks_of_prompts(pop, dtype, ydtype, window):
    rng = np.random.default_rng(window)
    for heads, n_kv, d, page, context, new in ((4, 4, 128, 16, [40, 7, 200, 90], [40, 3, 100, 1]), (6, 2, 64, 64, [130, 64, 33], [70, 64, 5]),
                                               (2, 1, 256, 16, [75], [75]), (5, 1, 128, 32, [300, 1], [150, 1])):
        c = Cached(pop, rng, context, n_kv, d, page)
        start = np.concatenate([[0], np.cumsum(new)])
        q = _queries(rng, start[-1], heads, d, dtype)
        y = _attend(pop, c, q, start, dtype, ydtype, heads, 0.07, window)
        _check(c, y, q, start, dtype, ydtype, 0.07, window)
        # sizes that the caller underestimates
        y = _attend(pop, c, q, start, dtype, ydtype, heads, 0.07, window, max_new=1, max_context=1)
        _check(c, y, q, start, dtype, ydtype, 0.07, window)


@pytest.mark.parametrize("dtype,ydtype", [(BF16, BF16), (F32, F32)])
@pytest.mark.parametrize("context,new", [([20000], [1]), ([5000, 300], [2, 1]), ([3000], [33])])
def test_long_sequences_are_split(pop, dtype, ydtype, context, new):
    rng = np.random.default_rng(context[0])
    c = Cached(pop, rng, context, 2, 128, 64)
    start = np.concatenate([[0], np.cumsum(new)])
    q = _queries(rng, start[-1], 4, 128, dtype)
    assert pop.pop_cache_attention_workspace(int(start[-1]), len(new), 4, 2, 128, max(new), max(context)) > 0
    y = _attend(pop, c, q, start, dtype, ydtype, 4, 128 ** -0.5)
    _check(c, y, q, start, dtype, ydtype, 128 ** -0.5)
    again = _attend(pop, c, q, start, dtype, ydtype, 4, 128 ** -0.5)
    assert torch.equal(y, again)


@pytest.mark.parametrize("dtype,ydtype", [(BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("window", [0, 333])
@pytest.mark.parametrize("heads,n_kv,d", [(4, 2, 128), (3, 1, 64), (2, 2, 256)])
def test_long_chunks_of_few_heads(pop, dtype, ydtype, window, heads, n_kv, d):
    """Chunks whose tokens are split over workgroups, with a hole, and sizes that the caller underestimates in part."""
    rng = np.random.default_rng(d + window)
    context, new = [2100, 900, 130], [130, 65, 130]
    c = Cached(pop, rng, context, n_kv, d, 32)
    table = c.table.copy()
    table[0, [5, 40]] = -1
    there = [np.repeat((t >= 0) & (t < c.n_pages), 32) for t in table]
    start = np.concatenate([[0], np.cumsum(new)])
    q = _queries(rng, start[-1], heads, d, dtype)
    for max_new, max_context in ((130, 2100), (70, 2100), (130, 1000), (64, 600)):
        y = _attend(pop, c, q, start, dtype, ydtype, heads, 0.08, window, max_new=max_new, max_context=max_context, table=table)
        _check(c, y, q, start, dtype, ydtype, 0.08, window, there=there)


@pytest.mark.parametrize("new", [1, 40])
def test_pages_that_are_none_and_rows_that_see_nothing(pop, new):
    rng = np.random.default_rng(new)
    c = Cached(pop, rng, [200, 150, 90, 60], 2, 128, 16)
    table = c.table.copy()
    table[0, 3], table[0, 12] = -1, c.n_pages  # a hole, and the last page
    table[1, :] = -1                           # nothing at all
    table[2, :2] = -7                          # pages that a window has left
    start = np.concatenate([[0], np.cumsum([new] * 4)])
    context = [200, 150, 90, new - 1 if new > 1 else 0]  # the last one is shorter than its new tokens
    q = _queries(rng, start[-1] + 2, 4, 128, BF16)
    there = [np.repeat((t >= 0) & (t < c.n_pages), 16) for t in table]
    for ydtype in (BF16, F32):
        y = _attend(pop, c, q, start, BF16, ydtype, 4, 0.1, table=table, context=context)
        _check(c, y, q, start, BF16, ydtype, 0.1, there=there, context=context)
        h = f64(y)
        assert (h[start[1]:start[2]] == 0).all() and (h[start[3]] == 0).all()
        assert (h[start[-1]:] == 7.0).all()  # rows of no sequence


def test_a_table_that_is_shorter_than_its_context(pop):
    rng = np.random.default_rng(8)
    c = Cached(pop, rng, [64], 1, 64, 16, spare=0)
    q = _queries(rng, 1, 1, 64, F32)
    y = _attend(pop, c, q, np.array([0, 1]), F32, F32, 1, 0.1, context=[5000])  # position 4999 sees the 64 tokens there are
    want = orc.attention(f64(q), c.k[0], c.v[0], 0.1, 4999)
    assert np.abs(f64(y) - want).max() < 1e-5


def test_large_and_small_scores(pop):
    """Maxima that move by more than the kernel's slack, from both ends, and a scale that makes all weights equal."""
    rng = np.random.default_rng(9)
    c = Cached(pop, rng, [333], 1, 128, 16)
    for scale in (0.0, 3.0, -3.0, 40.0):
        for dtype, ydtype in ((BF16, F32), (F32, F32)):
            q = _queries(rng, 5, 2, 128, dtype)
            y = _attend(pop, c, q, np.array([0, 5]), dtype, ydtype, 2, scale)
            _check(c, y, q, np.array([0, 5]), dtype, ydtype, scale)


def test_another_stream_and_a_replayed_graph(pop):
    rng = np.random.default_rng(10)
    c = Cached(pop, rng, [3000, 77], 2, 128, 16)
    start = np.array([0, 1, 2])
    q = _queries(rng, 2, 4, 128, BF16)
    want = _attend(pop, c, q, start, BF16, BF16, 4, 0.09)
    other = torch.cuda.Stream()
    assert torch.equal(_attend(pop, c, q, start, BF16, BF16, 4, 0.09, stream=other), want)
    torch.cuda.synchronize()
    # captured: plan, write, attention and selection of a step; new inputs before every replay
    ring, pool, pool2 = i32(np.arange(8)), i32([0, 8]), i32([0, 0])
    table = i32(np.full((1, 4), -1))
    cached, new = i32([0]), i32([20])
    ctx, st, slots, status = i32([0]), i32([0, 0]), i32(np.zeros(20)), i32([0])
    cache = torch.zeros(pop.pop_cache_bytes(1, 64, 16, 8), dtype=torch.uint8, device="cuda")
    kv = torch.zeros(20, 128, device="cuda")
    q1, y1 = torch.zeros(20, 2, 64, device="cuda"), torch.zeros(20, 2, 64, device="cuda")
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    logits, was = torch.zeros(2, 900, device="cuda"), torch.zeros(2, device="cuda")
    so, to, po = torch.zeros(3, device="cuda"), i32([0] * 3), i32([0] * 3)

    def step(s):
        pop.pop_cache_plan(cached, new, 1, 16, table, 4, ring, 8, pool, pool2, 20, ctx, st, slots, None, status, stream=s)
        pop.pop_cache_write(cache, 1, 64, 16, 8, kv[:, :64], kv[:, 64:], F32, slots, 20, stream=s)
        pop.pop_cache_attention(q1, F32, 20, cache, 1, 64, 16, 8, table, 4, st, ctx, 1, 2, 20, 20, 0.2, 0, y1, F32, ws, stream=s)
        pop.pop_beam_select(logits, F32, was, None, 1, 2, 900, 3, 0, so, to, po, ws, stream=s)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(torch.cuda.current_stream())
    for i in range(4):
        g = torch.Generator(device="cuda").manual_seed(i)
        for t in (kv, q1, logits, was):
            t.normal_(generator=g)
        new.fill_(17 + i)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y1[:17 + i], slots, so, to, po, cache)]
        for t in (y1, slots, so, to, po):
            t.zero_()
        step(torch.cuda.current_stream())
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (y1[:17 + i], slots, so, to, po, cache)))


LARGE = dict(max_new=2048, max_context=1 << 19)  # sizes for which blocks of 128 columns are taken, whatever the chunks really have


@pytest.mark.parametrize("window", [0, 60])
@pytest.mark.parametrize("heads,n_kv,d,page,context,new", [
    (4, 4, 128, 16, [240, 7, 400, 0], [200, 3, 380, 0]), (6, 2, 64, 64, [130, 64, 33], [70, 64, 5]), (5, 1, 128, 32, [300, 1], [150, 1]),
    (2, 1, 128, 64, [2900, 65], [130, 65]), (3, 3, 64, 32, [1500], [97]), (16, 1, 64, 16, [63, 64, 65, 127, 129], [9, 8, 7, 33, 5])])
def test_blocks_of_128_columns(pop, window, heads, n_kv, d, page, context, new):
    rng = np.random.default_rng(d + window + len(context))
    c = Cached(pop, rng, context, n_kv, d, page)
    start = np.concatenate([[0], np.cumsum(new)])
    q = _queries(rng, start[-1], heads, d, BF16)
    for scale in (0.07, -0.4, 0.0):
        y = _attend(pop, c, q, start, BF16, BF16, heads, scale, window, **LARGE)
        _check(c, y, q, start, BF16, BF16, scale, window)
    assert torch.equal(y, _attend(pop, c, q, start, BF16, BF16, heads, scale, window, **LARGE))
    # pages that are none, a context shorter than its new tokens
    table = c.table.copy()
    table[0, ::3] = -1
    there = [np.repeat((t >= 0) & (t < c.n_pages), page) for t in table]
    y = _attend(pop, c, q, start, BF16, BF16, heads, 0.07, window, table=table, **LARGE)
    _check(c, y, q, start, BF16, BF16, 0.07, window, there=there)
    short = [new[0] // 2] + context[1:]
    y = _attend(pop, c, q, start, BF16, BF16, heads, 0.07, window, context=short, **LARGE)
    _check(c, y, q, start, BF16, BF16, 0.07, window, context=short)
    assert (f64(y)[: new[0] - new[0] // 2] == 0).all()


@pytest.mark.parametrize("page,window", [(16, 0), (32, 77)])
def test_blocks_of_128_columns_with_the_widest_heads(pop, page, window):
    rng = np.random.default_rng(page + 1)
    c = Cached(pop, rng, [301, 200], 64, 256, page)
    start = np.array([0, 250, 450])
    q = _queries(rng, 450, 64, 256, BF16)
    table = c.table.copy()
    table[0, 64 // page] = -1
    there = [np.repeat((t >= 0) & (t < c.n_pages), page) for t in table]
    y = _attend(pop, c, q, start, BF16, BF16, 64, 0.06, window, table=table, **LARGE)
    _check(c, y, q, start, BF16, BF16, 0.06, window, there=there)


def test_blocks_of_128_columns_in_a_replayed_graph(pop):
    """Units that several workgroups share; other work uses the workspace in between."""
    rng = np.random.default_rng(13)
    c = Cached(pop, rng, [2900, 300], 2, 128, 32)
    start = np.array([0, 64, 94])
    q, y = _queries(rng, 94, 8, 128, BF16), torch.zeros(94, 8, 128, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(pop.pop_cache_attention_workspace(94, 2, 8, 2, 128, *LARGE.values()), dtype=torch.uint8, device="cuda")
    table, starts, context = i32(c.table), i32(start), i32(c.context)

    def attend(s):
        pop.pop_cache_attention(q, BF16, 94, c.cache, 2, 128, 32, c.n_pages, table, c.table.shape[1], starts, context, 2, 8, *LARGE.values(), 0.09, 0,
                                y, BF16, ws, stream=s)

    attend(torch.cuda.current_stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        attend(torch.cuda.current_stream())
    for i in range(4):
        q.normal_(generator=torch.Generator(device="cuda").manual_seed(i))
        ws.fill_(255 - i)
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        _check(c, got, q, start, BF16, BF16, 0.09)
        attend(torch.cuda.current_stream())
        torch.cuda.synchronize()
        assert torch.equal(got, y)


@pytest.mark.parametrize("dtype,ydtype", [(BF16, BF16), (F32, F32)])
@pytest.mark.parametrize("n_seq,longest,window", [(150, 0, 0), (150, 9000, 0), (40, 3000, 700), (70, 1100, 0), (260, 0, 31)])
def test_many_sequences(pop, dtype, ydtype, n_seq, longest, window):
    """Dealt by whole units and by pieces; several sequences to a lane; empty ones and ones without new tokens."""
    rng = np.random.default_rng(n_seq + longest)
    context = rng.integers(0, 300, n_seq)
    context[rng.integers(0, n_seq)] = max(longest, 1)
    new = np.minimum(rng.integers(0, 4, n_seq), context)
    c = Cached(pop, rng, context.tolist(), 3, 64, 16)
    start = np.concatenate([[0], np.cumsum(new)])
    q = _queries(rng, start[-1], 9, 64, dtype)
    y = _attend(pop, c, q, start, dtype, ydtype, 9, 0.125, window)
    _check(c, y, q, start, dtype, ydtype, 0.125, window)
    assert torch.equal(y, _attend(pop, c, q, start, dtype, ydtype, 9, 0.125, window))


@pytest.mark.parametrize("page,window", [(16, 0), (32, 77)])
def test_chunks_with_the_widest_heads(pop, page, window):
    """Units for every compute unit; a page that is none, a context shorter than the chunk, an empty sequence."""
    rng = np.random.default_rng(page)
    c = Cached(pop, rng, [401, 130, 0, 257], 64, 256, page)
    start = np.array([0, 129, 259, 259, 389])
    q = _queries(rng, 389, 64, 256, BF16)
    y = _attend(pop, c, q, start, BF16, BF16, 64, 0.06, window)
    _check(c, y, q, start, BF16, BF16, 0.06, window)
    table = c.table.copy()
    table[0, 64 // page] = -1
    there = [np.arange(n) // page != 64 // page if s == 0 else np.ones(n, dtype=bool) for s, n in enumerate(c.context)]
    y = _attend(pop, c, q, start, BF16, BF16, 64, 0.06, window, table=table)
    _check(c, y, q, start, BF16, BF16, 0.06, window, there)
    short = [401, 60, 0, 257]
    y = _attend(pop, c, q, start, BF16, BF16, 64, 0.06, window, context=short, max_new=130)
    _check(c, y, q, start, BF16, BF16, 0.06, window, context=short)


@pytest.mark.parametrize("new", [[1, 1], [64, 30]])
def test_pieces_are_joined_in_a_replayed_graph(pop, new):
    """Units that several workgroups share, captured; other work uses the workspace in between."""
    rng = np.random.default_rng(11)
    c = Cached(pop, rng, [2900, 300], 2, 128, 32)
    start = np.concatenate([[0], np.cumsum(new)])
    q, y = _queries(rng, start[-1], 8, 128, BF16), torch.zeros(start[-1], 8, 128, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(pop.pop_cache_attention_workspace(start[-1], 2, 8, 2, 128, max(new), 2900), dtype=torch.uint8, device="cuda")
    table, starts, context = i32(c.table), i32(start), i32(c.context)

    def attend(s):
        pop.pop_cache_attention(q, BF16, start[-1], c.cache, 2, 128, 32, c.n_pages, table, c.table.shape[1], starts, context, 2, 8, max(new), 2900,
                                0.09, 0, y, BF16, ws, stream=s)

    attend(torch.cuda.current_stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        attend(torch.cuda.current_stream())
    for i in range(4):
        q.normal_(generator=torch.Generator(device="cuda").manual_seed(i))
        ws.fill_(255 - i)
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        _check(c, got, q, start, BF16, BF16, 0.09)
        attend(torch.cuda.current_stream())
        torch.cuda.synchronize()
        assert torch.equal(got, y)


def test_offsets_beyond_32_bits(pop):
    """The last pages of a cache of more than 4 GB."""
    n_kv, d, page = 8, 128, 64
    n_pages = (5 << 30) // pop.pop_cache_bytes(n_kv, d, page, 1)
    rng = np.random.default_rng(12)
    c = Cached(pop, rng, [1], n_kv, d, page)
    c.n_pages = n_pages
    c.cache = torch.full((pop.pop_cache_bytes(n_kv, d, page, n_pages),), 0xFF, dtype=torch.uint8, device="cuda")
    length = 150
    c.context, c.table = [length], np.array([[n_pages - 1, n_pages - 3, n_pages - 2]])
    k, v = (rng.standard_normal((length, n_kv, d)).astype(np.float32) for _ in range(2))
    slots = c.table[0, np.arange(length) // page] * page + np.arange(length) % page
    pop.pop_cache_write(c.cache, n_kv, d, page, n_pages, torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), F32, i32(slots), length)
    c.k, c.v = [orc.decode(*orc.encode(k))], [orc.decode(*orc.encode(v))]
    ko, vo = torch.zeros(length, n_kv, d, device="cuda"), torch.zeros(length, n_kv, d, device="cuda")
    pop.pop_cache_read(c.cache, n_kv, d, page, n_pages, i32(slots), length, ko, vo, F32)
    assert np.array_equal(f64(ko), c.k[0]) and np.array_equal(f64(vo), c.v[0])
    for new in (1, 40):
        q = _queries(rng, new, 16, d, BF16)
        y = _attend(pop, c, q, np.array([0, new]), BF16, BF16, 16, 0.08)
        _check(c, y, q, np.array([0, new]), BF16, BF16, 0.08)
    pop.pop_cache_copy_pages(c.cache, n_kv, d, page, n_pages, i32([[n_pages - 1, n_pages - 9]]), 1)
    slots = slots[:page] - 8 * page
    pop.pop_cache_read(c.cache, n_kv, d, page, n_pages, i32(slots), page, ko[:page], vo[:page], F32)
    assert np.array_equal(f64(ko[:page]), c.k[0][:page])


# ---------------------------------------------------------------- beams

def _select(pop, logits, dtype, scores, done, beams, k, pad):
    r = logits.shape[0] // beams
    so = torch.full((r, k), 5.0, device="cuda")
    to, po = i32(np.full((r, k), 55)), i32(np.full((r, k), 55))
    ws = torch.full((pop.pop_beam_workspace(r, beams, logits.shape[1], k),), 0xFF, dtype=torch.uint8, device="cuda")
    pop.pop_beam_select(logits, dtype, scores, done, r, beams, logits.shape[1], k, pad, so, to, po, ws)
    return f64(so), ints(to), ints(po)


def _check_beams(logits, scores, done, beams, k, pad, got):
    """Scores: 32-bit sums of up to 2^24 terms in blocks (relative 2^-18 of the sum, absolute in its logarithm), and roundings of numbers
    of their size.  Order: exact wherever neighbouring scores differ by more than that or are equal in 64 bits."""
    x, was = f64(logits), f64(scores)
    dn = None if done is None else ints(done)
    for i in range(x.shape[0] // beams):
        rows = slice(i * beams, (i + 1) * beams)
        s, t, p = orc.beam_select(x[rows], was[rows], None if dn is None else dn[rows], k + 1, pad)
        n = min(k, len(s))
        fin = np.isfinite(s[:n])
        size = np.abs(was[rows][np.isfinite(was[rows])]).max(initial=0) + np.abs(np.where(np.isfinite(x[rows]), x[rows], 0)).max() + 20
        tol = 2.0 ** -18 + 2.0 ** -21 * size
        assert np.array_equal(np.isfinite(got[0][i][:n]), fin)
        assert (np.abs(got[0][i][:n] - s[:n])[fin] <= tol).all()
        gaps = s[:-1] - s[1:] if np.isfinite(s).all() else np.where(np.isfinite(s[:-1]) & np.isfinite(s[1:]), np.diff(-np.where(np.isfinite(s), s, 0)), 0)
        clear = (np.abs(gaps) > 2 * tol) | (gaps == 0)
        assert clear.all(), "the test's own scores nearly tie"
        assert np.array_equal(got[1][i][:n], t[:n]) and np.array_equal(got[2][i][:n], p[:n])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("requests,beams,vocab,k", [(1, 1, 1, 1), (1, 1, 7, 7), (2, 3, 100, 6), (1, 4, 2048, 4), (3, 4, 2049, 8), (2, 8, 8191, 16),
                                                    (5, 2, 32000, 64), (1, 16, 5003, 32), (300, 8, 2500, 8)])
def test_selection(pop, dtype, requests, beams, vocab, k):
    rng = np.random.default_rng(vocab)
    # logits on a grid, so that scores of one beam tie exactly or not at all; beams' own scores far from each other's sums
    x = np.round(rng.standard_normal((requests * beams, vocab)) * 16) / 8
    for row in x:  # a few that stand out, all different
        at = rng.permutation(vocab)[:min(vocab, 2 * k)]
        row[at] = 5.0 + rng.permutation(len(at)) / 16
    logits = torch.from_numpy(x.astype(np.float32)).cuda().to(DT[dtype])
    scores = torch.from_numpy((-0.0137 * rng.permutation(requests * beams) - 0.5).astype(np.float32)).cuda()
    done = torch.from_numpy((rng.random(requests * beams) < 0.15).astype(np.uint8)).cuda()
    for dn in (None, done):
        got = _select(pop, logits, dtype, scores, dn, beams, k, vocab // 2)
        try:
            _check_beams(logits, scores, dn, beams, k, vocab // 2, got)
        except AssertionError as e:
            if "nearly tie" not in str(e):
                raise
            scores2 = scores - 0.00071 * torch.arange(requests * beams, device="cuda") ** 1.5
            _check_beams(logits, scores2, dn, beams, k, vocab // 2, _select(pop, logits, dtype, scores2, dn, beams, k, vocab // 2))


@pytest.mark.parametrize("vocab", [50, 2500, 40001])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_equal_and_forbidden_logits(pop, dtype, vocab):
    """Rows of one value, rows with three allowed tokens or none, beams that are not alive, NaN."""
    x = torch.zeros(8, vocab)
    x[1] = -torch.inf
    x[1, [vocab - 1, 3, vocab // 2]] = torch.tensor([1.0, 1.0, 0.5])
    x[2] = -torch.inf
    x[3, ::2] = float("nan")
    x[4, -2:] = 1.0
    x[5] = torch.arange(vocab) % 7 / 8.0
    x = x.cuda().to(DT[dtype])
    was = torch.tensor([-1.0, -30.0, -2.0, -64.0, -90.0, -120.0, -torch.inf, -200.0], device="cuda")
    done = torch.tensor([0, 0, 0, 0, 0, 0, 0, 1], dtype=torch.uint8, device="cuda")
    for k in (1, 5, 16, 64):
        for beams in (1, 2, 8):
            if k > beams * vocab:
                continue
            got = _select(pop, x, dtype, was, done, beams, k, 4)
            _check_beams(x, was, done, beams, k, 4, got)


def test_selection_over_many_tiles_of_candidates(pop):
    """16 beams x many stretches x 64 candidates: the joining workgroup takes them in several tiles."""
    rng = np.random.default_rng(4)
    x = torch.from_numpy((np.round(rng.standard_normal((16, 150000)) * 64) / 64).astype(np.float32)).cuda()
    was = torch.from_numpy((-8.3 * np.arange(16)).astype(np.float32)).cuda()
    _check_beams(x, was, None, 16, 64, 0, _select(pop, x, F32, was, None, 16, 64, 0))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [70, 2500, 33001])
def test_logits_of_lowest_and_largest_values(pop, dtype, vocab):
    """Rows that are masked with finite values, whole and in part, rows far from zero, and a row of largest values."""
    low = float(torch.finfo(DT[dtype]).min)
    x = torch.zeros(8, vocab)
    x[0] = low                       # masked whole: every token is as likely as the others
    x[1] = low
    x[1, [3, vocab // 2, vocab - 1]] = torch.tensor([1.0, 0.5, 0.25])
    x[2] = -1e30
    x[3] = -1e10
    x[3, vocab // 3] = 0.0
    x[4] = -low
    x[5] = low / 2
    x[5, :vocab // 2] = low
    x[6] = -torch.inf
    x[6, 1:9] = low
    x[7, 5] = -low                   # the others' scores are lower than float32 goes
    x = x.cuda().to(DT[dtype])
    was = torch.tensor([-3.0, -9.0, -30.0, -50.0, -70.0, -90.0, -110.0, -130.0], device="cuda")
    h = f64(was)
    for beams in (1, 2, 8):
        for k in (1, 4, 16):
            so, to, po = _select(pop, x, dtype, was, None, beams, k, 0)
            for i in range(8 // beams):
                rows = slice(i * beams, (i + 1) * beams)
                s, t, p = orc.beam_select(f64(x[rows]), h[rows], None, k, 0)
                with np.errstate(over="ignore"):
                    s = s.astype(np.float32).astype(np.float64)
                assert np.array_equal(so[i] == -np.inf, s == -np.inf)
                fin = np.isfinite(s)
                # 32-bit sums of exponentials (2^-18 of the sum, as above) and roundings of the score
                assert (np.abs(so[i][fin] - s[fin]) <= 2.0 ** -18 + 2.0 ** -21 * np.abs(s[fin])).all()
                assert np.array_equal(to[i], t) and np.array_equal(po[i], p)


@pytest.mark.parametrize("length,page", [(-1, 16), (49, 16), (2147483647, 16), (-2147483648, 64)])
@pytest.mark.parametrize("groups,stride", [(1, 3), (3, 3), (2, 300)])
def test_reorder_says_which_lengths_are_wrong(pop, length, page, groups, stride):
    """Negative lengths and those that a table's row has no room for, in a row that goes on and in one that does not."""
    for at in (0, 2 * groups - 1):
        n = 2 * groups
        lengths = np.full(n, 20)
        lengths[at] = length if length != 49 else stride * page + 1
        table = np.arange(n * stride).reshape(n, stride)
        n_pages = n * stride + 4
        for parents in (np.zeros(n, int), np.ones(n, int), np.full(n, -1)):
            args = (table, lengths, parents, 2, page, np.concatenate([np.arange(n * stride, n_pages), np.zeros(n * stride, int)]), (0, 4))
            got = _run_reorder(pop, *args)
            assert got[-1] == 4
            _same(got, orc.reorder(*args))
            assert np.array_equal(got[1], lengths) and (got[2] == -1).all() and got[4] == (0, 4) and np.array_equal(got[3], args[5])


def test_reorder_of_last_pages_that_are_none(pop):
    """What a row did not see its children do not see: no page is taken to copy one that there is not."""
    table = np.array([[1, -1, -1], [1, 77, -1], [4, 5, 6], [4, 5, 7]])
    args = (table, np.array([20, 20, 40, 40]), np.array([0, 0, 1, 1]), 2, 16, np.array([0, 8, 2, 3, 0, 0, 0, 0, 0]), (0, 4))
    got = _run_reorder(pop, *args)
    _same(got, orc.reorder(*args))
    assert got[2].tolist() == [[-1, -1], [-1, -1], [-1, -1], [7, 0]] and got[0][1].tolist() == [1, -1, -1]
    # a ring that holds what is no page: the child has none either, and does not write to its parent's
    args = args[:5] + (np.array([-5, 8, 2, 3, 0, 0, 0, 0, 0]), (0, 4))
    got = _run_reorder(pop, *args)
    _same(got, orc.reorder(*args))
    assert got[0][3].tolist() == [4, 5, -5]


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype,ydtype", TYPES)
def test_scores_far_from_zero(pop, d, dtype, ydtype):
    """Keys of up to 1.5 x 2^116 in all tokens, or in one beside zeros: scores of 2^29 to 2^125, of either sign.  Products and their sums
    are exact in 32 bits, so that scores have no error (and stored values are written again as they are)."""
    rng = np.random.default_rng(d + 1)
    for heads, n_kv, new, kw in ((2, 1, 1, {}), (4, 2, 3, {}), (8, 1, 40, dict(max_new=2048, max_context=1 << 19))):
        c = Cached(pop, rng, [300, 2000], n_kv, d, 16)
        start = np.array([0, new, 2 * new])
        q = torch.ones(2 * new, heads, d, device="cuda", dtype=DT[dtype])
        for size in (1.5 * 2.0 ** 23, 1.5 * 2.0 ** 60, 1.5 * 2.0 ** 116):
            for alike in (False, True):
                for s, length in enumerate(c.context):
                    k = np.full((length, n_kv, d), size if alike else 0.0, dtype=np.float32)
                    if not alike:
                        k[length // 3], k[length // 2] = size, -size
                    t = np.arange(length)
                    slots = c.table[s, t // c.page] * c.page + t % c.page
                    kd, vd = (torch.from_numpy(x.astype(np.float32)).cuda() for x in (k, c.v[s]))
                    pop.pop_cache_write(c.cache, n_kv, d, c.page, c.n_pages, kd, vd, F32, i32(slots), length)
                    c.k[s] = k
                for scale in (1.0, -0.75):
                    h = f64(_attend(pop, c, q, start, dtype, ydtype, heads, scale, **kw))
                    for s, length in enumerate(c.context):
                        sizes = []
                        a, b = start[s], start[s + 1]
                        want = orc.attention(f64(q[a:b]), c.k[s], c.v[s], scale, length - new, 0, None, sizes)
                        bound = sizes[0] * ((length + 32) * 2.0 ** -24 + 2.0 ** -21) + 2.0 ** -23 * np.abs(want)  # (as in _check, of exact scores)
                        if ydtype == BF16:
                            bound = bound + 2.0 ** -8 * sizes[0] + 2.0 ** -8 * np.abs(want)
                        assert (np.abs(h[a:b] - want) <= bound + 1e-30).all(), (heads, size, alike, scale, s)


def test_pages_of_more_than_32_bits(pop):
    """Two pages of 4.3 GB, of which the second holds the tokens of three heads and zeros for the others."""
    n_kv, d, page = 62000, 256, 256
    rng = np.random.default_rng(14)
    cache = torch.zeros(pop.pop_cache_bytes(n_kv, d, page, 2), dtype=torch.uint8, device="cuda")
    assert cache.numel() > 2 << 32
    heads = [0, 30000, n_kv - 1]
    kh, vh = (rng.standard_normal((2, 3, d)).astype(np.float32) for _ in range(2))
    k, v = torch.zeros(2, n_kv, d, device="cuda"), torch.zeros(2, n_kv, d, device="cuda")
    k[:, heads], v[:, heads] = torch.from_numpy(kh).cuda(), torch.from_numpy(vh).cuda()
    pop.pop_cache_write(cache, n_kv, d, page, 2, k, v, F32, i32([page, page + 1]), 2)
    q = torch.zeros(1, n_kv, d, device="cuda")
    q[0, heads] = torch.from_numpy(rng.standard_normal((3, d)).astype(np.float32)).cuda()
    y = torch.full_like(q, 7.0)
    ws = torch.empty(pop.pop_cache_attention_workspace(1, 1, n_kv, n_kv, d, 1, 2), dtype=torch.uint8, device="cuda")
    pop.pop_cache_attention(q, F32, 1, cache, n_kv, d, page, 2, i32([[1]]), 1, i32([0, 1]), i32([2]), 1, n_kv, 1, 2, 0.1, 0, y, F32, ws)
    want = orc.attention(f64(q[:, heads]), orc.decode(*orc.encode(kh)), orc.decode(*orc.encode(vh)), 0.1, 1)
    # 32-bit sums of 256 products below 4 x 4, and two weights
    assert np.abs(f64(y[:, heads]) - want).max() < 1e-5
    y[:, heads] = 0
    assert not y.any()


@pytest.mark.parametrize("shape", [(5, 192), (5, 3, 64), (7, 192), (5, 128), (5, 2, 64), (10, 64), (1, 5, 2, 64), (1, 640), (640,), (9, 2, 64), (1, 5, 192)])
def test_write_takes_rows_as_a_tensor_has_them(pop, shape):
    """Contiguous tensors of 5 tokens of 2 heads of 64, some with longer rows or more of them, or with axes of their own."""
    x = torch.arange(int(np.prod(shape)), device="cuda").remainder(5).float().sub_(2.0).view(shape)  # (-2 .. 2: kept as they are)
    width = shape[-1] if shape[-1] == 192 else 192 if shape[1:] == (3, 64) else 128
    want = f64(x).reshape(-1, width)[:5, :128]
    cache = torch.zeros(pop.pop_cache_bytes(2, 64, 16, 1), dtype=torch.uint8, device="cuda")
    ko, vo = torch.zeros(5, 2, 64, device="cuda"), torch.zeros(5, 2, 64, device="cuda")
    slots = i32(np.arange(5))
    pop.pop_cache_write(cache, 2, 64, 16, 1, x, x, F32, slots, 5)
    pop.pop_cache_read(cache, 2, 64, 16, 1, slots, 5, ko, vo, F32)
    assert np.array_equal(f64(ko).reshape(5, 128), want) and np.array_equal(f64(vo).reshape(5, 128), want)


def _attend_in_blocks(pop, c, q, start, heads, scale, window=0, max_new=1 << 19, max_context=1 << 19, parts=None, **kw):
    """_attend with sizes that take blocks of 128 columns, which is asked of the library: a rule that changes does not take the test with it."""
    kind, got = pop.pop_cache_attention_kind(BF16, BF16, q.shape[0], len(c.context), heads, c.n_kv, c.d, max_new, max_context, window)
    assert kind == 2 and (parts is None or (got > 1) == parts), (kind, got)
    return _attend(pop, c, q, start, BF16, BF16, heads, scale, window, max_new=max_new, max_context=max_context, **kw)


@pytest.mark.parametrize("window", [1, 60, 333])
@pytest.mark.parametrize("heads,n_kv,d,page,context,new", [
    (4, 4, 128, 16, [240, 7, 400, 0], [200, 3, 380, 0]), (6, 2, 64, 64, [130, 64, 33], [70, 64, 5]), (5, 1, 128, 32, [300, 1], [150, 1]),
    (2, 1, 128, 64, [2900, 65], [130, 65]), (3, 3, 64, 32, [1500], [97]), (16, 1, 64, 16, [63, 64, 65, 127, 129], [9, 8, 7, 33, 5]),
    (4, 2, 128, 256, [2100, 900, 130], [130, 65, 130])])
def test_windows_in_blocks_of_128_columns(pop, window, heads, n_kv, d, page, context, new):
    """Blocks that begin behind the first token, whole and in parts; pages that are none; a context shorter than its new tokens."""
    rng = np.random.default_rng(d + window + len(context))
    c = Cached(pop, rng, context, n_kv, d, page)
    start = np.concatenate([[0], np.cumsum(new)])
    q = _queries(rng, start[-1], heads, d, BF16)
    for scale in (0.07, -0.4):
        y = _attend_in_blocks(pop, c, q, start, heads, scale, window, parts=True)
        _check(c, y, q, start, BF16, BF16, scale, window)
    assert torch.equal(y, _attend_in_blocks(pop, c, q, start, heads, -0.4, window))
    table = c.table.copy()
    table[0, ::3] = -1
    there = [np.repeat((t >= 0) & (t < c.n_pages), page) for t in table]
    y = _attend_in_blocks(pop, c, q, start, heads, 0.07, window, table=table)
    _check(c, y, q, start, BF16, BF16, 0.07, window, there=there)
    short = [new[0] // 2] + context[1:]
    y = _attend_in_blocks(pop, c, q, start, heads, 0.07, window, context=short)
    _check(c, y, q, start, BF16, BF16, 0.07, window, context=short)


@pytest.mark.parametrize("window", [0, 90])
@pytest.mark.parametrize("n_seq,heads,n_kv,d", [(65, 4, 1, 64), (150, 8, 2, 64), (129, 16, 4, 128)])
def test_many_sequences_in_blocks_of_128_columns(pop, n_seq, heads, n_kv, d, window):
    """Several sequences to a lane; empty ones, ones without new tokens, many of one length."""
    rng = np.random.default_rng(n_seq + window)
    context = rng.integers(0, 300, n_seq)
    context[rng.integers(0, n_seq, n_seq // 3)] = 200
    context[5] = 900
    new = np.minimum(rng.integers(0, 120, n_seq), context)
    new[context == 200] = 70
    c = Cached(pop, rng, context.tolist(), n_kv, d, 16)
    start = np.concatenate([[0], np.cumsum(new)])
    q = _queries(rng, start[-1], heads, d, BF16)
    y = _attend_in_blocks(pop, c, q, start, heads, 0.11, window)
    _check(c, y, q, start, BF16, BF16, 0.11, window)
    assert torch.equal(y, _attend_in_blocks(pop, c, q, start, heads, 0.11, window))


@pytest.mark.parametrize("page,window", [(16, 0), (32, 77)])
def test_widest_heads_in_blocks_of_128_columns(pop, page, window):
    rng = np.random.default_rng(page + 2)
    c = Cached(pop, rng, [401, 0, 257], 64, 256, page)
    start = np.array([0, 250, 250, 450])
    q = _queries(rng, 450, 64, 256, BF16)
    y = _attend_in_blocks(pop, c, q, start, 64, 0.06, window, parts=False)
    _check(c, y, q, start, BF16, BF16, 0.06, window)
    short = [401, 0, 150]
    y = _attend_in_blocks(pop, c, q, start, 64, 0.06, window, context=short)
    _check(c, y, q, start, BF16, BF16, 0.06, window, context=short)


@pytest.mark.parametrize("dtype,blocks", [(F32, False), (BF16, False), (BF16, True)])
def test_starts_that_do_not_ascend(pop, dtype, blocks):
    """Sequences whose rows are none or leave the tensors are left out; the others' rows, wherever they stand, are right."""
    rng = np.random.default_rng(15)
    c = Cached(pop, rng, [300, 200, 90, 64, 500, 7], 2, 64, 16)
    n = 150
    q = _queries(rng, n, 8, 64, dtype)
    for starts, kept in (([100, 140, 20, 60, 5000, 7000, -3], [0, 2]), ([150, 80, 149, 90, 2 ** 31 - 1, -2 ** 31, 0], [1]), ([-5, -1, 140, 3, 3, 10, 9], [4])):
        if blocks:
            h = f64(_attend_in_blocks(pop, c, q, starts, 8, 0.1, max_context=1 << 22))
        else:
            h = f64(_attend(pop, c, q, starts, dtype, dtype, 8, 0.1, max_new=40, max_context=500))
        written = np.zeros(n, bool)
        for s in kept:
            a, b = starts[s], starts[s + 1]
            written[a:b] = True
            sizes = []
            want = orc.attention(f64(q[a:b]), c.k[s], c.v[s], 0.1, c.context[s] - (b - a), 0, None, sizes)
            scores = (c.d + 8) * 2.0 ** -24 * sizes[1]
            bound = sizes[0] * (2 * scores + (c.context[s] + 32) * 2.0 ** -24 + 2.0 ** -21) + 2.0 ** -23 * np.abs(want)  # (as in _check)
            if dtype == BF16:
                bound = bound + 2.0 ** -8 * sizes[0] + 2.0 ** -8 * np.abs(want)
            assert (np.abs(h[a:b] - want) <= bound + 1e-30).all(), (starts, s)
        assert (h[~written] == 7.0).all()


def test_write_of_one_token_or_none_from_rows_of_any_length(pop):
    """Where there is no second row its distance says nothing, whatever 16 bytes make of it."""
    x = torch.arange(5 * 130, device="cuda").remainder(5).float().sub_(2.0).view(5, 130)
    cache = torch.zeros(pop.pop_cache_bytes(2, 64, 16, 1), dtype=torch.uint8, device="cuda")
    pop.pop_cache_write(cache, 2, 64, 16, 1, x, x, BF16, i32([0]), 0)
    assert not cache.any()
    pop.pop_cache_write(cache, 2, 64, 16, 1, x, x, F32, i32([3]), 1)
    ko, vo = torch.zeros(1, 2, 64, device="cuda"), torch.zeros(1, 2, 64, device="cuda")
    pop.pop_cache_read(cache, 2, 64, 16, 1, i32([3]), 1, ko, vo, F32)
    assert np.array_equal(f64(ko).ravel(), f64(x)[0, :128]) and np.array_equal(f64(vo).ravel(), f64(x)[0, :128])
