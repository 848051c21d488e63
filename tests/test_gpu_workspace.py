"""Attention over the cache writes nothing behind the workspace that it asked for: the calls of its tests with a guard there."""
import numpy as np
import pytest
import torch

import test_gpu_prefix as prefix
from test_gpu_decoder import BF16, F32, pop  # noqa: F401  (pop: the fixture)

pytestmark = pytest.mark.gpu
GUARD = 32 << 20  # more than any call's places for blocks of 128 columns


class Guarded:
    """The binding; attention gets a workspace of the size that it is given, with bytes behind it that have to stay."""

    def __init__(self, binding):
        self.binding, self.calls = binding, 0

    def __getattr__(self, name):
        entry = getattr(self.binding, name)
        if name not in ("pop_cache_attention", "pop_cache_attention_sinks", "pop_cache_attention_shared"):
            return entry

        def call(*args, **options):
            asked = args[-1].nbytes
            whole = torch.full((asked + GUARD,), 0xA5, dtype=torch.uint8, device="cuda")
            torch.cuda.synchronize()
            entry(*args[:-1], whole[:asked], **options)
            torch.cuda.synchronize()
            assert bool((whole[asked:] == 0xA5).all()), (name, args[13:], asked)
            self.calls += 1

        return call


@pytest.fixture
def guarded(pop):  # noqa: F811
    g = Guarded(pop)
    yield g
    assert g.calls > 0


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("rows,share", [(8, 2), (3, 11), (8, 5), (5, 9), (7, 8), (8, 8), (5, 13), (5, 25), (16, 8), (5, 26)])
def test_numbers_of_columns(guarded, d, rows, share):
    """16 columns of a pack to 130: blocks of 16, 32 and 128, the last of them nearly empty and full."""
    rng = np.random.default_rng(rows * share)
    c = prefix.Grouped(guarded, rng, [(1100, [1101 + 23 * i for i in range(rows)])], 2, d, 16)
    start = np.arange(rows + 1)
    for dtype in (BF16, F32):
        q = prefix.queries(rng, rows, 2 * share, d, dtype)
        y = prefix.attend_shared(guarded, c, q, start, dtype, dtype, 2 * share, d ** -0.5, kinds=(1, 2, 3) if d == 256 else (2, 3))
        prefix.check(c, y, q, start, dtype, d ** -0.5)


@pytest.mark.parametrize("dtype,ydtype", prefix.TYPES)
def test_shared(guarded, dtype, ydtype):
    prefix.test_shared_single_tokens(guarded, 64, dtype, ydtype)
    prefix.test_shared_long_prefixes(guarded, dtype, ydtype, 4, 2, 4)
    prefix.test_shared_chunks(guarded, dtype, ydtype, 6, 2, 64, 64)


@pytest.mark.parametrize("group,n_groups,heads,n_kv,d", [(65, 1, 4, 2, 64), (33, 5, 1, 1, 64), (2, 70, 3, 1, 64), (200, 1, 8, 1, 64)])
def test_shared_many_sequences(guarded, group, n_groups, heads, n_kv, d):
    prefix.test_shared_many_sequences(guarded, group, n_groups, heads, n_kv, d, BF16)


def test_shared_rows_of_several_sequences(guarded):
    for dtype in (BF16, F32):
        prefix.test_shared_rows_of_several_sequences(guarded, dtype)
        prefix.test_shared_starts_that_do_not_ascend(guarded, dtype)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_sinks(guarded, d):
    prefix.test_sinks_single_tokens(guarded, d, BF16, BF16)
    prefix.test_sinks_large_chunks(guarded, 16, 16, min(d, 128), 16, 300, 900, 333, 70)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_sinks_and_plain(guarded, dtype):
    prefix.test_sinks_chunks(guarded, dtype, dtype, 50, 64)
    prefix.test_sinks_long_sequences(guarded, dtype, dtype)
    prefix.test_sinks_without_a_window_or_without_tokens_are_plain_attention(guarded, dtype)
