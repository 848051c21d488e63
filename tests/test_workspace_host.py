"""Workspaces of attention over shared prefixes, on the host: what a call uses is never more than what it asks for."""
import random

import pytest


@pytest.fixture(scope="module")
def pop():
    from paper_2602_06822_amd import binding
    return binding


F32, BF16 = 0, 1
TYPES = [(BF16, BF16), (BF16, F32), (F32, F32)]


def fits(pop, asked, sizes):
    """Whether a workspace of so many bytes holds what calls of these sizes use, of whichever types."""
    return all(pop.pop_cache_attention_shared_used(*types, *sizes) <= asked for types in TYPES)


# tokens, sequences, group, heads, kv heads, channels, new tokens, context
@pytest.mark.parametrize("sizes", [
    (128, 128, 16, 32, 8, 64, 1, 20000), (256, 256, 16, 32, 8, 64, 1, 10000), (64, 64, 64, 32, 32, 64, 1, 40000), (48, 48, 48, 32, 32, 64, 1, 65536),
    (40, 40, 40, 40, 40, 64, 1, 32768), (8, 8, 8, 8, 1, 64, 1, 1 << 22), (9, 9, 9, 5, 1, 64, 1, 1 << 22), (64, 64, 64, 32, 8, 128, 1, 32768),
    (80, 40, 40, 16, 8, 64, 2, 60000), (12, 12, 12, 12, 4, 64, 1, 1 << 22), (8, 8, 8, 32, 4, 256, 1, 1 << 20)])
def test_calls_stay_within_their_workspace(pop, sizes):
    asked = pop.pop_cache_attention_shared_workspace(*sizes)
    assert pop.pop_cache_attention_shared_kind(BF16, BF16, *sizes) in (2, 3) and fits(pop, asked, sizes)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_every_number_of_columns(pop, d):
    """Calls that take narrow blocks and blocks of 128, on both sides of the border between them."""
    kinds = set()
    for columns in range(2, 300):
        for share, context in ((1, 1 << 22), (1, 70000), (2, 1 << 22), (7, 300000)):
            group = -(-columns // share)
            if group < 2:
                continue
            sizes = (group, group, group, 16 * share, 16, d, 1, context)
            kinds.add(pop.pop_cache_attention_shared_kind(BF16, BF16, *sizes))
            assert fits(pop, pop.pop_cache_attention_shared_workspace(*sizes), sizes), sizes
    assert kinds >= ({2, 3} if d < 256 else {2})


@pytest.mark.parametrize("d", [64, 128])
def test_blocks_that_are_at_most_half_full_are_not_taken(pop, d):
    """Blocks of 128 columns need more than 64; what they would use is not asked for then."""
    for rows in (33, 40, 48, 64):
        for groups, n_kv, context in ((1, 32, 1 << 22), (1, 32, 65536), (12, 8, 37128), (8, 8, 20000), (16, 16, 40000)):
            sizes = (groups * rows, groups * rows, rows, n_kv, n_kv, d, 1, context)
            assert pop.pop_cache_attention_shared_kind(BF16, BF16, *sizes) == 2, sizes
            row = 4 * (d + 4)
            assert pop.pop_cache_attention_shared_workspace(*sizes) <= max(512 * 32 * row + 2 * groups * rows * n_kv * row,
                                                                           pop.pop_cache_attention_workspace(*sizes[:2], *sizes[3:]))
    sizes = (96, 96, 48, 64, 32, d, 1, 1 << 20)
    assert pop.pop_cache_attention_shared_kind(BF16, BF16, *sizes) == 3


def test_random_sizes_and_all_smaller_ones(pop):
    rng = random.Random(7)

    def some(most):
        return max(1, min(most, int(2 ** rng.uniform(0, most.bit_length()))))

    kinds = [0] * 4
    for _ in range(6000):
        n_kv, group, d = rng.choice([1, 2, 3, 4, 8, 16, 32, 40]), some(200), rng.choice([64, 64, 128, 256])
        groups, share, max_new, max_context = some(max(1, min(65535 // (n_kv * group), 300))), rng.choice([1, 1, 2, 4, 5, 8, 16]), rng.choice([1, 1, 1, 2, 5, some(600)]), some(1 << 22)
        n_seq = group * groups
        n = some(n_seq * max_new) if rng.random() < 0.3 else n_seq * max_new
        if n * n_kv * share >= 1 << 30:
            continue
        sizes = (n, n_seq, group, n_kv * share, n_kv, d, max_new, max_context)
        asked = pop.pop_cache_attention_shared_workspace(*sizes)
        kinds[pop.pop_cache_attention_shared_kind(BF16, BF16, *sizes)] += 1
        assert fits(pop, asked, sizes), sizes
        for _ in range(4):
            less = (some(n), group * some(groups), group, n_kv * share, n_kv, d, some(max_new), some(max_context))
            assert pop.pop_cache_attention_shared_workspace(*less) <= asked and fits(pop, asked, less), (sizes, less)
    assert min(kinds[1:]) > 200  # (each implementation is among them often)


def test_used_refuses(pop):
    for status, args in (("POP_EINVAL", (2, BF16, 8, 8, 8, 8, 8, 64, 1, 100)), ("POP_EINVAL", (BF16, -1, 8, 8, 8, 8, 8, 64, 1, 100)),
                         ("POP_ESHAPE", (BF16, BF16, 8, 8, 3, 8, 8, 64, 1, 100)), ("POP_ESHAPE", (BF16, BF16, 8, 8, 8, 9, 8, 64, 1, 100)),
                         ("POP_EUNSUPPORTED", (BF16, BF16, 8, 8, 8, 8, 8, 96, 1, 100))):
        with pytest.raises(pop.PopError) as e:
            pop.pop_cache_attention_shared_used(*args)
        assert e.value.status == getattr(pop, status)
    assert pop.raw().pop_cache_attention_shared_used(1, 1, 8, 8, 8, 8, 8, 64, 1, 100, None) == pop.POP_EINVAL
    assert pop.pop_cache_attention_shared_used(1, 1, 0, 8, 8, 8, 8, 64, 1, 100) == 0 == pop.pop_cache_attention_shared_used(1, 1, 8, 0, 8, 8, 8, 64, 1, 100)
