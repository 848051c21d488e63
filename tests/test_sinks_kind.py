"""Which kernel a call with first tokens runs: they add to what a window sees."""
import numpy as np
import pytest

F32, BF16 = 0, 1
# 4 chunks of up to 100 tokens, 32 heads over 8: types, tokens, sequences, heads, kv heads, channels, new, context
CHUNKS = (BF16, BF16, 400, 4, 32, 8, 64, 100, 20000)


@pytest.fixture(scope="module")
def pop():
    from paper_2602_06822_amd import binding
    return binding


def test_first_tokens_count(pop):
    def kind(sizes, window, sinks):
        return pop.pop_cache_attention_sinks_kind(*sizes, window, sinks)

    assert kind(CHUNKS, 64, 4)[0] == 1 and kind(CHUNKS, 64, 5000)[0] == 2 and kind(CHUNKS, 5000, 4)[0] == 2
    assert kind((F32, F32, *CHUNKS[2:]), 64, 5000) == (1, 0)
    # none, or no window: what pop_cache_attention runs; as many as a wider window sees: what that runs
    for window in (0, 64, 1000, 5000):
        assert kind(CHUNKS, window, 0) == pop.pop_cache_attention_kind(*CHUNKS, window)
        for sinks in (32, 3200, 1 << 30):
            want = window + sinks if window else 0
            assert kind(CHUNKS, window, sinks) == pop.pop_cache_attention_kind(*CHUNKS, min(want, 1 << 30))
    assert kind(CHUNKS, 64, (1 << 31) - 1)[0] == 2
    for none in (dict(n=0), dict(n_seq=0)):
        sizes = list(CHUNKS)
        sizes[2 if "n" in none else 3] = 0
        assert kind(sizes, 64, 4) == (0, 0)


@pytest.mark.parametrize("status,at,value", [("POP_EINVAL", 0, 2), ("POP_EINVAL", 1, -1), ("POP_ESHAPE", 2, -1), ("POP_ESHAPE", 4, 33), ("POP_EUNSUPPORTED", 6, 96),
                                             ("POP_ESHAPE", 9, -1), ("POP_ESHAPE", 10, -1)])
def test_refusals(pop, status, at, value):
    args = [*CHUNKS, 64, 4]
    args[at] = value
    with pytest.raises(pop.PopError) as e:
        pop.pop_cache_attention_sinks_kind(*args)
    assert e.value.status == getattr(pop, status)


@pytest.mark.gpu
@pytest.mark.parametrize("window,sinks,kind", [(64, 4, 1), (64, 5000, 2), (700, 4001, 2)])
def test_both_kinds(pop, window, sinks, kind):
    """The call's own sizes, few and many first tokens; some of its rows and heads against the oracle."""
    import test_gpu_prefix as prefix
    from oracle import decoder_oracle as orc
    from test_gpu_decoder import Cached

    rng = np.random.default_rng(sinks)
    context, new = [7000, 5200, 6100, 300], [100, 97, 100, 100]
    c = Cached(pop, rng, context, 8, 64, 16)
    start = prefix.starts_of(new)
    q = prefix.queries(rng, start[-1], 32, 64, BF16)
    assert pop.pop_cache_attention_sinks_kind(BF16, BF16, len(q), 4, 32, 8, 64, 100, 7000, window, sinks)[0] == kind
    table = prefix.given_back(c, start, window, sinks)
    y, qh = prefix.f64(prefix.attend(pop, c, q, start, BF16, BF16, 32, 0.125, window, sinks, table=table)), prefix.f64(q)
    for s, length in enumerate(context):
        for i in range(0, new[s], 31):
            of, at = [], start[s] + i
            want = orc.attention(qh[at:at + 1], c.k[s], c.v[s], 0.125, length - new[s] + i, window, None, of, sinks)
            assert (np.abs(y[at] - want[0]) <= prefix.bound_of(want, of, 64, length, BF16)[0]).all(), (s, i)
