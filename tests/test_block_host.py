"""What stands around the FFN and its cache on the host: norms, rotary positions (frequencies), attention with first tokens and with a shared prefix;
refusals, pins of the 64-bit oracle."""
import math

import numpy as np
import pytest

from oracle import decoder_oracle as orc


@pytest.fixture(scope="module")
def pop():
    from paper_2602_06822_amd import binding
    return binding


A = 1 << 20  # an address that is never looked at
F = 0.25


def _with(base, /, **change):
    assert set(change) <= set(base)
    return [{**base, **change}[k] for k in base]


def _refused(pop, status, name, args):
    assert getattr(pop.raw(), name)(*args) == getattr(pop, status), (name, args)


NORM = dict(x=A, xdtype=0, x_stride=512, u=2 * A, dtype=1, u_stride=512, gate=3 * A, gate_rows=4, gate_stride=512, n=4, d=512, w_post=4 * A, w_pre=5 * A,
            post=1, offset=0.0, eps=1e-6, x_scale=1.0, u_scale=1.0, x_out=6 * A, x_out_stride=512, z=7 * A, z_stride=512, stream=None)
INF, NAN = math.inf, math.nan


@pytest.mark.parametrize("status,change", [
    ("POP_EINVAL", dict(x=None)), ("POP_EINVAL", dict(x_out=None, z=None)), ("POP_EINVAL", dict(xdtype=2)), ("POP_EINVAL", dict(dtype=-1)),
    ("POP_EINVAL", dict(eps=0.0)), ("POP_EINVAL", dict(eps=-1.0)), ("POP_EINVAL", dict(eps=NAN)), ("POP_EINVAL", dict(eps=INF)),
    ("POP_EINVAL", dict(offset=NAN)), ("POP_EINVAL", dict(x_scale=INF)), ("POP_EINVAL", dict(u_scale=NAN)),
    ("POP_EINVAL", dict(u=None)), ("POP_EINVAL", dict(u=None, post=0)), ("POP_EINVAL", dict(u=None, gate=None, gate_rows=0)),
    ("POP_EINVAL", dict(x=A + 2)), ("POP_EINVAL", dict(u=A + 1)), ("POP_EINVAL", dict(z=A + 1)), ("POP_EINVAL", dict(x_out=A + 2)),
    ("POP_EINVAL", dict(gate=A + 1)), ("POP_EINVAL", dict(w_pre=A + 1)), ("POP_EINVAL", dict(w_post=A + 1)),
    ("POP_EINVAL", dict(x_out=A, x_out_stride=1024)), ("POP_EINVAL", dict(z=A)), ("POP_EINVAL", dict(z=2 * A, z_stride=520)),
    ("POP_EINVAL", dict(x_out=2 * A)), ("POP_EINVAL", dict(x_out=7 * A)), ("POP_EINVAL", dict(z=3 * A)), ("POP_EINVAL", dict(z=5 * A)),
    ("POP_EINVAL", dict(x_out=4 * A)),
    ("POP_ESHAPE", dict(n=-1)), ("POP_ESHAPE", dict(d=0)), ("POP_ESHAPE", dict(x_stride=511)), ("POP_ESHAPE", dict(u_stride=0)),
    ("POP_ESHAPE", dict(x_out_stride=511)), ("POP_ESHAPE", dict(z_stride=-512)), ("POP_ESHAPE", dict(gate_rows=2)), ("POP_ESHAPE", dict(gate_rows=0)),
    ("POP_ESHAPE", dict(gate=None)), ("POP_ESHAPE", dict(gate_stride=511)),
    ("POP_EUNSUPPORTED", dict(d=65537)), ("POP_EUNSUPPORTED", dict(n=1 << 22)),
    ("POP_OK", dict(n=0, gate_rows=1)), ("POP_OK", dict(n=0, gate=None, gate_rows=0, x=None))])
def test_block_norm_refuses(pop, status, change):
    _refused(pop, status, "pop_block_norm", _with(NORM, **change))


ROTARY = dict(q=A, k=2 * A, dtype=1, n=4, n_heads=8, n_kv=2, d=64, r=64, layout=0, q_stride=512, k_stride=128, positions=A, turns=A, amplitude=1.0,
              q_out=3 * A, k_out=4 * A, q_out_stride=512, k_out_stride=128, stream=None)


@pytest.mark.parametrize("status,change", [
    ("POP_EINVAL", dict(q=None)), ("POP_EINVAL", dict(q_out=None)), ("POP_EINVAL", dict(k=None)), ("POP_EINVAL", dict(k_out=None)),
    ("POP_EINVAL", dict(positions=None)), ("POP_EINVAL", dict(turns=None)), ("POP_EINVAL", dict(dtype=3)), ("POP_EINVAL", dict(layout=2)),
    ("POP_EINVAL", dict(amplitude=NAN)), ("POP_EINVAL", dict(q=A + 1)), ("POP_EINVAL", dict(turns=A + 4)), ("POP_EINVAL", dict(positions=A + 2)),
    ("POP_EINVAL", dict(q_out=A, q_out_stride=640)), ("POP_EINVAL", dict(k_out=2 * A, k_out_stride=130)), ("POP_EINVAL", dict(k_out=A)),
    ("POP_EINVAL", dict(q_out=2 * A)), ("POP_EINVAL", dict(k_out=3 * A)),
    ("POP_ESHAPE", dict(n=-1)), ("POP_ESHAPE", dict(n_heads=0)), ("POP_ESHAPE", dict(n_kv=0)), ("POP_ESHAPE", dict(r=63)), ("POP_ESHAPE", dict(r=0)),
    ("POP_ESHAPE", dict(r=66)), ("POP_ESHAPE", dict(q_stride=511)), ("POP_ESHAPE", dict(k_stride=127)), ("POP_ESHAPE", dict(q_out_stride=0)),
    ("POP_ESHAPE", dict(k_out_stride=-128)),
    ("POP_EUNSUPPORTED", dict(d=2048, r=1026, q_stride=1 << 20, k_stride=1 << 20)), ("POP_EUNSUPPORTED", dict(n=1 << 22)),
    ("POP_EUNSUPPORTED", dict(n_heads=1 << 24, q_stride=1 << 30)), ("POP_EUNSUPPORTED", dict(n_heads=(1 << 20) - 2, q_stride=1 << 26)), ("POP_OK", dict(n=0)), ("POP_OK", dict(n=0, k=None, n_kv=0))])
def test_rotary_refuses(pop, status, change):
    _refused(pop, status, "pop_rotary", _with(ROTARY, **change))


SCALINGS = ["plain", "linear", "base", "bands", "ramp"]


@pytest.mark.parametrize("scaling", SCALINGS)
@pytest.mark.parametrize("r,base,factor,context,low,high", [(64, 1e4, 4.0, 4096, 1, 32), (128, 5e5, 8.0, 8192, 1, 4), (20, 1e4, 1.0, 2048, 1, 32),
                                                            (4, 100.0, 2.5, 7, 0.5, 0.6), (1024, 1e6, 32.0, 1e6, 1, 32), (64, 1e4, 4.0, 3, 1, 32)])
def test_frequencies(pop, scaling, r, base, factor, context, low, high):
    got, amplitude = pop.pop_rotary_frequencies(r, base, SCALINGS.index(scaling), factor, context, low, high)
    want, amp = orc.rotary_frequencies(r, base, scaling, factor, context, low, high)
    # powers, logarithms and a blend in 64 bits on either side; the exponent of a power times ln(base) <= 41 may lose that many steps
    assert np.allclose(got, want / (2 * np.pi), rtol=1e-13, atol=0)
    assert abs(amplitude - amp) <= 2.0 ** -24 * amp


def test_frequencies_by_hand(pop):
    assert pop.pop_rotary_frequencies(4, 100.0)[0] == pytest.approx([1 / (2 * math.pi), 0.1 / (2 * math.pi)], rel=1e-15)
    # the slowest is divided by the factor, the fastest stays
    got, _ = pop.pop_rotary_frequencies(64, 1e4, pop.POP_ROTARY_BASE, 8.0)
    plain, _ = pop.pop_rotary_frequencies(64, 1e4)
    assert got[0] == plain[0] and got[-1] == pytest.approx(plain[-1] / 8, rel=1e-12)
    got, amp = pop.pop_rotary_frequencies(64, 1e4, pop.POP_ROTARY_RAMP, 8.0, 4096, 1, 32)
    assert got[0] == plain[0] and got[-1] == pytest.approx(plain[-1] / 8, rel=1e-15) and amp == pytest.approx(1.2079442, rel=1e-6)


FREQUENCIES = dict(r=64, base=1e4, scaling=4, factor=2.0, context=4096.0, low=1.0, high=32.0)


@pytest.mark.parametrize("status,change", [
    ("POP_ESHAPE", dict(r=63)), ("POP_ESHAPE", dict(r=0)), ("POP_ESHAPE", dict(r=1026)), ("POP_ESHAPE", dict(r=2, scaling=2)),
    ("POP_EINVAL", dict(scaling=5)), ("POP_EINVAL", dict(scaling=-1)), ("POP_EINVAL", dict(base=1.0)), ("POP_EINVAL", dict(base=INF)),
    ("POP_EINVAL", dict(base=NAN)), ("POP_EINVAL", dict(factor=0.5)), ("POP_EINVAL", dict(factor=NAN)), ("POP_EINVAL", dict(context=0.0)),
    ("POP_EINVAL", dict(low=0.0)), ("POP_EINVAL", dict(low=32.0)), ("POP_EINVAL", dict(high=INF)), ("POP_EINVAL", dict(scaling=2, base=1e300, factor=1e300)),
    ("POP_EINVAL", dict(scaling=1, factor=0.0))])
def test_frequencies_refuse(pop, status, change):
    with pytest.raises(pop.PopError) as e:
        pop.pop_rotary_frequencies(*_with(FREQUENCIES, **change))
    assert e.value.status == getattr(pop, status)


def test_frequencies_refuse_no_place(pop):
    _refused(pop, "POP_EINVAL", "pop_rotary_frequencies", [64, 1e4, 0, 1.0, 0.0, 0.0, 0.0, None, None])


# ---------------------------------------------------------------- the oracle, pinned by hand

def test_oracle_norm_by_hand():
    x, u = np.array([[3.0, 0.0]]), np.array([[1.0, 4.0]])
    got, z = orc.block_norm(x, u, eps=0.0)
    assert np.array_equal(got, [[4.0, 4.0]]) and np.allclose(z, 1.0, rtol=1e-15)
    got, z = orc.block_norm(x, np.array([[5.0, 5.0]]), post=True, w_post=np.array([1.0, 3.0]), gate=np.array([[0.5, 1.0]]), offset=1.0, u_scale=2.0, eps=0.0)
    assert np.allclose(got, [[3 + 2 * 0.5 * 2, 2 * 4]], rtol=1e-15)
    assert np.allclose(z, got / np.sqrt((25 + 64) / 2), rtol=1e-15)


def test_oracle_rotary_by_hand():
    x = np.arange(1.0, 6.0).reshape(1, 1, 5)
    quarter = orc.rotary(x, [1], np.array([0.25, 0.5]), 2.0, True)  # a quarter and half a turn
    assert np.allclose(quarter, [[[-4, 2, -6, -8, 5]]], atol=1e-14)
    quarter = orc.rotary(x, [1], np.array([0.25, 0.5]), 1.0, False)  # pairs (0, 2) and (1, 3)
    assert np.allclose(quarter, [[[-3, -2, 1, -4, 5]]], atol=1e-14)
    assert np.array_equal(orc.rotary(x, [-1], np.array([0.25, 0.5]), 2.0, True), x)
    back = orc.rotary(orc.rotary(x, [12345], np.array([0.1, 0.37]), 1.0, True), [12345], np.array([-0.1, -0.37]), 1.0, True)
    assert np.allclose(back, x, rtol=1e-12)


# ---------------------------------------------------------------- attention with first tokens, and with a shared prefix

SINKS = dict(q=A, dtype=1, n=8, cache=A, n_kv=2, d=64, page=16, n_pages=100, table=A, stride=8, start=A, context=A, n_seq=4, heads=4, max_new=2, max_context=128,
             scale=0.1, window=20, sinks=4, y=A, ydtype=1, ws=A, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("status,change", [
    ("POP_EINVAL", dict(q=None)), ("POP_EINVAL", dict(y=None)), ("POP_EINVAL", dict(cache=A + 8)), ("POP_EINVAL", dict(scale=INF)), ("POP_EINVAL", dict(ws=None)),
    ("POP_ESHAPE", dict(sinks=-1)), ("POP_ESHAPE", dict(window=-1)), ("POP_ESHAPE", dict(heads=5)), ("POP_ESHAPE", dict(ws_bytes=0)),
    ("POP_EUNSUPPORTED", dict(d=96)), ("POP_EUNSUPPORTED", dict(page=17)), ("POP_OK", dict(n_seq=0)), ("POP_OK", dict(n=0))])
def test_sinks_refuse(pop, status, change):
    _refused(pop, status, "pop_cache_attention_sinks", _with(SINKS, **change))


SHARED = dict(q=A, dtype=1, n=8, cache=A, n_kv=2, d=64, page=16, n_pages=100, table=A, stride=8, start=A, context=A, n_seq=4, group=2, prefix=A, heads=4, max_new=2,
              max_context=128, scale=0.1, y=A, ydtype=1, ws=A, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("status,change", [
    ("POP_EINVAL", dict(q=None)), ("POP_EINVAL", dict(y=None)), ("POP_EINVAL", dict(prefix=None)), ("POP_EINVAL", dict(table=None)), ("POP_EINVAL", dict(start=None)),
    ("POP_EINVAL", dict(context=None)), ("POP_EINVAL", dict(cache=None)), ("POP_EINVAL", dict(cache=A + 8)), ("POP_EINVAL", dict(q=A + 8)), ("POP_EINVAL", dict(y=A + 2)),
    ("POP_EINVAL", dict(ws=A + 4)), ("POP_EINVAL", dict(scale=NAN)), ("POP_EINVAL", dict(ws=None)), ("POP_EINVAL", dict(dtype=2)), ("POP_EINVAL", dict(ydtype=-1)),
    ("POP_ESHAPE", dict(group=0)), ("POP_ESHAPE", dict(group=3)), ("POP_ESHAPE", dict(group=8)), ("POP_ESHAPE", dict(n_seq=-2)), ("POP_ESHAPE", dict(heads=5)),
    ("POP_ESHAPE", dict(ws_bytes=1000)), ("POP_ESHAPE", dict(stride=0)), ("POP_ESHAPE", dict(max_new=0)), ("POP_ESHAPE", dict(max_context=0)),
    ("POP_EUNSUPPORTED", dict(d=96)), ("POP_EUNSUPPORTED", dict(page=17)), ("POP_EUNSUPPORTED", dict(stride=1 << 27)), ("POP_EUNSUPPORTED", dict(n_seq=32768)),
    ("POP_EUNSUPPORTED", dict(n=1 << 27, stride=1 << 12)), ("POP_OK", dict(n_seq=0)), ("POP_OK", dict(n=0))])
def test_shared_refuses(pop, status, change):
    _refused(pop, status, "pop_cache_attention_shared", _with(SHARED, **change))


def test_shared_workspace(pop):
    sizes = dict(n=64, n_seq=64, group=8, heads=32, n_kv=8, d=128, max_new=1, max_context=40000)
    need = pop.pop_cache_attention_shared_workspace(*_with(sizes))
    _refused(pop, "POP_ESHAPE", "pop_cache_attention_shared", _with(dict(SHARED, n=64, n_seq=64, group=8, heads=32, n_kv=8, d=128, max_new=1, max_context=40000, page=64, stride=700),
                                                                    ws_bytes=need - 1))
    # of larger sizes it is enough for smaller ones
    for change in (dict(n=8, n_seq=8), dict(n=63), dict(max_context=1), dict(max_context=300), dict(n_seq=32, n=64), dict(n=1)):
        assert pop.pop_cache_attention_shared_workspace(*_with(sizes, **change)) <= need
    chunks = dict(sizes, n=2000, max_new=40)
    need = pop.pop_cache_attention_shared_workspace(*_with(chunks))
    for change in (dict(max_new=1), dict(max_new=3), dict(max_new=39), dict(n=64, max_new=1), dict(n=1999), dict(n_seq=8), dict(max_context=70)):
        assert pop.pop_cache_attention_shared_workspace(*_with(chunks, **change)) <= need
    wide = dict(sizes, n=160, n_seq=160, group=160, n_kv=32, max_context=200000)  # (a block of 128 columns, and a second one that is nearly empty)
    need = pop.pop_cache_attention_shared_workspace(*_with(wide))
    for n in range(1, 160, 7):
        assert pop.pop_cache_attention_shared_workspace(*_with(wide, n=n)) <= need
    with pytest.raises(pop.PopError) as e:
        pop.pop_cache_attention_shared_workspace(*_with(sizes, group=5))
    assert e.value.status == pop.POP_ESHAPE
    assert pop.pop_cache_attention_shared_workspace(*_with(sizes, n_seq=0)) == 0


def test_shared_kinds(pop):
    sizes = dict(dtype=1, ydtype=1, n=8, n_seq=8, group=8, heads=32, n_kv=32, d=128, max_new=1, max_context=4096)

    def kind(**change):
        return pop.pop_cache_attention_shared_kind(*_with(sizes, **change))

    assert kind(n=0) == 0 and kind(n_seq=0) == 0
    assert kind() == 2 and kind(group=1) == 1 and kind(max_context=100) == 1 and kind(max_new=2048, n=8 * 2048) == 1
    assert kind(group=2, n_seq=2, n=2, max_context=1000) == 1 and kind(group=2, n_seq=2, n=2, max_context=9000) == 2
    many = dict(n=64, n_seq=64, group=64, n_kv=8, max_context=40000)
    assert kind(**many) == 3 and kind(**many, dtype=0) == 2 and kind(**many, ydtype=0) == 2 and kind(**dict(many, group=8)) == 2 and kind(**dict(many, max_context=5000)) == 2
    for status, change in (("POP_EINVAL", dict(dtype=2)), ("POP_ESHAPE", dict(group=3)), ("POP_ESHAPE", dict(heads=33)), ("POP_EUNSUPPORTED", dict(d=80))):
        with pytest.raises(pop.PopError) as e:
            kind(**change)
        assert e.value.status == getattr(pop, status)


def test_oracle_attention_with_first_tokens():
    g = np.random.default_rng(2)
    q, k, v = g.standard_normal((3, 2, 8)), g.standard_normal((20, 1, 8)), g.standard_normal((20, 1, 8))
    y = orc.attention(q, k, v, 0.3, 17, 4, sinks=2)
    for i in range(3):
        seen = [0, 1] + list(range(14 + i, 18 + i))
        z = 0.3 * k[seen, 0] @ q[i, 1]
        w = np.exp(z - z.max())
        assert np.allclose(y[i, 1], (w / w.sum()) @ v[seen, 0], rtol=1e-13)
    assert np.array_equal(orc.attention(q, k, v, 0.3, 17, 0, sinks=2), orc.attention(q, k, v, 0.3, 17))
    assert np.array_equal(orc.attention(q, k, v, 0.3, 17, 4, sinks=30), orc.attention(q, k, v, 0.3, 17))
