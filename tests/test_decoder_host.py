"""The calls around the FFN (cache, attention, beams) on the host: sizes, refusals, and pins of their 64-bit oracle."""
import numpy as np
import pytest
import torch

from oracle import decoder_oracle as orc


@pytest.fixture(scope="module")
def pop():
    from paper_2602_06822_amd import binding
    return binding


# ---------------------------------------------------------------- the oracle, pinned by hand

def test_codes_at_ties_and_limits():
    """Blocks with a 4 in front have scale 1: halves go to the even code, 6 is the largest."""
    x = np.zeros(32)
    x[:16] = [4.0, 0.25, 0.2500001, 0.75, 1.25, 1.2500001, 1.75, 2.5, 2.5000001, 3.5, 5.0, 5.0000001, 6.9, -0.75, -2.5, -0.0]
    code, byte = orc.encode(x)
    assert byte.tolist() == [127]
    assert code[:16].tolist() == [6, 0, 1, 2, 2, 3, 4, 4, 5, 6, 6, 7, 7, 8 | 2, 8 | 4, 8]
    assert orc.decode(code, byte)[:4].tolist() == [4.0, 0.0, 0.5, 1.0]


@pytest.mark.parametrize("top,byte", [(4.0, 127), (6.999, 127), (7.0, 128), (7.9, 128), (8.0, 128), (1.0, 125), (0.0, 1),
                                      (1e-45, 1), (3.4028234e38, 252), (np.inf, 252), (2.0 ** -124, 1), (2.0 ** -123, 2)])
def test_scale_bytes(top, byte):
    x = np.zeros(32)
    x[3] = -top
    assert orc.encode(x)[1].tolist() == [byte]
    assert np.isfinite(orc.decode(*orc.encode(x))).all()


def test_no_stored_value_is_further_than_half_a_step():
    g = np.random.default_rng(3)
    x = g.standard_normal((400, 64)) * np.exp2(g.integers(-60, 60, (400, 1)))
    code, byte = orc.encode(x)
    y = orc.decode(code, byte)
    scale = np.repeat(np.exp2(byte - 127.0), 32, -1)
    # half the distance of neighbouring magnitudes (2 at the top); what lies in (6, 7) is cut by less than 1
    assert (np.abs(y - x) <= scale * 1.0 + 0).all()
    assert (np.abs(y - x)[np.abs(x) <= 2 * scale] <= 0.25 * scale[np.abs(x) <= 2 * scale]).all()
    assert np.isnan(orc.decode(*orc.encode(np.full(32, np.nan)))).sum() == 0


@pytest.mark.parametrize("d", [64, 128, 256])
def test_a_tile_holds_every_value_once(d):
    seen = set()
    for t in range(16):
        k, v, ks, vs = orc.byte_places(d, t)
        for place in [*k, *v, *[(i, s) for i in ks + vs for s in (0, 1)]]:
            assert place not in seen
            seen.add(place)
    assert len(seen) == 2 * orc.tile_bytes(d) and max(i for i, _ in seen) == orc.tile_bytes(d) - 1


def test_a_plan_by_hand():
    table = np.array([[7, 8, -1], [-1, -1, -1], [9, -1, -1]])
    ring = np.array([5, 6, 0, 1, 2, 3, 4, 0, 0, 0])
    t, ctx, start, slots, pos, pool, status = orc.plan([20, 0, 16], [1, 17, 1], 16, table, ring, (8, 5), 22)
    assert status == 0 and pool == (1, 2)
    assert t.tolist() == [[7, 8, -1], [0, 0, -1], [9, 5, -1]]
    assert ctx.tolist() == [21, 17, 17] and start.tolist() == [0, 1, 18, 19]
    assert slots[:3].tolist() == [8 * 16 + 4, 0, 1] and slots[18] == 5 * 16 and slots[19:].tolist() == [-1] * 3
    assert pos[:2].tolist() == [20, 0] and pos[18] == 16
    assert orc.plan([20, 0, 16], [1, 17, 1], 16, table, ring, (8, 2), 22)[-1] == 1


def test_a_reordering_by_hand():
    # two beams of 20 tokens share page 3; row 0 ends, row 1 goes on twice
    table = np.array([[3, 4, -1], [3, 5, -1]])
    new, length, copies, ring, pool, status = orc.reorder(table, [20, 20], [1, 1], 2, 16, np.array([0, 1, 2, 0, 0, 0]), (0, 3))
    assert status == 0 and new.tolist() == [[3, 5, -1], [3, 0, -1]] and length.tolist() == [20, 20]
    assert copies.tolist() == [[-1, -1], [5, 0]] and pool == (1, 3) and ring.tolist() == [0, 1, 2, 4, 0, 0]
    # released: the page they share goes back once
    new, length, copies, ring, pool, status = orc.reorder(table, [20, 20], [-1, 2], 2, 16, np.array([0, 1, 2, 0, 0, 0]), (0, 3))
    assert new.tolist() == [[-1] * 3] * 2 and pool == (0, 6) and ring[3:].tolist() == [3, 4, 5]


def test_oracle_attention_and_selection_against_torch():
    g = np.random.default_rng(5)
    q, k, v = g.standard_normal((3, 4, 8)), g.standard_normal((9, 2, 8)), g.standard_normal((9, 2, 8))
    y = orc.attention(q, k, v, 0.3, 6)
    tq, tk, tv = (torch.from_numpy(x) for x in (q, np.repeat(k, 2, 1), np.repeat(v, 2, 1)))
    s = torch.einsum("ihd,khd->hik", tq, tk) * 0.3
    s = s.masked_fill(torch.arange(9)[None, None] > 6 + torch.arange(3)[None, :, None], -torch.inf)
    assert np.allclose(y, torch.einsum("hik,khd->ihd", s.softmax(-1), tv).numpy(), rtol=0, atol=1e-13)
    x, was = g.standard_normal((3, 50)), np.array([-1.0, -np.inf, -2.5])
    score, token, parent = orc.beam_select(x, was, np.array([0, 0, 1]), 5, 7)
    ref = torch.from_numpy(was)[:, None] + torch.log_softmax(torch.from_numpy(x), -1)
    ref[2] = -torch.inf
    ref[2, 7] = -2.5
    top = torch.topk(ref.flatten(), 5)
    assert np.allclose(score, top.values.numpy(), rtol=0, atol=1e-13) and ((parent * 50 + token) == top.indices.numpy()).all()


# ---------------------------------------------------------------- sizes and refusals (nothing is launched)

def test_cache_bytes(pop):
    assert pop.pop_cache_bytes(32, 128, 16, 10) == 10 * 32 * 2176
    assert pop.pop_cache_bytes(1, 64, 64, 3) == 3 * 4 * 1088
    for bad in ((0, 128, 16, 1), (1, 128, 16, 0)):
        with pytest.raises(pop.PopError) as e:
            pop.pop_cache_bytes(*bad)
        assert e.value.status == pop.POP_ESHAPE
    for bad in ((1, 96, 16, 1), (1, 128, 24, 1), (1, 128, 8, 1), (1, 128, 512, 1), (1, 128, 16, 1 << 27)):
        with pytest.raises(pop.PopError) as e:
            pop.pop_cache_bytes(*bad)
        assert e.value.status == pop.POP_EUNSUPPORTED


A = 1 << 20  # an address that is aligned and never read: every call below is refused


def _refused(pop, status, name, args):
    assert getattr(pop.raw(), name)(*args) == getattr(pop, status), (name, args)


def _with(args, **changes):
    args = dict(args)
    args.update(changes)
    return list(args.values())


PLAN = dict(cached=A, new=A, n_seq=2, page=16, table=A, stride=4, ring=A, n_pages=8, pool=A, pool_out=A + 64, max_tokens=4,
            context=A + 128, start=A, slots=A, positions=None, status=A, stream=None)


@pytest.mark.parametrize("status,change", [
    ("POP_EINVAL", dict(cached=None)), ("POP_EINVAL", dict(new=None)), ("POP_EINVAL", dict(table=None)), ("POP_EINVAL", dict(ring=None)),
    ("POP_EINVAL", dict(pool=None)), ("POP_EINVAL", dict(pool_out=None)), ("POP_EINVAL", dict(pool_out=A)),
    ("POP_EINVAL", dict(context=A)), ("POP_EINVAL", dict(context=None)), ("POP_EINVAL", dict(start=None)),
    ("POP_EINVAL", dict(slots=None)), ("POP_EINVAL", dict(status=None)), ("POP_ESHAPE", dict(n_seq=-1)),
    ("POP_ESHAPE", dict(stride=0)), ("POP_ESHAPE", dict(n_pages=0)), ("POP_ESHAPE", dict(max_tokens=-1)),
    ("POP_EUNSUPPORTED", dict(page=17)), ("POP_EUNSUPPORTED", dict(n_pages=1 << 28)), ("POP_EUNSUPPORTED", dict(stride=1 << 28))])
def test_plan_refuses(pop, status, change):
    _refused(pop, status, "pop_cache_plan", _with(PLAN, **change))


WRITE = dict(cache=A, n_kv=2, d=128, page=16, n_pages=8, k=A, v=A, dtype=1, ks=256, vs=256, slots=A, n=3, stream=None)


@pytest.mark.parametrize("status,change", [
    ("POP_EINVAL", dict(cache=None)), ("POP_EINVAL", dict(k=None)), ("POP_EINVAL", dict(v=A + 8)), ("POP_EINVAL", dict(cache=A + 4)),
    ("POP_EINVAL", dict(slots=None)), ("POP_EINVAL", dict(dtype=2)), ("POP_ESHAPE", dict(ks=255)), ("POP_ESHAPE", dict(ks=260)),
    ("POP_ESHAPE", dict(vs=128)), ("POP_ESHAPE", dict(n=-1)), ("POP_ESHAPE", dict(n_kv=0)), ("POP_EUNSUPPORTED", dict(d=96)),
    ("POP_EUNSUPPORTED", dict(page=48)), ("POP_EUNSUPPORTED", dict(n=1 << 30)), ("POP_OK", dict(n=0, k=None))])
def test_write_refuses(pop, status, change):
    _refused(pop, status, "pop_cache_write", _with(WRITE, **change))


READ = dict(cache=A, n_kv=2, d=128, page=16, n_pages=8, slots=A, n=3, k=A, v=A, dtype=0, stream=None)


@pytest.mark.parametrize("status,change", [
    ("POP_EINVAL", dict(cache=None)), ("POP_EINVAL", dict(k=None)), ("POP_EINVAL", dict(v=A + 8)), ("POP_EINVAL", dict(slots=None)),
    ("POP_EINVAL", dict(dtype=-1)), ("POP_ESHAPE", dict(n=-1)), ("POP_EUNSUPPORTED", dict(d=32)), ("POP_OK", dict(n=0))])
def test_read_refuses(pop, status, change):
    _refused(pop, status, "pop_cache_read", _with(READ, **change))


ATTENTION = dict(q=A, dtype=1, n_tokens=4, cache=A, n_kv=2, d=128, page=16, n_pages=8, table=A, stride=4, start=A, context=A, n_seq=2,
                 n_heads=4, max_new=2, max_context=64, scale=0.1, window=0, y=A, ydtype=1, ws=A, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("status,change", [
    ("POP_EINVAL", dict(q=None)), ("POP_EINVAL", dict(cache=None)), ("POP_EINVAL", dict(table=None)), ("POP_EINVAL", dict(start=None)),
    ("POP_EINVAL", dict(context=None)), ("POP_EINVAL", dict(y=None)), ("POP_EINVAL", dict(q=A + 2)), ("POP_EINVAL", dict(y=A + 8)),
    ("POP_EINVAL", dict(dtype=7)), ("POP_EINVAL", dict(ydtype=-1)), ("POP_EINVAL", dict(scale=float("nan"))),
    ("POP_EINVAL", dict(scale=float("inf"))), ("POP_EINVAL", dict(ws=A + 1)), ("POP_ESHAPE", dict(n_heads=5)), ("POP_ESHAPE", dict(n_heads=0)),
    ("POP_ESHAPE", dict(n_seq=-1)), ("POP_ESHAPE", dict(n_tokens=-1)), ("POP_ESHAPE", dict(max_new=0)), ("POP_ESHAPE", dict(max_context=0)),
    ("POP_ESHAPE", dict(window=-1)), ("POP_ESHAPE", dict(stride=0)), ("POP_EUNSUPPORTED", dict(d=96)),
    ("POP_EUNSUPPORTED", dict(n_seq=40000)), ("POP_OK", dict(n_seq=0)), ("POP_OK", dict(n_tokens=0, q=None))])
def test_attention_refuses(pop, status, change):
    _refused(pop, status, "pop_cache_attention", _with(ATTENTION, **change))


def test_attention_refuses_a_small_workspace(pop):
    need = pop.pop_cache_attention_workspace(1, 1, 4, 2, 128, 1, 100000)
    assert need > 0
    one = dict(ATTENTION, n_tokens=1, n_seq=1, max_new=1, max_context=100000)
    _refused(pop, "POP_ESHAPE", "pop_cache_attention", _with(one, ws_bytes=need - 1))
    _refused(pop, "POP_EINVAL", "pop_cache_attention", _with(one, ws=None, ws_bytes=0))


@pytest.mark.parametrize("heads,n_kv", [(1, 1), (32, 32), (32, 8), (71, 1)])
def test_a_workspace_of_larger_sizes_is_enough(pop, heads, n_kv):
    sizes = [1, 2, 3, 8, 17, 64, 130, 600, 5000, 70000]
    for n_seq in (1, 4, 37, 256):
        for context in sizes:
            of_new = []
            for new in sizes:
                need = [pop.pop_cache_attention_workspace(n, n_seq, heads, n_kv, 128, new, context) for n in sizes]
                assert need == sorted(need)
                of_new.append(need)
            assert all(a <= b for few, more in zip(of_new, of_new[1:]) for a, b in zip(few, more))
    for new in sizes:
        need = [[pop.pop_cache_attention_workspace(3000, n_seq, heads, n_kv, 64, new, c) for c in sizes] for n_seq in (1, 2, 5, 30, 400)]
        assert all(row == sorted(row) for row in need)
        assert all(a <= b for few, more in zip(need, need[1:]) for a, b in zip(few, more))


BEAM = dict(logits=A, dtype=0, scores=A, done=None, requests=1, beams=4, vocab=100, k=4, pad=0, s=A + 64, t=A, p=A, ws=A,
            ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("status,change", [
    ("POP_EINVAL", dict(logits=None)), ("POP_EINVAL", dict(logits=A + 4)), ("POP_EINVAL", dict(scores=None)), ("POP_EINVAL", dict(s=None)),
    ("POP_EINVAL", dict(s=A)), ("POP_EINVAL", dict(t=None)), ("POP_EINVAL", dict(p=None)), ("POP_EINVAL", dict(ws=None)),
    ("POP_EINVAL", dict(dtype=3)), ("POP_ESHAPE", dict(pad=100)), ("POP_ESHAPE", dict(pad=-1)), ("POP_ESHAPE", dict(vocab=0)),
    ("POP_ESHAPE", dict(k=0)), ("POP_ESHAPE", dict(beams=1, vocab=3, pad=0)), ("POP_ESHAPE", dict(ws_bytes=16)),
    ("POP_ESHAPE", dict(requests=-1)), ("POP_EUNSUPPORTED", dict(beams=17)), ("POP_EUNSUPPORTED", dict(k=65)),
    ("POP_EUNSUPPORTED", dict(vocab=(1 << 24) + 1)), ("POP_OK", dict(requests=0))])
def test_beam_refuses(pop, status, change):
    _refused(pop, status, "pop_beam_select", _with(BEAM, **change))


REORDER = dict(table=A, length=A, parents=A, n_seq=8, beams=4, page=16, stride=8, new_table=A + 64, new_len=A + 64, copies=A, ring=A,
               n_pages=9, pool=A, pool_out=A + 64, ws=A, ws_bytes=1 << 20, status=A, stream=None)


@pytest.mark.parametrize("status,change", [
    ("POP_EINVAL", dict(table=None)), ("POP_EINVAL", dict(new_table=A)), ("POP_EINVAL", dict(new_len=A)), ("POP_EINVAL", dict(pool_out=A)),
    ("POP_EINVAL", dict(ws=None)), ("POP_EINVAL", dict(status=None)), ("POP_EINVAL", dict(copies=None)), ("POP_EINVAL", dict(parents=None)),
    ("POP_ESHAPE", dict(beams=3)), ("POP_ESHAPE", dict(n_seq=0)), ("POP_ESHAPE", dict(ws_bytes=0)), ("POP_ESHAPE", dict(stride=0)),
    ("POP_EUNSUPPORTED", dict(n_seq=34, beams=17)), ("POP_EUNSUPPORTED", dict(page=20))])
def test_reorder_refuses(pop, status, change):
    _refused(pop, status, "pop_cache_reorder", _with(REORDER, **change))


@pytest.mark.parametrize("status,change", [
    ("POP_EINVAL", dict(cache=None)), ("POP_EINVAL", dict(copies=None)), ("POP_EINVAL", dict(cache=A + 8)), ("POP_ESHAPE", dict(n=-1)),
    ("POP_EUNSUPPORTED", dict(d=100)), ("POP_OK", dict(n=0))])
def test_copy_pages_refuses(pop, status, change):
    _refused(pop, status, "pop_cache_copy_pages", _with(dict(cache=A, n_kv=2, d=64, page=16, n_pages=8, copies=A, n=2, stream=None), **change))


def test_binding_takes_device_tensors_only(pop):
    x = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        pop.pop_cache_plan(x, x, 4, 16, x, 1, x, 4, x, x, 0, x, x, x, x, x)
    with pytest.raises(ValueError):
        pop.pop_cache_write(0, 1, 64, 16, 1, torch.zeros(1, 64), torch.zeros(1, 64), 0, 0, 1)


@pytest.mark.parametrize("rows", [1 << 24, (1 << 24) + 16, 1 << 30])
def test_more_rows_than_a_grid_holds_are_refused(pop, rows):
    """A grid's axis counts threads in 32 bits: 2^24 workgroups of 256 would begin anew at zero."""
    _refused(pop, "POP_EUNSUPPORTED", "pop_beam_select", _with(BEAM, requests=rows // 4, beams=4, vocab=1, k=1))
    with pytest.raises(pop.PopError) as e:
        pop.pop_beam_workspace(rows // 4, 4, 1, 1)
    assert e.value.status == pop.POP_EUNSUPPORTED
    _refused(pop, "POP_EUNSUPPORTED", "pop_cache_reorder", _with(REORDER, n_seq=rows, beams=1, ws_bytes=1 << 40))
    with pytest.raises(pop.PopError) as e:
        pop.pop_cache_reorder_workspace(rows, 1, 8)
    assert e.value.status == pop.POP_EUNSUPPORTED
    _refused(pop, "POP_EUNSUPPORTED", "pop_cache_copy_pages", [A, 2, 64, 16, 8, A, rows, None])


def test_the_most_rows_have_a_workspace(pop):
    assert pop.pop_beam_workspace((1 << 20) - 1, 16, 1, 1) > 0 and pop.pop_cache_reorder_workspace((1 << 24) - 1, 1, 1) > 0


KIND = dict(dtype=1, ydtype=1, n_tokens=4096, n_seq=2, n_heads=32, n_kv=8, d=128, max_new=2048, max_context=6144, window=0, parts=None)


@pytest.mark.parametrize("status,change", [
    ("POP_EINVAL", dict(dtype=7)), ("POP_EINVAL", dict(ydtype=-1)), ("POP_ESHAPE", dict(n_heads=33)), ("POP_ESHAPE", dict(window=-1)),
    ("POP_ESHAPE", dict(max_new=0)), ("POP_EUNSUPPORTED", dict(d=96))])
def test_attention_kind_refuses(pop, status, change):
    _refused(pop, status, "pop_cache_attention_kind", _with(KIND, **change))


def test_attention_kinds(pop):
    def kind(**change):
        return pop.pop_cache_attention_kind(*_with(KIND, **change)[:-1])

    assert kind(n_seq=0) == (0, 0) and kind(n_tokens=0) == (0, 0)
    assert kind()[0] == 2
    for general in (dict(dtype=0), dict(ydtype=0), dict(n_tokens=2, max_new=1), dict(n_tokens=32, max_new=16), dict(d=256, n_tokens=128, max_new=64)):
        assert kind(**general) == (1, 0)
    few = dict(n_tokens=128, n_seq=1, n_heads=16, n_kv=4, max_new=128, max_context=60000)
    assert kind(**few)[1] > 1 and kind(**few, window=50) == (1, 0)


@pytest.mark.parametrize("change", [
    dict(n_seq=32768), dict(n_kv=65536, n_heads=65536, n_seq=1), dict(n_tokens=1 << 28), dict(n_tokens=1 << 26, stride=1 << 22),
    dict(n_tokens=1 << 20, n_seq=16, n_heads=64, n_kv=64, stride=1 << 26)])
def test_attention_refuses_what_it_does_not_count(pop, change):
    _refused(pop, "POP_EUNSUPPORTED", "pop_cache_attention", _with(ATTENTION, **change))


def test_write_and_read_refuse_what_a_grid_does_not_count(pop):
    _refused(pop, "POP_EUNSUPPORTED", "pop_cache_write", _with(WRITE, n=1 << 26))
    _refused(pop, "POP_EUNSUPPORTED", "pop_cache_read", _with(READ, n=1 << 26))
