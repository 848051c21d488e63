"""A decoder's step with everything around its projections from the library: norms, rotary positions, the cache, attention over a shared prompt or a window with
first tokens, the pruned FFN, selection and reordering."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def prompt_of(model, n):
    return torch.randint(0, model.vocab, (n,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(5))


ROOM = 40000  # tokens that a cache is made for: with that many, reading the prompt once for all beams pays


@pytest.mark.parametrize("beams,prompt_len,new,window,room", [(4, 40, 20, 0, 0), (3, 700, 30, 0, 0), (4, 700, 30, 0, ROOM), (8, 500, 12, 0, ROOM), (8, 100, 18, 33, 0),
                                                              (2, 300, 20, 64, 0)])
def test_beams_have_the_scores_of_their_tokens(beams, prompt_len, new, window, room):
    """As of the form in plain torch: beams that are replayed one by one, each in a row of its own, have the scores that the search reports."""
    import beam_decode as ex
    model = ex.Decoder(beams=beams, layers=3, max_tokens=room or prompt_len + new + 3, seed=beams, fused=True, window=window, sinks=4)
    assert not room or shared_kind(model) == 2
    try:
        prompt = prompt_of(model, prompt_len)
        history, scores = ex.beam_search(model, prompt, new)
        assert history.shape == (beams, new) and bool((scores[:-1] >= scores[1:]).all())
        again = ex.beam_search(model, prompt, new)
        assert torch.equal(history, again[0]) and torch.equal(scores, again[1])
        model.reset()
        logits = model.prompt(prompt)
        model.reorder(ex._int32(beams))
        total = torch.zeros(beams, device="cuda")
        for i in range(new):
            token = history[:, i].long()
            total += torch.log_softmax(logits.double(), -1).gather(1, token[:, None])[:, 0].float()
            if i + 1 < new:
                logits = model.step(history[:, i].contiguous())
        assert model.failed.tolist() == [0, 0]
        # the same rows in the same kernels, but in other places of the batch; sums of `new` float32 numbers of up to 20 each
        assert torch.allclose(total, scores, rtol=0, atol=1e-4 * new), (total - scores).abs().max()
    finally:
        model.close()


def shared_kind(model):
    import beam_decode as ex
    return ex.pop.pop_cache_attention_shared_kind(ex.BF16, ex.BF16, model.beams, model.beams, model.beams, model.heads, model.n_kv, model.head_dim, 1, model.max_tokens)


@pytest.mark.parametrize("window", [0, 50])
def test_both_forms_of_a_layer_agree(window):
    """One layer from the same cache and embedding.  The FFN's selection of channels may fall differently where hidden states differ by a rounding, so
    what is compared stands in front of it: the keys and values that the layer caches, and the residual stream after attention."""
    import beam_decode as ex
    pop = ex.pop
    n = 90
    seen = []
    for fused in (False, True):
        model = ex.Decoder(beams=2, layers=1, max_tokens=n + 4, seed=7, fused=fused, window=window, sinks=4)
        try:
            rows = []
            model._ffn = lambda layer, z, count, first: rows.append(z.clone()) or torch.zeros_like(z)
            model.prompt(prompt_of(model, n))
            slots = model.slots[:n].contiguous()
            k = torch.empty(n, model.n_kv, model.head_dim, device="cuda")
            v = torch.empty_like(k)
            pop.pop_cache_read(model.layers[0].cache, model.n_kv, model.head_dim, model.page, model.n_pages, slots, n, k, v, pop.POP_F32)
            seen.append((k, v, rows[0].float()))
        finally:
            model.close()
    (k0, v0, z0), (k1, v1, z1) = seen
    # The first norm's input is the embedding in both forms: keys and values differ where a rounding to bf16 (half a step, 2^-8) moves a number to the
    # neighbouring 4-bit code, which is up to a third of it; few do
    for a, b in ((k0, k1), (v0, v1)):
        moved = (a != b).float().mean()
        assert moved < 0.05 and bool(((a - b).abs() <= 0.5 * torch.maximum(a.abs(), b.abs()) + 1e-6).float().mean() > 0.99), float(moved)
    # the second norm's output has numbers of size 1
    assert float((z0 - z1).square().mean().sqrt()) < 0.05 * float(z0.square().mean().sqrt())


def test_fused_steps_in_a_replayed_graph():
    """A decode step of all of it, captured once and replayed with other tokens, against the same step run eagerly."""
    import beam_decode as ex
    model = ex.Decoder(beams=4, layers=2, max_tokens=ROOM, seed=11, fused=True)
    assert shared_kind(model) == 2
    try:
        prompt = prompt_of(model, 600)
        model.reset()
        model.prompt(prompt)
        model.reorder(ex._int32(4))
        tokens = torch.randint(0, model.vocab, (4,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
        model.plan(ex._int32(4, fill=1), 4)
        model.logits(model.forward(tokens, False))  # (warm)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):  # (the planned token is written anew by every replay)
            out = model.logits(model.forward(tokens, False))
        for i in range(3):
            tokens.copy_(torch.randint(0, model.vocab, (4,), device="cuda"))
            graph.replay()
            torch.cuda.synchronize()
            got = out.clone()
            want = model.logits(model.forward(tokens, False))
            torch.cuda.synchronize()
            assert torch.equal(got, want)
    finally:
        model.close()
