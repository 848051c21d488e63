"""The example that runs the operators together: its beams, replayed one by one without any selection, have the scores it reports."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("beams,prompt_len,new,eos", [(4, 40, 20, -1), (3, 16, 35, 7), (8, 100, 18, -1), (1, 5, 12, -1)])
def test_beams_have_the_scores_of_their_tokens(beams, prompt_len, new, eos):
    import beam_decode as ex
    model = ex.Decoder(beams=beams, layers=3, max_tokens=prompt_len + new + 3, seed=beams)
    try:
        g = torch.Generator(device="cuda").manual_seed(5)
        prompt = torch.randint(0, model.vocab, (prompt_len,), device="cuda", generator=g)
        history, scores = ex.beam_search(model, prompt, new, eos=eos)
        assert history.shape == (beams, new) and bool((scores[:-1] >= scores[1:]).all())
        assert len({tuple(r) for r in history.tolist()}) == beams
        again = ex.beam_search(model, prompt, new, eos=eos)
        assert torch.equal(history, again[0]) and torch.equal(scores, again[1])
        # every row goes its own way from the prompt on: one reordering that gives each a row, and none after it
        model.reset()
        logits = model.prompt(prompt)
        model.reorder(ex._int32(beams))
        total, ended = torch.zeros(beams, device="cuda"), torch.zeros(beams, dtype=torch.bool, device="cuda")
        for i in range(new):
            token = history[:, i].long()
            gain = torch.log_softmax(logits.double(), -1).gather(1, token[:, None])[:, 0].float()
            total += torch.where(ended, 0.0, gain)
            ended |= token == eos
            if i + 1 < new:
                logits = model.step(history[:, i].contiguous())
        assert model.failed.tolist() == [0, 0]
        # the same rows in the same kernels, but in other places of the batch; sums of `new` float32 numbers of up to 20 each
        assert torch.allclose(total, scores, rtol=0, atol=1e-4 * new), (total - scores).abs().max()
    finally:
        model.close()


def test_greedy_beam_is_argmax():
    import beam_decode as ex
    model = ex.Decoder(beams=1, layers=2, max_tokens=40, seed=3)
    try:
        prompt = torch.arange(10, device="cuda")
        history, _ = ex.beam_search(model, prompt, 8)
        model.reset()
        logits = model.prompt(prompt)
        for i in range(8):
            assert int(logits[0].argmax()) == int(history[0, i])
            logits = model.step(history[:, i].contiguous())
    finally:
        model.close()


def test_running_out_of_pages_is_reported():
    import beam_decode as ex
    model = ex.Decoder(beams=2, layers=1, max_tokens=64, pages=3, seed=3)  # (the prompt takes two)
    try:
        with pytest.raises(RuntimeError, match="pages"):
            ex.beam_search(model, torch.arange(20, device="cuda"), 20)
    finally:
        model.close()
