"""Beam search with a small decoder: pruned FFNs under the prompt's partition, attention over a 4-bit paged cache.

Random weights, one prompt, up to POP_MAX_BATCH beams.  The prompt determines every layer's partition
(pop_prefill_forward); the beams that grow from it share that partition, the batch of the decode steps.  A step is

    pop_cache_plan       pages and slots for every beam's next token
    per layer            pop_cache_write, pop_cache_attention, pop_decode_step
    pop_beam_select      the best (beam, token) pairs
    pop_cache_reorder    block tables after the selection; per layer pop_cache_copy_pages

Projections, norms and the rotary embedding are plain torch.  Needs one MI355X:  python examples/beam_decode.py
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2602_06822_amd import binding as pop  # noqa: E402

BF16 = pop.POP_BF16


def _int32(*shape, fill=0):
    return torch.full(shape, fill, dtype=torch.int32, device="cuda")


class Layer:
    def __init__(self, g, d, m, heads, n_kv, head_dim, max_tokens, beams, page, n_pages):
        def w(*shape):
            return (0.02 * torch.randn(*shape, generator=g, device="cuda")).bfloat16()

        self.norm1, self.norm2 = torch.ones(d, device="cuda").bfloat16(), torch.ones(d, device="cuda").bfloat16()
        self.wqkv, self.wo = w((heads + 2 * n_kv) * head_dim, d), w(d, heads * head_dim)
        self.ffn = pop.pop_layer_create(d, m, BF16, w(m, d), w(m, d), w(d, m), max_tokens, beams)
        self.cache = torch.zeros(pop.pop_cache_bytes(n_kv, head_dim, page, n_pages), dtype=torch.uint8, device="cuda")

    def close(self):
        pop.pop_layer_destroy(self.ffn)


class Decoder:
    """The model, the cache and the tables of one request's beams."""

    def __init__(self, *, d=512, m=1408, layers=4, heads=8, n_kv=4, head_dim=64, vocab=4000, beams=4, page=16, max_tokens=256,
                 pages=None, sparsity=0.35, gamma=0.1, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.d, self.m, self.heads, self.n_kv, self.head_dim = d, m, heads, n_kv, head_dim
        self.vocab, self.beams, self.page, self.max_tokens = vocab, beams, page, max_tokens
        self.n_ret, self.n_cand, _ = pop.pop_region_counts(m, 1 - sparsity - gamma / 2, gamma)
        self.k = pop.pop_k_for_ratio(m, sparsity, self.n_ret, self.n_cand)
        blocks = -(-max_tokens // page)
        self.n_pages = pages or beams * blocks + beams
        self.layers = [Layer(g, d, m, heads, n_kv, head_dim, max_tokens, beams, page, self.n_pages) for _ in range(layers)]
        self.embedding = (0.3 * torch.randn(vocab, d, generator=g, device="cuda")).bfloat16()
        self.head = (0.08 * torch.randn(vocab, d, generator=g, device="cuda")).bfloat16()
        # two of what the calls read and write anew: tables, lengths, the pool
        self.tables = [_int32(beams, blocks, fill=-1) for _ in range(2)]
        self.lengths = [_int32(beams) for _ in range(2)]
        self.pools = [_int32(2) for _ in range(2)]
        self.ring = torch.arange(self.n_pages, dtype=torch.int32, device="cuda")
        self.start, self.slots, self.positions = _int32(beams + 1), _int32(max_tokens), _int32(max_tokens)
        self.copies, self.status, self.failed = _int32(beams, 2), _int32(2), _int32(2)
        need = [pop.pop_cache_attention_workspace(n, beams, heads, n_kv, head_dim, new, max_tokens) for n, new in ((max_tokens, max_tokens), (beams, 1))]
        need += [pop.pop_beam_workspace(1, beams, vocab, beams), pop.pop_cache_reorder_workspace(beams, beams, blocks)]
        self.workspace = torch.empty(max(need), dtype=torch.uint8, device="cuda")
        self.turns = dict(tables=0, lengths=0, pools=0)
        self.reset()

    def close(self):
        for layer in self.layers:
            layer.close()

    def reset(self):
        self.now("tables").fill_(-1)
        self.now("lengths").zero_()
        self.failed.zero_()
        self.ring.copy_(torch.arange(self.n_pages, dtype=torch.int32))
        self.now("pools").copy_(torch.tensor([0, self.n_pages], dtype=torch.int32))

    def now(self, name):
        return getattr(self, name)[self.turns[name]]

    def next(self, name):
        return getattr(self, name)[1 - self.turns[name]]

    def turn(self, *names):
        for name in names:
            self.turns[name] ^= 1

    def plan(self, new_len, n_tokens):
        table = self.now("tables")
        pop.pop_cache_plan(self.now("lengths"), new_len, self.beams, self.page, table, table.shape[1], self.ring, self.n_pages,
                           self.now("pools"), self.next("pools"), n_tokens, self.next("lengths"), self.start, self.slots,
                           self.positions, self.status[:1])
        self.failed |= self.status  # (read when the search is over)
        self.turn("lengths", "pools")

    def reorder(self, parents):
        table, new = self.now("tables"), self.next("tables")
        pop.pop_cache_reorder(table, self.now("lengths"), parents, self.beams, self.beams, self.page, table.shape[1], new,
                              self.next("lengths"), self.copies, self.ring, self.n_pages, self.now("pools"), self.next("pools"),
                              self.workspace, self.status[1:])
        self.failed |= self.status
        self.turn("tables", "lengths", "pools")
        for layer in self.layers:
            pop.pop_cache_copy_pages(layer.cache, self.n_kv, self.head_dim, self.page, self.n_pages, self.copies, self.beams)

    def _norm(self, x, weight):
        f = x.float()
        return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + 1e-6)).bfloat16() * weight

    def _rotate(self, x, positions):
        half = self.head_dim // 2
        angle = positions[:, None].float() * torch.exp(torch.arange(half, device="cuda") * (-math.log(10000.0) / half))
        c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
        a, b = x.float().split(half, -1)
        return torch.cat([a * c - b * s, a * s + b * c], -1).bfloat16()

    def forward(self, tokens, prompt):
        """Hidden states of the planned tokens: a prompt (the first row's) or one token of every beam."""
        n = tokens.numel()
        x, positions, table = self.embedding[tokens], self.positions[:n], self.now("tables")
        h, kv, hd = self.heads, self.n_kv, self.head_dim
        for layer in self.layers:
            q, k, v = (self._norm(x, layer.norm1) @ layer.wqkv.T).split([h * hd, kv * hd, kv * hd], -1)
            q = self._rotate(q.reshape(n, h, hd), positions).contiguous()
            k = self._rotate(k.reshape(n, kv, hd), positions).contiguous()
            pop.pop_cache_write(layer.cache, kv, hd, self.page, self.n_pages, k, v, BF16, self.slots, n)
            y = torch.empty_like(q)
            pop.pop_cache_attention(q, BF16, n, layer.cache, kv, hd, self.page, self.n_pages, table, table.shape[1], self.start,
                                    self.now("lengths"), self.beams, h, n if prompt else 1, self.max_tokens, hd ** -0.5, 0, y,
                                    BF16, self.workspace)
            x = x + y.view(n, h * hd) @ layer.wo.T
            z = self._norm(x, layer.norm2)
            out = torch.empty_like(z)
            if prompt:
                pop.pop_prefill_forward(layer.ffn, z, n, self.n_ret, self.n_cand, self.k, out, BF16)
            else:
                pop.pop_decode_step(layer.ffn, z, n, self.k, out, BF16)
            x = x + out
        return x

    def logits(self, x):
        return (x @ self.head.T).float()

    def prompt(self, tokens):
        """Runs the prompt in the first row; logits behind its last token, for every row."""
        new = _int32(self.beams)
        new[0] = tokens.numel()
        self.plan(new, tokens.numel())
        return self.logits(self.forward(tokens, True)[-1:]).expand(self.beams, -1).contiguous()

    def step(self, tokens):
        self.plan(_int32(self.beams, fill=1), self.beams)
        return self.logits(self.forward(tokens, False))


def beam_search(model: Decoder, prompt, new_tokens: int, eos: int = -1, pad: int = 0):
    """The best sequences of new tokens [beams][new_tokens] and their scores [beams], best first.  eos: a token that ends
    a beam, which then goes on by `pad`."""
    w = model.beams
    model.reset()
    logits = model.prompt(prompt)
    scores = torch.full((w,), -math.inf, device="cuda")
    scores[0] = 0.0  # the only row so far
    done = torch.zeros(w, dtype=torch.uint8, device="cuda")
    chosen = [torch.empty(w, device="cuda"), _int32(w), _int32(w)]
    history = torch.empty(w, 0, dtype=torch.int32, device="cuda")
    for i in range(new_tokens):
        pop.pop_beam_select(logits, pop.POP_F32, scores, done, 1, w, model.vocab, w, pad, *chosen, model.workspace)
        scores, tokens, parents = (t.clone() for t in chosen)
        at = parents.long()
        history = torch.cat([history[at], tokens[:, None]], 1)
        done = ((done[at] != 0) | (tokens == eos)).to(torch.uint8)
        model.reorder(parents)
        if i + 1 < new_tokens:
            logits = model.step(tokens)
    status = model.failed.tolist()
    if any(status):
        raise RuntimeError(f"the cache ran out of pages or was given wrong lengths (status {status})")
    return history, scores


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--beams", type=int, default=4)
    p.add_argument("--prompt", type=int, default=100, help="tokens of the (random) prompt")
    p.add_argument("--tokens", type=int, default=32, help="new tokens")
    p.add_argument("--seed", type=int, default=0)
    a = p.parse_args()
    model = Decoder(beams=a.beams, seed=a.seed, max_tokens=a.prompt + a.tokens + 16)
    prompt = torch.randint(0, model.vocab, (a.prompt,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(a.seed + 1))
    history, scores = beam_search(model, prompt, a.tokens)
    for row, score in zip(history.tolist(), scores.tolist()):
        print("%9.3f  %s" % (score, " ".join(map(str, row))))
    model.close()


if __name__ == "__main__":
    main()
