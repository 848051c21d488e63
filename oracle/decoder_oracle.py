"""Plain 64-bit forms of the operators around the FFN: the 4-bit cache's format, block tables, attention, beam search.

Test infrastructure only, written from the definitions in include/pop.h with loops over sequences, heads and tokens; it
shares no code with the HIP path.  Everything is numpy on the host.
"""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


# ---------------------------------------------------------------- format

def encode(x):
    """x [..., D] (any float) -> codes [..., D] and scale bytes [..., D/32], by trying all eight magnitudes."""
    x = np.asarray(x, dtype=np.float64)
    x = np.where(np.isnan(x), 0.0, x)
    x = np.clip(x, -float(np.finfo(np.float32).max), float(np.finfo(np.float32).max))
    b = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    top = np.abs(b).max(-1)
    m, e = np.frexp(top)  # top = m 2^e, 1/2 <= m < 1
    e = np.where(top > 0, e - 1 + (m >= 0.875), -1000) - 2 + 127
    byte = np.clip(e, 1, 252).astype(np.int64)
    y = np.abs(b) * np.exp2(127.0 - byte)[..., None]
    dist = np.abs(y[..., None] - GRID)
    near = dist.min(-1, keepdims=True)
    # the nearest magnitude; of two that are as near, the one with an even code
    even_first = np.argsort(np.arange(8) % 2, kind="stable")
    code = even_first[np.argmax((dist == near)[..., even_first], axis=-1)]
    code = np.where(y > 6.0, 7, code) | (np.signbit(b).astype(np.int64) << 3)
    return code.reshape(x.shape), byte


def decode(code, byte):
    code, byte = np.asarray(code), np.asarray(byte)
    v = np.where(code & 8, -1.0, 1.0) * GRID[code & 7]
    v = v.reshape(*code.shape[:-1], code.shape[-1] // 32, 32) * np.exp2(byte - 127.0)[..., None]
    return v.reshape(code.shape)


def tile_bytes(d):
    return 16 * (d + d // 16)


def byte_places(d, t):
    """Where token t (0 .. 15) of a tile stands: byte and nibble of each channel's K and V code, and its scale bytes."""
    k, v, ks, vs = [], [], [], []
    w = d // 32
    for c in range(d):
        k.append((t * (d // 2) + c // 2, c % 2))
        lane, left = divmod(c, d // 16)
        v.append((8 * d + (((t // 4) * 16 + lane) * 4 + t % 4) * w + left // 2, left % 2))
    for b in range(w):
        ks.append(16 * d + t * w + b)
        vs.append(16 * d + 16 * w + ((t // 4) * w + b) * 4 + t % 4)
    return k, v, ks, vs


def store(cache, page_tokens, d, slot, head, k, v):
    """One token and head into cache (uint8 [pages][n_kv][page/16][tile])."""
    page, at = divmod(int(slot), page_tokens)
    tile = cache[page, head, at // 16]
    pk, pv, pks, pvs = byte_places(d, at % 16)
    for places, scales, x in ((pk, pks, k), (pv, pvs, v)):
        code, byte = encode(x)
        for c, (i, high) in enumerate(places):
            tile[i] = (tile[i] & 0x0F) | (code[c] << 4) if high else (tile[i] & 0xF0) | code[c]
        for b, i in enumerate(scales):
            tile[i] = byte[b]


def load(cache, page_tokens, d, slot, head):
    page, at = divmod(int(slot), page_tokens)
    tile = cache[page, head, at // 16].astype(np.int64)
    pk, pv, pks, pvs = byte_places(d, at % 16)
    out = []
    for places, scales in ((pk, pks), (pv, pvs)):
        code = np.array([(tile[i] >> 4) if high else (tile[i] & 15) for i, high in places])
        out.append(decode(code, tile[scales]))
    return out


# ---------------------------------------------------------------- tables

def plan(cached, new, page_tokens, table, ring, pool, max_tokens):
    """Sequence by sequence, token by token.  Returns (table, context, start, slots, positions, pool, status)."""
    n_pages, (head, count) = len(ring), pool
    table = table.copy()
    pages = lambda n: -(-int(n) // page_tokens)  # noqa: E731
    status = 0 if 0 <= head < n_pages and 0 <= count <= n_pages else 4
    need = tokens = 0
    for c, n in zip(cached, new):
        if c < 0 or n < 0 or pages(int(c) + int(n)) > table.shape[1]:
            status |= 4
            continue
        need += pages(int(c) + int(n)) - pages(c)
        tokens += int(n)
    status |= (1 if need > count else 0) | (2 if tokens > max_tokens else 0)
    slots, positions = np.full(max_tokens, -1), np.full(max_tokens, -1)
    if status:
        return table, np.array(cached), np.zeros(len(cached) + 1, int), slots, positions, tuple(pool), status
    start, t, taken = [0], 0, 0
    for s, (c, n) in enumerate(zip(cached, new)):
        for b in range(pages(c), pages(int(c) + int(n))):
            table[s, b] = ring[(head + taken) % n_pages]
            taken += 1
        for p in range(int(c), int(c) + int(n)):
            page = table[s, p // page_tokens]
            slots[t] = page * page_tokens + p % page_tokens if 0 <= page < n_pages else -1
            positions[t] = p
            t += 1
        start.append(t)
    return (table, np.array(cached) + np.array(new), np.array(start), slots, positions,
            ((head + taken) % n_pages, count - taken), 0)


def reorder(table, length, parents, n_beams, page_tokens, ring, pool):
    """Returns (new_table, new_len, copies, ring, pool, status)."""
    n_seq, stride = table.shape
    n_pages, (head, count) = len(ring), pool
    ring = ring.copy()
    blocks = [min(-(-max(int(x), 0) // page_tokens), stride) for x in length]
    new_table, new_len = np.full_like(table, -1), np.zeros(n_seq, int)
    copies = np.full((n_seq, 2), -1)
    taken = 0
    for g in range(0, n_seq, n_beams):
        goes_on = set()
        for c in range(n_beams):
            p = int(parents[g + c])
            if not 0 <= p < n_beams:
                continue
            old = g + p
            new_len[g + c] = length[old]
            new_table[g + c, :blocks[old]] = table[old, :blocks[old]]
            if length[old] > 0 and length[old] % page_tokens and p in goes_on and 0 <= table[old, blocks[old] - 1] < n_pages:
                fresh = ring[(head + taken) % n_pages]
                taken += 1
                copies[g + c] = table[old, blocks[old] - 1], fresh
                new_table[g + c, blocks[old] - 1] = fresh
            goes_on.add(p)
    wrong = any(x < 0 or -(-int(x) // page_tokens) > stride for x in length)
    if wrong or taken > count:
        same = np.full_like(table, -1)
        for r in range(n_seq):
            same[r, :blocks[r]] = table[r, :blocks[r]]
        return same, np.array(length), np.full((n_seq, 2), -1), ring, tuple(pool), 4 if wrong else 1
    freed = 0
    for g in range(0, n_seq, n_beams):
        keeps = {g + int(p) for p in parents[g:g + n_beams] if 0 <= p < n_beams}
        for j in range(stride):
            kept = {int(table[r, j]) for r in keeps if j < blocks[r]}
            for r in range(g, g + n_beams):
                if j < blocks[r] and 0 <= table[r, j] < n_pages and int(table[r, j]) not in kept:
                    ring[(head + count + freed) % n_pages] = table[r, j]
                    freed += 1
                    kept.add(int(table[r, j]))
    return new_table, new_len, copies, ring, ((head + taken) % n_pages, count - taken + freed), 0


# ---------------------------------------------------------------- attention

def attention(q, k, v, scale, first_pos, window=0, there=None, sizes=None):
    """One sequence: q [new][heads][D]; k, v [context][kv heads][D]; there [context]: tokens whose page exists.
    sizes: a list that gets (sum of weight |v|, largest sum |scale q k|), both [new][heads].., for error bounds."""
    new, heads, d = q.shape
    context, n_kv, _ = k.shape
    y, weight, product = np.zeros((new, heads, d)), np.zeros((new, heads, d)), np.zeros((new, heads, 1))
    if sizes is not None:
        sizes += [weight, product]
    key = np.arange(context)
    for i in range(new):
        pos = first_pos + i
        sees = key <= pos
        if window:
            sees &= key > pos - window
        if there is not None:
            sees &= there
        if not sees.any():
            continue
        for h in range(heads):
            kv = h // (heads // n_kv)
            z = scale * (k[sees, kv].astype(np.float64) @ q[i, h].astype(np.float64))
            p = np.exp(z - z.max())
            y[i, h] = (p / p.sum()) @ v[sees, kv].astype(np.float64)
            if sizes is not None:
                weight[i, h] = (p / p.sum()) @ np.abs(v[sees, kv].astype(np.float64))
                product[i, h] = (abs(scale) * (np.abs(k[sees, kv].astype(np.float64)) @ np.abs(q[i, h].astype(np.float64)))).max()
    return y


# ---------------------------------------------------------------- beams

def beam_select(logits, scores, done, k, pad):
    """One request: logits [beams][vocab].  Returns (scores, tokens, parents): the order is (score descending, place)."""
    beams, vocab = logits.shape
    out = np.full((beams, vocab), -np.inf)
    for b in range(beams):
        if done is not None and done[b]:
            out[b, pad] = scores[b]
            continue
        x = logits[b].astype(np.float64)
        x = np.where(np.isnan(x), -np.inf, x)
        if scores[b] == -np.inf or not np.isfinite(x).any():
            continue
        down = x - x.max()  # (first, so that the sum's logarithm is not lost beside masks of a type's lowest value)
        out[b] = np.where(np.isfinite(x), float(scores[b]) + (down - np.log(np.exp(down).sum())), -np.inf)
    flat = out.ravel()
    at = np.argsort(-flat, kind="stable")[:k]
    return flat[at], at % vocab, at // vocab
