"""Performance cases of the operators around the pruned FFN in a decoder that serves several beams of a prompt: block
tables and slot maps built from request lengths, a paged cache of keys and values held in 4 bits with the attention that
reads it, beam search's selection, and the reordering of the cached states that follows it.

`own` false: every operator in its plain form, elementary torch operations in 32 bits.  `own` true: the calls that a
program makes of the library.  Inputs do not depend on it.

The cache's format (one layer).  Values are e2m1 codes (sign, 2 bits of exponent, 1 of significand: 0 .5 1 1.5 2 3 4 6)
with one scale byte for 32 channels, 2^(byte - 127).  A page holds `page` tokens of all kv heads; one head's 16 tokens are a
tile of 16 (D + D/16) bytes: K codes [16 tokens][D/2], V codes [4 groups of 4 tokens][16][4 tokens][D/32] (the 16 are D/16
channels each), K scales [16 tokens][D/32], V scales [4 groups][D/32][4 tokens]; the lower channel of a byte is its low nibble.
The cache is [pages][kv heads][page/16][tile].  A token's slot is its page's number times `page` plus its place there.
Free pages stand in a ring of page numbers; `pool` holds the first free one's place and how many are free.
"""
import math

import torch

own = False

F32, BF16 = 0, 1
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
CODE = {"f32": F32, "bf16": BF16}


# ---------------------------------------------------------------- cases

def listed():
    return [
        # a decode step's plan: eight sequences, one new token each; latency
        dict(name="plan_step_b8", kind="plan", n_seq=8, cached=2000, new=1, page=16, decode=True),
        # prompts admitted next to running sequences: ragged lengths, a quarter of a million slots
        dict(name="plan_prompts_b256", kind="plan", n_seq=256, cached=4096, new=2048, page=16, decode=False),
        # one decode step of four beams, small float32 layer
        dict(name="write_step_f32", kind="write", dtype="f32", tokens=4, n_kv=8, head_dim=64, page=16),
        # a prompt's keys and values, taken out of the rows of one joint projection at the Llama-2-7B shape; odd length
        dict(name="write_7b_t8191", kind="write", dtype="bf16", tokens=8191, n_kv=32, head_dim=128, page=64),
        # one short float32 sequence under a sliding window: the smallest attention call
        dict(name="decode_small_f32", kind="attention", dtype="f32", ydtype="f32", n_seq=1, new=1, context=77, n_heads=4,
             n_kv=2, head_dim=64, page=16, window=50),
        # the headline: eight sequences decode at the Llama-2-7B shape (32 heads, no sharing), ragged up to 4096 tokens
        dict(name="decode_7b_b8", kind="attention", dtype="bf16", ydtype="bf16", n_seq=8, new=1, context=4096, n_heads=32,
             n_kv=32, head_dim=128, page=16, window=0),
        # two long documents, four query heads to a kv head: work split over the long axis
        dict(name="decode_long_gqa", kind="attention", dtype="bf16", ydtype="bf16", n_seq=2, new=1, context=131072,
             n_heads=32, n_kv=8, head_dim=128, page=64, window=0),
        # ragged chunks of prompts at the Llama-2-7B shape over what is cached already: matrix products bound it
        dict(name="prompt_7b_chunks", kind="attention", dtype="bf16", ydtype="bf16", n_seq=4, new=2048, context=6144,
             n_heads=32, n_kv=32, head_dim=128, page=64, window=0),
        # one request of four beams at the Llama-2 vocabulary: latency
        dict(name="beam_4_v32000", kind="beam", dtype="bf16", requests=1, beams=4, vocab=32000, k=4),
        # many requests of eight beams, float32 logits of a wide odd vocabulary, twice as many candidates as beams
        dict(name="beam_32x8_v131071", kind="beam", dtype="f32", requests=32, beams=8, vocab=131071, k=16),
        # the states of one request's four beams after its selection
        dict(name="reorder_4", kind="reorder", requests=1, beams=4, context=700, n_kv=8, head_dim=128, page=16),
        # the states of 64 requests of eight beams, long contexts, pages of 64 tokens
        dict(name="reorder_64x8", kind="reorder", requests=64, beams=8, context=16000, n_kv=4, head_dim=128, page=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["plan", "write", "attention", "attention", "attention", "beam", "reorder"])
    if kind == "plan":
        n_seq = _log_int(rng, 1, 1000)
        return dict(kind=kind, n_seq=n_seq, cached=_log_int(rng, 1, 8000), new=_log_int(rng, 1, 400000 // n_seq),
                    page=rng.choice([16, 32, 64, 128]), decode=rng.random() < 0.3)
    if kind == "write":
        n_kv, d = rng.choice([1, 2, 3, 4, 8, 32, 40]), rng.choice([64, 128, 128, 256])
        return dict(kind=kind, dtype=rng.choice(["f32", "bf16"]), tokens=_log_int(rng, 1, (8191 * 32 * 128) // (n_kv * d) // 2),
                    n_kv=n_kv, head_dim=d, page=rng.choice([16, 32, 64]))
    if kind == "beam":
        requests, beams = _log_int(rng, 1, 32), rng.randint(1, 8)
        return dict(kind=kind, dtype=rng.choice(["f32", "bf16"]), requests=requests, beams=beams,
                    vocab=_log_int(rng, 1000, 131071), k=rng.randint(beams, 2 * beams))
    if kind == "reorder":
        return dict(kind=kind, requests=_log_int(rng, 1, 64), beams=rng.randint(2, 8), context=_log_int(rng, 20, 16000),
                    n_kv=rng.choice([1, 2, 4]), head_dim=rng.choice([64, 128]), page=rng.choice([16, 32, 64]))
    n_kv, share = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 5, 8, 16])
    d, dtype = rng.choice([64, 128, 128, 256]), rng.choice(["bf16", "bf16", "bf16", "f32"])
    case = dict(kind=kind, dtype=dtype, ydtype=rng.choice([dtype, dtype, "f32"]), n_heads=n_kv * share, n_kv=n_kv, head_dim=d,
                page=rng.choice([16, 32, 64, 128]), window=rng.choice([0, 0, 0, _log_int(rng, 10, 4000)]))
    if rng.random() < 0.6:  # single tokens
        n_seq = _log_int(rng, 1, 32)
        most = min(131072, (2 * 131072 * 8 * 128) // (n_seq * n_kv * d))
        return dict(case, n_seq=n_seq, new=1, context=_log_int(rng, 1, max(most, 2)))
    n_seq, new, before = rng.randint(1, 4), _log_int(rng, 2, 2048), _log_int(rng, 1, 4096)
    room = 4 * 32 * 128 * 2048 * 6144 / (n_seq * n_kv * share * d)  # new (new + before) of the largest listed one
    new = min(new, int((math.sqrt(before * before + 4 * room) - before) / 2))
    return dict(case, n_seq=n_seq, new=new, context=new + before)


def work(case):
    """Each input read once, each output written once; products that the result needs."""
    c = case
    if c["kind"] == "plan":
        cached, new = _plan_lengths(c, 0)
        pages = int(((cached + new + c["page"] - 1) // c["page"] - (cached + c["page"] - 1) // c["page"]).sum())
        return dict(bytes=16 * c["n_seq"] + 8 * int(new.sum()) + 8 * pages, flops=0)
    if c["kind"] == "write":
        n = 2 * c["tokens"] * c["n_kv"] * c["head_dim"]
        size = 4 if c["dtype"] == "f32" else 2
        return dict(bytes=2 * n * size + 2 * n * 17 // 32 + 4 * c["tokens"], flops=0)
    if c["kind"] == "beam":
        n = c["requests"] * c["beams"]
        return dict(bytes=n * c["vocab"] * (4 if c["dtype"] == "f32" else 2) + 12 * c["requests"] * c["k"], flops=0)
    if c["kind"] == "reorder":
        rows, blocks = c["requests"] * c["beams"], -(-c["context"] // c["page"])
        values = rows * c["page"] * c["n_kv"] * c["head_dim"]  # of keys in the rows' last pages, and as many of values
        return dict(bytes=8 * rows * blocks + values * (17 / 16 + 17 / 16 + 4), flops=0)
    context, new = _attention_lengths(c, 0)
    seen, pairs = 0, 0
    for L, n in zip(context, new):
        w = c["window"] or L
        seen += min(L, w + n - 1)
        first = L - n + 1  # keys that the first new token may see
        full = max(0, min(n, w - first + 1))  # new tokens that see all keys up to their own
        pairs += full * first + full * (full - 1) // 2 + (n - full) * w
    d, size, ysize = c["head_dim"], 4 if c["dtype"] == "f32" else 2, 4 if c["ydtype"] == "f32" else 2
    return dict(bytes=seen * c["n_kv"] * d * 17 // 16 + sum(new) * c["n_heads"] * d * (size + ysize),
                flops=4 * d * c["n_heads"] * pairs)


# ---------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _int32(x):
    return torch.as_tensor(x, dtype=torch.int32, device="cuda")


def _plan_lengths(case, seed):
    """Host: cached and new tokens of each sequence.  The seed puts them in another order: sums and bounds stay."""
    g = torch.Generator().manual_seed(17)
    n = case["n_seq"]
    cached = torch.randint(0, case["cached"] + 1, (n,), generator=g)
    if case["decode"]:
        new = torch.full((n,), 1)
    else:  # half of the sequences go on by one token, the others bring prompts; some of all of them have nothing cached
        new = torch.randint(1, 2 * case["new"] + 1, (n,), generator=g)
        new = torch.where(torch.rand(n, generator=g) < 0.5, torch.ones_like(new), new)
        cached = torch.where(torch.rand(n, generator=g) < 0.2, torch.zeros_like(cached), cached)
    order = torch.randperm(n, generator=torch.Generator().manual_seed(seed))
    return cached[order], new[order]


def _attention_lengths(case, seed):
    """Host: tokens in reach and new tokens of each sequence.  The first sequence is the longest; lengths do not depend on
    the seed, as the bytes and products of a case do not."""
    g = torch.Generator().manual_seed(23)
    context, new = [], []
    for i in range(case["n_seq"]):
        share = 1.0 if i == 0 else 0.25 + 0.75 * float(torch.rand((), generator=g))
        n = max(1, int(case["new"] * share))
        context.append(max(n, int(case["context"] * share)))
        new.append(n)
    return context, new


def _codes(x):
    """x [..., D] float32 -> e2m1 codes [..., D] and scale bytes [..., D/32] (uint8).  The scale's exponent is that of the
    block's largest magnitude less two, and one more where its significand is 1.75 or more; a value goes to the nearest
    code, halves to the even one."""
    x = torch.nan_to_num(x, nan=0.0)
    b = x.unflatten(-1, (-1, 32))
    top = b.abs().amax(-1).view(torch.int32)
    byte = (((top + 0x200000) >> 23) - 2).clamp(1, 252)
    y = b.abs() * ((254 - byte) << 23).view(torch.float32).unsqueeze(-1)
    code = (y > 0.25).to(torch.uint8)
    for edge, upper in ((0.75, False), (1.25, True), (1.75, False), (2.5, True), (3.5, False), (5.0, True)):
        code += (y > edge) if upper else (y >= edge)
    return (code | (torch.signbit(b).to(torch.uint8) << 3)).flatten(-2), byte.to(torch.uint8)


def _packed(c):
    return c[..., 0::2] | (c[..., 1::2] << 4)


def _tiles(k, v):
    """k, v [pages][page][n_kv][D] float32 -> the cache's bytes [pages][n_kv][page/16][tile]."""
    n, page, h, d = k.shape
    kc, ks = _codes(k)
    vc, vs = _codes(v)
    kc = _packed(kc).view(n, page // 16, 16, h, d // 2).permute(0, 3, 1, 2, 4).flatten(3)
    ks = ks.view(n, page // 16, 16, h, d // 32).permute(0, 3, 1, 2, 4).flatten(3)
    vc = _packed(vc).view(n, page // 16, 4, 4, h, 16, d // 32).permute(0, 4, 1, 2, 5, 3, 6).flatten(3)
    vs = vs.view(n, page // 16, 4, 4, h, d // 32).permute(0, 4, 1, 2, 5, 3).flatten(3)
    return torch.cat([kc, vc, ks, vs], -1)


def _random_cache(g, n_pages, page, n_kv, d):
    """Keys with a few channels that are larger than the others, as keys have, and values; in parts, they are large."""
    out = torch.empty(n_pages, n_kv, page // 16, 16 * (d + d // 16), dtype=torch.uint8, device="cuda")
    gain = torch.ones(n_kv, d, device="cuda")
    gain[:, :: max(d // 4, 1)] = 4.0
    part = max(1, (1 << 26) // (page * n_kv * d))
    for i in range(0, n_pages, part):
        n = min(part, n_pages - i)
        k = torch.randn(n, page, n_kv, d, generator=g, device="cuda") * gain
        v = torch.randn(n, page, n_kv, d, generator=g, device="cuda")
        out[i:i + n] = _tiles(k, v)
    return out


def _table(g, lengths, page, n_pages, extra):
    """Block table of sequences of the given lengths over pages in random order, -1 behind a sequence's last; the pages that are left."""
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    blocks = -(-torch.as_tensor(lengths, device="cuda") // page)
    start = torch.cumsum(blocks, 0) - blocks
    j = torch.arange(int(blocks.max()) + extra, device="cuda")
    at = (start[:, None] + j).clamp(max=n_pages - 1)
    return torch.where(j < blocks[:, None], order[at], -1).to(torch.int32).contiguous(), order[int(blocks.sum()):]


def prepare(case, seed):
    c = dict(case)
    g = _gen(seed)
    page = c.get("page")
    if c["kind"] == "plan":
        cached, new = _plan_lengths(c, seed)
        blocks = int((-(-(cached + new) // page)).sum())
        n_pages = blocks + 37
        table, free = _table(g, cached.tolist(), page, n_pages, 0)
        stride = int((-(-(cached + new) // page)).max()) + 5
        wide = torch.full((c["n_seq"], stride), -1, dtype=torch.int32, device="cuda")
        wide[:, :min(stride, table.shape[1])] = table[:, :stride]
        head = int(torch.randint(0, n_pages, (1,), generator=g, device="cuda"))
        ring = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
        ring[(head + torch.arange(free.numel(), device="cuda")) % n_pages] = free
        tokens = int(new.sum()) + 3  # the slot map has room for a few tokens more
        out = dict(context=_int32([0] * c["n_seq"]), start=_int32([0] * (c["n_seq"] + 1)), slots=_int32([0] * tokens),
                   positions=_int32([0] * tokens), pool=_int32([0, 0]), status=_int32([0]))
        return dict(c, cached_len=_int32(cached), new_len=_int32(new), table=wide, ring=ring, n_pages=n_pages,
                    pool=_int32([head, free.numel()]), tokens=tokens, out=out)
    if c["kind"] == "write":
        t, h, d = c["tokens"], c["n_kv"], c["head_dim"]
        n_pages = -(-t // page) + 5
        pages = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
        at = torch.arange(t, device="cuda") + page // 2  # the first page is half full already
        slots = (pages[at // page] * page + at % page).to(torch.int32)
        slots[t // 2 + 1:t // 2 + 3] = -1  # padding of the batch
        # rows of one projection: [q | k | v], here with as many query heads as kv heads
        rows = torch.randn(t, 3 * h * d, generator=g, device="cuda")
        rows[:, ::97] *= 6.0
        rows = rows.to(TORCH[c["dtype"]])
        cache = torch.zeros(n_pages, h, page // 16, 16 * (d + d // 16), dtype=torch.uint8, device="cuda")
        k_out = torch.empty(t, h, d, dtype=rows.dtype, device="cuda")
        return dict(c, k=rows[:, h * d:2 * h * d], v=rows[:, 2 * h * d:], slots=slots, cache=cache, n_pages=n_pages,
                    k_out=k_out, v_out=torch.empty_like(k_out))
    if c["kind"] == "attention":
        context, new = _attention_lengths(c, seed)
        n_pages = sum(-(-x // page) for x in context) + 3
        table, _ = _table(g, context, page, n_pages, 2)
        cache = _random_cache(g, n_pages, page, c["n_kv"], c["head_dim"])
        tokens = sum(new)
        q = (1.5 * torch.randn(tokens, c["n_heads"], c["head_dim"], generator=g, device="cuda")).to(TORCH[c["dtype"]])
        start = [0]
        for n in new:
            start.append(start[-1] + n)
        y = torch.empty(tokens, c["n_heads"], c["head_dim"], dtype=TORCH[c["ydtype"]], device="cuda")
        # a program sizes the workspace once for its largest batch; this bound holds for every case here
        workspace = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
        return dict(c, q=q, cache=cache, table=table, context_len=_int32(context), start=_int32(start), tokens=tokens,
                    n_pages=n_pages, max_new=max(new), max_context=max(context), scale=c["head_dim"] ** -0.5, y=y,
                    workspace=workspace)
    if c["kind"] == "beam":
        r, w, v, k = c["requests"], c["beams"], c["vocab"], c["k"]
        logits = torch.empty(r * w, v, dtype=TORCH[c["dtype"]], device="cuda")
        scores = torch.empty(r, w, device="cuda")
        done = torch.rand(r, w, generator=g, device="cuda") < 0.1
        bad = torch.ones(r, dtype=torch.bool, device="cuda")
        pad = 2
        while bool(bad.any()):  # scores of different rows that nearly tie have no order that rounding keeps: drawn again
            n = int(bad.sum())
            x = 2.0 * torch.randn(n * w, v, generator=g, device="cuda")
            x[:, 5::211] += 5.0
            x[torch.rand(n * w, v, generator=g, device="cuda") < 0.01] = -math.inf  # tokens that a grammar forbids
            logits.view(r, w, v)[bad] = x.view(n, w, v).to(logits.dtype)
            scores[bad] = -20.0 * torch.rand(n, w, generator=g, device="cuda")
            if w > 1 and seed % 2:
                scores[:, -1] = -math.inf  # a beam that is not alive yet
            top, alive = _beam_near(logits.view(r, w, v)[bad], scores[bad], done[bad], pad, k + 1)
            gap = top[:, :-1] - top[:, 1:]
            bad[bad.clone()] = ((gap > 0) & (gap < 2e-4) & alive[:, 1:]).any(1)
        workspace = torch.zeros(16 << 20, dtype=torch.uint8, device="cuda")
        out = dict(scores=torch.empty(r, k, device="cuda"), tokens=torch.empty(r, k, dtype=torch.int32, device="cuda"),
                   parents=torch.empty(r, k, dtype=torch.int32, device="cuda"))
        return dict(c, logits=logits, scores=scores.flatten().contiguous(), done=done.flatten().to(torch.uint8), pad=pad, out=out,
                    workspace=workspace)
    # reorder: beams of a request hold the pages of its prompt together and their own behind it
    r, w, h, d = c["requests"], c["beams"], c["n_kv"], c["head_dim"]
    length = torch.randint((c["context"] + 1) // 2, c["context"] + 1, (r, 1), generator=g, device="cuda").expand(r, w).clone()
    blocks = -(-length // page)
    nb = -(-c["context"] // page) + 3
    j = torch.arange(nb, device="cuda")
    common = (length // page - torch.randint(0, 7, (r, w), generator=g, device="cuda")).clamp(min=0)
    shared = (j < common[..., None]) & (torch.arange(w, device="cuda")[:, None] > 0)
    own_page = (j < blocks[..., None]) & ~shared
    number = (torch.cumsum(own_page.flatten(), 0) - 1).view(r, w, nb)
    used = int(own_page.sum())
    n_pages = r * nb + 10 * r * w + 11  # a row has eight blocks of its own at most; two for each row are free
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.where(own_page, order[number], -1)
    table = torch.where(shared, table[:, :1], table).to(torch.int32)
    parents = (w * torch.rand(r, w, generator=g, device="cuda") ** 1.5).to(torch.int32)
    parents[torch.rand(r, w, generator=g, device="cuda") < 0.03] = -1  # a beam that ended
    head = int(torch.randint(0, n_pages, (1,), generator=g, device="cuda"))
    free = order[used:]
    ring = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    ring[(head + torch.arange(free.numel(), device="cuda")) % n_pages] = free
    n = r * w
    # read back: the tokens of the pages that the ring hands out next
    slots = (free[:n, None].to(torch.int64) * page + torch.arange(page, device="cuda")).flatten().to(torch.int32)
    k_out = torch.empty(slots.numel(), h, d, dtype=torch.bfloat16, device="cuda")
    out = dict(table=torch.zeros(n, nb, dtype=torch.int32, device="cuda"), length=_int32([0] * n),
               copies=_int32([[0, 0]] * n), pool=_int32([0, 0]), status=_int32([0]))
    return dict(c, table=table.view(n, nb).contiguous(), length=length.flatten().to(torch.int32),
                parents=parents.flatten().contiguous(), ring=ring, pool=_int32([head, free.numel()]), n_pages=n_pages,
                cache=_random_cache(g, n_pages, page, h, d), slots=slots, k_out=k_out, v_out=torch.empty_like(k_out),
                workspace=torch.zeros(1 << 20, dtype=torch.uint8, device="cuda"), out=out)


def _beam_near(logits, scores, done, pad, k):
    """The k best scores in 64 bits, and which of them are no -inf."""
    x = logits.double()
    s = x - torch.logsumexp(x, -1, keepdim=True) + scores.double()[..., None]
    s = torch.where(done[..., None], -math.inf, s)
    s[..., pad] = torch.where(done, scores.double(), s[..., pad])
    top = torch.topk(s.flatten(1), min(k, s.flatten(1).shape[1]), -1).values
    return top, top > -math.inf


# ---------------------------------------------------------------- plain forms

def _ceil_div(a, b):
    return (a + b - 1) // b


def _plain_plan(s):
    page, n_pages, tokens = s["page"], s["n_pages"], s["tokens"]
    cached, new, table, ring = s["cached_len"].long(), s["new_len"].long(), s["table"], s["ring"]
    head, count = s["pool"].long()
    have, need = _ceil_div(cached, page), _ceil_div(cached + new, page)
    pages = need - have
    wrong = ((cached < 0) | (new < 0) | (need > table.shape[1])).any()
    status = (pages.sum() > count) * 1 + (new.sum() > tokens) * 2 + wrong * 4
    new = new * (status == 0)
    start = torch.cat([torch.zeros_like(new[:1]), torch.cumsum(new, 0)])
    first = torch.cumsum(pages, 0) - pages
    t = torch.arange(tokens, device="cuda")
    seq = torch.searchsorted(start[1:].contiguous(), t, right=True).clamp(max=len(new) - 1)
    valid = t < start[-1]
    pos = cached[seq] + t - start[seq]
    block = pos // page
    fresh = block >= have[seq]
    taken = ring[(head + first[seq] + block - have[seq]) % n_pages]
    number = torch.where(fresh, taken, table[seq, block.clamp(max=table.shape[1] - 1)]).long()
    slots = torch.where(valid & (number >= 0) & (number < n_pages), number * page + pos % page, -1)
    opens = valid & fresh & (pos % page == 0)
    table[seq[opens], block[opens]] = taken[opens]
    took = torch.where(status == 0, pages.sum(), 0)
    return dict(table=table, context=(cached + new).int(), start=start.int(), slots=slots.int(),
                positions=torch.where(valid, pos, -1).int(), pool=torch.stack([(head + took) % n_pages, count - took]).int(),
                status=status.int().view(1))


def _places(slots, page, n_kv, d):
    """Byte offsets in the cache, for tokens at `slots`: of K codes and V codes [tokens][n_kv][D/2], and of K and V scales
    [tokens][n_kv][D/32]."""
    tile_bytes = 16 * (d + d // 16)
    slots = slots.long()
    at = slots % page
    tile = ((slots // page)[:, None] * n_kv + torch.arange(n_kv, device="cuda")) * (page // 16) + (at // 16)[:, None]
    base = (tile * tile_bytes)[..., None]
    t = (at % 16)[:, None, None]
    j = torch.arange(d // 2, device="cuda")
    b = torch.arange(d // 32, device="cuda")
    w = d // 32  # bytes of one lane's channels
    k = base + t * (d // 2) + j
    v = base + 8 * d + (t // 4) * (2 * d) + (j // w) * (4 * w) + (t % 4) * w + j % w
    ks = base + 16 * d + t * w + b
    vs = base + 16 * d + 16 * w + (t // 4) * (4 * w) + b * 4 + t % 4
    return k, v, ks, vs


def _values(codes, scales):
    """Bytes [..., D/2] of codes and scale bytes [..., D/32] -> float32 [..., D]."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    m = (c & 7).float()
    mag = torch.where(m < 2, 0.5 * m, (1.0 + 0.5 * (m % 2)) * torch.exp2(torch.floor(m / 2) - 1.0))
    x = torch.where(c > 7, -mag, mag)
    return (x.unflatten(-1, (-1, 32)) * (scales.int() << 23).view(torch.float32).unsqueeze(-1)).flatten(-2)


def _plain_read(cache, slots, page, n_kv, d, dtype):
    k, v, ks, vs = _places(slots.clamp(min=0), page, n_kv, d)
    flat, there = cache.view(-1), (slots >= 0)[:, None, None]
    return (torch.where(there, _values(flat[k], flat[ks]), 0.0).to(dtype),
            torch.where(there, _values(flat[v], flat[vs]), 0.0).to(dtype))


def _plain_write(s):
    h, d, page, slots = s["n_kv"], s["head_dim"], s["page"], s["slots"]
    there = slots >= 0
    kc, ks = _codes(s["k"].float().view(-1, h, d)[there])
    vc, vs = _codes(s["v"].float().view(-1, h, d)[there])
    flat = s["cache"].view(-1)
    for where, what in zip(_places(slots[there], page, h, d), (_packed(kc), _packed(vc), ks, vs)):
        flat[where] = what
    k, v = _plain_read(s["cache"], slots, page, h, d, s["k"].dtype)
    return dict(k=k, v=v)


def _plain_attention(s):
    h, d, page, n_seq = s["n_kv"], s["head_dim"], s["page"], s["n_seq"]
    share = s["n_heads"] // h
    tile = 16 * (d + d // 16)
    table, context, start = s["table"].long(), s["context_len"].long(), s["start"].long()
    blocks = _ceil_div(s["max_context"], page)
    table = table[:, :blocks]
    w = d // 32
    raw = s["cache"][table.clamp(min=0)].permute(0, 2, 1, 3, 4).reshape(n_seq, h, -1, tile)  # [seq][head][tile in order]
    kc, vc, ks, vs = raw.split([8 * d, 8 * d, 16 * w, 16 * w], -1)
    k = _values(kc.unflatten(-1, (16, d // 2)), ks.unflatten(-1, (16, w))).flatten(2, 3)
    vc = vc.unflatten(-1, (4, 16, 4, w)).transpose(4, 5).reshape(n_seq, h, -1, 16, d // 2)
    vs = vs.unflatten(-1, (4, w, 4)).transpose(4, 5).reshape(n_seq, h, -1, 16, w)
    v = _values(vc, vs).flatten(2, 3)
    # queries, padded to the longest sequence's
    new = start[1:] - start[:-1]
    i = torch.arange(s["max_new"], device="cuda")
    row = (start[:-1, None] + i).clamp(max=s["tokens"] - 1)
    q = s["q"].float()[row].view(n_seq, s["max_new"], h, share, d).permute(0, 2, 1, 3, 4).reshape(n_seq, h, -1, d)
    pos = (context - new)[:, None] + i  # [seq][new]
    key = torch.arange(blocks * page, device="cuda")
    sees = (key <= pos[..., None]) & (key < context[:, None, None]) & (table >= 0).repeat_interleave(page, 1)[:, None]
    if s["window"]:
        sees &= key > pos[..., None] - s["window"]
    sees = sees[:, None, :, None].expand(n_seq, 1, s["max_new"], share, key.numel()).reshape(n_seq, 1, -1, key.numel())
    p = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(s["scale"]).masked_fill_(~sees, -math.inf)
    top = p.amax(-1, keepdim=True)
    p = p.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
    total = p.sum(-1, keepdim=True)
    y = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    y = y.view(n_seq, h, s["max_new"], share, d).permute(0, 2, 1, 3, 4).reshape(n_seq, s["max_new"], h * share, d)
    return y[i < new[:, None]].to(s["y"].dtype)


def _plain_beam(s):
    r, w, v, k = s["requests"], s["beams"], s["vocab"], s["k"]
    x = s["logits"].float().view(r, w, v)
    top = x.amax(-1, keepdim=True)
    shift = torch.where(top > -math.inf, top, 0.0)
    lse = shift + torch.log(torch.exp(x - shift).sum(-1, keepdim=True))
    was, done = s["scores"].view(r, w, 1), s["done"].view(r, w, 1) > 0
    new = torch.where(x > -math.inf, was + (x - lse), -math.inf)
    only = torch.where(torch.arange(v, device="cuda") == s["pad"], was, -math.inf)
    new = torch.where(done, only, new).flatten(1)
    # scores as ordered whole numbers, and below them the place, the lowest first: no two are equal
    bits = (new + 0.0).view(torch.int32).long()
    key = torch.where(bits < 0, bits ^ 0x7fffffff, bits) * (1 << 32) + ((1 << 32) - 1 - torch.arange(w * v, device="cuda"))
    at = (1 << 32) - 1 - (torch.topk(key, k, -1).values & 0xffffffff)
    return dict(scores=new.gather(1, at), tokens=(at % v).int(), parents=(at // v).int())


def _plain_reorder(s):
    w, page, n_pages = s["beams"], s["page"], s["n_pages"]
    n, nb = s["table"].shape
    r = n // w
    table, length = s["table"].view(r, w, nb), s["length"].view(r, w).long()
    parent, ring = s["parents"].view(r, w).long(), s["ring"]
    head, count = s["pool"].long()
    parent = torch.where((parent >= 0) & (parent < w), parent, -1)
    lives, p = parent >= 0, parent.clamp(min=0)
    same = (parent[:, :, None] == parent[:, None, :]) & lives[:, :, None]  # [child][other child]
    first = ~(same & torch.ones(w, w, dtype=torch.bool, device="cuda").tril(-1)).any(-1)
    took_len = torch.where(lives, length.gather(1, p), 0)
    blocks = _ceil_div(took_len, page)
    copied = lives & (took_len % page != 0) & ~first
    total = copied.sum()
    status = (total > count).int()
    fine = status == 0
    # rows
    j = torch.arange(nb, device="cuda")
    rows = torch.where(j < blocks[..., None], table.gather(1, p[..., None].expand(r, w, nb)), -1)
    order = (torch.cumsum(copied.flatten(), 0) - 1).view(r, w)
    fresh = ring[(head + order.clamp(min=0)) % n_pages]
    last = j == (blocks - 1)[..., None]
    source = torch.where(last, rows, 0).sum(-1)
    rows = torch.where(last & copied[..., None], fresh[..., None], rows)
    copies = torch.where((copied & fine)[..., None], torch.stack([source, fresh], -1), -1)
    was = torch.where(j < _ceil_div(length, page)[..., None], table, -1)
    # pages that no row holds any more, by request, block and row
    held = (was >= 0) & (was < n_pages)
    parented = (torch.arange(w, device="cuda")[:, None] == parent[:, None, :]).any(-1)  # [row]: has a child
    match = was[:, :, None, :] == was[:, None, :, :]
    kept = (match & parented[:, None, :, None]).any(2)
    earlier = (match & torch.ones(w, w, dtype=torch.bool, device="cuda").tril(-1)[None, :, :, None]).any(2)
    freed = (held & ~kept & ~earlier & fine).transpose(1, 2)
    pages = was.transpose(1, 2)[freed]
    ring[(head + count + torch.arange(pages.numel(), device="cuda")) % n_pages] = pages
    took = torch.where(fine, total, 0)
    cache, src = s["cache"], copies.view(n, 2)[copies.view(n, 2)[:, 0] >= 0].long()
    cache[src[:, 1]] = cache[src[:, 0]]
    k, v = _plain_read(cache, s["slots"], page, s["n_kv"], s["head_dim"], torch.bfloat16)
    return dict(table=torch.where(fine, rows, was).view(n, nb).int(), length=torch.where(fine, took_len, length).flatten().int(),
                copies=copies.view(n, 2).int(), ring=ring, k=k, v=v, status=status.view(1),
                pool=torch.stack([(head + took) % n_pages, count - took + pages.numel()]).int())


PLAIN = dict(plan=_plain_plan, write=_plain_write, attention=_plain_attention, beam=_plain_beam, reorder=_plain_reorder)


# ---------------------------------------------------------------- the library's calls

def _own_plan(s, pop):
    o = s["out"]
    pop.pop_cache_plan(s["cached_len"], s["new_len"], s["n_seq"], s["page"], s["table"], s["table"].shape[1], s["ring"],
                       s["n_pages"], s["pool"], o["pool"], s["tokens"], o["context"], o["start"], o["slots"],
                       o["positions"], o["status"])
    return dict(table=s["table"], context=o["context"], start=o["start"], slots=o["slots"], positions=o["positions"],
                pool=o["pool"], status=o["status"])


def _own_write(s, pop):
    h, d, t = s["n_kv"], s["head_dim"], s["tokens"]
    pop.pop_cache_write(s["cache"], h, d, s["page"], s["n_pages"], s["k"], s["v"], CODE[s["dtype"]], s["slots"], t)
    pop.pop_cache_read(s["cache"], h, d, s["page"], s["n_pages"], s["slots"], t, s["k_out"], s["v_out"], CODE[s["dtype"]])
    return dict(k=s["k_out"], v=s["v_out"])


def _own_attention(s, pop):
    pop.pop_cache_attention(s["q"], CODE[s["dtype"]], s["tokens"], s["cache"], s["n_kv"], s["head_dim"], s["page"],
                            s["n_pages"], s["table"], s["table"].shape[1], s["start"], s["context_len"], s["n_seq"],
                            s["n_heads"], s["max_new"], s["max_context"], s["scale"], s["window"], s["y"],
                            CODE[s["ydtype"]], s["workspace"])
    return s["y"]


def _own_beam(s, pop):
    o = s["out"]
    pop.pop_beam_select(s["logits"], CODE[s["dtype"]], s["scores"], s["done"], s["requests"], s["beams"], s["vocab"], s["k"],
                        s["pad"], o["scores"], o["tokens"], o["parents"], s["workspace"])
    return o


def _own_reorder(s, pop):
    o, h, d = s["out"], s["n_kv"], s["head_dim"]
    n, nb = s["table"].shape
    pop.pop_cache_reorder(s["table"], s["length"], s["parents"], n, s["beams"], s["page"], nb, o["table"], o["length"],
                          o["copies"], s["ring"], s["n_pages"], s["pool"], o["pool"], s["workspace"], o["status"])
    pop.pop_cache_copy_pages(s["cache"], h, d, s["page"], s["n_pages"], o["copies"], n)
    pop.pop_cache_read(s["cache"], h, d, s["page"], s["n_pages"], s["slots"], s["slots"].numel(), s["k_out"], s["v_out"], BF16)
    return dict(table=o["table"], length=o["length"], copies=o["copies"], ring=s["ring"], k=s["k_out"], v=s["v_out"],
                status=o["status"], pool=o["pool"])


OWN = dict(plan=_own_plan, write=_own_write, attention=_own_attention, beam=_own_beam, reorder=_own_reorder)


def run(state):
    if own:
        from paper_2602_06822_amd import binding as pop
        return OWN[state["kind"]](state, pop)
    return PLAIN[state["kind"]](state)


# ---------------------------------------------------------------- 64 bits, from the definitions

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_round(x):
    """What the 4-bit format keeps of x [..., D], in 64 bits."""
    b = x.double().unflatten(-1, (-1, 32))
    top = b.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(top)  # top = m 2^e, m in [.5, 1)
    e = torch.where(top > 0, e - 1 + (m >= 0.875).to(e.dtype) - 2, -126).clamp(-126, 125)
    y = torch.ldexp(b, -e)
    step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0)).double()
    return torch.ldexp((torch.round(y / step) * step).clamp(-6.0, 6.0), e).flatten(-2)


def _exact_stored(cache, n_kv, head, d, page, pages, tokens, value):
    """Tokens 0 .. tokens - 1 of one kv head of a sequence whose pages are given, [tokens][D] in 64 bits."""
    grid = torch.tensor(GRID, dtype=torch.float64, device="cuda")
    grid = torch.cat([grid, -grid])
    t = torch.arange(tokens, device="cuda")
    flat = cache[pages.long(), head].reshape(-1, cache.shape[-1])[t // 16]  # the tile of each token
    u, c = (t % 16)[:, None], torch.arange(d, device="cuda")[None]
    if value:
        lane, left = c // (d // 16), c % (d // 16)
        at = 8 * d + (((u // 4) * 16 + lane) * 4 + u % 4) * (d // 32) + left // 2
        scale = 16 * d + d // 2 + ((u // 4) * (d // 32) + c // 32) * 4 + u % 4
    else:
        at, scale = u * (d // 2) + c // 2, 16 * d + u * (d // 32) + c // 32
    code = (flat.gather(1, at) >> (4 * (c % 2)).to(torch.uint8)) & 15
    return torch.ldexp(grid[code.long()], flat.gather(1, scale).int() - 127)


def _exact_attention(s):
    d, h, share = s["head_dim"], s["n_kv"], s["n_heads"] // s["n_kv"]
    start, context = s["start"].tolist(), s["context_len"].tolist()
    y = torch.zeros(s["tokens"], s["n_heads"], d, dtype=torch.float64, device="cuda")
    for i, length in enumerate(context):
        a, b = start[i], start[i + 1]
        pages = s["table"][i, :-(-length // s["page"])]
        pos = length - (b - a) + torch.arange(b - a, device="cuda")[:, None]
        for head in range(h):
            k = _exact_stored(s["cache"], h, head, d, s["page"], pages, length, False)
            v = _exact_stored(s["cache"], h, head, d, s["page"], pages, length, True)
            key = torch.arange(length, device="cuda")[None]
            sees = (key <= pos) & ((key > pos - s["window"]) if s["window"] else (key >= 0))
            for one in range(head * share, (head + 1) * share):
                z = torch.where(sees, s["scale"] * (s["q"][a:b, one].double() @ k.T), -math.inf)
                y[a:b, one] = torch.softmax(z, -1) @ v
    return y


def exact(case, seed):
    s = prepare(case, seed)
    if s["kind"] == "write":
        there = (s["slots"] >= 0)[:, None, None]
        shape = (-1, s["n_kv"], s["head_dim"])
        return {x: torch.where(there, _exact_round(s[x].reshape(shape)), 0.0) for x in ("k", "v")}
    if s["kind"] == "attention":
        return _exact_attention(s)
    if s["kind"] == "beam":
        r, w, v, k = s["requests"], s["beams"], s["vocab"], s["k"]
        top = []
        for i in range(r):
            x = s["logits"][i * w:(i + 1) * w].double()
            z = torch.log_softmax(x, -1) + s["scores"][i * w:(i + 1) * w].double()[:, None]
            over = s["done"][i * w:(i + 1) * w] > 0
            z[over] = -math.inf
            z[over, s["pad"]] = s["scores"][i * w:(i + 1) * w].double()[over]
            top.append(torch.topk(z.flatten(), k).values)
        return dict(scores=torch.stack(top), tokens=None, parents=None)
    if s["kind"] == "reorder":
        d, h, page = s["head_dim"], s["n_kv"], s["page"]
        # rows one by one: the second and later children of a partly filled page take the ring's next page each
        parents, length, table = s["parents"].tolist(), s["length"].tolist(), s["table"].cpu()
        ring, (head, _) = s["ring"].cpu(), s["pool"].tolist()
        holds, taken, seen = {}, 0, set()
        for row, p in enumerate(parents):
            if p < 0:
                continue
            old = row - row % s["beams"] + p
            if length[old] % page and old in seen:
                holds[int(ring[(head + taken) % s["n_pages"]])] = int(table[old, length[old] // page])
                taken += 1
            seen.add(old)
        pages = (s["slots"].view(-1, page)[:, 0] // page).tolist()
        source = torch.tensor([holds.get(x, x) for x in pages], device="cuda", dtype=torch.int32)
        n = source.numel() * page
        out = [torch.stack([_exact_stored(s["cache"], h, one, d, page, source, n, value) for one in range(h)], 1)
               for value in (False, True)]
        return dict(table=None, length=None, copies=None, ring=None, k=out[0], v=out[1], status=None, pool=None)
    return None
