"""Performance cases of what a decoder layer needs next to the pruned FFN, the 4-bit cache and its attention: residual sums with the norms around a
block, rotary positions, attention with a sliding window and a few first tokens that stay visible, and attention of sequences that share a prefix.

`own` false: every operator in its plain form, elementary torch operations in 32 bits (angles of positions in 64).  `own` true: the calls
that a program makes of the library.  Inputs do not depend on it.

The cache's format (one layer).  Values are e2m1 codes (sign, 2 bits of exponent, 1 of significand: 0 .5 1 1.5 2 3 4 6) with one scale
byte for 32 channels, 2^(byte - 127).  A page holds `page` tokens of all kv heads; one head's 16 tokens are a tile of 16 (D + D/16)
bytes: K codes [16 tokens][D/2], V codes [4 groups of 4 tokens][16][4 tokens][D/32] (the 16 are D/16 channels each), K scales [16
tokens][D/32], V scales [4 groups][D/32][4 tokens]; the lower channel of a byte is its low nibble.  The cache is [pages][kv
heads][page/16][tile]; a row of the block table names a sequence's pages in order, -1 for none.
"""
import math

import torch

own = False

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
CODE = {"f32": 0, "bf16": 1}
SIZE = {"f32": 4, "bf16": 2}
EPS = 1e-5


# ---------------------------------------------------------------- cases

def listed():
    return [
        # one step of four beams of a small layer: latency
        dict(name="norm_step_b4", kind="norm", tokens=4, d=512, xdtype="bf16", dtype="bf16", post=False, gate="none", offset=0.0),
        # a prompt at the Llama-2-7B width: residual sum and the next block's norm; odd length
        dict(name="norm_7b_t2047", kind="norm", tokens=2047, d=4096, xdtype="bf16", dtype="bf16", post=False, gate="none", offset=0.0),
        # a long prompt at the Llama-2-13B width: residual stream in float32, norms on both sides of the block, a gate of its own for each token
        dict(name="norm_both_13b", kind="norm", tokens=4096, d=5120, xdtype="f32", dtype="bf16", post=True, gate="tokens", offset=1.0),
        # one step of eight sequences, four query heads to a kv head: latency
        dict(name="rotary_step_b8", kind="rotary", tokens=8, n_heads=32, n_kv=8, head_dim=128, rotary=128, layout="halves", dtype="bf16",
             farthest=4096, stretch=1.0),
        # a long prompt at the Llama-2-7B shape out of the rows of one joint projection, frequencies scaled for eight times the context
        dict(name="rotary_7b_t8191", kind="rotary", tokens=8191, n_heads=32, n_kv=32, head_dim=128, rotary=128, layout="halves", dtype="bf16",
             farthest=65536, stretch=8.0),
        # part of each head, neighbouring channels turned, float32, positions of a million: what the angles cost
        dict(name="rotary_part_f32", kind="rotary", tokens=1001, n_heads=24, n_kv=3, head_dim=80, rotary=40, layout="pairs", dtype="f32",
             farthest=1 << 20, stretch=1.0),
        # one short float32 sequence: the smallest attention call
        dict(name="sinks_small_f32", kind="sinks", dtype="f32", ydtype="f32", n_seq=1, new=1, context=300, n_heads=4, n_kv=2, head_dim=64, page=16,
             window=50, sinks=4),
        # thirty-two long conversations decode with a window; pages between the first tokens and the window have been given back
        dict(name="sinks_step_b32", kind="sinks", dtype="bf16", ydtype="bf16", n_seq=32, new=1, context=131072, n_heads=32, n_kv=8, head_dim=128,
             page=64, window=4096, sinks=4),
        # chunks of prompts under a window of an odd size, more first tokens than a tile holds
        dict(name="sinks_chunks", kind="sinks", dtype="bf16", ydtype="bf16", n_seq=4, new=2048, context=16384, n_heads=32, n_kv=32, head_dim=128,
             page=64, window=1001, sinks=17),
        # four beams of one prompt, the float32 layer of a small decoder: the smallest call with a shared prefix
        dict(name="shared_small_f32", kind="shared", dtype="f32", ydtype="f32", groups=1, group=4, new=1, prefix=700, own=30, n_heads=8, n_kv=4,
             head_dim=64, page=16),
        # eight beams of a 4000-token prompt at the Llama-2-7B shape
        dict(name="shared_7b_b8", kind="shared", dtype="bf16", ydtype="bf16", groups=1, group=8, new=1, prefix=4000, own=200, n_heads=32, n_kv=32,
             head_dim=128, page=16),
        # sixty-four sequences that ask about one long document, four query heads to a kv head
        dict(name="shared_b64_gqa", kind="shared", dtype="bf16", ydtype="bf16", groups=1, group=64, new=1, prefix=32768, own=700, n_heads=32,
             n_kv=8, head_dim=128, page=64),
    ]


def _log_int(rng, lo, hi):
    hi = max(lo, hi)
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "rotary", "rotary", "sinks", "sinks", "shared", "shared", "shared"])
    if kind == "norm":
        d = rng.choice([_log_int(rng, 64, 16384), 8 * _log_int(rng, 8, 2048), rng.choice([512, 4096, 5120, 8192])])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        return dict(kind=kind, tokens=_log_int(rng, 1, 4096 * 5120 // (2 * d)), d=d, xdtype=rng.choice([dtype, "f32"]), dtype=dtype,
                    post=rng.random() < 0.4, gate=rng.choice(["none", "none", "channels", "tokens"]), offset=rng.choice([0.0, 1.0]))
    if kind == "rotary":
        n_kv, share = rng.choice([1, 2, 3, 8, 32]), rng.choice([1, 1, 4, 7])
        d = rng.choice([64, 80, 128, 128, 256, 96])
        return dict(kind=kind, tokens=_log_int(rng, 1, 8191 * 32 * 128 // (n_kv * (share + 1) * d)), n_heads=n_kv * share, n_kv=n_kv, head_dim=d,
                    rotary=rng.choice([d, d, d // 2, 2 * rng.randint(1, d // 2)]), layout=rng.choice(["halves", "halves", "pairs"]),
                    dtype=rng.choice(["bf16", "bf16", "f32"]), farthest=_log_int(rng, 100, 1 << 20), stretch=rng.choice([1.0, 1.0, 4.0, 32.0]))
    n_kv, share = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 5, 8])
    d, dtype = rng.choice([64, 128, 128, 256]), rng.choice(["bf16", "bf16", "bf16", "f32"])
    case = dict(kind=kind, dtype=dtype, ydtype=rng.choice([dtype, dtype, "f32"]), n_heads=n_kv * share, n_kv=n_kv, head_dim=d,
                page=rng.choice([16, 32, 64, 128]))
    if kind == "sinks":
        window, sinks = _log_int(rng, 10, 8192), rng.choice([1, 4, 4, 16, rng.randint(1, 200)])
        if rng.random() < 0.6:  # single tokens
            n_seq = _log_int(rng, 1, 32)
            return dict(case, n_seq=n_seq, new=1, context=_log_int(rng, 1, 131072), window=window, sinks=sinks)
        n_seq, new = rng.randint(1, 4), _log_int(rng, 2, 2048)
        room = 4 * 2048 * 1000 * 32 * 128 // (n_seq * new * n_kv * share * d)  # positions that a token may see, as in the largest listed one
        return dict(case, n_seq=n_seq, new=new, context=new + _log_int(rng, 1, 14000), window=max(min(window, room - sinks), 10), sinks=sinks)
    group, groups = _log_int(rng, 2, 64), rng.choice([1, 1, 1, 2, 3])
    new = rng.choice([1, 1, 1, 2, 5, 16])
    new = max(1, min(new, 256 // (group * groups)))
    prefix = _log_int(rng, 1, min(32768, 64 * 32 * 128 * 32768 // (groups * group * new * n_kv * share * d)))
    return dict(case, groups=groups, group=group, new=new, prefix=prefix, own=_log_int(rng, max(new, 1), 700))


def work(case):
    """Each input read once, each output written once; products that the result needs."""
    c = case
    if c["kind"] == "norm":
        n, rows = c["tokens"] * c["d"], dict(none=0, channels=1, tokens=c["tokens"])[c["gate"]]
        weights = (1 + c["post"] + rows) * c["d"] * SIZE[c["dtype"]]
        return dict(bytes=n * (2 * SIZE[c["xdtype"]] + 2 * SIZE[c["dtype"]]) + weights, flops=n * (10 if c["post"] else 7))
    if c["kind"] == "rotary":
        heads = c["n_heads"] + c["n_kv"]
        return dict(bytes=c["tokens"] * (2 * heads * c["head_dim"] * SIZE[c["dtype"]] + 4) + 4 * c["rotary"],
                    flops=3 * c["tokens"] * heads * c["rotary"])
    d, h = c["head_dim"], c["n_heads"]
    if c["kind"] == "sinks":
        context, new = _sinks_lengths(c)
        seen = pairs = 0
        for length, n in zip(context, new):
            lo = max(length - n - c["window"] + 1, 0)
            seen += length - lo + min(c["sinks"], lo)
            for p in range(length - n, length):
                lo = max(p + 1 - c["window"], 0)
                pairs += p + 1 - lo + min(c["sinks"], lo)
    else:
        prefix, length, new = _shared_lengths(c)
        seen = sum(prefix) + sum(n - prefix[i // c["group"]] for i, n in enumerate(length))
        pairs = sum(n * m - m * (m - 1) // 2 for n, m in zip(length, new))
    return dict(bytes=seen * c["n_kv"] * d * 17 // 16 + sum(new) * h * d * (SIZE[c["dtype"]] + SIZE[c["ydtype"]]), flops=4 * d * h * pairs)


# ---------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _int32(x):
    return torch.as_tensor(x, dtype=torch.int32, device="cuda")


def _sinks_lengths(case):
    """Host: tokens in reach and new tokens of each sequence; the first sequence is the longest.  They do not depend on the seed, as the
    bytes and products of a case do not."""
    g = torch.Generator().manual_seed(29)
    context, new = [], []
    for i in range(case["n_seq"]):
        share = 1.0 if i == 0 else 0.25 + 0.75 * float(torch.rand((), generator=g))
        n = max(1, int(case["new"] * share))
        context.append(max(n, int(case["context"] * share)))
        new.append(n)
    return context, new


def _shared_lengths(case):
    """Host: shared tokens of each group, tokens in all and new tokens of each sequence."""
    g = torch.Generator().manual_seed(31)
    prefix, length, new = [], [], []
    for i in range(case["groups"]):
        prefix.append(max(1, int(case["prefix"] * (1.0 if i == 0 else 0.25 + 0.75 * float(torch.rand((), generator=g))))))
        for j in range(case["group"]):
            share = 1.0 if j == 0 else float(torch.rand((), generator=g))
            new.append(max(1, int(case["new"] * (0.5 + 0.5 * share))))
            length.append(prefix[-1] + max(new[-1], int(case["own"] * share)))
    return prefix, length, new


def _codes(x):
    """x [..., D] float32 -> e2m1 codes [..., D] and scale bytes [..., D/32] (uint8).  The scale's exponent is that of the block's largest
    magnitude less two, and one more where its significand is 1.75 or more; a value goes to the nearest code, halves to the even one."""
    b = x.unflatten(-1, (-1, 32))
    byte = (((b.abs().amax(-1).view(torch.int32) + 0x200000) >> 23) - 2).clamp(1, 252)
    y = b.abs() * ((254 - byte) << 23).view(torch.float32).unsqueeze(-1)
    code = (y > 0.25).to(torch.uint8)
    for edge, upper in ((0.75, False), (1.25, True), (1.75, False), (2.5, True), (3.5, False), (5.0, True)):
        code += (y > edge) if upper else (y >= edge)
    return (code | (torch.signbit(b).to(torch.uint8) << 3)).flatten(-2), byte.to(torch.uint8)


def _random_cache(g, n_pages, page, n_kv, d):
    """Keys with a few channels that are larger than the others, as keys have, and values; made in parts, they are large."""
    out = torch.empty(n_pages, n_kv, page // 16, 16 * (d + d // 16), dtype=torch.uint8, device="cuda")
    gain = torch.ones(d, device="cuda")
    gain[:: max(d // 4, 1)] = 4.0
    part, w = max(1, (1 << 26) // (page * n_kv * d)), d // 32
    for i in range(0, n_pages, part):
        n = min(part, n_pages - i)
        kc, ks = _codes(torch.randn(n, n_kv, page // 16, 16, d, generator=g, device="cuda") * gain)
        vc, vs = _codes(torch.randn(n, n_kv, page // 16, 4, 4, d, generator=g, device="cuda"))
        kc, vc = (x[..., 0::2] | (x[..., 1::2] << 4) for x in (kc, vc))
        vc = vc.unflatten(-1, (16, w)).transpose(4, 5)  # [group][16][4 tokens][D/32]
        out[i:i + n] = torch.cat([kc.flatten(3), vc.flatten(3), ks.flatten(3), vs.transpose(4, 5).flatten(3)], -1)
    return out


def _starts(new):
    return _int32([0] + torch.cumsum(torch.tensor(new), 0).tolist())


def _attention_state(c, g, table, n_pages, context, new):
    d = c["head_dim"]
    q = 1.5 * torch.randn(sum(new), c["n_heads"], d, generator=g, device="cuda")
    # a program sizes the workspace once for its largest batch; this holds for every case here
    return dict(c, q=q.to(TORCH[c["dtype"]]), cache=_random_cache(g, n_pages, c["page"], c["n_kv"], d), table=table, n_pages=n_pages,
                start=_starts(new), context_len=_int32(context), n_seq=len(new), tokens=sum(new), max_new=max(new), max_context=max(context),
                scale=d ** -0.5, y=torch.empty(sum(new), c["n_heads"], d, dtype=TORCH[c["ydtype"]], device="cuda"),
                workspace=torch.zeros(256 << 20, dtype=torch.uint8, device="cuda"))


def prepare(case, seed):
    c = dict(case)
    g = _gen(seed)
    if c["kind"] == "norm":
        n, d = c["tokens"], c["d"]
        wide, narrow = TORCH[c["xdtype"]], TORCH[c["dtype"]]
        x = torch.randn(n, d, generator=g, device="cuda")
        x[:, 7::211] *= 30.0  # a residual stream has a few channels that are much larger than the others
        gate = None
        if c["gate"] != "none":
            rows = 1 if c["gate"] == "channels" else n
            gate = torch.sigmoid(torch.randn(rows, d, generator=g, device="cuda")).to(narrow)

        def weight():
            return (1.0 - c["offset"] + 0.2 * torch.randn(d, generator=g, device="cuda")).to(narrow)

        u = (0.5 * torch.randn(n, d, generator=g, device="cuda")).to(narrow)
        return dict(c, x=x.to(wide), u=u, gate=gate, w_post=weight() if c["post"] else None, w_pre=weight(), x_scale=1.0, u_scale=0.25,
                    x_out=torch.empty(n, d, dtype=wide, device="cuda"), z=torch.empty(n, d, dtype=narrow, device="cuda"))
    if c["kind"] == "rotary":
        n, h, kv, d, r = c["tokens"], c["n_heads"], c["n_kv"], c["head_dim"], c["rotary"]
        rows = torch.randn(n, (h + 2 * kv) * d, generator=g, device="cuda").to(TORCH[c["dtype"]])  # of one projection: [q | k | v]
        # positions that go on from some place, of several sequences; some rows are padding
        at = torch.randint(0, c["farthest"], (3,), generator=g, device="cuda")
        i = torch.arange(n, device="cuda")
        positions = (at[3 * i // n] + i).to(torch.int32)
        positions[n // 2 + 1:n // 2 + 3] = -1
        # revolutions a token, in 64 bits: base 10000, the slow ones as many times slower as the context is stretched
        turns = torch.exp(-math.log(1e4) * torch.arange(0, r, 2, device="cuda", dtype=torch.float64) / r) / (2 * math.pi)
        slow = ((4.0 - 4096.0 * turns) / 3.0).clamp(0.0, 1.0)
        turns = turns * (1.0 - slow) + turns / c["stretch"] * slow
        out = [torch.zeros(n, x, d, dtype=rows.dtype, device="cuda") for x in (h, kv)]
        return dict(c, q=rows[:, :h * d], k=rows[:, h * d:(h + kv) * d], positions=positions, turns=turns,
                    amplitude=0.1 * math.log(c["stretch"]) + 1.0, q_out=out[0], k_out=out[1])
    page = c["page"]
    if c["kind"] == "sinks":
        # the pages that hold tokens between the first ones and the window's are none: given back, or never brought
        context, new = _sinks_lengths(c)
        length, fresh = _int32(context).long()[:, None], _int32(new).long()[:, None]
        block = torch.arange(-(-max(context) // page) + 2, device="cuda")[None]
        lo = (length - fresh - c["window"] + 1).clamp(min=0)
        held = (block * page < length) & ((block * page < c["sinks"]) | ((block + 1) * page > lo))
        n_pages = int(held.sum()) + 3
        order = torch.randperm(n_pages, generator=g, device="cuda")
        number = (torch.cumsum(held.flatten(), 0) - 1).view(held.shape)
        table = torch.where(held, order[number.clamp(min=0)], -1).to(torch.int32).contiguous()
        return _attention_state(c, g, table, n_pages, context, new)
    # shared: the full pages of a group's prefix are the same in all its rows; the page that the prefix ends in is copied for each row
    prefix, length, new = _shared_lengths(c)
    first = torch.arange(len(length), device="cuda") // c["group"] * c["group"]
    shared = (torch.tensor(prefix, device="cuda") // page).repeat_interleave(c["group"])[:, None]
    block = torch.arange(-(-max(length) // page) + 2, device="cuda")[None]
    held = block * page < _int32(length).long()[:, None]
    mine = held & ((block >= shared) | (first == torch.arange(len(length), device="cuda"))[:, None])
    n_pages = int(mine.sum()) + 3
    order = torch.randperm(n_pages, generator=g, device="cuda")
    number = (torch.cumsum(mine.flatten(), 0) - 1).view(mine.shape)
    table = torch.where(mine, order[number.clamp(min=0)], -1)
    table = torch.where(held & (block < shared), table[first], table)
    s = _attention_state(c, g, table.to(torch.int32).contiguous(), n_pages, length, new)
    last = table.gather(1, shared)[:, 0]  # (a row's own tokens begin in it, as in its copies' of the first row)
    s["cache"][last] = s["cache"][last[first]]
    return dict(s, prefix_len=_int32(prefix), max_prefix=max(prefix), max_own=max(n - prefix[i // c["group"]] for i, n in enumerate(length)))


# ---------------------------------------------------------------- plain forms

def _plain_norm(s):
    def normed(v, w):
        return v * torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS) * (w.float() + s["offset"])

    u = s["u"].float()
    if s["post"]:
        u = normed(u, s["w_post"])
    if s["gate"] is not None:
        u = u * s["gate"].float()
    x = s["x_scale"] * s["x"].float() + s["u_scale"] * u
    return dict(x=x.to(s["x"].dtype), z=normed(x, s["w_pre"]).to(s["u"].dtype))


def _plain_rotary(s):
    n, d, r = s["tokens"], s["head_dim"], s["rotary"]
    turn = s["positions"].double()[:, None] * s["turns"]
    angle = (2 * math.pi) * (turn - torch.round(turn))
    c, t = (s["amplitude"] * f(angle).float()[:, None] for f in (torch.cos, torch.sin))

    def turned(x, out):
        x = x.float().view(n, -1, d)
        pair = x[..., :r].unflatten(-1, (2, r // 2) if s["layout"] == "halves" else (r // 2, 2))
        a, b = pair.unbind(-2 if s["layout"] == "halves" else -1)
        y = torch.stack([a * c - b * t, a * t + b * c], -2 if s["layout"] == "halves" else -1).flatten(-2)
        return torch.where((s["positions"] >= 0)[:, None, None], torch.cat([y, x[..., r:]], -1).to(out.dtype), out)

    return dict(q=turned(s["q"], s["q_out"]), k=turned(s["k"], s["k_out"]))


def _values(codes, scales):
    """Bytes [..., D/2] of codes and scale bytes [..., D/32] -> float32 [..., D]."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    m = (c & 7).float()
    size = torch.where(m < 2, 0.5 * m, (1.0 + 0.5 * (m % 2)) * torch.exp2(torch.floor(m / 2) - 1.0))
    x = torch.where(c > 7, -size, size)
    return (x.unflatten(-1, (-1, 32)) * (scales.int() << 23).view(torch.float32).unsqueeze(-1)).flatten(-2)


def _stored(s, table, t):
    """Keys and values of tokens t [rows][n] (below 0: none) of sequences with the given block table rows: [rows][n_kv][n][D] float32, and which are there."""
    h, d, page = s["n_kv"], s["head_dim"], s["page"]
    w, at = d // 32, t.clamp(min=0)
    number = table.long().gather(1, (at // page).clamp(max=table.shape[1] - 1))
    there = (t >= 0) & (at // page < table.shape[1]) & (number >= 0) & (number < s["n_pages"])
    number = torch.where(there, number, 0)
    tile = (number[:, None] * h + torch.arange(h, device="cuda")[:, None]) * (page // 16) + (at % page // 16)[:, None]
    base, u = (tile * (16 * (d + d // 16)))[..., None], (at % 16)[:, None, :, None]
    j, b, flat = torch.arange(d // 2, device="cuda"), torch.arange(w, device="cuda"), s["cache"].view(-1)
    k = _values(flat[base + u * (d // 2) + j], flat[base + 16 * d + u * w + b])
    v = _values(flat[base + 8 * d + (u // 4) * (2 * d) + (j // w) * (4 * w) + (u % 4) * w + j % w],
                flat[base + 16 * d + 16 * w + (u // 4) * (4 * w) + b * 4 + u % 4])
    return k, v, there


def _queries(s):
    """Query columns, padded to the longest sequence's: [seq][n_kv][new x share][D] float32, their positions [seq][new] (-1: none), and which rows are there."""
    n_seq, h, d = s["n_seq"], s["n_kv"], s["head_dim"]
    start, i = s["start"].long(), torch.arange(s["max_new"], device="cuda")
    new = (start[1:] - start[:-1])[:, None]
    q = s["q"].float()[(start[:-1, None] + i).clamp(max=s["tokens"] - 1)]
    q = q.view(n_seq, s["max_new"], h, -1, d).permute(0, 2, 1, 3, 4).reshape(n_seq, h, -1, d)
    return q, torch.where(i < new, s["context_len"].long()[:, None] - new + i, -1), i < new


def _columns(s, sees):
    """sees [seq][new][keys] -> [seq][1][new x share][keys]."""
    return sees.repeat_interleave(s["n_heads"] // s["n_kv"], 1)[:, None]


def _scores(s, q, k, sees):
    return torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(s["scale"]).masked_fill_(~sees, -math.inf)


def _rows(s, y, live):
    """Columns [seq][n_kv][new x share][D] -> the rows of y."""
    y = y.view(s["n_seq"], s["n_kv"], s["max_new"], -1, s["head_dim"]).permute(0, 2, 1, 3, 4).flatten(2, 3)
    return y[live].to(s["y"].dtype)


def _plain_sinks(s):
    q, pos, live = _queries(s)
    first = torch.where(live, pos, pos.amax()).amin(-1, keepdim=True)
    lo = (first - s["window"] + 1).clamp(min=0)
    begin, near = torch.arange(s["sinks"], device="cuda"), lo + torch.arange(min(s["window"] + s["max_new"], s["max_context"]), device="cuda")
    t = torch.cat([begin.expand(s["n_seq"], -1), torch.where(near >= s["sinks"], near, -1)], 1)
    k, v, there = _stored(s, s["table"], t)
    t, p = t[:, None], pos[..., None]
    sees = _columns(s, there[:, None] & (t <= p) & ((t < s["sinks"]) | (p - t < s["window"])))
    z = _scores(s, q, k, sees)
    top = z.amax(-1, keepdim=True)
    w = z.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
    total = w.sum(-1, keepdim=True)
    return _rows(s, torch.matmul(w, v) / torch.where(total > 0, total, 1.0), live)


def _plain_shared(s):
    groups, group, h, d = s["groups"], s["group"], s["n_kv"], s["head_dim"]
    q, pos, live = _queries(s)
    prefix = s["prefix_len"].long()
    own_first = prefix.repeat_interleave(group)[:, None]
    # the prefix, once a group, for the columns of all its sequences
    t = torch.arange(s["max_prefix"], device="cuda")
    t = torch.where(t < prefix[:, None], t, -1)
    k, v, there = _stored(s, s["table"].view(groups, group, -1)[:, 0], t)
    t, there = (x.repeat_interleave(group, 0)[:, None] for x in (t, there))
    sees = _columns(s, there & (t <= pos[..., None]))

    def of_group(x):
        return x.unflatten(0, (groups, group)).transpose(1, 2).flatten(2, 3)

    def of_sequences(x):
        return x.unflatten(2, (group, -1)).transpose(1, 2).flatten(0, 1)

    z1 = of_sequences(_scores(s, of_group(q).contiguous(), k, of_group(sees)))
    # and the tokens behind it
    t = own_first + torch.arange(s["max_own"], device="cuda")
    mine_k, mine_v, there = _stored(s, s["table"], torch.where(t < s["context_len"].long()[:, None], t, -1))
    z2 = _scores(s, q, mine_k, _columns(s, there[:, None] & (t[:, None] <= pos[..., None])))
    top = torch.maximum(z1.amax(-1, keepdim=True), z2.amax(-1, keepdim=True))
    top = torch.where(top > -math.inf, top, 0.0)
    w1, w2 = z1.sub_(top).exp_(), z2.sub_(top).exp_()
    total = w1.sum(-1, keepdim=True) + w2.sum(-1, keepdim=True)
    y = of_sequences(torch.matmul(of_group(w1).contiguous(), v)) + torch.matmul(w2, mine_v)
    return _rows(s, y / torch.where(total > 0, total, 1.0), live)


PLAIN = dict(norm=_plain_norm, rotary=_plain_rotary, sinks=_plain_sinks, shared=_plain_shared)


# ---------------------------------------------------------------- the library's calls

def _own_norm(s, pop):
    rows = 0 if s["gate"] is None else s["gate"].shape[0]
    pop.pop_block_norm(s["x"], CODE[s["xdtype"]], s["u"], CODE[s["dtype"]], s["tokens"], s["d"], s["x_out"], s["z"], s["w_pre"],
                       post_norm=s["post"], w_post=s["w_post"], gate=s["gate"], gate_rows=rows, weight_offset=s["offset"], eps=EPS,
                       x_scale=s["x_scale"], u_scale=s["u_scale"])
    return dict(x=s["x_out"], z=s["z"])


def _own_rotary(s, pop):
    layout = pop.POP_ROTARY_HALVES if s["layout"] == "halves" else pop.POP_ROTARY_PAIRS
    pop.pop_rotary(s["q"], s["k"], CODE[s["dtype"]], s["tokens"], s["n_heads"], s["n_kv"], s["head_dim"], s["rotary"], layout, s["positions"],
                   s["turns"], s["amplitude"], s["q_out"], s["k_out"])
    return dict(q=s["q_out"], k=s["k_out"])


def _own_sinks(s, pop):
    pop.pop_cache_attention_sinks(s["q"], CODE[s["dtype"]], s["tokens"], s["cache"], s["n_kv"], s["head_dim"], s["page"], s["n_pages"],
                                  s["table"], s["table"].shape[1], s["start"], s["context_len"], s["n_seq"], s["n_heads"], s["max_new"],
                                  s["max_context"], s["scale"], s["window"], s["sinks"], s["y"], CODE[s["ydtype"]], s["workspace"])
    return s["y"]


def _own_shared(s, pop):
    pop.pop_cache_attention_shared(s["q"], CODE[s["dtype"]], s["tokens"], s["cache"], s["n_kv"], s["head_dim"], s["page"], s["n_pages"],
                                   s["table"], s["table"].shape[1], s["start"], s["context_len"], s["n_seq"], s["group"], s["prefix_len"],
                                   s["n_heads"], s["max_new"], s["max_context"], s["scale"], s["y"], CODE[s["ydtype"]], s["workspace"])
    return s["y"]


OWN = dict(norm=_own_norm, rotary=_own_rotary, sinks=_own_sinks, shared=_own_shared)


def run(state):
    if own:
        from paper_2602_06822_amd import binding as pop
        return OWN[state["kind"]](state, pop)
    return PLAIN[state["kind"]](state)


# ---------------------------------------------------------------- 64 bits, from the definitions

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_stored(s, head, pages, tokens, value):
    """Tokens 0 .. tokens - 1 of one kv head of a sequence whose pages are given, [tokens][D] in 64 bits (of pages that are none: anything)."""
    grid = torch.tensor(GRID, dtype=torch.float64, device="cuda")
    grid, d = torch.cat([grid, -grid]), s["head_dim"]
    t = torch.arange(tokens, device="cuda")
    tiles = s["cache"][pages.long().clamp(min=0), head].reshape(-1, s["cache"].shape[-1])[t // 16]  # the tile of each token
    u, c = (t % 16)[:, None], torch.arange(d, device="cuda")[None]
    if value:
        at = 8 * d + (((u // 4) * 16 + c // (d // 16)) * 4 + u % 4) * (d // 32) + c % (d // 16) // 2
        scale = 16 * d + d // 2 + ((u // 4) * (d // 32) + c // 32) * 4 + u % 4
    else:
        at, scale = u * (d // 2) + c // 2, 16 * d + u * (d // 32) + c // 32
    code = (tiles.gather(1, at) >> (4 * (c % 2)).to(torch.uint8)) & 15
    return torch.ldexp(grid[code.long()], tiles.gather(1, scale).int() - 127)


def _exact_attention(s):
    """Every sequence by itself, from its own row of the table."""
    h, share = s["n_kv"], s["n_heads"] // s["n_kv"]
    start, context = s["start"].tolist(), s["context_len"].tolist()
    y = torch.zeros(s["tokens"], s["n_heads"], s["head_dim"], dtype=torch.float64, device="cuda")
    for i, length in enumerate(context):
        a, b = start[i], start[i + 1]
        pages = s["table"][i, :-(-length // s["page"])]
        key, pos = torch.arange(length, device="cuda")[None], length - (b - a) + torch.arange(b - a, device="cuda")[:, None]
        sees = (key <= pos) & (pages >= 0).repeat_interleave(s["page"])[:length]
        if s["kind"] == "sinks":
            sees &= (key > pos - s["window"]) | (key < s["sinks"])
        some = torch.nonzero(sees.any(0))[:, 0]  # (of a long context, few)
        for head in range(h):
            k, v = (_exact_stored(s, head, pages, length, value)[some] for value in (False, True))
            for one in range(head * share, (head + 1) * share):
                z = torch.where(sees[:, some], s["scale"] * (s["q"][a:b, one].double() @ k.T), -math.inf)
                y[a:b, one] = torch.softmax(z, -1) @ v
    return y


def exact(case, seed):
    s = prepare(case, seed)
    if s["kind"] == "norm":
        u, x = s["u"].double(), s["x"].double()
        if s["post"]:
            u = u / torch.sqrt(torch.linalg.vector_norm(u, dim=-1, keepdim=True) ** 2 / s["d"] + EPS) * (s["offset"] + s["w_post"].double())
        x = s["x_scale"] * x + s["u_scale"] * (u if s["gate"] is None else u * s["gate"].double())
        z = x / torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / s["d"] + EPS) * (s["offset"] + s["w_pre"].double())
        return dict(x=x, z=z)
    if s["kind"] == "rotary":
        # a turned pair is a product of complex numbers; the angle goes in two parts, so that far positions lose nothing
        p, r, out = s["positions"].double()[:, None], s["rotary"], {}
        high, low = torch.floor(p / 1024) * 1024, p % 1024
        unit = [torch.polar(torch.ones_like(x * s["turns"]), 2 * math.pi * (x * s["turns"] % 1.0)) for x in (high, low)]
        unit = s["amplitude"] * (unit[0] * unit[1])[:, None]
        for name in ("q", "k"):
            y = s[name].double().reshape(s["tokens"], -1, s["head_dim"]).clone()
            re, im = (slice(0, r // 2), slice(r // 2, r)) if s["layout"] == "halves" else (slice(0, r, 2), slice(1, r, 2))
            z = torch.complex(y[..., re].contiguous(), y[..., im].contiguous()) * unit
            y[..., re], y[..., im] = z.real, z.imag
            y[s["positions"] < 0] = 0.0  # (rows of padding are left as they were)
            out[name] = y
        return out
    return _exact_attention(s)
