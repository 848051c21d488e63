"""Norms around a block and rotary positions on the GPU against their 64-bit oracle."""
import numpy as np
import pytest
import torch

from oracle import decoder_oracle as orc

pytestmark = pytest.mark.gpu
F32, BF16 = 0, 1
DT = {F32: torch.float32, BF16: torch.bfloat16}
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}  # a rounding of the type: half a step
U = 2.0 ** -24


@pytest.fixture(scope="module")
def pop():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2602_06822_amd import binding
    return binding


def f64(t):
    torch.cuda.synchronize()
    return t.double().cpu().numpy()


def bits(t):
    torch.cuda.synchronize()
    return t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32).cpu().numpy()


def rows(rng, n, d, dtype, pad=0, size=1.0, at=0):
    """n rows of d on the device, `pad` elements between them and `at` in front of the first."""
    flat = torch.from_numpy((size * rng.standard_normal(at + n * (d + pad))).astype(np.float32)).cuda().to(DT[dtype])
    return flat[at:].view(n, d + pad)[:, :d]


# ---------------------------------------------------------------- norms

def norm_bounds(x, u, xo, z, dtype, xdtype, d, *, gate, w_post, w_pre, post, offset, x_scale, u_scale, eps):
    """How far x' and z may be off.  A sum of squares: a thread's 64 terms at most one by one, a tree of six, up to 16 waves: 86 roundings of
    positive terms; its mean, eps, root and inverse 4; halved by the root but for the last two: 48 in r.  u': product by r, by the weight (a sum
    with the offset and a product), by the gate, by the scale: 5 more.  x': the scaled x and the sum, 2 of their own sizes."""
    r = 48 * U
    x, u = np.abs(x.astype(np.float64)), None if u is None else u.astype(np.float64)
    sized = np.zeros_like(x)
    if u is not None:
        sized = np.abs(orc.block_norm(np.zeros_like(u), u, gate=gate, w_post=w_post, post=post, offset=offset, eps=eps, u_scale=u_scale)[0])
    ex = sized * ((r if post else 0) + 5 * U) + U * (np.abs(x_scale) * x * 2 + np.abs(xo))
    rz = 1.0 / np.sqrt((xo * xo).mean(-1, keepdims=True) + eps)
    w = np.ones(d) if w_pre is None else np.abs(w_pre.astype(np.float64) + offset)
    share = np.sqrt((ex * ex).sum(-1, keepdims=True) / np.maximum((xo * xo).sum(-1, keepdims=True), 1e-300))
    ez = (ex * rz + np.abs(xo) * rz * (r + share)) * w + 4 * U * np.abs(z)
    tiny = 2.0 ** -126
    return ex + HALF[xdtype] * np.abs(xo) + tiny, ez + HALF[dtype] * np.abs(z) * (1 + 1e-3) + tiny


def run_norm(pop, n, d, xdtype, dtype, *, gate="none", post=False, weights=True, offset=0.0, pad=0, at=0, seed=0, in_place=False, u_there=True,
             outs="xz", x_scale=1.0, u_scale=0.5, eps=1e-5, size=1.0):
    rng = np.random.default_rng(seed + 1000 * n + d)
    x, u = rows(rng, n, d, xdtype, pad, size, at), rows(rng, n, d, dtype, 2 * pad, size, at) if u_there else None
    x[:, ::53] *= 20.0
    g = None if gate == "none" else rows(rng, 1 if gate == "channels" else n, d, dtype, pad if gate == "tokens" else 0, 1.0, at)
    w_post, w_pre = ((rows(rng, 1, d, dtype, 0, 0.2, at) + (1.0 - offset)).view(-1) if weights else None for _ in range(2))
    h = {k: None if t is None else f64(t) for k, t in dict(x=x, u=u, gate=g, w_post=w_post if post else None, w_pre=w_pre).items()}
    args = dict(gate=h["gate"], w_post=h["w_post"], w_pre=h["w_pre"], post=post, offset=offset, eps=float(np.float32(eps)), x_scale=x_scale, u_scale=u_scale)
    want_x, want_z = orc.block_norm(h["x"], h["u"], **args)
    fill = lambda t: torch.full((at + n * (d + 3 * pad),), 7.0, dtype=DT[t], device="cuda")  # noqa: E731
    whole_x, whole_z = fill(xdtype), fill(dtype)
    x_out, z = (w[at:].view(n, d + 3 * pad)[:, :d] for w in (whole_x, whole_z))
    if in_place:
        x_out, z = x, u
    pop.pop_block_norm(x, xdtype, u, dtype, n, d, x_out if "x" in outs else None, z if "z" in outs else None, w_pre, post_norm=post,
                       w_post=w_post if post else None, gate=g, gate_rows=0 if g is None else g.shape[0], weight_offset=offset, eps=eps,
                       x_scale=x_scale, u_scale=u_scale)
    bx, bz = norm_bounds(h["x"], h["u"], want_x, want_z, dtype, xdtype, d, **args)
    if "x" in outs:
        assert (np.abs(f64(x_out) - want_x) <= bx).all(), np.max(np.abs(f64(x_out) - want_x) / bx)
    if "z" in outs:
        assert (np.abs(f64(z) - want_z) <= bz).all(), np.max(np.abs(f64(z) - want_z) / bz)
    if not in_place:  # what lies between the rows stays
        for w, o, name in ((whole_x, x_out, "x"), (whole_z, z, "z")):
            assert (f64(w[:at]) == 7.0).all() and (f64(w[at:].view(n, d + 3 * pad)[:, d:]) == 7.0).all()
            if name not in outs:
                assert (f64(w) == 7.0).all()
    return x_out, z


@pytest.mark.parametrize("d", [1, 7, 8, 63, 512, 513, 1000, 4096, 4099, 5120, 8192, 10240, 16384, 20001, 40000, 65535, 65536])
@pytest.mark.parametrize("xdtype,dtype", [(F32, F32), (F32, BF16), (BF16, BF16), (BF16, F32)])
def test_norm_widths(pop, d, xdtype, dtype):
    run_norm(pop, 3, d, xdtype, dtype)
    run_norm(pop, 1, d, xdtype, dtype, post=True, gate="tokens", offset=1.0, seed=1)


@pytest.mark.parametrize("n", [1, 2, 33, 700, 3001])
@pytest.mark.parametrize("d", [64, 65, 128, 129, 160, 256, 257, 520, 1003])
def test_norm_rows(pop, n, d):
    run_norm(pop, n, d, BF16, BF16)
    run_norm(pop, n, d, F32, BF16, post=True, gate="channels")


@pytest.mark.parametrize("pad,at", [(8, 0), (8, 8), (5, 0), (0, 1), (3, 3)])
@pytest.mark.parametrize("d", [512, 515])
@pytest.mark.parametrize("xdtype,dtype", [(F32, BF16), (BF16, BF16), (F32, F32)])
def test_norm_rows_apart_and_misaligned(pop, d, pad, at, xdtype, dtype):
    run_norm(pop, 9, d, xdtype, dtype, pad=pad, at=at, post=True, gate="tokens")


@pytest.mark.parametrize("d", [512, 4100])
@pytest.mark.parametrize("change", [dict(u_there=False), dict(outs="x"), dict(outs="z"), dict(weights=False), dict(weights=False, post=True, offset=1.0),
                                    dict(gate="channels"), dict(u_there=False, outs="z", x_scale=1.0), dict(x_scale=0.5, u_scale=-3.0), dict(u_scale=0.0),
                                    dict(size=1e-12, eps=1e-6), dict(size=1e12), dict(post=True, offset=1.0)])
def test_norm_parts(pop, d, change):
    run_norm(pop, 5, d, F32, BF16, **change)
    run_norm(pop, 5, d, BF16, BF16, **change)


@pytest.mark.parametrize("d", [512, 4096, 4099])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norm_in_place(pop, d, dtype):
    a = run_norm(pop, 40, d, dtype, dtype, post=True, gate="tokens", in_place=True)
    b = run_norm(pop, 40, d, dtype, dtype, post=True, gate="tokens")
    assert np.array_equal(bits(a[0]), bits(b[0])) and np.array_equal(bits(a[1]), bits(b[1]))


def test_norm_of_zeros_and_what_is_no_number(pop):
    x = torch.zeros(4, 512, device="cuda")
    x[1, 5], x[2, 6] = float("nan"), float("inf")
    x[3] = 1.0
    xo, z = torch.empty_like(x), torch.empty_like(x)
    pop.pop_block_norm(x, F32, None, F32, 4, 512, xo, z)
    z = f64(z)
    assert (z[0] == 0).all() and np.isnan(z[1]).all() and abs(z[3] - 1).max() < 1e-6  # rows do not touch each other
    assert np.array_equal(bits(xo), bits(x))


def test_norm_on_another_stream_and_in_a_replayed_graph(pop):
    d, n = 4096, 64
    rng = np.random.default_rng(5)
    x, u, w = rows(rng, n, d, F32), rows(rng, n, d, BF16), rows(rng, 1, d, BF16).view(-1)
    xo, z = torch.empty_like(x), torch.empty_like(u)

    def call():
        pop.pop_block_norm(x, F32, u, BF16, n, d, xo, z, w, post_norm=True, w_post=w)

    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        call()
    stream.synchronize()
    want = [bits(xo), bits(z)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(3):
        xo.fill_(0), z.fill_(0)
        graph.replay()
        assert np.array_equal(bits(xo), want[0]) and np.array_equal(bits(z), want[1])
        call()
        torch.cuda.synchronize()


# ---------------------------------------------------------------- rotary positions

def rotary_bound(x, positions, turns, amplitude, dtype, want):
    """Angles: a product in 64 bits (2^-53 of its revolutions), the rest below one half rounded to 32 (2^-26 revolutions); sine and cosine
    to 4 steps; the amplitude, two products and their sum 4 roundings."""
    p = np.abs(np.asarray(positions, dtype=np.float64))[:, None, None]
    angle = 2 * np.pi * (2.0 ** -26 + p * np.abs(turns).max() * 2.0 ** -52)
    size = np.abs(x).max(-1, keepdims=True)  # (of any of the head's channels)
    return 2 * size * abs(amplitude) * (angle + (4 + 4) * U) + HALF[dtype] * np.abs(want) * (1 + 1e-3)


def run_rotary(pop, n, heads, n_kv, d, r, pairs, dtype, positions, *, amplitude=1.0, pad=0, in_place=False, at=0, seed=0):
    rng = np.random.default_rng(seed + n + d + r)
    width = (heads + 2 * n_kv) * d
    joint = rows(rng, n, width, dtype, pad, 3.0, at)
    q, k = joint[:, :heads * d], joint[:, heads * d:(heads + n_kv) * d] if n_kv else None
    turns = torch.from_numpy(1e4 ** (-np.arange(0, r, 2) / r) / (2 * np.pi)).cuda()
    pos = torch.from_numpy(np.asarray(positions, dtype=np.int32)).cuda()
    ins = [f64(q).reshape(n, heads, d)] + ([f64(k).reshape(n, n_kv, d)] if n_kv else [])
    outs = [q, k] if in_place else [torch.full((n, h, d), 7.0, dtype=DT[dtype], device="cuda") if h else None for h in (heads, n_kv)]
    before = f64(joint)
    pop.pop_rotary(q, k, dtype, n, heads, n_kv, d, r, pop.POP_ROTARY_PAIRS if pairs else pop.POP_ROTARY_HALVES, pos, turns, amplitude, *outs)
    amp, left = float(np.float32(amplitude)), np.asarray(positions) < 0
    for x, out in zip(ins, outs):
        want, got = orc.rotary(x, positions, f64(turns), amp, pairs), f64(out).reshape(x.shape)
        bound = rotary_bound(x, positions, f64(turns), amp, dtype, want)
        assert (np.abs(got - want) <= bound)[~left].all(), np.max((np.abs(got - want) / bound)[~left])
        assert np.array_equal(got[~left][..., r:], x[~left][..., r:])
        assert (got[left] == (x[left] if in_place else 7.0)).all()
    if in_place:  # what is neither q nor k stays
        assert np.array_equal(f64(joint)[:, (heads + n_kv) * d:], before[:, (heads + n_kv) * d:])
    return outs


def some_positions(rng, n, most):
    p = rng.integers(0, most, n)
    p[rng.random(n) < 0.1] = -1
    return p


@pytest.mark.parametrize("d,r", [(64, 64), (80, 40), (80, 80), (128, 128), (128, 46), (128, 64), (96, 2), (3, 2), (256, 256), (33, 32), (1100, 1024), (128, 2), (128, 126), (64, 6), (1024, 1000), (2400, 500), (4096, 34), (8200, 20)])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rotary_shapes(pop, d, r, pairs, dtype):
    rng = np.random.default_rng(d * r)
    for n, heads, n_kv in ((1, 4, 1), (37, 3, 3), (5, 9, 0)):
        run_rotary(pop, n, heads, n_kv, d, r, pairs, dtype, some_positions(rng, n, 5000), amplitude=1.2)


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rotary_far_positions(pop, pairs, dtype):
    run_rotary(pop, 7, 2, 1, 64, 64, pairs, dtype, [0, 1, 131071, 1 << 20, (1 << 30) + 1, (1 << 31) - 1, -(1 << 31)])


@pytest.mark.parametrize("pad,at", [(8, 0), (5, 0), (8, 8), (0, 1), (4, 4)])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rotary_rows_apart_misaligned_and_in_place(pop, pad, at, in_place, pairs, dtype):
    run_rotary(pop, 19, 5, 2, 64, 48, pairs, dtype, some_positions(np.random.default_rng(3), 19, 1 << 17), pad=pad, at=at, in_place=in_place)


@pytest.mark.parametrize("n,heads,n_kv,d,r", [(3000, 32, 8, 128, 128), (1500, 7, 1, 80, 20), (300, 71, 1, 64, 64), (2, 128, 128, 128, 128), (3000, 32, 8, 128, 46), (2000, 8, 8, 256, 250), (700, 2, 1, 2048, 1000)])
@pytest.mark.parametrize("pairs", [False, True])
def test_rotary_many_tokens(pop, n, heads, n_kv, d, r, pairs):
    run_rotary(pop, n, heads, n_kv, d, r, pairs, BF16, some_positions(np.random.default_rng(n), n, 1 << 20))


def test_rotary_angles_depend_on_distances_only(pop):
    """q k of turned heads: the same for the same distance, near or far."""
    turns, amplitude = pop.pop_rotary_frequencies(128, 10000.0, pop.POP_ROTARY_RAMP, 8.0, 4096, 1, 32)
    turns = torch.tensor(turns, dtype=torch.float64, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    x, y = (torch.randn(1, 1, 128, generator=g, device="cuda").expand(6, 1, 128).contiguous() for _ in range(2))
    at = torch.tensor([0, 5, 77, 4096, 131072, 1 << 20], dtype=torch.int32, device="cuda")
    a, b = torch.empty_like(x), torch.empty_like(y)
    pop.pop_rotary(x, None, F32, 6, 1, 0, 128, 128, pop.POP_ROTARY_HALVES, at, turns, amplitude, a, None)
    pop.pop_rotary(y, None, F32, 6, 1, 0, 128, 128, pop.POP_ROTARY_HALVES, at + 300, turns, amplitude, b, None)
    s = (f64(a) * f64(b)).sum(-1)[:, 0]
    # 128 products of sizes |x||y|, each with two turned channels that are off by the bound above
    bound = 4 * amplitude ** 2 * float(x[0].norm() * y[0].norm()) * (2 * np.pi * 2.0 ** -26 + 10 * U) * 2
    assert np.abs(s - s[0]).max() <= bound


def test_rotary_on_another_stream_and_in_a_replayed_graph(pop):
    rng = np.random.default_rng(9)
    q, k = rows(rng, 50, 8 * 128, BF16), rows(rng, 50, 2 * 128, BF16)
    pos = torch.arange(50, dtype=torch.int32, device="cuda")
    turns = torch.tensor(pop.pop_rotary_frequencies(128)[0], dtype=torch.float64, device="cuda")
    qo, ko = torch.empty_like(q), torch.empty_like(k)

    def call():
        pop.pop_rotary(q, k, BF16, 50, 8, 2, 128, 128, pop.POP_ROTARY_HALVES, pos, turns, 1.0, qo, ko)

    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        call()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(3):  # positions move on between replays, as from step to step
        qo.fill_(0)
        graph.replay()
        got = [bits(qo), bits(ko)]
        call()
        assert np.array_equal(bits(qo), got[0]) and np.array_equal(bits(ko), got[1])
        pos += 50
        torch.cuda.synchronize()
