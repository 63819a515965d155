"""The operators around the cache (rotary positions, norms with rotation, packed caches, attention over them) against plain implementations in
64 bits and more, through the C ABI.  Tolerances count roundings: half a step of a type is finfo.eps / 2 relative, H below is float32's."""
import os

import numpy as np
import pytest
import torch

from paper_2504_09261_amd.binding import Cache, Hack, HackError, PackedCache, Rope, packed_bytes

pytestmark = pytest.mark.gpu

H = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
DEV = "cuda:0"


@pytest.fixture(scope="module")
def contexts():
    made = {}

    def get(heads, d, dtype, units=64, queries=4096, form=0):
        key = (heads, d, dtype, units, queries, form)
        if key not in made:
            os.environ["HACK_ATTN_PACKED_QUERIES"] = str(form)      # read when a context is created
            try:
                made[key] = Hack(heads, d, dtype, units, 1024, queries)
            finally:
                del os.environ["HACK_ATTN_PACKED_QUERIES"]
        return made[key]
    yield get
    for h in made.values():
        h.close()


def to64(t):
    return t.detach().double().cpu().numpy()


# ---- rotary positions, norms -------------------------------------------------
TWO_PI = np.longdouble("6.283185307179586476925286766559")


def turned(x, pos, freq, gain, rot, axes, layout):
    """Rotation of x [B, heads, N, d] (float64) at pos [B, axes, N]; also the sum of the magnitudes that enter each element."""
    out, mag = x.copy(), np.abs(x)
    S = rot // axes
    for a in range(axes):
        for i in range(S // 2):
            p, q = (i, i + S // 2) if layout == "half" else (2 * i, 2 * i + 1)
            p, q = p + a * S, q + a * S
            ang = np.fmod(pos[:, a].astype(np.longdouble) * np.longdouble(freq[a * S // 2 + i]), TWO_PI)
            c, s = (gain * f(ang).astype(np.float64)[:, None] for f in (np.cos, np.sin))
            out[..., p], out[..., q] = x[..., p] * c - x[..., q] * s, x[..., p] * s + x[..., q] * c
            mag[..., p] = mag[..., q] = gain * (np.abs(x[..., p]) + np.abs(x[..., q]))
    return out, mag


def check_rows(got, want, mag, dtype, roundings):
    err = np.abs(to64(got) - want)
    tol = HALF_STEP[dtype] * 1.01 * np.abs(want) + roundings * H * mag
    assert (err <= tol).all(), (float((err / np.maximum(tol, 1e-300)).max()), np.unravel_index(np.argmax(err / np.maximum(tol, 1e-300)), err.shape))


# cos and sin: the fraction of a turn is cut at 2^-32, converted, scaled (three roundings of an angle below pi / 4), the polynomials end with two
# roundings of their own, the gain is rounded and multiplied: 7 H and 2e-9; the products and the sum: 3 H.  10 H of |a| + |b|.
ROTATION = 10.1

ROPES = [   # head_dim, rot_dim, axes, layout
    (128, 128, 1, "half"), (128, 128, 1, "interleaved"), (64, 64, 1, "half"), (64, 64, 1, "interleaved"), (128, 128, 2, "half"), (64, 64, 2, "interleaved"),
    (128, 32, 1, "half"), (128, 96, 1, "interleaved"), (64, 16, 1, "half"), (64, 32, 2, "half"), (128, 96, 2, "half"), (128, 32, 2, "interleaved"),
]


def rows_in(shape, how, dtype, g):
    """[B, heads, N, d] as the batch, a projection or a part of a wider tensor holds them."""
    B, h, N, d = shape
    if how == "plain":
        return torch.randn(shape, generator=g, device=DEV).to(TYPES[dtype])
    if how == "projection":
        return torch.randn((B, N, 3 * h, d), generator=g, device=DEV).to(TYPES[dtype])[:, :, h:2 * h].transpose(1, 2)
    return torch.randn((N + 2, h, B, d + 16), generator=g, device=DEV).to(TYPES[dtype])[1:-1, :, :, 8:8 + d].permute(2, 1, 0, 3)   # "part"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d, rot, axes, layout", ROPES)
def test_rotate(contexts, dtype, d, rot, axes, layout):
    g = torch.Generator(DEV).manual_seed(rot + axes)
    rng = np.random.default_rng(d + rot)
    for (B, h, N), how in (((1, 1, 1), "plain"), ((3, 5, 7), "projection"), ((2, 3, 65), "part"), ((2, 9, 130), "plain"), ((1, 40, 33), "projection")):
        hk = contexts(1, d, dtype)
        x = rows_in((B, h, N, d), how, dtype, g)
        far = np.array([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 1000003])
        pos = rng.integers(-(1 << 20), 1 << 20, (B, axes, N)).astype(np.int32)
        pos.reshape(-1)[:far.size] = far[:pos.size]
        gain = 1.25 if N == 7 else 1.0
        freq = np.concatenate([10000.0 ** (-2 * np.arange(rot // axes // 2) / (rot // axes)) / (1 + a) for a in range(axes)])
        if N == 65:
            freq[0], freq[1] = -2.5, 9.0     # backwards, more than a turn per position
        rope = Rope(freq, rot, axes, layout, gain)
        out = torch.full((B, h, N, d), 7.0, dtype=TYPES[dtype], device=DEV)
        hk.rotate(x, rope, out, pos=torch.from_numpy(pos).to(DEV))
        want, mag = turned(to64(x), pos, freq, gain, rot, axes, layout)
        check_rows(out, want, mag, dtype, ROTATION)
        assert torch.equal(out[..., rot:], x[..., rot:])
        # the same positions for every batch element
        hk.rotate(x, rope, out, pos=torch.from_numpy(pos[0]).to(DEV))
        want, mag = turned(to64(x), np.repeat(pos[:1], B, 0), freq, gain, rot, axes, layout)
        check_rows(out, want, mag, dtype, ROTATION)
        # in place
        y = x.contiguous().clone()
        hk.rotate(y, rope, y, pos=torch.from_numpy(pos[0]).to(DEV))
        assert torch.equal(y, out)


@pytest.mark.parametrize("d, axes, layout", [(128, 1, "half"), (64, 1, "interleaved"), (128, 2, "half")])
def test_rotate_backwards_at_far_positions(contexts, d, axes, layout):
    """Small frequencies below zero are as exact as those above, and undo them."""
    hk = contexts(1, d, "f32")
    g = torch.Generator(DEV).manual_seed(d)
    S = d // axes
    x = torch.randn((1, 3, 6, d), generator=g, device=DEV)
    pos = np.repeat(np.array([2 ** 31 - 1, -2 ** 31, 2 ** 31 - 12345, 2 ** 30 + 1, -2 ** 31 + 7, 1])[None, None], axes, 1).astype(np.int32)
    freq = -np.tile(10000.0 ** (-2 * np.arange(S // 2) / S), axes)
    out, back = torch.empty_like(x), torch.empty_like(x)
    hk.rotate(x, Rope(freq, d, axes, layout), out, pos=torch.from_numpy(pos).to(DEV))
    want, mag = turned(to64(x), pos, freq, 1.0, d, axes, layout)
    check_rows(out, want, mag, "f32", ROTATION)
    hk.rotate(out, Rope(-freq, d, axes, layout), back, pos=torch.from_numpy(pos).to(DEV))
    check_rows(back, to64(x), 2 * np.abs(to64(x)).max() * np.ones(x.shape), "f32", ROTATION * 2.5)


def test_rotate_numbers_rows_without_positions_and_turns_back(contexts):
    hk = contexts(1, 128, "f32")
    g = torch.Generator(DEV).manual_seed(3)
    x = torch.randn((2, 3, 77, 128), generator=g, device=DEV)
    rope = Rope.scaled(128)
    a, b = torch.empty_like(x), torch.empty_like(x)
    hk.rotate(x, rope, a, pos0=-40)
    pos = torch.arange(-40, 37, dtype=torch.int32, device=DEV)
    hk.rotate(x, rope, b, pos=pos)
    assert torch.equal(a, b)
    hk.rotate(a, rope, b, pos=-pos)
    # two rotations' roundings of |a| + |b| at most, which a rotation makes at most sqrt 2 larger
    check_rows(b, to64(x), 2 * np.abs(to64(x)).max() * np.ones(x.shape), "f32", ROTATION * 2.5)


def test_rotate_keeps_what_does_not_rotate_and_spreads_nan_to_its_pair_only(contexts):
    hk = contexts(1, 64, "bf16")
    x = torch.ones((1, 2, 3, 64), dtype=torch.bfloat16, device=DEV)
    x[0, 0, 1, 3] = float("nan")
    x[0, 1, 2, 50] = float("inf")
    out = torch.empty_like(x)
    hk.rotate(x, Rope.scaled(32), out, pos0=5)
    bad = torch.zeros(x.shape, dtype=torch.bool, device=DEV)
    bad[0, 0, 1, 3] = bad[0, 0, 1, 19] = True
    assert torch.equal(torch.isnan(out), bad)
    assert out[0, 1, 2, 50] == float("inf") and torch.equal(out[..., 32:50], x[..., 32:50])


@pytest.mark.parametrize("dtype, d, rot, layout", [("bf16", 128, 128, "half"), ("bf16", 64, 32, "interleaved"), ("f32", 64, 64, "half"), ("f32", 128, 32, "interleaved"), ("f32", 64, 16, "half")])
def test_large_outputs_are_those_of_their_parts(contexts, dtype, d, rot, layout):
    """Beyond 32 MB of output stores take another way."""
    hk = contexts(1, d, dtype)
    g = torch.Generator(DEV).manual_seed(8)
    heads, N = 10, 4001
    B = (40 << 20) // (heads * N * d * TYPES[dtype].itemsize) + 1
    x, k = rows_in((B, heads, N, d), "projection", dtype, g), rows_in((B, 3, N, d), "plain", dtype, g)
    rope, pos = Rope.scaled(rot, 1, layout), torch.arange(N, dtype=torch.int32, device=DEV) * 77
    out, part = torch.empty((B, heads, N, d), dtype=x.dtype, device=DEV), torch.empty((1, heads, N, d), dtype=x.dtype, device=DEV)
    hk.rotate(x, rope, out, pos=pos)
    for b in range(B):
        hk.rotate(x[b:b + 1], rope, part, pos=pos)
        assert torch.equal(part[0], out[b])
    ko, kp = torch.empty_like(k), torch.empty_like(k[:1])
    hk.norm_rotate(x, k, "rms", 1e-6, None, None, rope, out, ko, pos=pos)
    for b in range(B):
        hk.norm_rotate(x[b:b + 1], k[b:b + 1], "rms", 1e-6, None, None, rope, part, kp, pos=pos)
        assert torch.equal(part[0], out[b]) and torch.equal(kp[0], ko[b])


# The sum of squares: chains of 16 and three more sums, half of it in the root, 10 H; root, reciprocal, mean and eps 4 H; the two products 2 H.
NORM = 17.0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d, rot, axes, layout", [ROPES[i] for i in (0, 3, 4, 7, 9)])
@pytest.mark.parametrize("norm", ["rms", "l2"])
def test_norm_rotate(contexts, dtype, d, rot, axes, layout, norm):
    g = torch.Generator(DEV).manual_seed(rot)
    rng = np.random.default_rng(rot)
    for i, ((B, hq, hk_, N), how) in enumerate((((1, 1, 1, 1), "plain"), ((5, 8, 2, 1), "projection"), ((2, 6, 6, 33), "part"), ((1, 12, 4, 130), "projection"))):
        hk = contexts(1, d, dtype)
        q, k = rows_in((B, hq, N, d), how, dtype, g), rows_in((B, hk_, N, d), how, dtype, g)
        q[0, 0, 0] = 0
        qw = None if i == 0 else 1 + torch.randn((d,) if i == 1 else (hq, d), generator=g, device=DEV) / 3
        kw = None if i == 2 else 1 + torch.randn((hk_, d) if i == 1 else (d,), generator=g, device=DEV) / 3
        pos = rng.integers(-9, 1 << 17, (B, axes, N)).astype(np.int32)
        rope = Rope.scaled(rot, axes, layout, "linear", factor=3.0)
        qo, ko = torch.empty((B, hq, N, d), dtype=q.dtype, device=DEV), torch.empty((B, hk_, N, d), dtype=q.dtype, device=DEV)
        hk.norm_rotate(q, k, norm, 1e-5, qw, kw, rope, qo, ko, pos=torch.from_numpy(pos).to(DEV))
        no_rope_q, no_rope_k = torch.empty_like(qo), torch.empty_like(ko)
        hk.norm_rotate(q, k, norm, 1e-5, qw, kw, None, no_rope_q, no_rope_k)
        for x, w, o, plain in ((q, qw, qo, no_rope_q), (k, kw, ko, no_rope_k)):
            y = to64(x)
            ss = (y * y).sum(-1, keepdims=True)
            eps = float(np.float32(1e-5))
            y = y / np.sqrt(ss / d + eps) if norm == "rms" else y / np.maximum(np.sqrt(ss), eps)
            if w is not None:
                y = y * to64(w if w.dim() == 1 else w[:, None])
            check_rows(plain, y, np.abs(y), dtype, NORM)
            want, mag = turned(y, pos, rope.freq, 1.0, rot, axes, layout)
            check_rows(o, want, mag, dtype, ROTATION + NORM)
        # queries alone
        alone = torch.empty_like(qo)
        hk.norm_rotate(q, None, norm, 1e-5, qw, None, rope, alone, None, pos=torch.from_numpy(pos).to(DEV))
        assert torch.equal(alone, qo)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("norm", ["rms", "l2"])
@pytest.mark.parametrize("eps", [2.0 ** -149, 2.0 ** -127, 1e-30, 2.0 ** -51, 2.0 ** -49, 1e-6, 1e30])
def test_norms_of_rows_whose_squares_leave_float32(contexts, dtype, d, norm, eps):
    """Rows of any finite magnitude, zero ones too, for every eps above zero.  Scaling by a power of two adds no rounding to NORM's; elements below 2^-149 of a row's
    largest, and results below the smallest normal number, may lose what falls off there: half of float32's smallest step in either place (bf16: its own)."""
    hk = contexts(1, d, dtype)
    g = torch.Generator(DEV).manual_seed(d)
    exps = [-149, -140, -133, -126, -120, -101, -76, -75, -74, -64, -63, -62, -51, -50, -49, -30, 0, 40, 59, 60, 61, 62, 63, 64, 65, 100, 124]
    x = torch.randn((1, 2, len(exps) + 1, d), generator=g, device=DEV, dtype=torch.float64).clamp_(-4, 4)
    x[:, :, :-1] *= torch.exp2(torch.tensor(exps, dtype=torch.float64, device=DEV))[:, None]
    x[:, :, -1] = 0
    x[:, 1, :, 1:] *= 0.0                     # the second head: one element alone
    x = x.to(TYPES[dtype])
    out = torch.empty_like(x)
    hk.norm_rotate(x, None, norm, eps, None, None, None, out, None)
    y = to64(x)
    e = float(np.float32(eps))
    ss = (y * y).sum(-1, keepdims=True)
    want = y / np.sqrt(ss / d + e) if norm == "rms" else y / np.maximum(np.sqrt(ss), e)
    tiny = 2.0 ** -149 + (2.0 ** -134 if dtype == "bf16" else 0.0)
    err = np.abs(to64(out) - want)
    tol = HALF_STEP[dtype] * 1.01 * np.abs(want) + NORM * H * np.abs(want) + tiny
    assert (err <= tol).all(), (float((err / tol).max()), np.unravel_index(np.argmax(err / tol), err.shape))
    assert not to64(out)[:, :, -1].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d, rot, axes, layout", [(128, 128, 1, "half"), (64, 32, 2, "half"), (64, 16, 1, "interleaved"), (128, 96, 2, "interleaved")])
@pytest.mark.parametrize("hq, hk_", [(1, 1), (3, 1), (10, 2), (1, 5), (17, 33)])
def test_any_number_of_heads_gives_what_each_gives_alone(contexts, dtype, d, rot, axes, layout, hq, hk_):
    """How many rows of a head a work-group takes follows from the heads of each tensor; what becomes of a row does not."""
    hk = contexts(1, d, dtype)
    g = torch.Generator(DEV).manual_seed(hq)
    B, N = 2, 67
    q, k = rows_in((B, hq, N, d), "projection", dtype, g), rows_in((B, hk_, N, d), "part", dtype, g)
    w = [1 + torch.randn((h, d), generator=g, device=DEV) / 3 for h in (hq, hk_)]
    rope = Rope.scaled(rot, axes, layout)
    pos = torch.randint(0, 9000, (B, axes, N), generator=g, device=DEV, dtype=torch.int32)
    out = [torch.full((B, h, N, d), 7.0, dtype=q.dtype, device=DEV) for h in (hq, hk_)]
    hk.norm_rotate(q, k, "rms", 1e-6, *w, rope, *out, pos=pos)
    alone = torch.empty((B, 1, N, d), dtype=q.dtype, device=DEV)
    for x, weight, o in zip((q, k), w, out):
        for h in range(x.shape[1]):
            hk.norm_rotate(x[:, h:h + 1], None, "rms", 1e-6, weight[h].contiguous(), None, rope, alone, None, pos=pos)
            assert torch.equal(alone[:, 0], o[:, h])


# ---- packed caches -----------------------------------------------------------
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def nearest(x):
    """Rows [n, d] (float64 of bf16 or float32 numbers) as a packed cache holds them: by search over exponents and values."""
    n, d = x.shape
    g = x.reshape(n, -1, 32)
    top = np.abs(g).max(-1)
    bad = ~np.isfinite(top)
    top = np.where(bad, 1.0, top)
    s = np.full(top.shape, 252)
    for e in range(252, 2, -1):
        s = np.where(top <= 7 * 2.0 ** (e - 127), e, s)
    y = np.where(bad[..., None], 0.0, g) / 2.0 ** (s - 127)[..., None]
    a = np.minimum(np.abs(y), 6.0)
    dist = np.abs(a[..., None] - GRID)
    best = dist.min(-1, keepdims=True)
    code = np.where(dist == best, np.arange(8) + np.where(np.arange(8) % 2, 8, 0), 99).argmin(-1)   # of two at the same distance the even code
    v = np.sign(y) * GRID[code] * 2.0 ** (s - 127)[..., None]
    return np.where(bad[..., None], np.nan, v).reshape(n, d)


def offsets(lens, step, gap=0, order=None):
    order = range(len(lens)) if order is None else order
    off, at = np.zeros(len(lens), np.int64), 0
    for u in order:
        off[u] = at
        at += (int(lens[u]) + step - 1) // step * step + gap
    return off, at


def packed(lens, d, fill=0, gap=0, order=None, with_pos=False):
    """An empty packed cache with room for lens rows of each unit."""
    off, rows = offsets(lens, 64, gap, order)
    k, v = (torch.full((rows // 64, 34 * d), fill, dtype=torch.uint8, device=DEV) for _ in range(2))
    return PackedCache(k, v, off, lens, torch.full((rows,), -7, dtype=torch.int32, device=DEV) if with_pos else None)


def same(a, b):
    return np.array_equal(a, b, equal_nan=True)


def read_back(hk, B, pc, lens, dtype, first=None):
    off, rows = offsets(lens, 8)
    out = Cache(*(torch.full((rows, pc.head_dim), 3.5, dtype=TYPES[dtype], device=DEV) for _ in range(2)), off, lens,
                torch.full((rows,), -9, dtype=torch.int32, device=DEV))
    hk.unpack(B, pc, out, first=first)
    return [(to64(out.k[o:o + n]), to64(out.v[o:o + n]), out.pos[o:o + n].cpu().numpy()) for o, n in zip(off, lens)], out


def hard_rows(n, d, dtype, g):
    """Rows with every rounding: powers of two apart, exact ties, zeros, the smallest and largest numbers, NaN and infinities."""
    x = torch.randn((n, d), generator=g, device=DEV) * torch.exp2(torch.randint(-20, 20, (n, 1), generator=g, device=DEV).float())
    for i, row in enumerate(x):
        if i % 11 == 1:
            row[:32] = 0
        if i % 11 == 2:   # ties and steps of the unit 1
            row[:32] = torch.tensor([6, 5, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25] * 4, device=DEV) * (1 - 2 * (torch.arange(32, device=DEV) % 2))
        if i % 11 == 3:   # the largest at the border between two units
            row[:32] = row[:32].clamp(-1, 1)
            row[5] = 7.0 if i % 2 else 7.03125
        if i % 11 == 4:
            row *= 1e-37
        if i % 11 == 5:
            row[32:64] = row[32:64].sign() * 3e38
        if i % 11 == 6:
            row[7] = float("nan")
        if i % 11 == 7:
            row[40] = -float("inf")
        if i % 11 == 8:
            row[:32] = 2.0 ** -126 * row[:32].sign()
    return x.to(TYPES[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_pack_rounds_to_the_nearest_value_and_reads_back_exactly(contexts, dtype, d):
    hk = contexts(1, d, dtype, units=8)
    g = torch.Generator(DEV).manual_seed(d)
    lens = np.array([1, 130, 64, 63, 65, 1000, 16, 17])
    off, rows = offsets(lens, 8)
    k, v = hard_rows(rows, d, dtype, g), hard_rows(rows, d, dtype, g)
    pos = torch.arange(rows, dtype=torch.int32, device=DEV)
    pc = packed(lens, d, fill=0xEE, with_pos=True, order=[3, 1, 0, 2, 7, 6, 5, 4])
    hk.pack(8, 0, pc, cache_in=Cache(k, v, off, lens, pos))
    got, back = read_back(hk, 8, pc, lens, dtype)
    with np.errstate(invalid="ignore"):
        for o, n, (gk, gv, gp) in zip(off, lens, got):
            assert same(gk, nearest(to64(k[o:o + n]))) and same(gv, nearest(to64(v[o:o + n])))
            assert np.array_equal(gp, np.arange(o, o + n))
    # packed again: the same bytes
    again = packed(lens, d, fill=0xEE, with_pos=True, order=[3, 1, 0, 2, 7, 6, 5, 4])
    hk.pack(8, 0, again, cache_in=back)
    finite = [u for u in range(8) if np.isfinite(got[u][0]).all() and np.isfinite(got[u][1]).all()]
    for u in range(8):
        b0, b1 = pc.off[u] // 64, (pc.off[u] + lens[u] + 63) // 64
        for a, b in ((pc.k, again.k), (pc.v, again.v)):
            assert torch.equal(a[b0:b1], b[b0:b1]), u
    assert finite


@pytest.mark.parametrize("dtype, d", [("bf16", 128), ("f32", 64), ("bf16", 64)])
def test_pack_appends_behind_what_is_there_and_touches_nothing_else(contexts, dtype, d):
    heads, B = 5, 3
    hk = contexts(heads, d, dtype, units=heads * B)
    g = torch.Generator(DEV).manual_seed(1)
    rng = np.random.default_rng(5)
    cap = np.full(heads * B, 200)
    pc = packed(cap, d, fill=0xAB, with_pos=True)
    have = [np.zeros((2, 0, d)) for _ in cap]
    at = np.zeros(heads * B, np.int64)
    for step, n in enumerate([1, 1, 30, 1, 33, 64, 1, 7]):
        kn, vn = (torch.randn((B, heads, n, d), generator=g, device=DEV).to(TYPES[dtype]) for _ in range(2))
        takes = rng.integers(0, 2, heads * B) * n if step == 3 else np.full(heads * B, n)     # some units take nothing
        pc.len = (at + takes).astype(np.int32)
        hk.pack(B, n, pc, k_new=kn, v_new=vn, pos_new=1000 * step, at=at)
        for u in range(heads * B):
            if takes[u]:
                new = np.stack([nearest(to64(x[u // heads, u % heads])) for x in (kn, vn)])
                have[u] = np.concatenate([have[u], new], 1)
        at = at + takes
        got, _ = read_back(hk, B, pc, at, dtype)
        for u in range(heads * B):
            assert same(got[u][0], have[u][0]) and same(got[u][1], have[u][1])
            assert (got[u][2][len(got[u][2]) - takes[u]:] == 1000 * step + np.arange(takes[u])).all()
    # rows behind the last one: their bytes are as they were
    ref = packed(cap, d, fill=0xAB)
    zero = Cache(*(torch.zeros((int(at.sum()) + 8 * len(at), d), dtype=TYPES[dtype], device=DEV) for _ in range(2)), offsets(at, 8)[0], at)
    for p in (pc, ref):     # the written rows the same in both: what differs then is elsewhere
        p.len = at.astype(np.int32)
        hk.pack(B, 0, p, cache_in=zero)
    assert torch.equal(pc.k, ref.k) and torch.equal(pc.v, ref.v)
    tail = pc.pos.cpu().numpy().reshape(len(cap), -1)
    assert all((tail[u, at[u]:] == -7).all() for u in range(len(cap)))


def test_pack_through_kept_lists(contexts):
    heads, B, d, N = 3, 2, 128, 37
    hk = contexts(heads, d, "bf16", units=6)
    g = torch.Generator(DEV).manual_seed(2)
    rng = np.random.default_rng(2)
    cached = np.array([100, 0, 64, 1, 333, 20])
    off, rows = offsets(cached, 8, gap=8)
    k, v = (torch.randn((rows, d), generator=g, device=DEV).bfloat16() for _ in range(2))
    pos = torch.arange(rows, dtype=torch.int32, device=DEV) + 5000
    kn, vn = (torch.randn((B, heads, N, d), generator=g, device=DEV).bfloat16() for _ in range(2))
    n_kept = np.array([70, 37, 1, 38, 200, 3])
    kept = torch.full((6, 256), 1 << 30, dtype=torch.int32, device=DEV)
    lists = []
    for u in range(6):
        i = np.sort(rng.choice(cached[u] + N, n_kept[u], replace=False))
        if u == 5:
            i = np.array([22, 22, 4])      # in any order, the same row twice
        lists.append(i)
        kept[u, :len(i)] = torch.from_numpy(i).to(DEV)
    first = np.array([0, 5, 63, 64, 1, 0])
    pc = packed(first + n_kept, d, with_pos=True)
    hk.pack(B, N, pc, cache_in=Cache(k, v, off, cached, pos), kept_idx=kept, k_new=kn, v_new=vn, pos_new=77, at=first)
    got, _ = read_back(hk, B, pc, n_kept, "bf16", first=first)
    for u, i in enumerate(lists):
        for a, new, x in ((k, kn, got[u][0]), (v, vn, got[u][1])):
            both = np.concatenate([to64(a[off[u]:off[u] + cached[u]]), to64(new[u // heads, u % heads])])
            assert same(x, nearest(both[i]))
        assert np.array_equal(got[u][2], np.where(i < cached[u], 5000 + off[u] + i, 77 + i - cached[u]))
    # positions of cached rows stay as they are where the cache has none
    pc.pos.fill_(-3)
    hk.pack(B, N, pc, cache_in=Cache(k, v, off, cached), kept_idx=kept, k_new=kn, v_new=vn, pos_new=77, at=first)
    got, _ = read_back(hk, B, pc, n_kept, "bf16", first=first)
    for u, i in enumerate(lists):
        assert np.array_equal(got[u][2], np.where(i < cached[u], -3, 77 + i - cached[u]))


@pytest.mark.parametrize("dtype, d", [("bf16", 128), ("f32", 64)])
def test_many_rows_read_back_as_their_parts(contexts, dtype, d):
    """Beyond 32 MB of output stores take another way."""
    hk = contexts(1, d, dtype, units=8)
    g = torch.Generator(DEV).manual_seed(1)
    lens = np.array([30001, 1, 17000, 20003, 64, 9999, 22222, 5000])
    off, rows = offsets(lens, 8)
    assert 2 * rows * d * TYPES[dtype].itemsize > 50 << 20
    k, v = (torch.randn((rows, d), generator=g, device=DEV).to(TYPES[dtype]) for _ in range(2))
    pc = packed(lens, d)
    hk.pack(8, 0, pc, cache_in=Cache(k, v, off, lens))
    out, part = (Cache(torch.zeros_like(k), torch.zeros_like(v), off, lens) for _ in range(2))
    hk.unpack(8, pc, out)
    for a in range(0, 30001, 9000):     # rows a .. of every unit
        n = np.minimum(np.maximum(lens - a, 0), 9000)
        some, at = Cache(torch.zeros_like(k), torch.zeros_like(v), off, n), np.minimum(lens, a)
        hk.unpack(8, pc, some, first=at)
        for u in range(8):
            part.k[off[u] + at[u]:off[u] + at[u] + n[u]] = some.k[off[u]:off[u] + n[u]]
            part.v[off[u] + at[u]:off[u] + at[u] + n[u]] = some.v[off[u]:off[u] + n[u]]
    assert torch.equal(out.k, part.k) and torch.equal(out.v, part.v)
    assert same(to64(out.k[off[3]:off[3] + 200]), nearest(to64(k[off[3]:off[3] + 200])))


def test_a_unit_of_more_rows_than_a_launch_takes(contexts):
    """More than 2^28 rows of 128, read back at both ends and where launches of 2^27 rows meet; K and V are the same 69 GB."""
    hk = contexts(1, 128, "bf16", units=8)
    g = torch.Generator(DEV).manual_seed(28)
    n, period = 2 ** 28 + 1000, 1 << 16
    some = torch.randn((period, 128), generator=g, device=DEV).bfloat16()
    k = torch.empty((n, 128), dtype=torch.bfloat16, device=DEV)
    k[:2 ** 28].view(-1, period, 128).copy_(some)
    k[2 ** 28:].copy_(some[:1000])
    pc = PackedCache(*(torch.empty(((n + 63) // 64, 34 * 128), dtype=torch.uint8, device=DEV) for _ in range(2)), [0], [n])
    hk.pack(1, 0, pc, cache_in=Cache(k, k, [0], [n]))
    want = nearest(to64(some))
    for at in (0, 2 ** 27 - 500, 2 ** 28 - 500, n - 1000):
        out = Cache(torch.zeros((1000, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((1000, 128), dtype=torch.bfloat16, device=DEV), [0], [1000])
        hk.unpack(1, pc, out, first=np.array([at], np.int32))
        i = (at + np.arange(1000)) % period
        assert same(to64(out.k), want[i]) and same(to64(out.v), want[i])
    del k, pc
    torch.cuda.empty_cache()


def test_packed_sizes():
    assert packed_bytes(128, 64) == 34 * 128 and packed_bytes(64, 1) == 34 * 64
    with pytest.raises(HackError):
        packed_bytes(96, 64)
    pc = PackedCache.empty(64, [1, 65, 0, 64], device=DEV, with_pos=True)
    assert list(pc.off) == [0, 64, 192, 192] and pc.rows == 256 and list(pc.len) == [0, 0, 0, 0] and pc.pos.numel() == 256


# ---- attention ----------------------------------------------------------------
def filled(hk, B, lens, d, g, order=None):
    """A packed cache of random rows over memory that holds NaN everywhere else, and its rows."""
    pc = packed(lens, d, fill=0xFF, order=order, gap=64)
    off, rows = offsets(lens, 8)
    k, v = (torch.randn((rows, d), generator=g, device=DEV).to(hk.torch_dtype) for _ in range(2))
    hk.pack(B, 0, pc, cache_in=Cache(k, v, off, lens))
    return pc, [r[:2] for r in read_back(hk, B, pc, np.asarray(lens), hk.dtype)[0]]


def check_attention(q, rows, scale, out):
    """q, out [units, n, d]; rows: (K, V) of every unit.  Against softmax in float64.  Probabilities are rounded to bf16 where they are multiplied and
    where they are summed: 2 2^-8 of sum p |v|; a score of d products is summed in float32: (d + 4) 2^-24 of sum |q k|, and an error of s is a factor
    e^s on its probability and on the sum; exponentials and sums in float32: 1e-5; the output: half a step.
    Probabilities are taken against a reference that lies up to 2^15 above the largest (many queries), and what is below 2^-126 then, float32's and bf16's
    smallest normal number, may be zero: 2^-111 of each |v|.
    float32: queries and probabilities are three exact pieces, so a score sums 3 d products, and the sums over T keys have 3 T / 32 steps of a matrix
    instruction and 40 more of the merges, H each on the output and on the normaliser; the scale times log2 e is rounded twice: 2 H of a score on its exponent."""
    exact = q.dtype == torch.float32
    q, o = to64(q), to64(out)
    d = q.shape[-1]
    for u, (k, v) in enumerate(rows):
        s = q[u] @ k.T * scale
        p = np.exp(s - s.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        want = p @ v
        slack = scale * ((3 * d if exact else d) + 4) * H * (np.abs(q[u]) @ np.abs(k).T).max(-1, keepdims=True)
        rounding = 2 * (3 * len(k) / 32 + 40) * H + 4 * H * np.abs(s).max(-1, keepdims=True) if exact else 2 * 2.0 ** -8
        half = HALF_STEP["f32" if exact else "bf16"]
        tol = (rounding + 2 * slack + 1e-5) * (p @ np.abs(v)) * 1.01 + half * 1.01 * np.abs(want) + 2.0 ** -111 * (1 + np.abs(v).sum(0))
        err = np.abs(o[u] - want)
        assert (err <= tol).all(), (u, k.shape, float((err / tol).max()))


LENGTHS = [[1, 2, 3, 15, 16, 17], [31, 32, 33, 63, 64, 65], [100, 511, 512, 513, 1, 64], [1000, 2000, 129, 900, 30, 4001], [20000, 1, 20001, 64, 7, 640]]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", LENGTHS, ids=lambda l: "-".join(map(str, l)))
@pytest.mark.parametrize("n", [1, 16, 40])
def test_float32_attention_over_a_packed_cache(contexts, d, lens, n):
    hk = contexts(3, d, "f32")
    g = torch.Generator(DEV).manual_seed(n)
    pc, rows = filled(hk, 2, np.array(lens), d, g, order=[4, 2, 0, 1, 5, 3])
    q = 2 * torch.randn((2, 3, n, d), generator=g, device=DEV)
    out = torch.full_like(q, 9.0)
    hk.attn_packed(q, pc, d ** -0.5, out)
    check_attention(q.flatten(0, 1), rows, float(np.float32(d ** -0.5)), out.flatten(0, 1))
    again = torch.full_like(q, -9.0)
    hk.attn_packed(q, pc, d ** -0.5, again)
    assert torch.equal(out, again)


def test_float32_attention_of_odd_numbers(contexts):
    """Queries that need all of their bits, are tiny, huge or no numbers: what is finite is right, the rest is NaN."""
    hk = contexts(3, 64, "f32")
    g = torch.Generator(DEV).manual_seed(2)
    pc, rows = filled(hk, 1, np.array([70, 200, 33]), 64, g)
    q = torch.randn((1, 3, 6, 64), generator=g, device=DEV)
    q[0, :, 1] *= 1e-30
    q[0, :, 2] = torch.nextafter(torch.ones(64, device=DEV), torch.full((64,), 2.0, device=DEV))
    q[0, 0, 3, 5] = float("nan")
    q[0, 1, 4, 6] = float("inf")
    out = torch.empty_like(q)
    hk.attn_packed(q, pc, 0.125, out)
    bad = torch.zeros((3, 6), dtype=torch.bool, device=DEV)
    bad[0, 3] = bad[1, 4] = True
    assert torch.equal(torch.isnan(out[0]).all(-1), bad) and torch.isfinite(out[0][~bad]).all()
    for u in range(3):
        fine = ~bad[u].cpu()
        check_attention(q[0, u][fine][None], [rows[u]], 0.125, out[0, u][fine][None])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", LENGTHS, ids=lambda l: "-".join(map(str, l)))
@pytest.mark.parametrize("n, form", [(1, 0), (1, 128), (4, 0), (16, 0), (17, 0), (17, 16), (17, 128), (33, 0), (129, 16), (129, 32), (129, 128)])
def test_attention_over_a_packed_cache(contexts, d, lens, n, form):
    hk = contexts(3, d, "bf16", form=form)
    g = torch.Generator(DEV).manual_seed(n)
    pc, rows = filled(hk, 2, np.array(lens), d, g, order=[4, 2, 0, 1, 5, 3])
    q = (2 * torch.randn((2, 3, n, d), generator=g, device=DEV)).bfloat16()
    out = torch.full_like(q, 9.0)
    hk.attn_packed(q, pc, d ** -0.5, out)
    check_attention(q.flatten(0, 1), rows, float(np.float32(d ** -0.5)), out.flatten(0, 1))
    again = torch.full_like(q, -9.0)
    hk.attn_packed(q, pc, d ** -0.5, again)
    assert torch.equal(out, again)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_of_few_queries_over_one_long_cache(contexts, dtype, d):
    """One unit in hundreds of chunks: the merge has more of them than it loads ahead."""
    hk = contexts(1, d, dtype)
    g = torch.Generator(DEV).manual_seed(d)
    pc, rows = filled(hk, 1, np.array([140001]), d, g)
    for n in (1, 5):
        q = (2 * torch.randn((1, 1, n, d), generator=g, device=DEV)).to(TYPES[dtype])
        out = torch.full_like(q, 9.0)
        hk.attn_packed(q, pc, d ** -0.5, out)
        check_attention(q[0], rows, float(np.float32(d ** -0.5)), out[0])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n, form", [(300, 0), (1000, 0), (1000, 32), (1000, 128)])
def test_attention_of_many_queries_over_a_packed_cache(contexts, d, n, form):
    hk = contexts(3, d, "bf16", form=form)
    g = torch.Generator(DEV).manual_seed(n)
    for lens in ([1, 700, 33], [64, 4000, 129], [2500, 2500, 2500], [9000, 1, 260]):
        pc, rows = filled(hk, 1, np.array(lens), d, g)
        q = (3 * torch.randn((1, 3, n, d), generator=g, device=DEV)).bfloat16()
        out = torch.full_like(q, 9.0)
        hk.attn_packed(q, pc, d ** -0.5, out)
        check_attention(q[0], rows, float(np.float32(d ** -0.5)), out[0])


@pytest.mark.parametrize("form", [16, 32, 128])
def test_attention_where_the_largest_score_comes_late_or_alone(contexts, form):
    hk = contexts(3, 128, "bf16", form=form)
    g = torch.Generator(DEV).manual_seed(9)
    lens = np.array([700, 5000, 65])
    off, rows = offsets(lens, 8)
    k, v = torch.randn((rows, 128), generator=g, device=DEV), torch.randn((rows, 128), generator=g, device=DEV)
    q = torch.randn((1, 3, 20, 128), generator=g, device=DEV)
    for u in range(3):     # the last key, and one in the middle, far above all others
        k[off[u] + lens[u] - 1] = 6 * q[0, u, 0]
        k[off[u] + lens[u] // 2] = 4 * q[0, u, 1]
    for first in (False, True):
        if first:
            for u in range(3):
                k[off[u]] = 8 * q[0, u, 0]
        pc = packed(lens, 128, fill=0xFF)
        hk.pack(1, 0, pc, cache_in=Cache(k.bfloat16(), v.bfloat16(), off, lens))
        kv = [r[:2] for r in read_back(hk, 1, pc, lens, "bf16")[0]]
        qb, out = q.bfloat16(), torch.empty((1, 3, 20, 128), dtype=torch.bfloat16, device=DEV)
        hk.attn_packed(qb, pc, 0.5, out)
        check_attention(qb[0], kv, 0.5, out[0])


def test_heads_that_share_a_cache(contexts):
    kv_heads, group, B, n, d = 2, 4, 3, 3, 64
    hk = contexts(kv_heads, d, "bf16")
    g = torch.Generator(DEV).manual_seed(4)
    lens = np.array([70, 1, 200, 64, 33, 1500])
    pc, rows = filled(hk, B, lens, d, g)
    q = torch.randn((B, kv_heads * group, n, d), generator=g, device=DEV).bfloat16()
    out = torch.empty_like(q)
    hk.attn_packed(q, pc, 0.125, out)
    for b in range(B):
        for h in range(kv_heads * group):
            check_attention(q[b, h][None], [rows[b * kv_heads + h // group]], 0.125, out[b, h][None])


@pytest.mark.parametrize("form", [16, 32, 128])
def test_attention_says_nan_where_a_row_holds_one(contexts, form):
    hk = contexts(3, 64, "bf16", form=form)
    g = torch.Generator(DEV).manual_seed(6)
    lens = np.array([90, 90, 90])
    off, rows = offsets(lens, 8)
    k, v = (torch.randn((rows, 64), generator=g, device=DEV).bfloat16() for _ in range(2))
    k[off[1] + 3, 7] = float("nan")
    v[off[2] + 80, 40] = float("inf")
    pc = packed(lens, 64)
    hk.pack(1, 0, pc, cache_in=Cache(k, v, off, lens))
    q = torch.randn((1, 3, 5, 64), generator=g, device=DEV).bfloat16()
    out = torch.empty_like(q)
    hk.attn_packed(q, pc, 0.125, out)
    assert torch.isfinite(out[0, 0]).all() and torch.isnan(out[0, 1]).all()
    assert torch.isnan(out[0, 2, :, 32:]).all() and torch.isfinite(out[0, 2, :, :32]).all()


def test_many_units(contexts):
    """More units than a launch takes, on a stream of their own."""
    heads, B, d = 20, 70, 64
    hk = contexts(heads, d, "bf16", units=1400)
    g = torch.Generator(DEV).manual_seed(8)
    lens = np.array([1 + u * 31 % 150 for u in range(heads * B)])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pc, rows = filled(hk, B, lens, d, g)
        q = torch.randn((B, heads, 2, d), generator=g, device=DEV).bfloat16()
        out = torch.empty_like(q)
        hk.attn_packed(q, pc, 0.125, out)
    side.synchronize()
    check_attention(q.flatten(0, 1), rows, 0.125, out.flatten(0, 1))


# ---- together -----------------------------------------------------------------
def test_a_schedule_over_a_packed_cache(contexts):
    """Projection -> norm and rotation -> score, select and pack where the cache would outgrow its budget, pack alone before -> attention, for some steps;
    rows and outputs against plain arithmetic on what the step before has left."""
    heads, B, d, budget = 4, 2, 64, 96
    hk = Hack(heads, d, "bf16", heads * B, 512, 128)
    U = heads * B
    g = torch.Generator(DEV).manual_seed(12)
    rope = Rope.scaled(d, axes=2)
    w = 1 + torch.randn((heads, d), generator=g, device=DEV) / 4
    types = np.array([0, 1, 0, 1], np.uint8)
    pc = [packed(np.full(U, budget + 64), d, fill=0xFF) for _ in range(2)]
    lens, compressed = np.zeros(U, np.int64), 0
    for step, side in enumerate([2, 4, 5, 7, 8, 6, 3]):
        n = side * side
        proj = torch.randn((B, n, 3 * heads, d), generator=g, device=DEV).bfloat16().transpose(1, 2)
        q, k_new = (torch.empty((B, heads, n, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        v_new = proj[:, 2 * heads:].contiguous()
        pos = torch.stack([torch.arange(n) // side, torch.arange(n) % side]).int().to(DEV)
        hk.norm_rotate(proj[:, :heads], proj[:, heads:2 * heads], "l2", 1e-6, 8 * w, w, rope, q, k_new, pos=pos)
        t_in = lens + n
        cur, nxt = pc
        if t_in.max() <= budget:
            cur.len = t_in.astype(np.int32)
            hk.pack(B, n, cur, k_new=k_new, v_new=v_new, at=lens)
            lens = t_in
        else:
            compressed += 1
            cur.len = lens.astype(np.int32)
            _, plain = read_back(hk, B, cur, lens, "bf16")
            imp = torch.zeros((U, 512), device=DEV)
            kept = torch.zeros((U, 512), dtype=torch.int32, device=DEV)
            hk.score(q, plain, d ** -0.5, imp, k_new=k_new, n_obs=min(32, n))
            out_len = hk.select(B, imp, t_in, types, np.full(U, budget), 4, min(n, 20), kept)
            nxt.len = out_len.copy()
            hk.pack(B, n, nxt, cache_in=plain, kept_idx=kept, k_new=k_new, v_new=v_new)
            for u in range(U):
                both = np.concatenate([to64(plain.k[plain.off[u]:plain.off[u] + lens[u]]), to64(k_new[u // heads, u % heads])])
                i = kept[u, :out_len[u]].cpu().numpy()
                assert (np.diff(i) > 0).all() and i[-1] < t_in[u] and len(i) == budget
                rows = read_back(hk, B, nxt, out_len.astype(np.int64), "bf16")[0][u]
                assert same(rows[0], nearest(both[i]))
                assert same(rows[0][i < lens[u]], both[i][i < lens[u]])     # kept rows are not rounded again
            lens = out_len.astype(np.int64)
            pc = [nxt, cur]
        cur = pc[0]
        out = torch.empty_like(q)
        hk.attn_packed(q, cur, d ** -0.5, out)
        rows = [r[:2] for r in read_back(hk, B, cur, lens, "bf16")[0]]
        check_attention(q.flatten(0, 1), rows, float(np.float32(d ** -0.5)), out.flatten(0, 1))
    assert compressed >= 3
    torch.cuda.synchronize()
    hk.check()
    hk.close()


@pytest.mark.parametrize("B", [6, 20])
def test_graph_replays_and_eager_calls_in_turn(contexts, B):
    """A serving step captured once: norms and rotation, the new row packed, attention; replayed with eager work and other inputs between."""
    heads, d = 4, 128
    hk = contexts(heads, d, "bf16", units=4 * B, queries=64)
    g = torch.Generator(DEV).manual_seed(3)
    lens = np.array([1 + 97 * u for u in range(heads * B)])
    pc, _ = filled(hk, B, lens, d, g)
    pc.len = (lens + 1).astype(np.int32)      # capacity: the rows beyond are in the gap behind every unit
    proj = torch.empty((B, 1, 3 * heads, d), dtype=torch.bfloat16, device=DEV)
    p = proj.transpose(1, 2)
    q, k, out = (torch.empty((B, heads, 1, d), dtype=torch.bfloat16, device=DEV) for _ in range(3))
    v = torch.empty_like(k)
    pos = torch.zeros((B, 1, 1), dtype=torch.int32, device=DEV)
    rope = Rope.scaled(d)

    def step():
        hk.norm_rotate(p[:, :heads], p[:, heads:2 * heads], "rms", 1e-6, None, None, rope, q, k, pos=pos)
        v.copy_(p[:, 2 * heads:])
        hk.pack(B, 1, pc, k_new=k, v_new=v, at=lens)
        hk.attn_packed(q, pc, d ** -0.5, out)
        return out

    def feed(i):
        proj.copy_(torch.randn(proj.shape, generator=torch.Generator(DEV).manual_seed(100 + i), device=DEV))
        pos.fill_(50 + i)

    feed(0)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        feed(i)
        graph.replay()
        torch.cuda.synchronize()
        replayed, bytes_k = out.clone(), pc.k.clone()
        feed(50 + i)
        step()                      # eager, other inputs, the same workspace
        torch.cuda.synchronize()
        feed(i)
        out.zero_()
        step()
        torch.cuda.synchronize()
        assert torch.equal(out, replayed) and torch.equal(pc.k, bytes_k)
