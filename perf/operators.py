"""The operators around the cache that this library is timed on beside its steps: rotary positions, the norms of queries
and keys with the rotation in the same pass, rows packed into a 4-bit cache and read back, and attention over such a
cache; over sizes from one token to whole images and long caches.

With `own` false `run` computes them in plain torch operations, with `own` true it calls the library.
"""
from __future__ import annotations

import functools
import math

import numpy as np
import torch

own = False

GROUP = 32           # elements that share a scale
BLOCK = 64           # rows of a block of a packed cache
THRESHOLDS = ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False))
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---- cases -----------------------------------------------------------------
def _rotate(name, dtype, heads, head_dim, batch, n, layout="half", rot=None, axes=1, scaling="plain", factor=1.0, first=0, strided=False):
    """first: position of the first row; strided: rows as a projection leaves them, [batch, n, heads, head_dim]."""
    return dict(name=name, kind="rotate", dtype=dtype, heads=heads, head_dim=head_dim, batch=batch, n=n, layout=layout, rot=rot or head_dim,
                axes=axes, scaling=scaling, factor=factor, first=first, strided=strided)


def _norm(name, dtype, heads, kv_heads, head_dim, batch, n, norm="rms", per_head=False, **rope):
    """Queries and keys where one projection for q, k and v has left them: [batch, n, (heads + 2 kv_heads) head_dim]."""
    c = _rotate(name, dtype, heads, head_dim, batch, n, **rope)
    return dict(c, kind="norm", kv_heads=kv_heads, norm=norm, per_head=per_head, strided=True)


def _pack(name, dtype, heads, head_dim, batch, lo, hi, n, keep):
    """Units of lo to hi cached rows and n new ones.  keep > 0: a share of them all goes to a cache of its own, through kept lists, as hack_compact
    does it; keep 0: the new rows go behind the cached ones."""
    return dict(name=name, kind="pack", dtype=dtype, heads=heads, head_dim=head_dim, batch=batch, lo=lo, hi=hi, n=n, keep=keep)


def _attn(name, heads, kv_heads, head_dim, batch, lo, hi, n):
    """n queries of each of `heads` heads, which share kv_heads caches of lo to hi rows."""
    return dict(name=name, kind="attn", dtype="bf16", heads=heads, kv_heads=kv_heads, head_dim=head_dim, batch=batch, lo=lo, hi=hi, n=n)


def listed():
    return [
        # keys of one token of each of eight sequences, far into a long context whose frequencies are scaled by parts: latency
        _rotate("rotate-one-token", "bf16", 16, 128, 8, 1, scaling="parts", factor=8.0, first=100000),
        # queries of the last scale of a 1024^2 image, one prompt with guidance, rows and columns as two axes
        _rotate("rotate-1024-image", "bf16", 16, 128, 2, 4096, axes=2, strided=True),
        # float32, an odd side (37^2 tokens), a quarter of the head, pairs side by side
        _rotate("rotate-f32-part", "f32", 20, 64, 3, 1369, layout="interleaved", rot=16, scaling="linear", factor=4.0, first=70000),
        # one token of each of 64 sequences, grouped heads, from one projection: what a serving step begins with
        _norm("norm-one-token", "bf16", 32, 8, 128, 64, 1, first=9000),
        # a prompt of a long context, base raised
        _norm("norm-long-prompt", "bf16", 32, 8, 128, 1, 16384, scaling="base", factor=4.0),
        # 256^2 images, unit norms with a scale for each head, the last scale of a batch of 16 with guidance
        _norm("norm-256-batch", "bf16", 30, 30, 64, 32, 256, norm="l2", per_head=True, axes=2),
        # the new row of each of 64 sequences behind its cached ones: latency
        _pack("pack-one-token", "bf16", 8, 128, 64, 900, 4000, 1, 0.0),
        # a compressing step of a 1024^2 image: kept rows of each head, cached and new ones, into a packed cache
        _pack("pack-1024-compact", "bf16", 16, 128, 2, 1943, 3885, 2304, 0.5),
        # one token, 64 sequences of different lengths, four heads to a cache: an ordinary serving step
        _attn("attn-one-token", 32, 8, 128, 64, 900, 4000, 1),
        # one sequence over a long cache, eight heads to a cache: few units, work split over the keys
        _attn("attn-long-cache", 64, 8, 128, 1, 131071, 131071, 1),
        # the last scale of a 1024^2 image over compressed caches of two lengths: matrix products
        _attn("attn-1024-image", 16, 16, 128, 2, 1943, 3885, 4096),
        # a middle scale of 256^2 images, narrow heads, odd lengths, a batch: many short units
        _attn("attn-256-batch", 30, 30, 64, 16, 61, 293, 100),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "norm", "pack", "attn", "attn"])
    d = rng.choice([64, 128])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    scaling = rng.choice(["plain", "linear", "base", "parts"])
    axes = rng.choice([1, 1, 2])
    rope = dict(layout=rng.choice(["half", "interleaved"]), rot=rng.choice([d, d, d // 2, 16 * axes]), axes=axes, scaling=scaling,
                factor=1.0 if scaling == "plain" else rng.choice([2.0, 4.0, 8.0]), first=_log(rng, 1, 200000) - 1)
    while True:
        heads, batch = _log(rng, 1, 40), _log(rng, 1, 64)
        if kind == "rotate":
            c = _rotate("", dtype, heads, d, batch, _log(rng, 1, 16384), strided=rng.random() < 0.5, **rope)
        elif kind == "norm":
            kv = rng.choice([k for k in range(1, heads + 1) if heads % k == 0])
            c = _norm("", dtype, heads, kv, d, batch, _log(rng, 1, 16384), norm=rng.choice(["rms", "l2"]), per_head=rng.random() < 0.5, **rope)
        elif kind == "pack":
            hi = _log(rng, 1, 6000)
            c = _pack("", dtype, heads, d, batch, rng.randint(1, hi), hi, _log(rng, 1, 3000), rng.choice([0.0, 0.1, 0.3, 0.7]))
        else:
            kv = rng.choice([k for k in range(1, heads + 1) if heads % k == 0])
            hi = _log(rng, 1, 131071)
            c = _attn("", heads, kv, d, batch, rng.randint(max(1, hi // 3), hi), hi, _log(rng, 1, 4096) if rng.random() < 0.6 else 1)
            if c["n"] * heads // kv > 4096:
                continue
        w = work(c)
        if w["bytes"] <= 400e6 and w["flops"] <= 2e11:
            del c["name"]
            return c


# ---- what a case is made of ------------------------------------------------
def _lengths(lo, hi, units):
    """Lengths of the units, spread over lo..hi in an order of their own."""
    if units == 1:
        return np.array([hi], np.int64)
    return np.array([lo + (hi - lo) * ((u * 7919) % units) // (units - 1) for u in range(units)], np.int64)


def _kept(c):
    units = c["batch"] * c["heads"]
    cached = _lengths(c["lo"], c["hi"], units)
    return cached, np.maximum(1, (c["keep"] * (cached + c["n"])).astype(np.int64)) if c["keep"] else np.full(units, c["n"], np.int64)


def _offsets(lengths, step):
    rows = (lengths + step - 1) // step * step
    return np.concatenate([[0], np.cumsum(rows)[:-1]]), int(rows.sum())


def _type(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _positions(c):
    """[axes, n]: token numbers, or rows and columns of a square image (in two axes) of the nearest side."""
    i = np.arange(c["n"], dtype=np.int64)
    if c["axes"] == 1:
        return (i + c["first"]).astype(np.int32)[None]
    side = max(1, math.isqrt(c["n"]))
    return np.stack([i // side, i % side]).astype(np.int32)


def _frequencies(c):
    """Radians per position of the pairs of each axis, one after the other, and the factor on cosine and sine."""
    size, base, f = c["rot"] // c["axes"], 10000.0, c["factor"]
    i = np.arange(size // 2, dtype=np.float64)
    if c["scaling"] == "base" and size > 2:
        base *= f ** (size / (size - 2))
    freq, gain = base ** (-2 * i / size), 1.0
    if c["scaling"] == "linear":
        freq = freq / f
    if c["scaling"] == "parts":   # pairs that turn often over the length trained on stay, slow ones are stretched
        at = lambda turns: size * math.log(4096 / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        low, high = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), size - 1)
        ramp = np.clip((i - low) / max(high - low, 0.001), 0, 1)
        freq, gain = freq * (1 - ramp) + freq / f * ramp, 0.1 * math.log(f) + 1.0
    return np.tile(freq, c["axes"]), gain


def _split(x):
    """Scale exponents and codes (sign in bit 3) of the groups of x, in float32."""
    g = x.float().unflatten(-1, (-1, GROUP))
    most = g.abs().amax(-1, keepdim=True)
    fine = torch.isfinite(most)
    m, e = torch.frexp(torch.where(fine, most, 1.0))           # most = m 2^e, m in [0.5, 1)
    e = (e - 3 + (m > 0.875)).clamp(3 - 127, 252 - 127)        # the largest lies in (3.5, 7] 2^e
    e = torch.where(most == 0, 3 - 127, e)
    y = torch.ldexp(torch.where(fine, g, 0.0), -e)
    a = y.abs()
    code = sum((a >= t if up else a > t).to(torch.uint8) for t, up in THRESHOLDS) + 8 * (y < 0).to(torch.uint8)
    return torch.where(fine, e + 127, 255).squeeze(-1).to(torch.uint8), code


def _join(scale, code):
    """The values that scale exponents and codes stand for, in float32."""
    mags = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device=code.device)
    return torch.ldexp(mags[code.int()], scale.int().unsqueeze(-1) - 127).flatten(-2)


def _to_blocks(scale, code):
    """Bytes of a packed tensor [rows / 64, 34 head_dim] from those of its rows: codes of 16 rows and a quarter of the head side by side, then scales."""
    rows, d = code.shape[0], code.shape[1] * GROUP
    c = code.view(rows, d // 2, 2)
    c = (c[..., 0] | c[..., 1] << 4).view(rows // BLOCK, -1, 128 // d, 16, 4, d // 8)    # block, pair of 16s, 16 rows, row, quarter, bytes
    s = scale.view(rows // BLOCK, 4, 16, d // GROUP).permute(0, 3, 2, 1)
    return torch.cat([c.permute(0, 1, 4, 3, 2, 5).reshape(rows // BLOCK, -1), s.reshape(rows // BLOCK, -1)], 1).contiguous()


def _from_blocks(mem, d):
    """Scale exponents and codes of the rows of a packed tensor."""
    n = mem.shape[0]
    c = mem[:, : 32 * d].view(n, -1, 4, 16, 128 // d, d // 8).permute(0, 1, 4, 3, 2, 5).reshape(n * BLOCK, d // 2)
    s = mem[:, 32 * d :].view(n, d // GROUP, 16, 4).permute(0, 3, 2, 1).reshape(n * BLOCK, d // GROUP)
    return s, torch.stack([c & 15, c >> 4], -1).view(n * BLOCK, d // GROUP, GROUP)


def _keys(shape, g, dev):
    """Rows as keys have them: some elements of the head much larger than the others."""
    x = torch.randn(shape, generator=g, device=dev)
    return x * (1 + 5 * (torch.rand(shape[-1], generator=g, device=dev) < 0.06))


def prepare(case, seed):
    c, dev = case, torch.device("cuda", 0)
    g = torch.Generator(device=dev).manual_seed(seed)
    st = dict(case=c)
    t, d, B, H = _type(c), c["head_dim"], c["batch"], c["heads"]
    if c["kind"] in ("rotate", "norm"):
        st["pos"] = torch.from_numpy(_positions(c)).to(dev)
        st["freq"], st["gain"] = _frequencies(c)
    if c["kind"] == "rotate":
        shape = (B, c["n"], H, d) if c["strided"] else (B, H, c["n"], d)
        x = torch.randn(shape, generator=g, device=dev).to(t)
        st["x"] = x.transpose(1, 2) if c["strided"] else x
        st["out"] = torch.empty((B, H, c["n"], d), dtype=t, device=dev)
    elif c["kind"] == "norm":
        K = c["kv_heads"]
        proj = torch.randn((B, c["n"], H + 2 * K, d), generator=g, device=dev).mul_(2.5).to(t).transpose(1, 2)
        st["q"], st["k"] = proj[:, :H], proj[:, H : H + K]
        st["q_w"], st["k_w"] = (1 + 0.3 * torch.randn((h, d) if c["per_head"] else (d,), generator=g, device=dev) for h in (H, K))
        st["q_out"], st["k_out"] = (torch.empty((B, h, c["n"], d), dtype=t, device=dev) for h in (H, K))
    elif c["kind"] == "pack":
        cached, kept = _kept(c)
        st["kept_len"], st["cached"] = kept, cached
        st["k_new"], st["v_new"] = _keys((B, H, c["n"], d), g, dev).to(t), torch.randn((B, H, c["n"], d), generator=g, device=dev).to(t)
        if c["keep"]:
            st["in_off"], rows = _offsets(cached, 8)
            st["k_in"], st["v_in"] = _keys((rows, d), g, dev).to(t), torch.randn((rows, d), generator=g, device=dev).to(t)
            total = torch.from_numpy(cached + c["n"]).to(dev)[:, None]
            pri = torch.rand((B * H, int(cached.max()) + c["n"]), generator=g, device=dev)
            pri[torch.arange(pri.shape[1], device=dev) >= total] = -1.0
            top = pri.argsort(1, descending=True)[:, : int(kept.max())]
            top[torch.arange(top.shape[1], device=dev) >= torch.from_numpy(kept).to(dev)[:, None]] = 1 << 30
            st["kept"] = top.sort(1).values.int().contiguous()
            st["at"] = np.zeros(B * H, np.int64)
        else:
            st["at"] = cached
        st["off"], rows = _offsets(st["at"] + kept, BLOCK)
        st["k_mem"], st["v_mem"] = (torch.zeros((rows // BLOCK, 34 * d), dtype=torch.uint8, device=dev) for _ in range(2))
        st["out_off"], rows = _offsets(kept, 8)
        st["k_out"], st["v_out"] = (torch.zeros((rows, d), dtype=t, device=dev) for _ in range(2))
    else:
        n = _lengths(c["lo"], c["hi"], B * c["kv_heads"])
        st["len"] = n
        st["off"], rows = _offsets(n, BLOCK)
        st["k_mem"] = _to_blocks(*_split(_keys((rows, d), g, dev)))
        st["v_mem"] = _to_blocks(*_split(torch.randn((rows, d), generator=g, device=dev)))
        st["q"] = (2 * torch.randn((B, H, c["n"], d), generator=g, device=dev)).to(t)
        st["out"] = torch.empty_like(st["q"])
    return st


# ---- plain forms -----------------------------------------------------------
def _turn(x, c, st):
    """x (float32, [B, H, n, head_dim]) turned."""
    size, half = c["rot"] // c["axes"], c["rot"] // c["axes"] // 2
    angle = st["pos"].double().unsqueeze(-1) * torch.from_numpy(st["freq"]).to(x.device).view(c["axes"], 1, half)      # axes, n, pairs
    cos, sin = ((st["gain"] * f(angle)).float().transpose(0, 1) for f in (torch.cos, torch.sin))        # n, axes, pairs
    y = x[..., : c["rot"]].unflatten(-1, (c["axes"], 2, half) if c["layout"] == "half" else (c["axes"], half, 2))
    a, b = y.unbind(-2 if c["layout"] == "half" else -1)
    y = torch.stack([a * cos - b * sin, a * sin + b * cos], -2 if c["layout"] == "half" else -1)
    return torch.cat([y.flatten(-3), x[..., c["rot"] :]], -1)


def _normed(x, w, c):
    """RMS or unit norm of float32 rows with a weight for each element, eps 1e-6."""
    w = w.view(1, -1, 1, x.shape[-1])
    s = (x * x).sum(-1, keepdim=True)
    return x * torch.rsqrt(s / x.shape[-1] + 1e-6) * w if c["norm"] == "rms" else x / s.sqrt().clamp_min(1e-6) * w


def _plain(st):
    c = st["case"]
    t, d = _type(c), c["head_dim"]
    if c["kind"] == "rotate":
        return _turn(st["x"].float(), c, st).to(t)
    if c["kind"] == "norm":
        return {"q": _turn(_normed(st["q"].float(), st["q_w"], c), c, st).to(t), "k": _turn(_normed(st["k"].float(), st["k_w"], c), c, st).to(t)}
    dev = st["k_mem"].device
    at = lambda a: torch.from_numpy(a).to(dev)  # noqa: E731
    if c["kind"] == "pack":
        units, n = c["batch"] * c["heads"], int(st["kept_len"].max())
        i = torch.arange(n, device=dev)
        there = i < at(st["kept_len"])[:, None]
        unit = torch.arange(units, device=dev)[:, None]
        if c["keep"]:
            new = st["kept"] - at(st["cached"])[:, None]
            src = torch.where(new < 0, at(st["in_off"])[:, None] + st["kept"], st["k_in"].shape[0] + unit * c["n"] + new)[there]
            rows = [torch.cat([a, b.reshape(-1, d)])[src] for a, b in ((st["k_in"], st["k_new"]), (st["v_in"], st["v_new"]))]
        else:
            rows = [st["k_new"].reshape(-1, d), st["v_new"].reshape(-1, d)]
        to = (at(st["out_off"])[:, None] + i)[there]
        for out, x in zip((st["k_out"], st["v_out"]), rows):
            out[to] = _join(*_split(x)).to(t)
        return {"k": st["k_out"], "v": st["v_out"]}
    # attention: units padded to the longest
    units, n = len(st["len"]), int(st["len"].max())
    i = torch.arange(n, device=dev)
    there = i < at(st["len"])[:, None]
    row = torch.where(there, at(st["off"])[:, None] + i, 0)
    k, v = (_join(*_from_blocks(st[m], d))[row] for m in ("k_mem", "v_mem"))
    s = torch.matmul(st["q"].float().reshape(units, -1, d), k.transpose(1, 2).contiguous()) * d ** -0.5
    s.masked_fill_(~there[:, None], -math.inf)
    p = s.sub_(s.amax(-1, keepdim=True)).exp_()
    return (torch.matmul(p, v) / p.sum(-1, keepdim=True)).reshape(st["q"].shape).to(t)


# ---- the library's calls ---------------------------------------------------
@functools.lru_cache(maxsize=None)
def _context(heads, head_dim, dtype, units, queries):
    from paper_2504_09261_amd.binding import Hack
    return Hack(heads, head_dim, dtype, units, 64, queries)


def _own(st):
    from paper_2504_09261_amd.binding import Cache, PackedCache, Rope
    c = st["case"]
    d, B, H = c["head_dim"], c["batch"], c["heads"]
    if c["kind"] in ("rotate", "norm"):
        hk = _context(H, d, c["dtype"], B * H, c["n"])
        if "rope" not in st:
            st["rope"] = Rope(st["freq"], c["rot"], c["axes"], c["layout"], st["gain"])
        if c["kind"] == "rotate":
            hk.rotate(st["x"], st["rope"], st["out"], pos=st["pos"])
            return st["out"]
        hk.norm_rotate(st["q"], st["k"], c["norm"], 1e-6, st["q_w"], st["k_w"], st["rope"], st["q_out"], st["k_out"], pos=st["pos"])
        return {"q": st["q_out"], "k": st["k_out"]}
    if c["kind"] == "pack":
        hk = _context(H, d, c["dtype"], B * H, c["n"])
        if "packed" not in st:
            st["packed"] = PackedCache(st["k_mem"], st["v_mem"], st["off"], st["at"] + st["kept_len"])
            st["rows"] = Cache(st["k_out"], st["v_out"], st["out_off"], st["kept_len"])
            st["cache"] = Cache(st["k_in"], st["v_in"], st["in_off"], st["cached"]) if c["keep"] else None
        hk.pack(B, c["n"], st["packed"], cache_in=st["cache"], kept_idx=st.get("kept"), k_new=st["k_new"], v_new=st["v_new"], at=st["at"])
        hk.unpack(B, st["packed"], st["rows"], first=st["at"])
        return {"k": st["k_out"], "v": st["v_out"]}
    hk = _context(c["kv_heads"], d, c["dtype"], B * c["kv_heads"], c["n"] * H // c["kv_heads"])
    if "packed" not in st:
        st["packed"] = PackedCache(st["k_mem"], st["v_mem"], st["off"], st["len"])
    hk.attn_packed(st["q"], st["packed"], d ** -0.5, st["out"])
    return st["out"]


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    c, d, e = case, case["head_dim"], 4 if case["dtype"] == "f32" else 2
    if c["kind"] in ("rotate", "norm"):
        rows = c["batch"] * c["n"] * (c["heads"] + c.get("kv_heads", 0))
        return {"bytes": 2 * rows * d * e + 4 * c["axes"] * c["n"], "flops": rows * (3 * c["rot"] + (4 * d if c["kind"] == "norm" else 0))}
    if c["kind"] == "pack":   # K and V: rows read, packed, read packed, written; lists
        rows = int(_kept(c)[1].sum())
        return {"bytes": rows * (4 * d * (e + 17 / 32) + (4 if c["keep"] else 0)), "flops": rows * 2 * d * 4}
    keys, queries = int(_lengths(c["lo"], c["hi"], c["batch"] * c["kv_heads"]).sum()), c["n"] * c["heads"] // c["kv_heads"]
    return {"bytes": keys * 2 * d * 17 / 32 + 4 * c["batch"] * c["heads"] * c["n"] * d, "flops": 4 * queries * keys * d}


# ---- the definitions in 64 bits --------------------------------------------
def _nearest(x):
    """x in 4 bits: the nearest value of the grid that the group's largest magnitude sets, ties to the even one."""
    g = x.double().reshape(*x.shape[:-1], -1, GROUP)
    top = g.abs().amax(-1, keepdim=True).clamp_min(2.0 ** -200)
    e = torch.floor(torch.log2(top)) - 2
    e = torch.where(torch.exp2(e + 3) <= top, e + 1, torch.where(torch.exp2(e + 2) > top, e - 1, e))      # where log2 rounded
    e = (e + (top > 7 * torch.exp2(e))).clamp(-124, 125)
    y = g / torch.exp2(e)
    step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0))
    return (torch.round(y / step) * step).clamp(-6, 6).mul(torch.exp2(e)).reshape(x.shape)


def _turned(x, c):
    freq, gain = _frequencies(c)
    pos, size = _positions(c), c["rot"] // c["axes"]
    out = x.clone()
    for a in range(c["axes"]):
        for i in range(size // 2):
            p, q = (i, i + size // 2) if c["layout"] == "half" else (2 * i, 2 * i + 1)
            p, q = p + a * size, q + a * size
            angle = pos[a].astype(np.float64) * freq[a * size // 2 + i]
            cos, sin = (torch.from_numpy(gain * f(angle)).to(x.device) for f in (np.cos, np.sin))
            out[..., p] = x[..., p] * cos - x[..., q] * sin
            out[..., q] = x[..., p] * sin + x[..., q] * cos
    return out


def exact(case, seed):
    st, c, d = prepare(case, seed), case, case["head_dim"]
    if c["kind"] == "rotate":
        return _turned(st["x"].double(), c)
    if c["kind"] == "norm":
        got = {}
        for name in ("q", "k"):
            x, w = st[name].double(), st[name + "_w"].double()
            size = x.square().sum(-1, keepdim=True)
            size = (size / d + 1e-6).sqrt() if c["norm"] == "rms" else size.sqrt().clamp_min(1e-6)
            got[name] = _turned(x / size * (w[:, None] if c["per_head"] else w), c)
        return got
    if c["kind"] == "pack":
        got = {}
        for name in ("k", "v"):
            out = torch.zeros(st[name + "_out"].shape, dtype=torch.float64, device=st[name + "_out"].device)
            new = st[name + "_new"].flatten(0, 1)
            for u, n in enumerate(st["kept_len"].tolist()):
                rows = new[u]
                if c["keep"]:
                    lo = int(st["in_off"][u])
                    rows = torch.cat([st[name + "_in"][lo : lo + int(st["cached"][u])], rows])[st["kept"][u, :n].long()]
                out[int(st["out_off"][u]) : int(st["out_off"][u]) + n] = _nearest(rows)
            got[name] = out
        return got
    out = torch.empty(st["q"].shape, dtype=torch.float64, device=st["q"].device)
    q = st["q"].double().view(len(st["len"]), -1, d)
    flat = out.view(q.shape)
    grid = torch.tensor([m * s for s in (1.0, -1.0) for m in MAGNITUDES], dtype=torch.float64, device=q.device)
    for u, n in enumerate(st["len"].tolist()):
        kv = []
        for name in ("k_mem", "v_mem"):
            scale, code = _from_blocks(st[name][int(st["off"][u]) // BLOCK : -(-(int(st["off"][u]) + n) // BLOCK)], d)
            kv.append((grid[code.long()] * torch.exp2(scale.double() - 127)[..., None]).flatten(-2)[:n])
        flat[u] = torch.softmax(q[u] @ kv[0].T * (1.0 / math.sqrt(d)), -1) @ kv[1]
    return out
