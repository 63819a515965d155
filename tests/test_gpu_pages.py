"""Caches in pages (appending with norm and rotation, attention for tokens, scales and causal prompts, shared prefixes) against plain implementations in
64 bits, through the C ABI.  Tolerances count roundings: half a step of a type is finfo.eps / 2 relative, H below is float32's."""
import os

import numpy as np
import pytest
import torch

from paper_2504_09261_amd.binding import Hack, HackError, PagedCache, Rope
from tests.test_gpu_operators import DEV, H, HALF_STEP, NORM, ROTATION, TYPES, check_rows, rows_in, to64, turned

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def contexts():
    made = {}

    def get(heads, d, dtype, units=64, queries=4096, shared=None):
        key = (heads, d, dtype, units, queries, shared)
        if key not in made:
            if shared is not None:
                os.environ["HACK_ATTN_PAGES_SHARED"] = str(shared)      # read when a context is created
            try:
                made[key] = Hack(heads, d, dtype, units, 64, queries)
            finally:
                os.environ.pop("HACK_ATTN_PAGES_SHARED", None)
        return made[key]
    yield get
    for h in made.values():
        h.close()


class Pool:
    """Sequences in pages of a pool that holds NaN everywhere else; entries of tables behind a sequence's last page are no page numbers."""

    def __init__(self, hk, lens, page, g, by_head=False, layout="rows", shared=(), extra=0, scale=1.0):
        lens = np.asarray(lens)                     # [B] or, by head, [B, heads]
        B, K, d = lens.shape[0], hk.heads, hk.head_dim
        per, in_page = (K, 1) if by_head else (1, K)
        lens = lens.reshape(B, per)
        need = -(-(lens + extra) // page)
        table = np.full((B, per, max(1, int(need.max())) + 2), 1 << 30, np.int64)
        n = 0
        for b in range(B):
            common = next(((f, r // page) for f, c, r in shared if f < b < f + c), (0, 0))
            for u in range(per):
                have = min(common[1], int(need[b, u]))
                table[b, u, :have] = table[common[0], u, :have]
                k = int(need[b, u]) - have
                table[b, u, have:have + k] = np.arange(n, n + k)
                n += k
        self.n_pages = n + 2
        order = torch.randperm(self.n_pages, generator=torch.Generator().manual_seed(n)).numpy()
        used = table < 1 << 30
        table[used] = order[table[used]]
        shape = {"rows": (self.n_pages, page, in_page, d), "heads": (self.n_pages, in_page, page, d), "turns": (self.n_pages, 2, page, in_page, d)}[layout]
        if layout == "turns":
            kv = torch.full(shape, float("nan"), dtype=hk.torch_dtype, device=DEV)
            self.k, self.v = kv[:, 0], kv[:, 1]
        else:
            self.k, self.v = (torch.full(shape, float("nan"), dtype=hk.torch_dtype, device=DEV) for _ in range(2))
            if layout == "heads":
                self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        self.np_table, self.page, self.by_head, self.lens, self.heads = table, page, by_head, lens, K
        self.table = torch.from_numpy(table.astype(np.int32)).reshape(B * per, -1).to(DEV)
        self.len = torch.from_numpy(lens.astype(np.int32)).reshape(-1).to(DEV)
        self.cache = PagedCache(self.k, self.v, self.table, self.len)
        for b in range(B):
            for h in range(K):
                at = self.where(b, h, 0, int(lens[b, h if by_head else 0]))
                for m, s in ((self.k, scale), (self.v, 1.0)):
                    old = m[at]
                    new = (s * torch.randn(old.shape, generator=g, device=DEV)).to(m.dtype)
                    m[at] = torch.where(torch.isnan(old), new, old)
        for f, c, r in shared:                      # rows of a page that is not shared as a whole
            for b in range(f + 1, f + c):
                for h in range(K):
                    n = min(r, int(lens[b, h if by_head else 0]))
                    for m in (self.k, self.v):
                        m[self.where(b, h, 0, n)] = m[self.where(f, h, 0, n)]

    def where(self, b, h, lo, hi):
        r = np.arange(lo, hi)
        page = self.np_table[b, h if self.by_head else 0][r // self.page]
        t = lambda x: torch.from_numpy(np.asarray(x, np.int64)).to(DEV)  # noqa: E731
        return t(page), t(r % self.page), torch.full((len(r),), 0 if self.by_head else h, dtype=torch.int64, device=DEV)

    def rows(self, b, h, n=None):
        at = self.where(b, h, 0, int(self.lens[b, h if self.by_head else 0]) if n is None else n)
        return self.k[at].double(), self.v[at].double()


def check_attention(pool, q, out, scale, causal=False, fresh=None, untouched=9.0):
    """Against softmax in float64, query by query over the rows that it sees.  Probabilities are rounded to bf16 where they are multiplied and where they are
    summed: 2 2^-8 of sum p |v|; a score of d products is summed in float32: (d + 4) 2^-24 of sum |q k|, and an error of s is a factor e^s on its probability
    and on the sum; exponentials and sums in float32: 1e-5; the output: half a step.  A probability is taken against a reference at most 2^15 above the row's
    largest, and what is below 2^-126 then, float32's and bf16's smallest normal number, may be zero: 2^-111 of each |v|.
    float32: sums over T keys have T / 4 steps of a matrix instruction and 60 more of the merges at most, H each on the output and on the normaliser; the
    scale times log2 e is rounded twice: 2 H of a score on its exponent, on the output and on the normaliser."""
    B, heads, N, d = q.shape
    G, exact = heads // pool.heads, q.dtype == torch.float32
    half = HALF_STEP["f32" if exact else "bf16"]
    for b in range(B):
        f = N if fresh is None else int(fresh[b])
        assert (out[b, :, f:] == untouched).all()
        for h in range(pool.heads):
            n = int(pool.lens[b, h if pool.by_head else 0])
            k, v = pool.rows(b, h)
            x, got = q[b, h * G:(h + 1) * G, :f].double().reshape(-1, d), out[b, h * G:(h + 1) * G, :f].double().reshape(-1, d)
            sees = torch.full((f,), n, device=DEV) if not causal else (n - f + 1 + torch.arange(f, device=DEV)).clamp_min(0)
            sees = sees.repeat(G)[:, None]
            gone = torch.arange(n, device=DEV) >= sees
            s = (x @ k.T.contiguous() * scale).masked_fill(gone, -float("inf"))
            p = torch.exp(s - s.amax(-1, keepdim=True)) if n else s
            p = torch.where(sees > 0, p / p.sum(-1, keepdim=True), 0.0)
            v = torch.where(torch.isfinite(v), v, 0.0)
            want = p @ v
            seen = torch.where(gone, 0.0, s.abs())
            size = torch.where(gone, 0.0, x.abs() @ k.abs().T.contiguous()).amax(-1, keepdim=True) if n else torch.zeros_like(x[:, :1])
            slack = scale * (d + 4) * H * size
            top = seen.amax(-1, keepdim=True) if n else torch.zeros_like(x[:, :1])
            rounding = 2 * (n / 4 + 60) * H + 4 * H * top if exact else 2 * 2.0 ** -8
            tol = (rounding + 2 * slack + 1e-5) * (p @ v.abs()) * 1.01 + half * 1.01 * want.abs() + 2.0 ** -111 * (1 + v.abs().sum(0))
            err = (got - want).abs()
            assert (err <= tol).all(), (b, h, n, f, float((err / tol).max()))
            assert (got[(sees <= 0)[:, 0]] == 0).all()


def queries(shape, dtype, g, size=2.0):
    return (size * torch.randn(shape, generator=g, device=DEV)).to(TYPES[dtype])


# ---- attention ----------------------------------------------------------------
LENGTHS = [[1, 2, 17], [16, 0, 33], [63, 64, 65], [1000, 31, 129], [2500, 1, 300]]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", LENGTHS, ids=lambda l: "-".join(map(str, l)))
@pytest.mark.parametrize("n, group, page", [(1, 1, 16), (1, 4, 64), (3, 2, 32), (16, 1, 128), (17, 1, 16), (40, 3, 64), (130, 1, 64), (300, 2, 16)])
def test_attention(contexts, dtype, d, lens, n, group, page):
    hk = contexts(2, d, dtype)
    g = torch.Generator(DEV).manual_seed(n)
    pool = Pool(hk, lens, page, g)
    q = queries((3, 2 * group, n, d), dtype, g)
    out = torch.full_like(q, 9.0)
    hk.attn_pages(q, pool.cache, d ** -0.5, out)
    check_attention(pool, q, out, float(np.float32(d ** -0.5)))
    again = torch.full_like(q, -9.0)
    hk.attn_pages(q, pool.cache, d ** -0.5, again)
    assert torch.equal(out, again)
    hk.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d, page, layout, by_head", [(64, 16, "rows", False), (128, 64, "heads", False), (64, 32, "turns", True), (128, 16, "rows", True)])
@pytest.mark.parametrize("n, fresh", [(1, None), (7, [7, 0, 3, 7]), (33, [1, 33, 20, 32]), (200, None), (257, [257, 255, 3, 130])])
def test_causal_attention_of_ragged_batches(contexts, dtype, d, page, layout, by_head, n, fresh):
    hk = contexts(2, d, dtype)
    g = torch.Generator(DEV).manual_seed(n)
    # a sequence shorter than its new rows: its first queries see nothing
    lens = np.array([n + 700, n, max(n // 2, 1), n + 31])
    if by_head:
        lens = np.stack([lens, lens[::-1] + 5], 1)
    pool = Pool(hk, lens, page, g, by_head, layout)
    q = queries((4, 6, n, d), dtype, g)
    out = torch.full_like(q, 9.0)
    f = None if fresh is None else torch.tensor(fresh, dtype=torch.int32, device=DEV)
    hk.attn_pages(q, pool.cache, 0.2, out, causal=True, fresh=f)
    check_attention(pool, q, out, float(np.float32(0.2)), True, fresh)
    out.fill_(9.0)
    hk.attn_pages(q, pool.cache, 0.2, out, fresh=f)
    check_attention(pool, q, out, float(np.float32(0.2)), False, fresh)
    hk.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d, page, by_head", [(64, 16, False), (128, 64, False), (128, 32, True)])
@pytest.mark.parametrize("n, group", [(1, 1), (1, 8), (5, 3), (40, 1), (60, 2)])
def test_shared_rows(contexts, dtype, d, page, by_head, n, group):
    hk = contexts(2, d, dtype, shared=0)
    g = torch.Generator(DEV).manual_seed(n + group)
    # groups of four and two, the rest alone; shared rows that end inside a page, an element shorter than what it shares
    lens = np.array([700, 513, 600, 530, 90, 200, 333, 64]) + n
    shared = [(0, 4, 512), (6, 2, 48)]
    pool = Pool(hk, np.stack([lens, lens + 3], 1) if by_head else lens, page, g, by_head, shared=shared)
    q = queries((8, 2 * group, n, d), dtype, g)
    for groups in (shared, [(0, 4, 501), (6, 2, 17)], [(0, 2, 512), (2, 2, 512), (6, 1, 20)], [(0, 4, 1)], []):
        for causal in (False, True):
            out = torch.full_like(q, 9.0)
            hk.attn_pages(q, pool.cache, d ** -0.5, out, causal=causal, shared=groups)
            check_attention(pool, q, out, float(np.float32(d ** -0.5)), causal)
    short = np.array([700, 100, 600, 0, 90, 200, 333, 64])
    pool.lens = np.stack([short, short], 1) if by_head else short[:, None]
    pool.len.copy_(torch.from_numpy(pool.lens.reshape(-1).astype(np.int32)))
    out = torch.full_like(q, 9.0)
    hk.attn_pages(q, pool.cache, d ** -0.5, out, causal=True, shared=shared)
    check_attention(pool, q, out, float(np.float32(d ** -0.5)), True)
    hk.check()


@pytest.mark.parametrize("dtype, d, batch, group, prefix", [("bf16", 128, 24, 8, 4100), ("f32", 64, 10, 4, 3000), ("bf16", 64, 3, 1, 9000)])
def test_long_shared_prefix(contexts, dtype, d, batch, group, prefix):
    """Many queries of many elements over one prefix, cut into chunks, and ragged rows of their own."""
    hk = contexts(2, d, dtype, shared=0)
    g = torch.Generator(DEV).manual_seed(batch)
    lens = prefix + (np.arange(batch) * 37) % 400
    pool = Pool(hk, lens, 64, g, shared=[(0, batch, prefix // 64 * 64)])
    q = queries((batch, 2 * group, 1, d), dtype, g)
    out = torch.full_like(q, 9.0)
    hk.attn_pages(q, pool.cache, d ** -0.5, out, shared=[(0, batch, prefix // 64 * 64)])
    check_attention(pool, q, out, float(np.float32(d ** -0.5)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("by_head", [False, True])
@pytest.mark.parametrize("n, n_groups", [(1, 3), (1, 40), (40, 40)])
def test_many_sequences_and_groups(contexts, dtype, by_head, n, n_groups):
    """More sequences than a wave keeps the blocks of, more groups than it looks through one by one, a few long caches that are cut."""
    batch = 300
    hk = contexts(2, 64, dtype, units=2 * batch, shared=0)
    g = torch.Generator(DEV).manual_seed(n_groups)
    lens = 70 + (np.arange(batch) * 29) % 60
    lens[[7, 150, 260, 299]] = (2900, 1777, 3100, 2500)
    shared = [(7 * i + 1, 5, 64 if i % 3 else 48) for i in range(n_groups)]
    pool = Pool(hk, np.stack([lens, lens[::-1]], 1) if by_head else lens, 16, g, by_head, shared=shared)
    q = queries((batch, 4, n, 64), dtype, g)
    for groups in (shared, None):
        out = torch.full_like(q, 9.0)
        hk.attn_pages(q, pool.cache, 0.125, out, causal=True, shared=groups)
        check_attention(pool, q, out, 0.125, True)
    hk.check()


@pytest.mark.parametrize("d, n, longest", [(64, 65, 300), (128, 65, 300), (128, 130, 2500), (64, 100, 2500)])
def test_more_queries_than_the_device_holds_at_once(contexts, d, n, longest):
    """Queries of so many caches that they are taken in the largest tiles, whole and cut; a value that is no number reaches the queries behind it only."""
    batch, heads = 66, 8
    hk = contexts(heads, d, "bf16", units=batch * heads)
    g = torch.Generator(DEV).manual_seed(n)
    lens = n + (np.arange(batch) * 37) % 150
    lens[[5, 40]] = (longest, n // 2)
    fresh = np.full(batch, n)
    fresh[::7] = np.arange(len(fresh[::7])) * 6 % (n + 1)
    pool = Pool(hk, lens, 32, g)
    q = queries((batch, heads, n, d), "bf16", g)
    f = torch.from_numpy(fresh.astype(np.int32)).to(DEV)
    fine = torch.full_like(q, 9.0)
    hk.attn_pages(q, pool.cache, 0.1, fine, causal=True, fresh=f)
    check_attention(pool, q, fine, float(np.float32(0.1)), True, fresh)
    out = torch.full_like(q, 9.0)
    hk.attn_pages(q, pool.cache, 0.1, out)
    check_attention(pool, q, out, float(np.float32(0.1)))
    places = [pool.where(b, 3, int(lens[b]) - n + 30, int(lens[b]) - n + 31) for b in (5, 9)]   # new row 30 of each
    values = [pool.v[p].clone() for p in places]
    for page, at, head in places:
        pool.v[page, at, head, 7] = float("nan")
    out.fill_(9.0)
    hk.attn_pages(q, pool.cache, 0.1, out, causal=True, fresh=f)
    same = torch.ones_like(out, dtype=torch.bool)
    for b in (5, 9):
        same[b, 3, :, 7] = False
        assert fresh[b] == n and torch.isnan(out[b, 3, 30:, 7]).all()
        out[b, 3, 30:, 7] = fine[b, 3, 30:, 7]
    assert torch.equal(out[same], fine[same])
    for p, v in zip(places, values):
        pool.v[p] = v
    check_attention(pool, q, out, float(np.float32(0.1)), True, fresh)   # queries in front of it: summed again in float32, so within the roundings
    hk.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 40])
def test_largest_pages(contexts, dtype, n):
    hk = contexts(2, 64, dtype)
    g = torch.Generator(DEV).manual_seed(n)
    pool = Pool(hk, [65536 + 300, 41], 65536, g)
    q = queries((2, 4, n, 64), dtype, g)
    out = torch.full_like(q, 9.0)
    hk.attn_pages(q, pool.cache, 0.125, out, causal=True)
    check_attention(pool, q, out, 0.125, True)
    hk.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_few_queries_over_one_long_cache(contexts, dtype, d):
    hk = contexts(1, d, dtype)
    g = torch.Generator(DEV).manual_seed(d)
    pool = Pool(hk, [70001], 64, g)
    for n, causal in ((1, False), (5, True)):
        q = queries((1, 1, n, d), dtype, g)
        out = torch.full_like(q, 9.0)
        hk.attn_pages(q, pool.cache, d ** -0.5, out, causal=causal)
        check_attention(pool, q, out, float(np.float32(d ** -0.5)), causal)


@pytest.mark.parametrize("dtype, d, n, group", [("bf16", 128, 1000, 2), ("bf16", 64, 777, 1), ("f32", 128, 400, 1)])
def test_long_causal_prompts(contexts, dtype, d, n, group):
    hk = contexts(2, d, dtype)
    g = torch.Generator(DEV).manual_seed(n)
    pool = Pool(hk, [n, n + 1777], 64, g)
    q = queries((2, 2 * group, n, d), dtype, g)
    out = torch.full_like(q, 9.0)
    hk.attn_pages(q, pool.cache, d ** -0.5, out, causal=True)
    check_attention(pool, q, out, float(np.float32(d ** -0.5)), True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n, old, shared", [(9, 40, 0), (150, 40, 0), (9, 3000, 0), (150, 3000, 0), (150, 2000, 1008)])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_what_is_not_seen_does_not_matter(contexts, dtype, d, n, old, shared, value):
    """A new row that is no number reaches the queries from it on, and none before; in a whole result and in the parts of a cut one."""
    hk = contexts(2, d, dtype, shared=0)
    g = torch.Generator(DEV).manual_seed(n)
    groups = [(0, 2, shared)] if shared else []
    pool = Pool(hk, [n + old + 60, n + old], 16, g, shared=groups)
    at = n // 2 + 1
    clean = queries((2, 2, n, d), dtype, g)
    fine = torch.full_like(clean, 9.0)
    hk.attn_pages(clean, pool.cache, 0.1, fine, causal=True, shared=groups)
    page, row, head = pool.where(1, 1, old + at, old + at + 1)
    old = pool.v[page, row, head].clone()
    pool.v[page, row, head, 5] = value
    out = torch.full_like(clean, 9.0)
    hk.attn_pages(clean, pool.cache, 0.1, out, causal=True, shared=groups)
    same = torch.ones_like(out, dtype=torch.bool)
    same[1, 1, :, 5] = False
    assert torch.equal(out[same], fine[same]), (out[same] != fine[same]).sum()
    hit = out[1, 1, at:, 5].clone()
    assert torch.isnan(hit).all() if np.isnan(value) else (hit == value).all(), hit
    pool.v[page, row, head] = old
    out[1, 1, at:, 5] = fine[1, 1, at:, 5]
    check_attention(pool, clean, out, float(np.float32(0.1)), True)
    pool.k[page, row, head, 5] = value            # a score that is no number, or infinite
    hk.attn_pages(clean, pool.cache, 0.1, out, causal=True, shared=groups)
    same[1, 1, :, 5] = True
    same[1, 1, at:] = False
    assert torch.equal(out[same], fine[same])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_of_minus_infinity_are_not_an_empty_row(contexts, dtype):
    """All keys of a query at minus infinity: softmax has no value; a query that sees no key gives zeros."""
    hk = contexts(1, 64, dtype)
    g = torch.Generator(DEV).manual_seed(1)
    pool = Pool(hk, [5, 0], 16, g)
    at = pool.where(0, 0, 0, 5)
    pool.k[at] = 1.0
    pool.k[at[0], at[1], at[2], 0] = -float("inf")
    q = torch.ones((2, 1, 1, 64), dtype=TYPES[dtype], device=DEV)
    out = torch.full_like(q, 9.0)
    hk.attn_pages(q, pool.cache, 0.1, out)
    assert torch.isnan(out[0]).all() and (out[1] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n, length", [(1, 200), (40, 200), (1, 5000), (40, 5000)])
def test_pages_and_lengths_that_are_none(contexts, dtype, n, length):
    """Rows in a page that is none are left out, lengths are brought into range, and both are reported once."""
    hk = contexts(2, 128, dtype)
    g = torch.Generator(DEV).manual_seed(3)
    pool = Pool(hk, [300, length], 32, g)
    hole = Pool(hk, [300, length - 32], 32, g)   # the second sequence of `pool` without its page 2
    for h in range(2):
        for m, o in ((pool.k, hole.k), (pool.v, hole.v)):
            rows = m[pool.where(1, h, 0, length)]
            o[hole.where(1, h, 0, length - 32)] = torch.cat([rows[:64], rows[96:]])
    q = queries((2, 4, n, 128), dtype, g)
    for bad in (-1, pool.n_pages, 1 << 30):
        pool.table[1, 2] = bad
        out = torch.full_like(q, 9.0)
        hk.attn_pages(q, pool.cache, 0.1, out)
        torch.cuda.synchronize()
        with pytest.raises(HackError) as e:
            hk.check()
        assert e.value.status == -1
        hk.check()
        hole_q = torch.full_like(q, 9.0)
        hk.attn_pages(q, hole.cache, 0.1, hole_q)
        half = HALF_STEP[dtype]
        assert torch.allclose(out[1].double(), hole_q[1].double(), rtol=8 * half, atol=16 * half)
    pool.table[1, 2] = int(pool.np_table[1, 0, 2])
    pool.len[0] = -5
    pool.len[1] = 1 << 30                        # taken as max_len, whose last pages are no pages either
    out = torch.full_like(q, 9.0)
    hk.attn_pages(q, pool.cache, 0.1, out)
    torch.cuda.synchronize()
    with pytest.raises(HackError):
        hk.check()
    assert (out[0] == 0).all()
    pool.len.copy_(torch.tensor([300, length]))
    for fresh in ([n + 1, n], [n, -1]):
        hk.attn_pages(q, pool.cache, 0.1, out, fresh=torch.tensor(fresh, dtype=torch.int32, device=DEV))
        torch.cuda.synchronize()
        with pytest.raises(HackError):
            hk.check()
    pool.len.copy_(torch.tensor([300, length]))
    hk.attn_pages(q, pool.cache, 0.1, out)
    check_attention(pool, q, out, float(np.float32(0.1)))
    hk.check()


def test_rows_beyond_four_gigabytes(contexts):
    hk = contexts(1, 128, "bf16")
    g = torch.Generator(DEV).manual_seed(5)
    pages, page = 300000, 64                     # 4.9 GB of K, and of V
    k, v = (torch.empty((pages, page, 1, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    where = torch.tensor([[pages - 1, 3, 270000]], dtype=torch.int32, device=DEV)
    n = 150
    rows = [torch.randn((1, 1, n, 128), generator=g, device=DEV).bfloat16() for _ in range(2)]
    cache = PagedCache(k, v, where, torch.tensor([n], dtype=torch.int32, device=DEV))
    hk.append_pages(rows[0], rows[1], cache)
    for m, r in ((k, rows[0]), (v, rows[1])):
        assert torch.equal(torch.cat([m[p, :, 0] for p in where[0].tolist()])[:n], r[0, 0])
    q = queries((1, 2, 1, 128), "bf16", g)
    out, want = torch.empty_like(q), torch.empty_like(q)
    hk.attn_pages(q, cache, 0.1, out)
    small = PagedCache(k[where[0].long()], v[where[0].long()], torch.tensor([[0, 1, 2]], dtype=torch.int32, device=DEV), cache.len)
    hk.attn_pages(q, small, 0.1, want)
    assert torch.equal(out, want)
    del k, v, cache
    torch.cuda.empty_cache()


# ---- appending ----------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d, rot, axes, layout", [(128, 128, 1, "half"), (64, 64, 1, "interleaved"), (64, 32, 2, "half"), (128, 96, 1, "half"), (128, 32, 2, "interleaved")])
@pytest.mark.parametrize("norm", [None, "rms", "l2"])
@pytest.mark.parametrize("pages, by_head", [("rows", False), ("heads", False), ("turns", True)])
def test_append(contexts, dtype, d, rot, axes, layout, norm, pages, by_head):
    g = torch.Generator(DEV).manual_seed(rot)
    rng = np.random.default_rng(rot)
    for i, ((B, hq, hkv, N), how, page) in enumerate((((1, 1, 1, 1), "plain", 16), ((5, 8, 2, 1), "projection", 64), ((2, 6, 3, 33), "part", 32),
                                                      ((3, 4, 4, 130), "projection", 16))):
        hk = contexts(hkv, d, dtype)
        fresh = rng.integers(0, N + 1, B) if i >= 2 else None
        f = np.full(B, N) if fresh is None else fresh
        old = rng.integers(0, 90, (B, hkv if by_head else 1))
        if i == 2:
            old[0] = -5                          # fewer rows than new ones: the first ones have no place
        lens = np.maximum(old + f[:, None], 0)
        pool = Pool(hk, lens if by_head else lens[:, 0], page, g, by_head, pages)
        q, k, v = (rows_in((B, h, N, d), how, dtype, g) for h in (hq, hkv, hkv))
        qw = None if norm is None or i == 0 else 1 + torch.randn((d,) if i == 1 else (hq, d), generator=g, device=DEV) / 3
        kw = None if norm is None or i == 2 else 1 + torch.randn((hkv, d) if i == 1 else (d,), generator=g, device=DEV) / 3
        own = axes == 1 and not by_head
        first = lens - f[:, None]
        pos = np.repeat(rng.integers(-9, 1 << 17, (B, axes, 1)) + np.arange(N), 1, 0) if not own else first[:, :1, None] + np.arange(N)
        pos = pos.astype(np.int32)
        rope = Rope.scaled(rot, axes, layout, "linear", factor=3.0)
        q_out = torch.full((B, hq, N, d), 9.0, dtype=TYPES[dtype], device=DEV)
        before = [pool.k.clone(), pool.v.clone()]
        wrote = torch.zeros(pool.k.shape[:3], dtype=torch.bool, device=DEV)
        hk.append_pages(k, v, pool.cache, rope=rope, pos=None if own else torch.from_numpy(pos).to(DEV),
                        fresh=None if fresh is None else torch.from_numpy(fresh.astype(np.int32)).to(DEV), q=q, q_out=q_out, norm=norm, eps=1e-5, q_weight=qw,
                        k_weight=kw)
        eps, results = float(np.float32(1e-5)), []
        for x, w in ((q, qw), (k, kw)):
            y = to64(x)
            ss = (y * y).sum(-1, keepdims=True)
            if norm:
                y = y / np.sqrt(ss / d + eps) if norm == "rms" else y / np.maximum(np.sqrt(ss), eps)
            if w is not None:
                y = y * to64(w if w.dim() == 1 else w[:, None])
            results.append(turned(y, pos, rope.freq, 1.0, rot, axes, layout))
        roundings = ROTATION + (NORM if norm else 0)
        for b in range(B):
            n = int(f[b])
            check_rows(q_out[b, :, :n], results[0][0][b, :, :n], results[0][1][b, :, :n], dtype, roundings)
            assert (q_out[b, :, n:] == 9.0).all()
            for h in range(hkv):
                lo = int(first[b, h if by_head else 0])
                skip = max(0, -lo)
                at = pool.where(b, h, lo + skip, lo + n)
                wrote[at] = True
                check_rows(pool.k[at], results[1][0][b, h, skip:n], results[1][1][b, h, skip:n], dtype, roundings)
                assert torch.equal(pool.v[at], v[b, h, skip:n])
        for m, o in zip((pool.k, pool.v), before):
            assert torch.equal(m[~wrote].nan_to_num(7.0), o[~wrote].nan_to_num(7.0))
        # without queries, and the keys alone as the rotation writes them
        pool.k.copy_(before[0])
        pool.v.copy_(before[1])
        hk.append_pages(k, v, pool.cache)
        if fresh is None:
            for b in range(B):
                for h in range(hkv):
                    lo = int(first[b, h if by_head else 0])
                    assert torch.equal(pool.k[pool.where(b, h, lo, lo + N)], k[b, h]) and torch.equal(pool.v[pool.where(b, h, lo, lo + N)], v[b, h])
        torch.cuda.synchronize()
        hk.check()


def test_append_is_the_rotation_of_the_same_rows(contexts):
    """Bit for bit what norm_rotate writes, small outputs and ones beyond 32 MB."""
    for B, N in ((2, 50), (3, 6000)):
        hk = contexts(8, 128, "bf16", queries=8192)
        g = torch.Generator(DEV).manual_seed(N)
        proj = torch.randn((B, N, 32, 128), generator=g, device=DEV).bfloat16().transpose(1, 2)
        q, k, v = proj[:, :16], proj[:, 16:24], proj[:, 24:]
        rope = Rope.scaled(128, scaling="base", factor=2.0)
        pos = torch.arange(N, dtype=torch.int32, device=DEV)
        qo, ko, qo2 = (torch.empty((B, h, N, 128), dtype=torch.bfloat16, device=DEV) for h in (16, 8, 16))
        hk.norm_rotate(q, k, "rms", 1e-6, None, None, rope, qo, ko, pos=pos)
        pool = Pool(hk, np.full(B, N), 64, g)
        hk.append_pages(k, v, pool.cache, rope=rope, q=q, q_out=qo2, norm="rms")
        assert torch.equal(qo, qo2)
        for b in range(B):
            for h in range(8):
                at = pool.where(b, h, 0, N)
                assert torch.equal(pool.k[at], ko[b, h]) and torch.equal(pool.v[at], v[b, h])


def test_append_to_pages_that_are_none(contexts):
    hk = contexts(2, 64, "bf16")
    g = torch.Generator(DEV).manual_seed(2)
    pool = Pool(hk, [100, 70], 16, g)
    before = [pool.k.clone(), pool.v.clone()]
    pool.table[0, 5] = pool.n_pages
    pool.table[1, 4] = -3
    pool.len[1] = 1 << 20                        # out of range: nothing of it is stored
    k, v = (torch.randn((2, 2, 40, 64), generator=g, device=DEV).bfloat16() for _ in range(2))
    hk.append_pages(k, v, pool.cache)
    torch.cuda.synchronize()
    with pytest.raises(HackError):
        hk.check()
    hk.check()
    for m, o, x in ((pool.k, before[0], k), (pool.v, before[1], v)):
        want = o.clone()
        for h in range(2):
            at = pool.where(0, h, 60, 100)
            keep = torch.from_numpy(np.arange(60, 100) // 16 != 5).to(DEV)
            want[at[0][keep], at[1][keep], at[2][keep]] = x[0, h][keep]
        assert torch.equal(m.nan_to_num(7.0), want.nan_to_num(7.0))
    # numbers of new rows
    pool.table[0, 5] = int(pool.np_table[0, 0, 5])
    pool.len.copy_(torch.tensor([100, 70]))
    before = [pool.k.clone(), pool.v.clone()]
    for fresh in ([41, -1], [-1, 1 << 30]):
        hk.append_pages(2 * k, 2 * v, pool.cache, fresh=torch.tensor(fresh, dtype=torch.int32, device=DEV))
        torch.cuda.synchronize()
        with pytest.raises(HackError):
            hk.check()
        for m, o in zip((pool.k, pool.v), before):
            assert torch.equal(m.nan_to_num(7.0), o.nan_to_num(7.0))


def test_views(contexts):
    """Tables with rows apart, a bound on lengths, queries in place, heads of a wider pool, another stream."""
    hk = contexts(2, 64, "bf16")
    g = torch.Generator(DEV).manual_seed(6)
    pool = Pool(hk, [90, 300, 7], 16, g)
    q = queries((3, 4, 5, 64), "bf16", g)
    want, out = torch.empty_like(q), torch.empty_like(q)
    hk.attn_pages(q, pool.cache, 0.1, want, causal=True)
    wide = torch.full((3, 50), -1, dtype=torch.int32, device=DEV)
    wide[:, 3:3 + pool.table.shape[1]] = pool.table
    for table, most in ((wide[:, 3:3 + pool.table.shape[1]], 0), (wide[:, 3:22], 300), (wide[:, 3:22], 304)):
        cache = PagedCache(pool.k, pool.v, table, pool.len, most)
        hk.attn_pages(q, cache, 0.1, out, causal=True)
        assert torch.equal(out, want)
    cache = PagedCache(pool.k, pool.v, wide[:, 3:21], pool.len)      # 288 rows: one length is out of range
    hk.attn_pages(q, cache, 0.1, out, causal=True)
    torch.cuda.synchronize()
    with pytest.raises(HackError):
        hk.check()
    assert torch.equal(out[::2], want[::2])
    # two of four heads of a pool
    four = [torch.full((pool.n_pages, 16, 4, 64), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    four[0][:, :, 1:3], four[1][:, :, 1:3] = pool.k, pool.v
    hk.attn_pages(q, PagedCache(four[0][:, :, 1:3], four[1][:, :, 1:3], pool.table, pool.len), 0.1, out, causal=True)
    assert torch.equal(out, want)
    # queries turned in place
    rope = Rope.scaled(64)
    k, v = (torch.randn((3, 2, 5, 64), generator=g, device=DEV).bfloat16() for _ in range(2))
    x, y = q.clone(), torch.empty_like(q)
    hk.append_pages(k, v, pool.cache, rope=rope, q=q, q_out=y)
    hk.append_pages(k, v, pool.cache, rope=rope, q=x, q_out=x)
    assert torch.equal(x, y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        hk.attn_pages(q, pool.cache, 0.1, out, causal=True)
    side.synchronize()
    hk.attn_pages(q, pool.cache, 0.1, want, causal=True)
    assert torch.equal(out, want)
    hk.check()


# ---- a run of both, graphs, streams ---------------------------------------------
@pytest.mark.parametrize("dtype, d, prefix", [("bf16", 128, 0), ("bf16", 64, 160), ("f32", 64, 64)])
def test_serving_run(contexts, dtype, d, prefix):
    """A shared prefix, prompts of different lengths, then tokens: queries and keys of one projection, appended, then attended to; the tokens in a captured graph,
    whose lengths grow in device memory, with eager work between replays."""
    B, K, G, N, tokens = 3, 2, 2, 50, 40
    hk = contexts(K, d, dtype, shared=0)
    g = torch.Generator(DEV).manual_seed(d)
    fresh = np.array([50, 13, 31])
    pool = Pool(hk, prefix + fresh, 16, g, shared=[(0, B, prefix)] if prefix else (), extra=tokens)
    shared = [(0, B, prefix)] if prefix else None
    rope, scale = Rope.scaled(d), float(np.float32(d ** -0.5))

    def projection(n):
        x = torch.randn((B, n, (G + 2) * K, d), generator=g, device=DEV).to(TYPES[dtype]).transpose(1, 2)
        return x[:, :G * K], x[:, G * K:-K], x[:, -K:]

    def turn(x, first):
        pos = (first[:, None, None] + np.arange(x.shape[2])).astype(np.int32)
        out = torch.empty(x.shape, dtype=x.dtype, device=DEV)
        hk.rotate(x, rope, out, pos=torch.from_numpy(pos).to(DEV))
        return out
    q, k, v = projection(N)
    f = torch.from_numpy(fresh.astype(np.int32)).to(DEV)
    qo = torch.full((B, G * K, N, d), 9.0, dtype=q.dtype, device=DEV)
    out = torch.full_like(qo, 9.0)
    hk.append_pages(k, v, pool.cache, rope=rope, fresh=f, q=q, q_out=qo)
    hk.attn_pages(qo, pool.cache, d ** -0.5, out, causal=True, fresh=f, shared=shared)
    ko = turn(k, np.full(B, prefix))
    for b in range(B):
        for h in range(K):
            at = pool.where(b, h, prefix, prefix + int(fresh[b]))
            assert torch.equal(pool.k[at], ko[b, h, :fresh[b]]) and torch.equal(pool.v[at], v[b, h, :fresh[b]])
    check_attention(pool, qo, out, scale, True, fresh)
    # one token at a time; a graph of the step that makes room, appends and attends
    q, k, v = (x.contiguous() for x in projection(1))
    qo, out = (torch.empty((B, G * K, 1, d), dtype=q.dtype, device=DEV) for _ in range(2))

    def step():
        pool.len.add_(1)
        hk.append_pages(k, v, pool.cache, rope=rope, q=q, q_out=qo)
        hk.attn_pages(qo, pool.cache, d ** -0.5, out, causal=True, shared=shared)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    pool.lens = pool.lens + 1
    check_attention(pool, qo, out, scale, True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(6):
        for dst, src in zip((q, k, v), projection(1)):
            dst.copy_(src)
        before = pool.lens.copy()
        out.fill_(9.0)
        graph.replay()
        pool.lens = before + 1
        assert pool.len.tolist() == pool.lens.reshape(-1).tolist()
        ko = turn(k, before[:, 0])
        for b in range(B):
            for h in range(K):
                at = pool.where(b, h, int(before[b, 0]), int(before[b, 0]) + 1)
                assert torch.equal(pool.k[at][0], ko[b, h, 0]) and torch.equal(pool.v[at][0], v[b, h, 0])
        check_attention(pool, qo, out, scale, True)
        got = out.clone()
        eager = torch.full_like(out, -9.0)
        hk.attn_pages(qo, pool.cache, d ** -0.5, eager, causal=True, shared=shared)
        assert torch.equal(got, eager)
        torch.cuda.synchronize()
    hk.check()


def test_refusals_through_the_binding(contexts):
    hk = contexts(2, 64, "bf16")
    g = torch.Generator(DEV).manual_seed(1)
    pool = Pool(hk, [40, 9], 16, g)
    q = queries((2, 4, 1, 64), "bf16", g)
    out, k = torch.empty_like(q), torch.zeros((2, 2, 1, 64), dtype=torch.bfloat16, device=DEV)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    for bad in (dict(fresh=i32(1)), dict(fresh=i32(1, 1).long()), dict(shared=[(0, 2)]), dict(shared=[(0, 1, 1)] * 257), dict(fresh=i32(1, 1).cpu())):
        with pytest.raises(AssertionError):
            hk.attn_pages(q, pool.cache, 0.1, out, **bad)
    with pytest.raises(OverflowError):
        hk.attn_pages(q, pool.cache, 0.1, out, shared=[(0, 1, 1 << 40)])
    with pytest.raises(HackError):
        hk.attn_pages(q, pool.cache, 0.1, out, shared=[(1, 2, 16)])
    with pytest.raises(HackError):
        hk.attn_pages(q, pool.cache, -0.1, out)
    for x, y in ((q[:, :3].contiguous(), out), (q, out[:, :2].contiguous()), (q.float(), out), (q.transpose(0, 1), out), (q[:1], out[:1])):
        with pytest.raises(AssertionError):
            hk.attn_pages(x, pool.cache, 0.1, y)
    for a in ((k[:1], k), (k, k[:, :1]), (k.float(), k), (k.cpu(), k)):
        with pytest.raises((AssertionError, HackError)):
            hk.append_pages(*a, pool.cache)
    with pytest.raises(HackError):
        hk.append_pages(k, k, pool.cache, k_weight=torch.ones(64, device=DEV))
    with pytest.raises(KeyError):
        hk.append_pages(k, k, pool.cache, norm="layer")
    with pytest.raises(AttributeError):
        pool.cache.len = pool.len
    for bad in (dict(table=pool.table.long()), dict(length=pool.len[:1]), dict(k=pool.k[:, :, :, :32]), dict(v=pool.v.transpose(1, 2).contiguous().transpose(1, 2)),
                dict(max_len=-1), dict(k=pool.k.cpu())):
        args = dict(k=pool.k, v=pool.v, table=pool.table, length=pool.len)
        with pytest.raises(AssertionError):
            PagedCache(**{**args, **bad})
    hk.check()
