"""Caches in pages where rows hold values that are no numbers, pages are none or lengths are out of range: what reaches a query, what is stored, and that such a
call stays about as fast as another one.  Plain implementations in 64 bits; the tolerances are those of tests/test_gpu_pages.py."""
import numpy as np
import pytest
import torch

from paper_2504_09261_amd.binding import HackError, PagedCache, Rope
from tests.test_gpu_operators import DEV, H, HALF_STEP
from tests.test_gpu_pages import Pool, check_attention, contexts, queries  # noqa: F401

pytestmark = pytest.mark.gpu
INF = float("inf")


def scale_of(d):
    return float(np.float32(d ** -0.5))


def put(pool, b, h, row, col, value):
    """An element of V, in every sequence's page of that row; what was there."""
    at = pool.where(b, h, row, row + 1)
    old = pool.v[at].clone()
    pool.v[at[0], at[1], at[2], col] = value
    return lambda: pool.v.__setitem__(at, old)


def median_ms(call, times=5):
    ms = []
    for _ in range(times):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        call()
        b.record()
        torch.cuda.synchronize()
        ms.append(a.elapsed_time(b))
    return sorted(ms)[len(ms) // 2]


# ---- rows that all queries see, in blocks that end or begin with rows that none sees ----
@pytest.mark.parametrize("value", [INF, -INF])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [16, 40, 130])
@pytest.mark.parametrize("length, prefix", [(1, 0), (17, 0), (65, 0), (81, 0), (3009, 0), (3025, 0), (3025, 1009), (1100, 1025), (1057, 1041)])
def test_infinities_that_all_queries_see(contexts, value, d, n, length, prefix):  # noqa: F811
    """An infinity in a row that every query sees is the result's, not a NaN, wherever the row lies: at the end of a sequence or on either side of a shared prefix's
    end; the other elements stay as they are."""
    hk = contexts(2, d, "bf16", shared=0)
    g = torch.Generator(DEV).manual_seed(length + n)
    groups = [(0, 2, prefix)] if prefix else []
    lens = [length, length + 7 if prefix else length // 2 + 3]
    pool = Pool(hk, lens, 16, g, shared=groups)
    q = queries((2, 4, n, d), "bf16", g)
    fine, out = torch.full_like(q, 9.0), torch.full_like(q, 9.0)
    hk.attn_pages(q, pool.cache, d ** -0.5, fine, shared=groups)
    check_attention(pool, q, fine, scale_of(d))
    rows = sorted({r for r in (0, length - 1, (length - 1) // 16 * 16, (length - 1) // 32 * 32, prefix - 1, prefix) if 0 <= r < length})
    for i, r in enumerate(rows):                 # each in a column of its own
        for b in ((0, 1) if r < prefix else (0,)):
            put(pool, b, 1, r, 3 * i, value)
    hk.attn_pages(q, pool.cache, d ** -0.5, out, shared=groups)
    same = torch.ones_like(out, dtype=torch.bool)
    for i, r in enumerate(rows):
        for b in ((0, 1) if r < prefix else (0,)):
            assert (out[b, 2:, :, 3 * i] == value).all(), (b, r, out[b, 2:, :, 3 * i].unique())
            same[b, 2:, :, 3 * i] = False
    assert torch.equal(out[same], fine[same])
    hk.check()


# ---- rows behind a prompt ----
def nan_behind_a_prompt(contexts, d, heads, row):  # noqa: F811
    """A NaN in V reaches the queries that see its row and no other, and the call takes about as long as without it; four heads: in tiles of 64 queries, many: of 128."""
    n, length = 1000, 3000
    hk = contexts(heads, d, "bf16", units=128)
    g = torch.Generator(DEV).manual_seed(row)
    pool = Pool(hk, [length], 64, g)
    q = queries((1, heads, n, d), "bf16", g)
    fine, out = torch.full_like(q, 9.0), torch.full_like(q, 9.0)

    def call(to):
        hk.attn_pages(q, pool.cache, d ** -0.5, to, causal=True)
    call(fine)
    clean = median_ms(lambda: call(fine))
    back = put(pool, 0, 1, row, 5, float("nan"))
    call(out)
    strange = median_ms(lambda: call(out))
    same = torch.ones_like(out, dtype=torch.bool)
    same[0, 1, :, 5] = False
    assert torch.equal(out[same], fine[same])
    first = max(0, row - (length - n))           # the first query that sees it
    assert torch.isnan(out[0, 1, first:, 5]).all()
    out[0, 1, first:, 5] = fine[0, 1, first:, 5]
    back()
    check_attention(pool, q, out, scale_of(d), True)
    hk.check()
    assert strange < 8 * clean + 0.3, (clean, strange)


HEADS = pytest.mark.parametrize("d, heads", [(64, 4), (128, 4), (64, 72), (128, 40)])


@HEADS
def test_a_nan_that_all_queries_see(contexts, d, heads):  # noqa: F811
    nan_behind_a_prompt(contexts, d, heads, 0)


# ---- rows that are masked for some queries ----
@HEADS
@pytest.mark.parametrize("row", [1999, 2500, 2999])
def test_a_nan_that_some_queries_see(contexts, d, heads, row):  # noqa: F811
    nan_behind_a_prompt(contexts, d, heads, row)


# ---- pages that are none ----
def check_without(pool, q, out, scale, causal, gone):
    """As check_attention, with rows that are left out: gone[b] is a list of rows of batch element b."""
    B, heads, N, d = q.shape
    G = heads // pool.heads
    for b in range(B):
        for h in range(pool.heads):
            k, v = pool.rows(b, h)
            n = k.shape[0]
            x, got = (t[b, h * G:(h + 1) * G].double().reshape(-1, d) for t in (q, out))
            sees = (n - N + 1 + torch.arange(N, device=DEV) if causal else torch.full((N,), n, device=DEV)).repeat(G)[:, None]
            hidden = torch.arange(n, device=DEV) >= sees
            hidden[:, torch.tensor(gone[b], dtype=torch.int64, device=DEV)] = True
            p = torch.softmax((x @ k.T.contiguous() * scale).masked_fill(hidden, -INF), -1)
            size = torch.where(hidden, 0.0, x.abs() @ k.abs().T.contiguous()).amax(-1, keepdim=True)
            want = p @ v
            tol = (2 * 2.0 ** -8 + 2 * scale * (d + 4) * H * size + 1e-5) * (p @ v.abs()) * 1.01 + HALF_STEP["bf16"] * 1.01 * want.abs() + 2.0 ** -111 * (1 + v.abs().sum(0))
            err = (got - want).abs()
            assert (err <= tol).all(), (b, h, float((err / tol).max()))


@HEADS
@pytest.mark.parametrize("page", [0, 20, 46])
def test_prompt_over_a_page_that_is_none(contexts, d, heads, page):  # noqa: F811
    """Its rows are left out, the other elements of the batch are as they were, and the call takes about as long as another one."""
    n, lens = 500, [3000, 1300]
    hk = contexts(heads, d, "bf16", units=144)
    g = torch.Generator(DEV).manual_seed(page)
    pool = Pool(hk, lens, 64, g)
    q = queries((2, heads, n, d), "bf16", g)
    fine, out = torch.full_like(q, 9.0), torch.full_like(q, 9.0)

    def call(to):
        hk.attn_pages(q, pool.cache, d ** -0.5, to, causal=True)
    call(fine)
    clean = median_ms(lambda: call(fine))
    rows = [list(range(64 * page, min(64 * page + 64, 3000))), []]
    pool.table[0, page] = pool.n_pages
    call(out)
    torch.cuda.synchronize()
    with pytest.raises(HackError):
        hk.check()
    check_without(pool, q, out, scale_of(d), True, rows)
    assert torch.equal(out[1], fine[1])

    def again():
        call(out)
        torch.cuda.synchronize()
        with pytest.raises(HackError):
            hk.check()
    assert median_ms(again) < 16 * clean + 0.5, clean
    hk.check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n, length", [(1, 1500), (16, 1500), (40, 1500), (130, 1500), (130, 40)])
def test_shared_pages_that_are_none(contexts, d, n, length):  # noqa: F811
    """A page of the shared rows, and one of an element's own."""
    prefix = 1024
    hk = contexts(2, d, "bf16", shared=0)
    g = torch.Generator(DEV).manual_seed(n)
    groups = [(0, 2, prefix)]
    pool = Pool(hk, [prefix + length, prefix + length + 9], 16, g, shared=groups)
    q = queries((2, 4, n, d), "bf16", g)
    out = torch.full_like(q, 9.0)
    pool.table[0, 5] = -1                        # rows that all read by the first element's table
    pool.table[1, prefix // 16 + 1] = 1 << 30
    hk.attn_pages(q, pool.cache, d ** -0.5, out, shared=groups)
    torch.cuda.synchronize()
    with pytest.raises(HackError):
        hk.check()
    common = list(range(80, 96))
    check_without(pool, q, out, scale_of(d), False, [common, common + list(range(prefix + 16, prefix + 32))])


# ---- appending with lengths or numbers of new rows that are out of range ----
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("given", [False, True])
def test_queries_of_sequences_out_of_range_are_left(contexts, dtype, given):  # noqa: F811
    """Appending stores nothing of such a sequence, its queries included, so a caller that turns them in place still has them."""
    hk = contexts(2, 64, dtype)
    g = torch.Generator(DEV).manual_seed(3)
    pool = Pool(hk, [100, 70, 90], 16, g)
    rope, n = Rope.scaled(64), 40
    q, k, v = (queries((3, h, n, 64), dtype, g, 1.0) for h in (4, 2, 2))
    pos = torch.arange(n, dtype=torch.int32, device=DEV) if given else None
    want = torch.full_like(q, 9.0)
    hk.append_pages(k, v, pool.cache, rope=rope, pos=pos, q=q, q_out=want, norm="rms")
    hk.check()
    for lens, fresh in (([100, 1 << 20, 90], None), ([100, -1, 90], None), ([100, 70, 90], [n, n + 1, n]), ([100, 70, 90], [n, -1, n])):
        pool.len.copy_(torch.tensor(lens))
        f = None if fresh is None else torch.tensor(fresh, dtype=torch.int32, device=DEV)
        before = [pool.k.clone(), pool.v.clone()]
        for in_place in (False, True):
            x = q.clone()
            out = x if in_place else torch.full_like(q, 9.0)
            hk.append_pages(k, v, pool.cache, rope=rope, pos=pos, fresh=f, q=x, q_out=out, norm="rms")
            torch.cuda.synchronize()
            with pytest.raises(HackError):
                hk.check()
            assert torch.equal(out[::2], want[::2])
            assert torch.equal(out[1], q[1]) if in_place else (out[1] == 9.0).all()
        for m, o in zip((pool.k, pool.v), before):
            assert torch.equal(m.nan_to_num(7.0), o.nan_to_num(7.0))
    hk.check()


# ---- groups whose partial results find no room ----
@pytest.mark.parametrize("dtype, d, batch, heads, group, n", [("bf16", 128, 64, 8, 4, 33), ("bf16", 64, 64, 8, 4, 33), ("f32", 64, 256, 8, 4, 1)])
def test_groups_without_room(contexts, dtype, d, batch, heads, group, n):  # noqa: F811
    """Every element reads the shared rows by itself then, and they are the same; half of the batch in a group finds room."""
    hk = contexts(heads, d, dtype, units=batch * heads, shared=0)
    g = torch.Generator(DEV).manual_seed(batch)
    prefix, lens = 64, 70 + n + (np.arange(batch) * 29) % 200
    pool = Pool(hk, lens, 16, g, shared=[(0, batch, prefix)])
    q = queries((batch, group * heads, n, d), dtype, g)
    for count in (batch, batch // 4):
        out = torch.full_like(q[:count], 9.0)
        cache = PagedCache(pool.k, pool.v, pool.table[:count], pool.len[:count])
        hk.attn_pages(q[:count], cache, 0.125, out, causal=True, shared=[(0, count, prefix)])
        check_attention(pool, q[:count], out, 0.125, True)
    hk.check()


# ---- float32 scores ----
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 16])
def test_small_products_beside_a_large_one(contexts, d, n):  # noqa: F811
    """A float32 score of 2^20 and d - 1 products of 3 2^-8, of which not even four reach half a step of 2^20 (2^-4): only those in the sum of a quarter that the large
    product is in are lost, (d / 4 - 1) 3 2^-8 of the score, and the three additions of the quarters round by 2^-4 at most.  Beside it a key whose score is 2^20, and whose
    value is 0: the result is the weight of the first one."""
    hk = contexts(1, d, "f32")
    g = torch.Generator(DEV).manual_seed(d)
    pool = Pool(hk, [2], 16, g)
    pool.k[pool.where(0, 0, 0, 2)] = 0.0
    page, row, head = pool.where(0, 0, 0, 2)
    pool.k[page[0], row[0], head[0]] = 3 * 2.0 ** -8
    pool.k[page, row, head, 0] = 2.0 ** 20
    pool.v[page, row, head] = torch.tensor([[1.0], [0.0]], device=DEV)
    q = torch.ones((1, 1, n, d), device=DEV)
    out = torch.full_like(q, 9.0)
    hk.attn_pages(q, pool.cache, 2.0, out)
    more, off = (d - 1) * 3 * 2.0 ** -8, (d / 4 - 1) * 3 * 2.0 ** -8 + 3 * 2.0 ** -4
    lo, hi = (1 / (1 + np.exp(-2.0 * x)) for x in (more - off, more + off))
    assert (out >= lo - 1e-5).all() and (out <= hi + 1e-5).all(), (float(out[0, 0, 0, 0]), lo, hi)
