"""A cache that compression left, with a length for every head, viewed as a cache in pages of one head: attended to, appended to and attended to again."""
import numpy as np
import pytest
import torch

from paper_2504_09261_amd.binding import Cache, PagedCache, Rope
from tests.test_gpu_operators import DEV, TYPES
from tests.test_gpu_pages import check_attention, contexts, queries  # noqa: F401

pytestmark = pytest.mark.gpu
PAGE = 16


class Units:
    """Rows of a compacted cache, as check_attention reads them."""

    by_head = True

    def __init__(self, cache, off, lens):
        self.cache, self.off, self.lens, self.heads = cache, off, lens, lens.shape[1]

    def rows(self, b, h):
        at, n = int(self.off[b, h]), int(self.lens[b, h])
        return self.cache.k[at:at + n].double(), self.cache.v[at:at + n].double()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_compacted_heads_as_pages(contexts, dtype, d):  # noqa: F811
    B, H, G, N, T = 2, 3, 2, 25, 304
    hk = contexts(H, d, dtype)
    g = torch.Generator(DEV).manual_seed(d)
    rng = np.random.default_rng(d)
    budget = np.array([[17, 300, 64], [1, 123, 32]])
    rand = lambda *shape: torch.randn(shape, generator=g, device=DEV).to(TYPES[dtype])  # noqa: E731
    full = Cache(rand(B * H * T, d), rand(B * H * T, d), np.arange(B * H) * T, np.full(B * H, T))
    kept = np.zeros((B * H, T), np.int32)
    for u, n in enumerate(budget.reshape(-1)):
        kept[u, :n] = np.sort(rng.permutation(T)[:n])
    # every unit has whole pages of 16 rows, with room for the new ones
    pages = -(-(budget + N) // PAGE)
    first = (np.cumsum(pages) - pages.reshape(-1)).reshape(B, H)
    rows = int(pages.sum()) * PAGE
    small = Cache(*(torch.full((rows, d), float("nan"), dtype=TYPES[dtype], device=DEV) for _ in range(2)), first.reshape(-1) * PAGE, budget.reshape(-1))
    hk.compact(B, 1, full, torch.from_numpy(kept).to(DEV), small, k_new=rand(B, H, 1, d), v_new=rand(B, H, 1, d))
    for u, n in enumerate(budget.reshape(-1)):
        at = int(small.off[u])
        assert torch.equal(small.k[at:at + n], full.k[T * u + torch.from_numpy(kept[u, :n]).long().to(DEV)])

    table = torch.zeros((B * H, int(pages.max())), dtype=torch.int32, device=DEV)
    for u, (p, n) in enumerate(zip(first.reshape(-1), pages.reshape(-1))):
        table[u, :n] = torch.arange(int(p), int(p + n), device=DEV)
    length = torch.from_numpy(budget.reshape(-1).astype(np.int32)).to(DEV)
    paged = PagedCache(small.k.view(-1, PAGE, 1, d), small.v.view(-1, PAGE, 1, d), table, length)
    q = queries((B, G * H, N, d), dtype, g)
    out = torch.full_like(q, 9.0)
    scale = float(np.float32(d ** -0.5))
    hk.attn_pages(q, paged, d ** -0.5, out)
    check_attention(Units(small, first * PAGE, budget), q, out, scale)
    own = torch.full_like(q[:, ::G], 9.0)
    hk.attn(q[:, ::G].contiguous(), small, d ** -0.5, own)     # the kernels over contiguous rows take a query head a cache
    check_attention(Units(small, first * PAGE, budget), q[:, ::G].contiguous(), own, scale)

    # a scale's new rows behind them, turned by their place in the image
    k, v = rand(B, H, N, d), rand(B, H, N, d)
    pos = torch.stack([torch.arange(N, device=DEV) // 5, torch.arange(N, device=DEV) % 5]).int()
    rope, turned = Rope.scaled(d, 2), torch.empty_like(k)
    length.add_(N)
    hk.append_pages(k, v, paged, rope=rope, pos=pos)
    hk.rotate(k, rope, turned, pos=pos)
    for b in range(B):
        for h in range(H):
            at = int(first[b, h]) * PAGE + int(budget[b, h])
            assert torch.equal(small.k[at:at + N], turned[b, h]) and torch.equal(small.v[at:at + N], v[b, h])
    for causal in (False, True):
        out.fill_(9.0)
        hk.attn_pages(q, paged, d ** -0.5, out, causal=causal)
        check_attention(Units(small, first * PAGE, budget + N), q, out, scale, causal)
    hk.check()
