"""Pages behind the first 4 GiB of a cache's codes: copied, moved and attended to like those in front."""
import pytest
import torch

from paper_2604_03950_amd import binding as dma

pytestmark = pytest.mark.gpu
HKV, P, D, PAGES = 32, 256, 128, 4400               # pages of 1 MiB each in K and V


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.fixture(scope="module")
def large():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("16 GiB of memory are needed")
    table = torch.full((24, 40), -1, dtype=torch.int32, device="cuda")
    cache = dma.KVCache.empty(table, PAGES, HKV, D, P)
    assert cache.k_codes.numel() > 1 << 32
    return cache


def fill(cache, pages, seed):
    """Numbers of all kinds in these pages; returns their bytes."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    for t in (cache.k_codes, cache.v_codes):
        for p in pages:
            t[p] = torch.randint(0, 0x60, t.shape[1:], generator=g, device="cuda", dtype=torch.uint8) | torch.randint(0, 2, t.shape[1:], generator=g, device="cuda", dtype=torch.uint8) << 7
    for t in (cache.k_scales, cache.v_scales):
        t[pages] = torch.randint(112, 118, (len(pages), HKV), generator=g, device="cuda", dtype=torch.uint8)
    return held(cache, pages)


def held(cache, pages):
    return [torch.stack([t[p] for p in pages]) for t in (cache.k_codes, cache.v_codes, cache.k_scales, cache.v_scales)]


def equal(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_reserve(large):
    """A shared page and its copy, both far back."""
    large.page_table.fill_(-1)
    want = fill(large, [4301, 4388], 1)
    large.page_table[:2, 0] = 4301
    large.page_table[2, 0] = 4388
    refs = torch.ones(PAGES, dtype=torch.int32, device="cuda")
    refs[4301], refs[4399] = 2, 0
    missing = dma.dma_kv_reserve(large, refs, i32([100] + [-1] * 23), 1)
    assert not missing.any() and large.page_table[0, 0] == 4399 and refs[4301] == 1 and refs[4399] == 1
    assert equal(held(large, [4399, 4388]), want) and equal(held(large, [4301]), [x[:1] for x in want])


def test_compact(large):
    """Pages from the back to places in front of and behind the border."""
    large.page_table.fill_(-1)
    refs = torch.ones(PAGES, dtype=torch.int32, device="cuda")
    refs[[7, 4200]] = 0
    refs[4396:] = 0
    refs[[4396, 4398]] = i32([3, 1])
    want = fill(large, [4396, 4398], 2)
    large.page_table[:3, 1] = 4396
    large.page_table[5, 39] = 4398
    used, moved = dma.dma_kv_compact(large, refs)
    assert used.item() == PAGES - 4 and moved[[7, 4200, 4396, 4398, 4399]].tolist() == [-1, -1, 7, 4200, -1]
    assert large.page_table[:3, 1].tolist() == [7] * 3 and large.page_table[5, 39] == 4200
    assert refs[[7, 4200]].tolist() == [3, 1] and not refs[PAGES - 4:].any()
    assert equal(held(large, [7, 4200]), want)


@pytest.mark.parametrize("N", [1, 6])
def test_attention(large, N):
    """The same pages in a small cache: the same bits."""
    common, own = [4390, 4100, 4320], list(range(4340, 4364))
    small = dma.KVCache.empty(torch.full((24, 40), -1, dtype=torch.int32, device="cuda"), 30, HKV, D, P)
    fill(large, common + own, 3)
    for x, y in ((large.k_codes, small.k_codes), (large.v_codes, small.v_codes), (large.k_scales, small.k_scales), (large.v_scales, small.v_scales)):
        for k, p in enumerate(common + own):
            y[k] = x[p]
    for cache, name in ((large, lambda k: (common + own)[k]), (small, lambda k: k)):
        cache.page_table.copy_(i32([[name(0), name(1), name(2), name(3 + b)] + [-1] * 36 for b in range(24)]))
    assert dma.dma_cache_attn_shared_workspace_bytes(large, 128, N, 1) != dma.dma_cache_attn_workspace_bytes(large, 128, N)
    q = torch.randn((24, 128, N, D), generator=torch.Generator(device="cuda").manual_seed(4), device="cuda").to(torch.bfloat16)
    start = i32([3 * P + (37 * b) % (P - N) for b in range(24)])
    a, b = (dma.dma_cache_attn_shared(q, cache, start, i32([0, 24]), i32([3 * P])) for cache in (large, small))
    assert torch.isfinite(a.float()).all() and torch.equal(a, b)
    one = dma.dma_cache_attn(q, large, start).float()
    assert (a.float() - one).norm() <= 4 * 2.0**-8 * one.norm()             # two results and their probabilities, each rounded to bf16
