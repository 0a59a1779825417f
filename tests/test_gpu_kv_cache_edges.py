"""The paged 8-bit key / value cache where its pages, scales and lengths end: scale bytes that nobody should see, pages that are missing
between others, writes into pages that hold nothing, NaN over all kinds of pages, infinities and large values, every key counted, batches of a
million."""
import numpy as np
import pytest
import torch

import kv_plain as plain
from kv_counts import channel, counts, wrong
from paper_2604_03950_amd import binding as dma
from test_gpu_kv_cache import FMT, Pair, bf16, i32, table_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def library():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dma.load()


def compare(pair, q, start, n=None, window=0, sinks=0):
    """Every row that exists against the definition, NaN for NaN; the others left as they were."""
    B, _, N, _ = q.shape
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    got = dma.dma_cache_attn(q.cuda(), pair.gpu, i32(start), i32(n), window=window, sink_tokens=sinks, out=out).double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        want, bound = pair.cpu.attn(q.double().numpy(), start, n, window, sinks)
    count = np.full(B, N) if n is None else np.clip(n, 0, N)
    exists = (np.arange(N) < np.where(np.asarray(start) < 0, 0, count)[:, None])[:, None, :, None] & np.ones(q.shape, bool)
    assert (got[~exists] == 7).all()
    np.testing.assert_array_equal(np.isnan(got[exists]), np.isnan(want[exists]))
    fine = exists & ~np.isnan(want)
    assert (np.abs(got - want)[fine] <= bound[fine]).all(), np.nanmax((np.abs(got - want) / bound)[fine])
    return want, exists


# ------------------------------------------------------------------------------- what lies where nothing has been written
# rows per kv head: 4, 25 and 48 (one and two tiles of the kernel for few rows), 160
ROWS = [(1, 4), (5, 5), (3, 16), (40, 4)]


@pytest.mark.parametrize("N,G", ROWS)
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("fmt,D,P", [("e4m3", 128, 16), ("e5m2", 64, 32), ("e4m3", 64, 64), ("e5m2", 128, 64), ("e4m3", 128, 256)])
def test_scales_that_nobody_should_see(fmt, D, P, wide, N, G):
    """The scale of every page that nothing was written to is 255, the byte of no number: page 0, which no table names and which entries
    without a page must not be mistaken for, pages handed out beyond the last token, and a page missing in the middle."""
    rng = np.random.default_rng(N + D + P)
    lens = [N, 3 * P, 2 * P + 63, 300, P + 40 if P < 256 else 300]
    used = [-(-n // P) for n in lens]
    order, at = 1 + rng.permutation(sum(used) + 3 * len(lens)), 0
    table = np.full((len(lens), max(used) + 3 + (2048 // P if wide else 0)), -1, np.int32)
    for b, u in enumerate(used):
        table[b, :u + 3] = order[at:at + u + 3]
        at += u + 3
    table[2, 1] = -1
    table[3, 300 // P - 1 if P < 256 else 0] = 1 << 30
    pair = Pair(rng, None, 2, P, D, fmt, table, 1 + len(order))
    pair.gpu.k_scales.fill_(255)
    pair.gpu.v_scales.fill_(255)
    S = max(lens)
    pair.write(bf16(rng, len(lens), 2, S, D), bf16(rng, len(lens), 2, S, D), [0] * len(lens), lens)
    q = bf16(rng, len(lens), 2 * G, N, D)
    for window, sinks in ((0, 0), (70, 5)):
        want, exists = compare(pair, q, np.array(lens) - N, None, window, sinks)
        assert not np.isnan(want[exists]).any()


@pytest.mark.parametrize("byte", [0, 16, 247, 255])
@pytest.mark.parametrize("fmt,P,D", [("e4m3", 16, 64), ("e5m2", 64, 128), ("e4m3", 256, 128)])
def test_written_from_the_middle(fmt, P, D, byte):
    """A first write that starts inside a page whose scale no write has left: the page holds nothing, and takes its scale from the new
    tokens alone; the next ones go on from there."""
    rng = np.random.default_rng(P + byte)
    pair = Pair(rng, [P + 9] * 3, 2, P, D, fmt)
    pair.gpu.k_scales.fill_(byte)
    pair.gpu.v_scales.fill_(byte)
    pair.cpu.ks[...] = pair.cpu.vs[...] = 0
    start = np.array([5, P - 1, 1])
    for n, size in ((3, 1.0), (1, 2.0 ** 9), (2, 2.0 ** -7)):
        pair.write(bf16(rng, 3, 2, n, D) * size, bf16(rng, 3, 2, n, D) / size, start)
        pair.same()
        start = start + n


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_empty_cache_holds_nothing(fmt):
    """A new cache's memory is that of tensors freed before it; its pages hold nothing all the same."""
    rng = np.random.default_rng(3)
    Hkv, P, D = 2, 32, 64
    table, pages = table_of(rng, [40, 40], P)
    for byte in (255, 200, 1):
        freed = [torch.full((pages, Hkv), byte, dtype=torch.uint8, device="cuda") for _ in range(8)]
        del freed
        cache = dma.KVCache.empty(torch.from_numpy(table).cuda(), pages, Hkv, D, P, FMT[fmt])
        k, v = bf16(rng, 2, Hkv, 4, D), bf16(rng, 2, Hkv, 4, D)
        dma.dma_kv_write(cache, k.cuda(), v.cuda(), i32([7, 20]))
        for b in range(2):
            for h in range(Hkv):
                assert int(cache.k_scales[table[b, 0], h]) == plain.needed(float(k[b, h].abs().max()), fmt)
                assert int(cache.v_scales[table[b, 0], h]) == plain.needed(float(v[b, h].abs().max()), fmt)


@pytest.mark.parametrize("N,G", ROWS)
@pytest.mark.parametrize("fmt,D,P", [("e4m3", 64, 16), ("e5m2", 128, 32), ("e4m3", 128, 64), ("e5m2", 64, 128), ("e4m3", 64, 256)])
def test_pages_missing_between_others(fmt, D, P, N, G):
    """Steps with a page and steps without, in any order, among them rows that see nothing at all."""
    rng = np.random.default_rng(N + P)
    lens, Hkv = [700, 700, 513, 700], 2
    wide = -(-700 // P)
    table = rng.permutation(4 * wide).reshape(4, wide).astype(np.int32)
    table[0, ::2] = -1
    table[1, 1:-1] = -1
    table[2, :] = -1                                            # nothing anywhere
    table[3, -2:] = 4 * wide
    pair = Pair(rng, None, Hkv, P, D, fmt, table, 4 * wide)
    pair.gpu.k_scales.fill_(255)
    pair.gpu.v_scales.fill_(255)
    pair.write(bf16(rng, 4, Hkv, 700, D), bf16(rng, 4, Hkv, 700, D), [0] * 4, lens)
    q = bf16(rng, 4, Hkv * G, N, D)
    for start in (np.array(lens) - N, np.array([0, P - 1, 2 * P, 333])):
        for window, sinks in ((0, 0), (90, 3)):
            want, exists = compare(pair, q, start, None, window, sinks)
            assert not want[2].any()


# ------------------------------------------------------------------------------------------------------ not a number
@pytest.mark.parametrize("window,sinks", [(0, 0), (2, 0), (70, 0), (20, 41)])
@pytest.mark.parametrize("B,Hkv,G,N", [(2, 1, 4, 3), (2, 1, 2, 20), (2, 2, 2, 100)])
@pytest.mark.parametrize("fmt,D,P", [("e4m3", 64, 16), ("e5m2", 128, 16), ("e5m2", 64, 32), ("e4m3", 128, 32), ("e4m3", 64, 64), ("e5m2", 128, 128), ("e5m2", 64, 256),
                                     ("e4m3", 128, 256)])
def test_nan_over_all_kinds_of_pages(fmt, D, P, B, Hkv, G, N, window, sinks):
    """A NaN key or value reaches the queries that see it, under a window and among the sinks too, and no others."""
    rng = np.random.default_rng(N + P + D)
    S = 300
    pair = Pair(rng, [S] * B, Hkv, P, D, fmt)
    k, v = bf16(rng, B, Hkv, S, D), bf16(rng, B, Hkv, S, D)
    nan = float("nan")
    v[0, 0, S - N + N // 2, 5] = v[0, 0, S - N + N // 2, D - 1] = v[0, 0, 40, 33] = nan
    v[1, 0, S - N - 1, 17] = v[1, 0, S - 1, 6] = nan
    k[1, Hkv - 1, S - max(N // 2, 1), 3] = nan
    pair.write(k, v, [0] * B)
    pair.same()
    want, exists = compare(pair, bf16(rng, B, Hkv * G, N, D), [S - N] * B, None, window, sinks)
    assert np.isnan(want).any() and not np.isnan(want).all()


@pytest.mark.parametrize("N,G", ROWS)
@pytest.mark.parametrize("P", [16, 64])
def test_infinities_of_others(P, N, G):
    """E5M2 codes of infinities, which no write leaves: not finite in the channels of the rows that see one, nothing for the rest."""
    rng = np.random.default_rng(N + P)
    S, D = 200, 64
    pair = Pair(rng, [S, S], 1, P, D, "e5m2")
    pair.write(bf16(rng, 2, 1, S, D), bf16(rng, 2, 1, S, D), [0, 0])
    for b, t, d, code in ((0, S - N + N // 2, 5, 0x7c), (0, 60, 9, 0xfc), (1, S - 1, 63, 0xfc)):
        page, u = pair.cpu.place(b, t)
        pair.cpu.v[page, 0, d, u] = code
        pair.gpu.v_codes[page, 0, d, u] = code
    q = bf16(rng, 2, G, N, D)
    for window in (0, 30):
        got = dma.dma_cache_attn(q.cuda(), pair.gpu, i32([S - N] * 2), window=window).double().cpu().numpy()
        with np.errstate(invalid="ignore"):
            want, bound = pair.cpu.attn(q.double().numpy(), [S - N] * 2, None, window)
        fine = np.isfinite(want)                                # the definition's table has NaN for an infinity
        np.testing.assert_array_equal(np.isfinite(got), fine)
        assert not fine.all() and (np.abs(got - want) <= bound)[fine].all()


# ------------------------------------------------------------------------------------------------------- every key once
# few rows with eight waves and with four, in one tile and in two; many rows in pieces and whole; B, Hkv, G, N, the longest
SHAPES = [(1, 2, 4, 1, 4000), (40, 4, 2, 1, 3000), (1, 2, 8, 4, 4000), (2, 2, 5, 12, 2000), (70, 4, 8, 3, 2500), (1, 2, 4, 40, 4000), (70, 4, 2, 70, 1500),
          (3, 2, 4, 1, 1200)]


def counting_cache(rng, lens, Hkv, P, D, fmt, wide=0):
    """Values of one in one channel of every position, kv heads by turns in either pattern."""
    table, pages = table_of(rng, lens, P)
    if wide:
        big = torch.full((len(lens), wide), -1, dtype=torch.int32, device="cuda")
        big[:, :table.shape[1]] = torch.from_numpy(table).cuda()
    cache = dma.KVCache.empty(big if wide else torch.from_numpy(table).cuda(), pages, Hkv, D, P, FMT[fmt])
    S = max(lens)
    t = torch.arange(S, device="cuda")
    v = torch.zeros((1, Hkv, S, D), dtype=torch.bfloat16, device="cuda")
    for h in range(Hkv):
        v[0, h, t, channel(t, D, h & 1)] = 1
    k = torch.randn((1, Hkv, S, D), device="cuda").to(torch.bfloat16)
    dma.dma_kv_write(cache, k.expand(len(lens), -1, -1, -1), v.expand(len(lens), -1, -1, -1), i32([0] * len(lens)), i32(lens))
    return cache


def count_all(cache, G, N, start, window, sinks):
    B, Hkv, D = cache.B, cache.Hkv, cache.D
    q = torch.zeros((B, Hkv * G, N, D), dtype=torch.bfloat16, device="cuda")
    got = dma.dma_cache_attn(q, cache, i32(start), window=window, sink_tokens=sinks)
    got = got.view(B, Hkv // 2, 2, G, N, D)
    assert (got == got[:, :1, :, :1]).all()                     # heads of a pattern are alike
    got = got[:, 0, :, 0].double().cpu().numpy()                # [B, 2, N, D]
    for b in range(B):
        for i in range(N):
            count, n = counts(D, int(start[b]) + i, window, sinks)
            assert not wrong(got[b, :, i], count, n).any(), (b, i, int(start[b]) + i)


@pytest.mark.parametrize("window,sinks", [(0, 0), (700, 70), (1300, 5)])
@pytest.mark.parametrize("fmt,D,P", [("e4m3", 128, 64), ("e5m2", 64, 16), ("e4m3", 64, 256), ("e5m2", 128, 32)])
@pytest.mark.parametrize("B,Hkv,G,N,longest", SHAPES)
def test_every_key_counts_once(B, Hkv, G, N, longest, fmt, D, P, window, sinks):
    rng = np.random.default_rng(B + N + P + window)
    lens = np.concatenate([[longest, 1300 if longest > 1300 else N, 1281 if longest > 1300 else 65, longest - 63][:B], rng.integers(N, longest, max(B - 4, 0))])
    lens = np.maximum(lens, N)
    cache = counting_cache(rng, list(lens), Hkv, P, D, fmt)
    count_all(cache, G, N, lens - N, window, sinks)


@pytest.mark.parametrize("N", [1, 12])
def test_every_key_counts_once_in_a_line_of_coarse_units(N):
    """More than 2^31 steps by the sizes alone: the line of steps is cut in units of several."""
    rng = np.random.default_rng(N)
    lens = list(rng.integers(N, 3000, 64))
    cache = counting_cache(rng, lens, 2, 256, 128, "e4m3", wide=(1 << 22) - 1)
    count_all(cache, 2, N, np.array(lens) - N, 0, 0)


# --------------------------------------------------------------------------------------------------------- magnitudes
@pytest.mark.parametrize("N,G", ROWS)
def test_large_values(N, G):
    """Values up to 2^121 / (512 + 64), the largest whose sums are said to stay in binary32, with scores that rise from key to key so that
    the running maximum stays behind."""
    rng = np.random.default_rng(N)
    S, D = 512, 64
    pair = Pair(rng, [S], 1, 64, D, "e4m3")
    k, v = bf16(rng, 1, 1, S, D) * 0.01, (1 + bf16(rng, 1, 1, S, D).abs().clamp(max=0.9).double()) * 2.0 ** 110
    k[0, 0, :, 0] = torch.arange(S) // 8                       # base 2: 16 / 8 * log2(e) / 8 = 0.36 from a group of 8 keys to the next
    pair.write(k.to(torch.bfloat16), v.to(torch.bfloat16), [0])
    q = bf16(rng, 1, G, N, D) * 0.01
    q[..., 0] = 2.0
    want, _ = compare(pair, q.to(torch.bfloat16), [S - N])
    assert np.isfinite(want).all()


# ------------------------------------------------------------------------------------------------------------- batches
@pytest.mark.parametrize("B,G", [(1 << 20, 1), (1 << 19, 20)])
@pytest.mark.parametrize("pages", [1, 81])
def test_a_million_sequences(B, G, pages):
    """Sequences of one token, with a table that holds little and one that may hold long ones: each sees its own key alone."""
    D, P, held = 64, 16, 1000
    table = torch.full((B, pages), -1, dtype=torch.int32, device="cuda")
    table[:, 0] = torch.arange(B, device="cuda") % held
    cache = dma.KVCache.empty(table, held, 1, D, P)
    first = dma.KVCache(cache.k_codes, cache.v_codes, cache.k_scales, cache.v_scales, table[:held].contiguous())
    k, v = (torch.randn((held, 1, 1, D), device="cuda").to(torch.bfloat16) for _ in range(2))
    zeros = torch.zeros(B, dtype=torch.int32, device="cuda")
    dma.dma_kv_write(first, k, v, zeros[:held])
    v = dma.dma_kv_read(first, zeros[:held], 1)[1]
    out = dma.dma_cache_attn(k[:1].expand(B, G, 1, D), cache, zeros)
    for at in range(0, B, 1 << 16):
        assert torch.equal(out[at:at + (1 << 16)], v[torch.arange(at, at + (1 << 16), device="cuda") % held].expand(-1, G, -1, -1)), at
