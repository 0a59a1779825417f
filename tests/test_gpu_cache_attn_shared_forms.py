"""Attention over the cache behind shared prefixes, every call of these in its own kernel (asserted with the call's window and sinks): windows with
tiles of 16 and of 32 rows, NaN and missing pages under them, keys counted where sinks and windows are cut between prefix and own part; more groups
than a wave looks at together and than are held in LDS; more sequences than a wave holds, with either tile.  Against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import kv_counts
import kv_rows
from paper_2604_03950_amd import binding as dma
from test_gpu_cache_attn_shared import Family
from test_gpu_kv_cache import FMT, bf16, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def library():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dma.load()


def shared(f, q, start, n=None, window=0, sinks=0, bounds=None, common=None, **kw):
    """The call, in the kernel for shared prefixes."""
    bounds, common = f.bounds if bounds is None else bounds, f.shared if common is None else common
    Hq, N = q.shape[1:3]
    assert dma.dma_cache_attn_shared_workspace_bytes(f.gpu, Hq, N, len(common), window, sinks) != dma.dma_cache_attn_workspace_bytes(f.gpu, Hq, N, window, sinks)
    return dma.dma_cache_attn_shared(q.cuda(), f.gpu, i32(start), i32(bounds), i32(np.array(common, int)), i32(n), window=window, sink_tokens=sinks, **kw)


def check(f, q, start, n=None, window=0, sinks=0, **kw):
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    got = shared(f, q, start, n, window, sinks, out=out, **kw).double().cpu().numpy()
    want, bound, exists = kv_rows.attn(f.cpu, q.double().numpy(), start, n, window, sinks)
    rows = np.broadcast_to(exists[:, None, :, None], q.shape)
    assert (got[~rows] == 7).all()
    np.testing.assert_array_equal(np.isnan(got)[rows], np.isnan(want)[rows])
    fine = rows & ~np.isnan(want)
    assert (np.abs(got - want)[fine] <= bound[fine]).all(), np.nanmax((np.abs(got - want) / bound)[fine])
    return np.isnan(want) & rows


# (sequences - groups) * (window + sinks) * 2 * kv heads * D >= 1e8 brings a call to the kernel
WINDOWS = [("e4m3", 128, 64, 8, 4, 5, 172, 310, 0), ("e5m2", 128, 16, 16, 2, 10, 86, 310, 5), ("e4m3", 64, 32, 32, 1, 17, 86, 300, 70), ("e5m2", 64, 256, 16, 4, 8, 172, 290, 130),
           ("e4m3", 128, 32, 32, 1, 3, 86, 150, 200)]


@pytest.mark.parametrize("fmt,D,P,Hkv,G,N,B,window,sinks", WINDOWS)
def test_windows(fmt, D, P, Hkv, G, N, B, window, sinks):
    """Far ends of windows in the prefix, behind it, before the sequence, of one sequence or of several in a tile; sinks up to and past the prefix's end;
    ragged numbers of tokens; a NaN of the prefix that some windows hold, a page that is missing for all, one for a single sequence, own NaN."""
    rng = np.random.default_rng(B + P + N)
    prefix, cut = 384, B // 3
    lens = [prefix + N + int(x) for x in rng.integers(0, 300, B)]
    f = Family(rng, [(cut, prefix), (B - cut - 2, prefix // 2), (2, -1)], lens, Hkv, P, D, fmt, wide=False)
    n = np.maximum(rng.integers(0, N + 1, B), [N] * 12 + [0] * (B - 12))
    start = np.array(lens) - n
    start[:6] = 0, 100, 191, 192, prefix - 1, 250
    start[cut:cut + 3] = prefix // 2 - 1, 5, -1
    q = bf16(rng, B, Hkv * G, N, D)
    check(f, q, start, n, window, sinks)
    for page, where, codes in ((f.cpu.table[0, 100 // P], (1, 7, 100 % P), "v"), (f.cpu.table[0, 200 // P], (0, 200 % P, 31), "k"), (f.cpu.table[cut, 130 // P], (2, 3, 130 % P), "v"),
                               (f.cpu.table[7, (start[7] - 1) // P], (3, 9, (start[7] - 1) % P), "v")):
        getattr(f.cpu, codes)[(page, *where)] = 0x7f
        getattr(f.gpu, codes + "_codes")[(int(page), *where)] = 0x7f
    for at in ((slice(0, cut), 300 // P), (9, (start[9] - 1) // P), (slice(cut, B - 2), 64 // P)):
        f.cpu.table[at] = -1
        f.gpu.page_table[at] = -1
    none = check(f, q, start, n, window, sinks)
    assert none[:, :4 * G].any() and not none[:, 4 * G:].any()


@pytest.mark.parametrize("D,P,fmt", [(128, 64, "e4m3"), (64, 16, "e5m2")])
@pytest.mark.parametrize("B,N,G,prefix,window,sinks", [(60, 1, 4, 6000, 5900, 100), (60, 9, 2, 3000, 2500, 1000), (100, 20, 1, 2000, 1800, 2300), (60, 3, 3, 4000, 4200, 70)])
def test_every_key_once_under_a_window(D, P, fmt, B, N, G, prefix, window, sinks):
    """Attention as counting (kv_counts): windows that begin in the prefix and sinks that end in it, behind it or in the window."""
    rng = np.random.default_rng(B + prefix)
    prefix, Hkv = prefix // P * P, 2 * 128 // D
    lens = [prefix + N + int(x) for x in rng.integers(0, 700, B)]
    f = Family(rng, [(B, prefix)], lens, Hkv, P, D, fmt, write=False, wide=False)
    one = 0x38 if fmt == "e4m3" else 0x3c
    table = f.gpu.page_table.cpu().numpy()
    f.gpu.k_codes.zero_()
    f.gpu.k_scales.fill_(127)
    f.gpu.v_scales.fill_(127)
    for odd in (0, 1):
        v = torch.zeros_like(f.gpu.v_codes).cpu().numpy()
        for b in range(B):
            t = np.arange(lens[b])
            v[table[b, t // P], :, kv_counts.channel(t, D, odd), t % P] = one
        f.gpu.v_codes.copy_(torch.from_numpy(v))
        got = shared(f, torch.zeros((B, Hkv * G, N, D), dtype=torch.bfloat16), np.array(lens) - N, None, window, sinks)
        assert (got == got[:, :1]).all()
        got = got[:, 0].double().cpu().numpy()
        for b in range(B):
            for i in range(N):
                count, total = kv_counts.counts(D, lens[b] - N + i, window, sinks)
                assert not kv_counts.wrong(got[b, i], count[odd], total).any(), (b, i)


def family_of_many(rng, sizes, alone, Hkv, P, D, fmt, N, prefixes):
    """Groups of these sizes (0 among them), with sequences of no group before and behind."""
    groups = [(alone, -1)] + [(s, int(rng.choice(prefixes))) for s in sizes] + [(alone, -1)]
    lens = np.concatenate([np.full(s, max(c, 0)) for s, c in groups]).astype(int)
    lens += rng.integers(N, 90, len(lens))
    f = Family(rng, groups, [int(x) for x in lens], Hkv, P, D, fmt)
    # a table so wide that so many sequences and groups come to the kernel
    columns, g = int(2e10 / ((len(lens) - len(f.shared)) * P * 2 * Hkv * D)) + 1, f.gpu
    f.gpu = dma.KVCache(g.k_codes, g.v_codes, g.k_scales, g.v_scales, torch.nn.functional.pad(g.page_table, (0, columns), value=-1), FMT[fmt])
    return f, lens


@pytest.mark.parametrize("fmt,D,P,Hkv,G,N", [("e4m3", 128, 64, 1, 4, 1), ("e5m2", 64, 32, 2, 5, 5), ("e4m3", 128, 16, 1, 1, 20)])
@pytest.mark.parametrize("groups", [63, 64, 65, 100, 129])
def test_many_groups(fmt, D, P, Hkv, G, N, groups):
    """As many groups as a wave looks at together, one more, several times as many; among them empty ones, of one sequence, and one that fills
    several tiles."""
    rng = np.random.default_rng(groups + N)
    sizes = rng.integers(0, 5, groups)
    sizes[groups // 2], sizes[-1] = 150, 3
    f, lens = family_of_many(rng, sizes, 3, Hkv, P, D, fmt, N, [70, 130, 300])
    check(f, bf16(rng, len(lens), Hkv * G, N, D), lens - N)


@pytest.mark.parametrize("fmt,D,P,Hkv,G,N", [("e4m3", 64, 64, 1, 2, 1), ("e5m2", 128, 32, 1, 3, 8)])
@pytest.mark.parametrize("groups", [511, 512, 513, 600])
def test_more_groups_than_lds_holds(fmt, D, P, Hkv, G, N, groups):
    """Bounds of 512 groups are held in LDS; with more they are read where they are needed."""
    rng = np.random.default_rng(groups + N)
    sizes = rng.integers(0, 6, groups)
    f, lens = family_of_many(rng, sizes, 5, Hkv, P, D, fmt, N, [64, 100, 200])
    check(f, bf16(rng, len(lens), Hkv * G, N, D), lens - N)


@pytest.mark.parametrize("fmt,D,P,G,N", [("e4m3", 128, 64, 1, 17), ("e5m2", 64, 16, 4, 5), ("e4m3", 64, 128, 8, 4), ("e5m2", 128, 32, 4, 16)])
@pytest.mark.parametrize("B", [256, 257, 520])
def test_large_batches_of_several_tokens(fmt, D, P, G, N, B):
    """As many sequences as a wave holds, one more, more than twice as many, in tiles of 32 rows; some without tokens."""
    rng = np.random.default_rng(B + N)
    sizes = [B // 2, 3, 0, 40]
    f, lens = family_of_many(rng, sizes + [B - sum(sizes) - 4], 2, 1, P, D, fmt, N, [200, 400])
    n = np.where(rng.random(B) < 0.2, 0, rng.integers(1, N + 1, B))
    check(f, bf16(rng, B, G, N, D), lens - N, n)


@pytest.mark.parametrize("fmt,D,P,Hkv,G,N", [("e4m3", 64, 64, 8, 2, 1), ("e5m2", 128, 32, 4, 4, 5)])
@pytest.mark.parametrize("B", [700, 1537])
def test_several_parts_of_large_batches_for_a_wave(fmt, D, P, Hkv, G, N, B):
    """More parts of sequences' own than there are waves, in batches of 256 sequences that a wave goes on through; sequences without tokens, among
    them whole batches at the front, in the middle and at the end."""
    rng = np.random.default_rng(B + N)
    sizes = [300, 1, 0, 90]
    f, lens = family_of_many(rng, sizes + [B - sum(sizes) - 6], 3, Hkv, P, D, fmt, N, [64, 130])
    for gone in ([], [(256, 600)], [(0, 300), (B - 260, B)]):
        n = np.where(rng.random(B) < 0.1, 0, rng.integers(1, N + 1, B))
        for lo, hi in gone:
            n[lo:hi] = 0
        check(f, bf16(rng, B, Hkv * G, N, D), lens - N, n)
