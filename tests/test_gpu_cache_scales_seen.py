"""Scales of value and key pages that no write leaves, on pages that some rows of a tile see and others do not: 255, with which every element
is NaN, and the largest ones, with which large elements pass what bf16 holds.  The rows that see such a page have its NaN or infinities, the
others their results, within the bound of kv_plain.  In the definition the page holds codes of NaN in the same places."""
import numpy as np
import pytest
import torch

import kv_rows
from paper_2604_03950_amd import binding as dma
from test_gpu_cache_attn_shared import Family
from test_gpu_kv_cache import Pair, bf16, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def library():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dma.load()


NAN = 0x7f


def spoil(pair, page, h, kind):
    """The page's scale of kv head h becomes 255, for values or keys; or 254, with one large value among zeros."""
    cpu, gpu, page = pair.cpu, pair.gpu, int(page)
    if kind == "large":
        cpu.v[page, h], cpu.vs[page, h] = 0, 127
        cpu.v[page, h, 7, -1] = cpu.v[page, h, 50, 0] = NAN
        gpu.v_codes[page, h] = 0
        gpu.v_codes[page, h, 7, -1] = gpu.v_codes[page, h, 50, 0] = 0x7e if cpu.fmt == "e4m3" else 0x7b
        gpu.v_scales[page, h] = 254
    else:
        getattr(cpu, kind)[page, h] = NAN
        getattr(gpu, kind + "_scales")[page, h] = 255


def compare(pair, got, q, start, n=None, window=0, sinks=0):
    want, bound, exists = kv_rows.attn(pair.cpu, q.double().numpy(), start, n, window, sinks)
    got = got.double().cpu().numpy()
    rows = np.broadcast_to(exists[:, None, :, None], q.shape)
    np.testing.assert_array_equal(np.isfinite(got)[rows], ~np.isnan(want)[rows])
    fine = rows & ~np.isnan(want)
    assert (np.abs(got - want)[fine] <= bound[fine]).all(), np.nanmax((np.abs(got - want) / bound)[fine])
    assert (~fine & rows).any() and fine.any()


# rows per kv head: 12, 25 and 48 (one and two tiles of the kernel for few rows), 160
ROWS = [(3, 4), (5, 5), (16, 3), (40, 4)]


@pytest.mark.parametrize("kind", ["v", "k", "large"])
@pytest.mark.parametrize("window,sinks", [(False, 0), (True, 0), (True, 3)])
@pytest.mark.parametrize("N,G", ROWS)
@pytest.mark.parametrize("fmt,D,P", [("e4m3", 128, 16), ("e5m2", 64, 32), ("e4m3", 64, 64), ("e5m2", 128, 64), ("e4m3", 128, 256)])
def test_tokens_of_a_sequence(fmt, D, P, N, G, window, sinks, kind):
    """A page that begins with one of the last tokens, so that those before it do not see it; under a window one that ends where it begins
    for one of them."""
    rng = np.random.default_rng(N + P + sinks)
    half, j = N // 2, max(300 // P, 2)
    start = [j * P - half, j * P - half - 1, j * P - N]           # the third sequence is as it should be
    pair = Pair(rng, [s + N for s in start], 2, P, D, fmt)
    S = max(start) + N
    pair.write(bf16(rng, 3, 2, S, D), bf16(rng, 3, 2, S, D), [0] * 3, [s + N for s in start])
    W = start[0] + half - ((j - 1) * P - 1) if window else 0      # token `half` of the first sequence sees nothing of page j - 2
    for b in range(2):
        spoil(pair, pair.cpu.table[b, j], b, kind)
        if window:
            spoil(pair, pair.cpu.table[b, j - 2], 1 - b, kind)
    q = bf16(rng, 3, 2 * G, N, D)
    compare(pair, dma.dma_cache_attn(q.cuda(), pair.gpu, i32(start), window=W, sink_tokens=sinks), q, start, None, W, sinks)


@pytest.mark.parametrize("kind", ["v", "k", "large"])
@pytest.mark.parametrize("fmt,D,P,N,G", [("e4m3", 128, 64, 1, 4), ("e5m2", 128, 16, 3, 2), ("e4m3", 64, 32, 9, 5), ("e5m2", 64, 128, 4, 8), ("e4m3", 128, 64, 20, 1)])
def test_sequences_behind_a_prefix(fmt, D, P, N, G, kind):
    """A page of a common prefix, which sequences that stand in it before the page do not see; a page of a sequence's own."""
    rng = np.random.default_rng(N + P)
    B, prefix = 7, 384
    f = Family(rng, [(B, prefix)], [prefix + P + N + 3] * B, 2, P, D, fmt)
    page = 2 * max(P, 64) // P                                    # begins at 128 or 256
    at, own = page * P, prefix // P + 1
    start = np.array([prefix + 2, at - N, at - 40, at - N + (N > 1), 5, at + 1, own * P - N // 2])
    spoil(f, f.cpu.table[0, page], 1, kind)
    spoil(f, f.cpu.table[6, own], 0, kind)
    f.served_together(2 * G, N)
    q = bf16(rng, B, 2 * G, N, D)
    got = dma.dma_cache_attn_shared(q.cuda(), f.gpu, i32(start), i32(f.bounds), i32(f.shared))
    compare(f, got, q, start)


@pytest.mark.parametrize("kind", ["v", "large"])
@pytest.mark.parametrize("fmt,D,P,Hkv,G,N,B,window,sinks", [("e4m3", 128, 64, 32, 1, 2, 43, 310, 0), ("e5m2", 128, 16, 32, 2, 1, 43, 310, 5), ("e4m3", 64, 32, 32, 1, 20, 84, 300, 70)])
def test_prefix_under_a_window(fmt, D, P, Hkv, G, N, B, window, sinks, kind):
    """A page of a common prefix that the windows of some sequences hold and those of others do not."""
    rng = np.random.default_rng(B + P)
    prefix = 384
    lens = [prefix + N + int(x) for x in rng.integers(0, 300, B)]
    f = Family(rng, [(B, prefix)], lens, Hkv, P, D, fmt, wide=False)
    assert dma.dma_cache_attn_shared_workspace_bytes(f.gpu, Hkv * G, N, 1, window, sinks) != dma.dma_cache_attn_workspace_bytes(f.gpu, Hkv * G, N, window, sinks)
    start = np.array(lens) - N
    start[1], start[2] = 100, 190
    for h in (0, 5):
        spoil(f, f.cpu.table[0, 192 // P + h // 5], h, kind)
    q = bf16(rng, B, Hkv * G, N, D)
    got = dma.dma_cache_attn_shared(q.cuda(), f.gpu, i32(start), i32(f.bounds), i32(f.shared), window=window, sink_tokens=sinks)
    compare(f, got, q, start, None, window, sinks)
