"""Attention over the cache behind shared prefixes, on the GPU against its definition in 64 bits (kv_plain): the same as attention over
the cache row by row, within the bound that kv_plain derives for every element.  Joining pieces of a row's sums multiplies each by one factor
that exp2 gives, which the bound's count of 32 units beside the number of keys covers, as for pieces of long sequences.

Where little would be read twice the call is served by the kernels of dma_cache_attn; what it goes by is the reach of the page table, so tables
with many empty columns (wide) bring short sequences to the kernel for shared prefixes."""
import numpy as np
import pytest
import torch

import kv_counts
import kv_plain as plain
from paper_2604_03950_amd import binding as dma
from test_gpu_kv_cache import Pair, bf16, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def library():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dma.load()


class Family(Pair):
    """Sequences of groups: sizes and common lengths of these (positions, taken down to whole pages), lens[b] positions in all; -1 as
    a common length: sequences of no group."""

    def __init__(self, rng, groups, lens, Hkv, P, D, fmt, write=True, spare=1, wide=True):
        self.wide = wide
        wide = max(-(-n // P) for n in lens) + spare
        table, at, b, self.bounds, self.shared = np.full((len(lens), wide), -1, np.int32), 0, 0, [], []
        order = rng.permutation(sum(-(-n // P) for n in lens) + 3)
        leaders = []
        for size, common in groups:
            k = max(common, 0) // P
            if common >= 0:
                if not self.bounds:
                    self.bounds.append(b)
                assert self.bounds[-1] == b
                self.bounds.append(b + size)
                self.shared.append(common)
            for i in range(size):
                u = -(-lens[b + i] // P)
                first = min(k, u) if i else 0
                table[b + i, :first] = table[b, :first]
                table[b + i, first:u] = order[at:at + u - first]
                at += u - first
                leaders.append((b, first * P))
            b += size
        self.shared = [s // P * P for s in self.shared]
        assert b == len(lens)
        super().__init__(rng, None, Hkv, P, D, fmt, table, len(order))
        self.together = self.wide and len(lens) > len(self.shared) > 0
        if self.together:                                          # empty columns, on the GPU alone
            columns = int(2e8 / ((len(lens) - len(self.shared)) * P * 2 * Hkv * D)) + 1
            g = self.gpu
            self.gpu = dma.KVCache(g.k_codes, g.v_codes, g.k_scales, g.v_scales, torch.nn.functional.pad(g.page_table, (0, columns), value=-1), g.fmt[0] if isinstance(g.fmt, tuple) else g.fmt)
        if write:
            start = np.array([own for _, own in leaders])
            n = np.maximum(np.array(lens) - start, 0)
            self.write(bf16(rng, b, Hkv, n.max(), D), bf16(rng, b, Hkv, n.max(), D), start, n)

    def attn(self, q, start, n=None, window=0, sinks=0, out=None, shared=None, bounds=None, **kw):
        got = dma.dma_cache_attn_shared(q.cuda() if not q.is_cuda else q, self.gpu, i32(start), i32(self.bounds or [0] if bounds is None else bounds),
                                        i32(np.array(self.shared if shared is None else shared, int)), i32(n), window=window, sink_tokens=sinks, out=out, **kw)
        if self.together and bounds is None and not window and q.shape[1] // self.cpu.Hkv * q.shape[2] <= 64:
            self.served_together(q.shape[1], q.shape[2])
        want, bound = self.cpu.attn(q.double().cpu().numpy(), start, n, window, sinks)
        rows = np.isfinite(want)
        off = np.abs(got.double().cpu().numpy() - want)[rows]
        assert not np.isnan(off).any()
        worst = (off - bound[rows]).max(initial=-1)
        assert worst <= 0, (worst, off.max(), (off / bound[rows]).max())
        return got, rows

    def served_together(self, Hq, N):
        assert dma.dma_cache_attn_shared_workspace_bytes(self.gpu, Hq, N, len(self.shared)) != dma.dma_cache_attn_workspace_bytes(self.gpu, Hq, N)


FORMS = [("e4m3", 128, 64, 2, 4, 1), ("e5m2", 128, 16, 1, 1, 1), ("e4m3", 64, 32, 3, 5, 1), ("e5m2", 64, 256, 2, 8, 1), ("e4m3", 128, 128, 1, 16, 1),
         ("e4m3", 128, 64, 2, 4, 3), ("e4m3", 64, 16, 1, 1, 17), ("e5m2", 128, 128, 2, 5, 7), ("e4m3", 128, 32, 1, 4, 33), ("e5m2", 64, 64, 1, 8, 20),
         ("e4m3", 128, 64, 1, 4, 8), ("e5m2", 64, 32, 2, 8, 8), ("e4m3", 128, 16, 1, 5, 13), ("e4m3", 64, 256, 1, 4, 16), ("e5m2", 128, 256, 1, 3, 21)]


@pytest.mark.parametrize("fmt,D,P,Hkv,G,N", FORMS)
@pytest.mark.parametrize("groups", [[(1, 100)], [(7, 300)], [(2, -1), (3, 70), (0, 9), (5, 513), (1, 0), (2, -1)], [(4, 0)], [(3, -1)]])
@pytest.mark.parametrize("window,sinks,wide", [(0, 0, True), (50, 0, True), (150, 70, True), (1 << 30, 0, True), (150, 70, False)])
def test_groups(fmt, D, P, Hkv, G, N, groups, window, sinks, wide):
    rng = np.random.default_rng(D + P + N + len(groups) + window)
    lens = []
    for size, common in groups:
        lens += [max(common, 0) + N + int(x) for x in rng.integers(0, 200, size)]
    f = Family(rng, groups, lens, Hkv, P, D, fmt, wide=wide)
    B = len(lens)
    n = np.full(B, N) if N == 1 else np.maximum(rng.integers(0, N + 1, B), [N] + [0] * (B - 1))
    out = torch.full((B, Hkv * G, N, D), 7.0, dtype=torch.bfloat16, device="cuda")
    got, rows = f.attn(bf16(rng, B, Hkv * G, N, D), np.array(lens) - n, n, window, sinks, out=out)
    assert got is out and (got.float().cpu().numpy()[~rows] == 7).all()


@pytest.mark.parametrize("fmt,D,P,Hkv,G,N,B,prefix,own,window,sinks", [
    ("e4m3", 128, 64, 32, 1, 1, 43, 320, 300, 310, 0), ("e4m3", 128, 16, 32, 2, 1, 43, 300, 200, 310, 5), ("e5m2", 128, 32, 32, 1, 2, 58, 256, 150, 210, 70),
    ("e5m2", 64, 64, 32, 1, 2, 62, 400, 100, 420, 500), ("e4m3", 64, 256, 32, 1, 3, 84, 512, 200, 300, 0), ("e4m3", 128, 128, 32, 1, 1, 240, 64, 40, 50, 4)])
def test_windows(fmt, D, P, Hkv, G, N, B, prefix, own, window, sinks):
    """Windows whose far end lies in the prefix, behind it, before the sequence; sinks in the prefix and beyond it.  What no row sees may be anything.
    (Enough heads and sequences for the kernel for shared prefixes.)"""
    rng = np.random.default_rng(B + prefix)
    lens = [prefix + N + int(x) for x in rng.integers(0, own, B)]
    cut = B // 3
    f = Family(rng, [(cut, prefix), (B - cut, prefix // 2)], lens, Hkv, P, D, fmt, wide=False)
    assert dma.dma_cache_attn_shared_workspace_bytes(f.gpu, Hkv * G, N, 2, window, sinks) != dma.dma_cache_attn_workspace_bytes(f.gpu, Hkv * G, N, window, sinks)
    start = np.array(lens) - N
    start[:4] = 0, prefix // 3, prefix // 2, prefix - 1
    start[cut:cut + 3] = prefix // 2 - 1, 5, -1
    seen = set()
    for b in range(B):
        if start[b] >= 0:
            for j in range((start[b] + N - 1) // P + 1):
                if (j + 1) * P > start[b] - window + 1 or j * P < sinks:
                    seen.add(int(f.cpu.table[b, j]))
    for p in set(range(f.cpu.pages)) - seen:
        f.gpu.k_codes[p], f.gpu.v_codes[p], f.gpu.k_scales[p], f.gpu.v_scales[p] = 0x7f, 0x7f, 255, 255
    f.attn(bf16(rng, B, Hkv * G, N, D), start, None, window, sinks)


@pytest.mark.parametrize("N,G", [(1, 4), (5, 2)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (30, 4), (2000, 0)])
def test_rows_inside_the_prefix(N, G, window, sinks):
    """Queries that stand inside what their group shares (a prompt seen again), at its first position, without tokens, before the sequence."""
    rng = np.random.default_rng(N + window)
    f = Family(rng, [(9, 640), (3, 320)], [700] * 9 + [400] * 3, 2, 32, 128, "e4m3")
    start = np.array([0, 1, 63, 64, 300, 639, 650, -1, 5, 0, 319, 399 - N])
    n = np.array([N] * 12)
    n[8] = 0
    out = torch.full((12, 2 * G, N, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    got, rows = f.attn(bf16(rng, 12, 2 * G, N, 128), start, n, window, sinks, out=out)
    assert (got.float().cpu().numpy()[~rows] == 7).all() and not rows[7].any() and not rows[8].any()


@pytest.mark.parametrize("shared", [[0], [1], [63], [64], [65], [500], [513], [-5], [-(1 << 31)]])
def test_any_part_of_what_is_common(shared):
    """Fewer positions than the rows have in common may be named."""
    rng = np.random.default_rng(3)
    f = Family(rng, [(6, 520)], [600, 530, 521, 700, 650, 520], 1, 16, 64, "e5m2")
    f.attn(bf16(rng, 6, 5, 2, 64), np.array([598, 528, 519, 698, 648, 518]), shared=shared)


def test_bounds_of_groups():
    """Bounds outside the batch, groups of nothing, far more groups than sequences: the sequences in none are by themselves."""
    rng = np.random.default_rng(4)
    f = Family(rng, [(8, 260)], [300] * 8, 2, 32, 64, "e4m3")
    for bounds, shared in (([-3, 5], [256]), ([2, 99], [256]), ([0, 0, 0, 8, 8], [9, 9, 256, 9]), ([3, 3], [256]), ([0, 2, 4, 6, 8], [256, 200, 0, 64]), ([8, 8], [256]),
                           ([0] * 500 + [4] * 700 + [8] * 300, [256] * 1499), ([0], []), ([5, 1 << 30], [128])):
        f.attn(bf16(rng, 8, 4, 1, 64), [299] * 8, bounds=bounds, shared=shared)


@pytest.mark.parametrize("B,Hkv", [(5, 1), (430, 4)])
def test_shared_beyond_the_table(B, Hkv):
    """A shared length at the end of its type: all rows name the same pages as far as the table goes, the tokens themselves among them.  (So
    many rows of a short table are enough for the kernel for shared prefixes.)"""
    rng = np.random.default_rng(5)
    f = Family(rng, [(B, 256)], [256] * B, Hkv, 64, 128, "e4m3", spare=0, wide=False)
    if B > 5:
        f.served_together(Hkv, 1)
    for shared in (256, (1 << 31) - 1):
        f.attn(bf16(rng, B, Hkv, 1, 128), [255, 255, 100, 255, 3] * (B // 5), shared=[shared])
        f.attn(bf16(rng, B, Hkv, 2, 128), [300, (1 << 31) - 1, 254, 1 << 30, 255] * (B // 5), None, 250, 3, shared=[shared])


@pytest.mark.parametrize("fmt,D,G,N,P", [("e4m3", 128, 4, 1, 64), ("e5m2", 64, 2, 3, 16), ("e4m3", 128, 1, 1, 128)])
def test_large_batches(fmt, D, G, N, P):
    """More sequences than a workgroup has threads: one large group, many small ones, some alone."""
    rng = np.random.default_rng(G + N)
    groups = [(290, 400)] + [(3, 200)] * 40 + [(4, -1)]
    lens = np.concatenate([np.full(s, max(c, 0)) for s, c in groups]) + rng.integers(N, 90, 414)
    f = Family(rng, groups, [int(x) for x in lens], 1, P, D, fmt)
    f.attn(bf16(rng, 414, G, N, D), lens - N)


@pytest.mark.parametrize("D,P,fmt", [(128, 64, "e4m3"), (64, 16, "e5m2")])
@pytest.mark.parametrize("B,N,G,prefix,window,sinks", [(2, 1, 1, 20000, 0, 0), (33, 1, 4, 9000, 0, 0), (70, 1, 8, 4097, 0, 0), (6, 20, 2, 5000, 0, 0), (33, 2, 3, 6000, 5900, 100),
                                                     (12, 1, 8, 3000, 0, 0)])
def test_every_key_once(D, P, fmt, B, N, G, prefix, window, sinks):
    """Attention as counting (kv_counts): a key left out, or taken both for all and for one, shows."""
    rng = np.random.default_rng(B + prefix)
    prefix = prefix // P * P
    lens = [prefix + N + int(x) for x in rng.integers(0, 700, B)]
    f = Family(rng, [(B, prefix)], lens, 1, P, D, fmt, write=False)
    one = 0x38 if fmt == "e4m3" else 0x3c
    table = f.gpu.page_table.cpu().numpy()
    f.gpu.k_codes.zero_()
    for odd in (0, 1):
        v = torch.zeros_like(f.gpu.v_codes).cpu().numpy()
        for b in range(B):
            t = np.arange(lens[b])
            v[table[b, t // P], 0, kv_counts.channel(t, D, odd), t % P] = one
        f.gpu.v_codes.copy_(torch.from_numpy(v))
        f.gpu.k_scales.fill_(127)
        f.gpu.v_scales.fill_(127)
        q = torch.zeros((B, G, N, D), dtype=torch.bfloat16, device="cuda")
        got = dma.dma_cache_attn_shared(q, f.gpu, i32(np.array(lens) - N), i32([0, B]), i32([prefix]), window=window, sink_tokens=sinks).double().cpu().numpy()
        for b in range(B):
            for i in range(N):
                count, n = kv_counts.counts(D, lens[b] - N + i, window, sinks)
                assert not kv_counts.wrong(got[b, :, i], count[odd], n).any(), (b, i)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("N,G", [(1, 4), (9, 5)])
def test_nan_reaches_only_who_sees_it(fmt, N, G):
    """A NaN among the shared keys or values and among a sequence's own."""
    rng = np.random.default_rng(40 + N)
    D, P, B = 128, 32, 6
    f = Family(rng, [(B, 320)], [360] * B, 2, P, D, fmt)
    for page, where, codes in ((f.cpu.table[0, 3], (1, 77, 5), "v"), (f.cpu.table[0, 9], (0, 127, 31), "v"), (f.cpu.table[2, 10], (0, 3, 6), "v"), (f.cpu.table[4, 11], (1, 2, 9), "k")):
        getattr(f.cpu, codes)[(page, *where)] = 0x7f
        getattr(f.gpu, codes + "_codes")[(int(page), *where)] = 0x7f
    start = np.array([350, 200, 345, 100, 348, 316])
    for window in (0, 2, 40, 250):
        q = bf16(rng, B, 2 * G, N, D)
        got = dma.dma_cache_attn_shared(q.cuda(), f.gpu, i32(start), i32([0, B]), i32([320]), window=window).double().cpu().numpy()
        with np.errstate(invalid="ignore"):
            want, bound = f.cpu.attn(q.double().numpy(), start, None, window)
        np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
        fine = ~np.isnan(want)
        assert (np.abs(got - want) <= bound)[fine].all()


def test_pages_that_are_missing():
    """Entries without a page in what is shared and behind it; nothing to see at all."""
    rng = np.random.default_rng(41)
    for holes in ([(slice(None), 1), (slice(None), 3), (2, 7)], [(slice(None), slice(0, 6)), (1, slice(None))], [(slice(None), slice(None))]):
        f = Family(rng, [(5, 96)], [140, 97, 128, 130, 111], 2, 16, 64, "e4m3")
        for at in holes:
            f.cpu.table[at] = -1
            f.gpu.page_table[at] = -1
        start = np.array([139, 96, 127, 129, 110])
        got, rows = f.attn(bf16(rng, 5, 4, 1, 64), start)
        f.attn(bf16(rng, 5, 4, 3, 64), start - 2, None, 20, 2)
        if holes[0] == (slice(None), slice(None)):
            assert not got.any() and rows.all()


@pytest.mark.parametrize("N", [1, 6])
@pytest.mark.parametrize("fill", [0x7f, 0xff])
def test_unseen_places_may_hold_anything(N, fill):
    """Codes of NaN and scales of 255 behind the tokens, before the window, in pages of nobody (page 0 among them)."""
    rng = np.random.default_rng(42)
    P, D, B = 64, 128, 5
    lens = [330, 300, 257, 400, 299]
    f = Family(rng, [(B, 256)], lens, 1, P, D, "e4m3")
    start = np.array(lens) - N
    used = np.unique(f.cpu.table[f.cpu.table >= 0])
    for p in set(range(f.cpu.pages)) - set(used.tolist()):
        f.gpu.k_codes[p], f.gpu.v_codes[p], f.gpu.k_scales[p], f.gpu.v_scales[p] = fill, fill, 255, 255
    for b in range(B):
        page, at = f.cpu.table[b, (lens[b] - 1) // P], (lens[b] - 1) % P + 1
        f.gpu.k_codes[int(page), :, at:] = fill
        f.gpu.v_codes[int(page), :, :, at:] = fill
    f.attn(bf16(rng, B, 4, N, D), start)
    f.gpu.k_codes[int(f.cpu.table[0, 0])], f.gpu.v_codes[int(f.cpu.table[0, 0])] = fill, fill
    f.gpu.k_scales[int(f.cpu.table[0, 0])], f.gpu.v_scales[int(f.cpu.table[0, 0])] = 255, 255
    f.attn(bf16(rng, B, 4, N, D), start, None, 150)


def test_sequences_that_ended():
    """Sequences without tokens have no say: the first of a group has lost its pages, queries of rows that do not exist are NaN and infinite."""
    rng = np.random.default_rng(48)
    f = Family(rng, [(3, 320), (60, 512)], [400] * 3 + [600 + i for i in range(60)], 1, 32, 128, "e4m3")
    gone = [0, 3, 4, 5, 60, 62]
    f.cpu.table[gone] = -1
    f.gpu.page_table[gone] = -1
    start, n = np.array([399, 398, 397] + [598 + i for i in range(60)]), np.full(63, 2)
    start[gone[:3]] = -1
    n[gone[3:]] = 0
    n[30:50] = 1
    q = bf16(rng, 63, 4, 2, 128)
    clean, _ = f.attn(q, start, n)
    q[gone], q[30:40, :, 1], q[40:50, :, 1] = float("nan"), float("inf"), float("nan")
    got = dma.dma_cache_attn_shared(q.cuda(), f.gpu, i32(start), i32(f.bounds), i32(f.shared), i32(n))
    assert torch.equal(got, clean)


def test_strides_and_streams():
    """Queries and results as views of larger tensors, on a stream of their own."""
    rng = np.random.default_rng(43)
    f = Family(rng, [(4, 200), (2, 64)], [230, 220, 260, 210, 100, 70], 2, 32, 64, "e5m2")
    start = np.array([227, 217, 257, 207, 97, 67])
    q = bf16(rng, 6, 3, 2, 10, 64).cuda()[:, :, 0].transpose(1, 2)                     # [6, 10, 3, 64] of a projection
    whole = torch.full((6, 10, 5, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got, _ = f.attn(q, start, out=whole[:, :, 1:4, 64:])
    stream.synchronize()
    plain_out, _ = f.attn(q.contiguous(), start)
    assert torch.equal(got, plain_out)
    whole[:, :, 1:4, 64:] = 3
    assert (whole == 3).all()


def test_equal_calls_equal_bits():
    rng = np.random.default_rng(44)
    f = Family(rng, [(40, 900)], [int(x) for x in rng.integers(905, 1400, 40)], 2, 64, 128, "e4m3")
    q, start = bf16(rng, 40, 8, 1, 128).cuda(), i32([900 + b for b in range(40)])
    call = lambda: dma.dma_cache_attn_shared(q, f.gpu, start, i32([0, 40]), i32([896])).view(torch.int16)  # noqa: E731  (bits: what lies behind the tokens may be NaN)
    first = call()
    for _ in range(5):
        assert torch.equal(first, call())


def test_workspaces():
    """A workspace of the caller's, of just the bytes that are asked for, full of NaN; what lies behind it stays."""
    rng = np.random.default_rng(45)
    f = Family(rng, [(20, 640)], [int(x) for x in rng.integers(650, 900, 20)], 2, 64, 128, "e4m3")
    for N in (1, 4):
        need = dma.dma_cache_attn_shared_workspace_bytes(f.gpu, 8, N, 1)
        ws = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")
        f.attn(bf16(rng, 20, 8, N, 128), [645] * 20, workspace=ws[:need])
        assert (ws[need:] == 255).all()


def test_graph():
    """Recorded and replayed with other lengths, groups and pages; each replay against the call by itself, with work in between."""
    rng = np.random.default_rng(46)
    f = Family(rng, [(6, 320), (6, 640)], [400] * 6 + [700] * 6, 2, 32, 128, "e4m3")
    q = bf16(rng, 12, 8, 2, 128).cuda()
    start, n, bounds, shared = i32([350] * 12), i32([2] * 12), i32([0, 6, 12]), i32([320, 320])
    out = torch.zeros((12, 8, 2, 128), dtype=torch.bfloat16, device="cuda")
    need = dma.dma_cache_attn_shared_workspace_bytes(f.gpu, 8, 2, 2)
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dma.dma_cache_attn_shared(q, f.gpu, start, bounds, shared, n, out=out, workspace=ws)
    for s, k, lo, sh in (([350] * 12, [2] * 12, [0, 6, 12], [320, 320]), ([390] * 6 + [690] * 6, [1] * 12, [0, 6, 12], [320, 640]),
                         ([0] * 12, [2] * 12, [0, 0, 12], [0, 0]), ([7, 399, -1, 200, 64, 63] * 2, [2, 1, 2, 0, 2, 2] * 2, [6, 12, 12], [320, 5])):
        for t, x in zip((start, n, bounds, shared), (s, k, lo, sh)):
            t.copy_(i32(x))
        q.copy_(bf16(rng, 12, 8, 2, 128))
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        alone, _ = f.attn(q, s, np.array(k), out=torch.full_like(out, 7), bounds=lo, shared=sh)
        assert torch.equal(got, alone)


def test_samples_from_prompt_to_compaction():
    """The calls together, as a program has them: a prompt, samples of it that part inside a page, tokens written and attended to
    behind the common prefix, drafts taken back, sequences that end, the rest compacted; the definition follows with plain pages."""
    rng = np.random.default_rng(47)
    P, D, Hkv, G, B, prompt = 32, 128, 2, 4, 6, 150
    table = np.full((B, 8), -1, np.int32)
    f = Pair(rng, None, Hkv, P, D, "e4m3", table, 40)
    refs = i32([0] * 40)
    follow = lambda: f.cpu.table.__setitem__(slice(None), f.gpu.page_table.cpu().numpy())  # noqa: E731

    def attend(start, N, shared):
        q = bf16(rng, B, Hkv * G, N, D)
        got = dma.dma_cache_attn_shared(q.cuda(), f.gpu, i32(start), i32([0, B]), i32([shared])).double().cpu().numpy()
        want, bound = f.cpu.attn(q.double().numpy(), start)
        rows = np.isfinite(want)
        assert (np.abs(got - want) <= bound)[rows].all()
        return q.cuda(), got

    n = [prompt] + [0] * (B - 1)
    assert not dma.dma_kv_reserve(f.gpu, refs, i32([0] * B), prompt, i32(n)).any()
    follow()
    f.write(bf16(rng, B, Hkv, prompt, D), bf16(rng, B, Hkv, prompt, D), [0] * B, n)
    dma.dma_kv_fork(f.gpu, refs, i32([0] * B), i32([prompt] * B))
    assert refs.sum() == B * 5 and refs.max() == B
    length = np.full(B, prompt)
    for N in (1, 3, 20):
        before = f.gpu.page_table.cpu().numpy()
        assert not dma.dma_kv_reserve(f.gpu, refs, i32(length), N).any()
        now = f.gpu.page_table.cpu().numpy()
        for b in range(B):                                       # the definition's copies: what a sequence held where it got another page
            for j in np.nonzero((before[b] != now[b]) & (before[b] >= 0))[0]:
                for x in (f.cpu.k, f.cpu.v, f.cpu.ks, f.cpu.vs, f.cpu.written):
                    x[now[b, j]] = x[before[b, j]]
        follow()
        f.write(bf16(rng, B, Hkv, N, D), bf16(rng, B, Hkv, N, D), length)
        f.same()
        attend(length, N, prompt // P * P)
        length = length + N
    # the last 7 tokens were drafts; two sequences end; another takes over a row
    length = length - 7
    length[4] = length[1]
    dma.dma_kv_fork(f.gpu, refs, i32([0, 1, -1, 3, 1, -1]), i32(length))
    follow()
    held = f.gpu.page_table.cpu().numpy()
    assert np.array_equal(np.bincount(held[held >= 0], minlength=40), refs.cpu().numpy())
    start = np.where(np.isin(np.arange(B), [2, 5]), -1, length - 1)
    q, got = attend(start, 1, prompt // P * P)
    used, moved = dma.dma_kv_compact(f.gpu, refs)
    assert used.item() == (refs > 0).sum() and not (refs[used.item():] > 0).any()
    after = f.gpu.page_table.cpu().numpy()
    assert np.array_equal(after, np.where(held >= 0, moved.cpu().numpy()[held], -1)) and after.max() < used.item()
    # the same pages in other places: the same bits
    again = dma.dma_cache_attn_shared(q, f.gpu, i32(start), i32([0, B]), i32([prompt // P * P]))
    assert torch.equal(again.double().cpu(), torch.from_numpy(got))
