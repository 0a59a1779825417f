"""Forking, reserving and compacting pages of the 8-bit cache on the GPU against the definition (kv_pages_plain): everything has to be equal."""
import copy

import numpy as np
import pytest
import torch

import kv_pages_plain as plain
from paper_2604_03950_amd import binding as dma

pytestmark = pytest.mark.gpu
FMT = {"e4m3": dma.FMT_MXFP8_E4M3, "e5m2": dma.FMT_MXFP8_E5M2}


@pytest.fixture(scope="module", autouse=True)
def library():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dma.load()


def i32(x):
    return None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


class Held:
    """A cache with random bytes on the GPU, its table and refs on both sides."""

    def __init__(self, rng, table, pages, Hkv=1, P=16, D=64, fmt="e4m3"):
        self.table, self.refs, self.P = [[int(p) for p in row] for row in table], plain.count(table, pages), P
        self.cache = dma.KVCache.empty(i32(table), pages, Hkv, D, P, FMT[fmt])
        for t in self.bytes():
            t.copy_(torch.from_numpy(rng.integers(0, 256, tuple(t.shape), dtype=np.uint8)))
        self.gpu_refs = i32(self.refs)
        self.want = [t.cpu().numpy().copy() for t in self.bytes()]         # codes, then scales

    def bytes(self):
        return self.cache.k_codes, self.cache.v_codes, self.cache.k_scales, self.cache.v_scales

    def moved(self, moves, wiped=()):
        for x in self.want[2:]:
            x[list(wiped)] = 255
        for x in self.want:
            was = x.copy()
            for a, b in moves:
                x[b] = was[a]

    def fork(self, src, length=None):
        self.table = plain.fork(self.table, len(self.refs), self.P, src, length)
        self.refs = plain.count(self.table, len(self.refs))
        dma.dma_kv_fork(self.cache, self.gpu_refs, i32(src), i32(length))

    def reserve(self, start, N, n=None, **kw):
        counts = [N if n is None else min(max(int(x), 0), N) for x in (n if n is not None else start)]
        missing, copies, wiped = plain.reserve(self.table, self.refs, self.P, [int(x) for x in start], counts)
        self.moved(copies, wiped)
        got = dma.dma_kv_reserve(self.cache, self.gpu_refs, i32(start), N, i32(n), **kw)
        assert got.tolist() == missing
        return missing, copies, wiped

    def compact(self):
        used, moved, moves = plain.compact(self.table, self.refs)
        self.moved(moves)
        got = dma.dma_kv_compact(self.cache, self.gpu_refs)
        assert got[0].tolist() == [used] and got[1].tolist() == moved
        return used, moves

    def same(self):
        assert torch.equal(self.cache.page_table.cpu(), torch.tensor(self.table, dtype=torch.int32).view(self.cache.page_table.shape))
        assert self.gpu_refs.tolist() == self.refs
        for t, x in zip(self.bytes(), self.want):
            assert np.array_equal(t.cpu().numpy(), x)


def random_table(rng, B, wide, pages, holes=0.3):
    """Rows of pages and -1, some pages named several times."""
    t = rng.integers(0, max(pages, 1), (B, wide))
    t[rng.random((B, wide)) < holes] = -1
    return t if pages else np.full((B, wide), -1)


# ---------------------------------------------------------------------------------------------------------------- fork
@pytest.mark.parametrize("B,wide", [(1, 1), (1, 70), (3, 17), (64, 33), (300, 129), (1025, 20), (2049, 9), (3000, 7), (5000, 3), (8192, 2)])
@pytest.mark.parametrize("P", [16, 256])
def test_fork(B, wide, P):
    """Sources of every kind, several rows of one source, rows that are both; lengths of none, one, borders, beyond the table."""
    rng = np.random.default_rng(B + wide)
    h = Held(rng, random_table(rng, B, wide, B * 2 + 1), B * 2 + 1, P=16)
    h.P, h.cache = P, h.cache if P == 16 else dma.KVCache.empty(h.cache.page_table, B * 2 + 1, 1, 64, P)
    h.want = [t.cpu().numpy().copy() for t in h.bytes()]
    for _ in range(2):
        src = rng.integers(-1, B + 1, B)
        src[rng.random(B) < 0.2] = rng.integers(0, B)
        length = rng.integers(-2, wide * P + 40, B)
        length[rng.random(B) < 0.3] = P * rng.integers(0, wide + 1)
        h.fork(src, length)
        h.same()
    h.fork(rng.permutation(B))
    h.same()
    h.fork([-1] * B, [0] * B)
    h.same()
    assert not any(h.refs)


def test_fork_extremes():
    """Entries that are no page, sources and lengths at the ends of their type."""
    rng = np.random.default_rng(1)
    lo, hi = -(1 << 31), (1 << 31) - 1
    table = np.array([[0, 5, -7, 2, 6], [hi, 1, lo, 3, -1], [4, 4, 4, 7, 0]])
    h = Held(rng, table, 6)
    h.fork([2, 0, 1], [hi, hi, hi])
    h.same()
    h.fork([0, lo, hi], [lo, hi, hi])
    h.same()
    assert [p for row in h.table for p in row] == [-1] * 15


def test_fork_no_pages():
    h = Held(np.random.default_rng(2), np.full((3, 4), -1), 0)
    h.fork([1, 1, 1])
    h.same()
    none = Held(np.random.default_rng(2), np.zeros((3, 0), int), 5)
    none.fork([1, 1, 1])
    none.same()


# ------------------------------------------------------------------------------------------------------------- reserve
@pytest.mark.parametrize("fmt,D,P,Hkv", [("e4m3", 128, 64, 3), ("e5m2", 64, 16, 1), ("e4m3", 64, 256, 2), ("e5m2", 128, 32, 5), ("e4m3", 128, 128, 2)])
@pytest.mark.parametrize("N", [1, 7, 300])
def test_reserve(fmt, D, P, Hkv, N):
    """Batches whose rows share pages in families, tokens at borders and inside pages, from their first position and behind the table."""
    rng = np.random.default_rng(D + P + N)
    B, wide = 11, 9
    for spare in (40, 3, 0):
        table = np.full((B, wide), -1)
        start, at = rng.integers(0, 4 * P, B), 0
        start[[0, 1]] = 2 * P, 0
        for b in range(B):
            if b % 3:
                start[b], table[b] = start[b - 1], table[b - 1]
            else:
                k = -(-int(start[b]) // P)
                table[b, :k] = np.arange(at, at + k)
                at += k
        pages = at + spare
        order = rng.permutation(pages)
        table = np.where(table >= 0, order[table], -1)
        h = Held(rng, table, pages, Hkv, P, D, fmt)
        start[9:] = -1, wide * P + 3
        n = rng.integers(-1, N + 3, B)
        n[:3] = N
        missing, copies, wiped = h.reserve(start, N, n)
        h.same()
        if spare == 40 and N == 7 and P > 16:
            assert copies and wiped
        if spare == 0:
            assert any(missing)
        h.reserve(np.minimum(start + 1, wide * P), N)          # what is theirs already stays
        h.same()


def test_reserve_many_entries():
    """More entries than a workgroup takes at a time, more pages than it looks through, few of them free."""
    rng = np.random.default_rng(5)
    B, wide, pages = 37, 70, 20000
    table = np.full((B, wide), -1)
    other = np.full((250, 70), -1)                             # rows of other sequences hold most of the pages
    other.ravel()[:] = rng.permutation(pages)[:250 * 70]
    h = Held(rng, np.concatenate([table, other]), pages)
    start = np.concatenate([rng.integers(0, 200, B), np.full(250, -1)])
    missing, _, wiped = h.reserve(start, 900, np.concatenate([rng.integers(800, 900, B), np.zeros(250, int)]))
    h.same()
    assert len(wiped) > 2000 and not any(missing)
    h.reserve(np.concatenate([rng.integers(0, 300, B) * 0 + 40, np.full(250, -1)]), 1 << 20)
    h.same()


def test_reserve_a_batch_of_many():
    rng = np.random.default_rng(6)
    B = 9001
    table = np.full((B, 2), -1)
    table[::3, 0] = rng.permutation(3100)[:len(table[::3])]
    h = Held(rng, table, 9100)
    h.reserve(rng.integers(0, 32, B), 1)
    h.same()


def test_reserve_after_fork():
    """Samples of one prompt part inside a page: each gets a copy, the page is free behind the last of them; then all is theirs."""
    rng = np.random.default_rng(7)
    table = np.full((6, 4), -1)
    table[0, :2] = 3, 5
    h = Held(rng, table, 12, 2, 32, 128)
    h.fork([0] * 6, [40] * 6)
    assert h.refs[3] == h.refs[5] == 6
    missing, copies, _ = h.reserve([40] * 6, 1)
    h.same()
    assert len(copies) == 6 and h.refs[5] == 0 and h.refs[3] == 6 and not any(missing)
    assert h.reserve([41] * 6, 23)[1:] == ([], [])
    h.same()
    # at a border nothing is copied; a sequence that goes back to a shared page's first position takes one that holds nothing
    h.reserve([64, -1, -1, 0, 32, -1], 1)
    h.same()
    # pages are given out again: the one that was left first
    h.fork([-1, 1, 2, 3, 4, 5])
    h.same()


def test_reserve_nothing():
    rng = np.random.default_rng(8)
    h = Held(rng, np.full((2, 3), -1), 4)
    for start, n in (([-1, -1], None), ([0, 0], [0, -4]), ([48, 1 << 30], None), ([(1 << 31) - 1, -(1 << 31)], None)):
        assert h.reserve(start, 5, n)[0] == [0, 0]
        h.same()
    none = Held(rng, np.full((2, 3), -1), 0)
    assert none.reserve([0, 20], 30)[0] == [2, 2]              # [20, 50): pages 1 and 2 of 3
    none.same()
    narrow = Held(rng, np.zeros((2, 0), int), 4)
    assert narrow.reserve([0, 0], 5)[0] == [0, 0]


# ------------------------------------------------------------------------------------------------------------- compact
@pytest.mark.parametrize("pages,share", [(1, 1.0), (2, 0.5), (7, 0.4), (300, 0.5), (1030, 0.1), (4097, 0.7), (9000, 0.02), (9000, 0.98), (12300, 0.5), (500, 0.0)])
@pytest.mark.parametrize("fmt,D,P,Hkv", [("e4m3", 64, 16, 1), ("e5m2", 128, 16, 3)])
def test_compact(pages, share, fmt, D, P, Hkv):
    rng = np.random.default_rng(pages)
    wide = 40
    B = pages // 40 + 3
    names = rng.permutation(pages)[:int(round(share * pages))]
    table = np.full(B * wide, -1)
    table[rng.permutation(B * wide)[:len(names)]] = names
    table = table.reshape(B, wide)
    table[B // 2] = table[0]                                   # shared
    h = Held(rng, table, pages, Hkv, P, D, fmt)
    used, _ = h.compact()
    h.same()
    assert all(r > 0 for r in h.refs[:used]) and not any(h.refs[used:])
    assert h.compact() == (used, [])
    h.same()


@pytest.mark.parametrize("P,D,Hkv", [(64, 128, 8), (256, 128, 5), (32, 64, 2), (128, 64, 1)])
def test_compact_large_pages(P, D, Hkv):
    """Pages of one slice, of several and of a part of one; the last page to the first place."""
    rng = np.random.default_rng(P)
    table = np.array([[30, 7, -1], [-1, 7, 29], [2, 18, 19]])
    h = Held(rng, table, 31, Hkv, P, D)
    assert h.compact()[0] == 6
    h.same()


# --------------------------------------------------------------------------------------------------- graphs and streams
def test_graph_and_stream():
    """The three calls recorded on a side stream and replayed: they follow the values of their arguments from replay to replay."""
    rng = np.random.default_rng(9)
    table = np.full((4, 6), -1)
    table[0, :3] = 9, 2, 17
    table[1, :2] = 4, 11
    h = Held(rng, table, 20, 2, 32, 64)
    src, length, start, n = i32([0] * 4), i32([70] * 4), i32([70] * 4), i32([1] * 4)
    missing, used, moved = i32([0] * 4), i32([0]), i32([0] * 20)
    ws = [torch.empty(max(k, 1), dtype=torch.uint8, device="cuda") for k in (dma.dma_kv_reserve_workspace_bytes(h.cache, 40), dma.dma_kv_compact_workspace_bytes(h.cache))]
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        dma.dma_kv_fork(h.cache, h.gpu_refs, src, length)
        dma.dma_kv_reserve(h.cache, h.gpu_refs, start, 40, n, missing=missing, workspace=ws[0])
        dma.dma_kv_compact(h.cache, h.gpu_refs, used=used, moved=moved, workspace=ws[1])
    h.same()                                                   # recorded, not run
    for args in (([0] * 4, [70] * 4, [70] * 4, [1] * 4), ([1, 0, 3, 2], [71] * 4, [71] * 4, [40] * 4), ([3, -1, 3, 0], [75, 0, 80, 64], [75, 5, 80, 64], [1, 2, 3, 4]),
                 ([0, 1, 2, 3], [0, 99, 0, 99], [0, 8, -1, 99], [9, 1, 1, 60])):
        for t, x in zip((src, length, start, n), args):
            t.copy_(i32(x))
        graph.replay()
        torch.cuda.synchronize()
        h.table = plain.fork(h.table, 20, 32, args[0], args[1])
        h.refs = plain.count(h.table, 20)
        want, copies, wiped = plain.reserve(h.table, h.refs, 32, args[2], args[3])
        h.moved(copies, wiped)
        total, where, moves = plain.compact(h.table, h.refs)
        h.moved(moves)
        h.same()
        assert missing.tolist() == want and used.tolist() == [total] and moved.tolist() == where
    # eager, on a stream of its own
    with torch.cuda.stream(stream):
        h.fork([2, 2, 2, 2], [20] * 4)
        h.reserve([20] * 4, 2)
        h.compact()
    stream.synchronize()
    h.same()


def test_equal_calls_equal_results():
    rng = np.random.default_rng(10)
    for _ in range(5):
        table = random_table(rng, 50, 12, 400)
        h = Held(rng, table, 500)
        other = Held(rng, table, 500)
        for x in (h, other):
            x.fork((np.arange(50) * 7) % 50, np.arange(50) * 5)
            x.reserve(np.arange(50) * 3, 20)
            x.compact()
        assert torch.equal(h.cache.page_table, other.cache.page_table) and torch.equal(h.gpu_refs, other.gpu_refs)
