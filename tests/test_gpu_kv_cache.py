"""The paged 8-bit key / value cache on the GPU against its definition in 64 bits (kv_plain): codes, scales and values read
back have to be equal, the attention within the bound that kv_plain derives for every element."""
import numpy as np
import pytest
import torch

import kv_plain as plain
from paper_2604_03950_amd import binding as dma

pytestmark = pytest.mark.gpu
FMT = {"e4m3": dma.FMT_MXFP8_E4M3, "e5m2": dma.FMT_MXFP8_E5M2}


@pytest.fixture(scope="module", autouse=True)
def library():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dma.load()


def bf16(rng, *shape, loud=0.02):
    """bf16 values with a few loud channels, as float64."""
    x = rng.standard_normal(shape) * np.where(rng.random(shape[-1]) < loud, 14.0, 1.0)
    return torch.from_numpy(x).to(torch.bfloat16)


def table_of(rng, lens, P, extra=2, spare=1):
    """A page table for sequences of these lengths, the pages in no order; (table, pages)."""
    used = [-(-n // P) for n in lens]
    pages = sum(used) + extra
    order, wide = rng.permutation(pages), max(used + [0]) + spare
    table, at = np.full((len(lens), wide), plain.NONE, np.int32), 0
    for b, u in enumerate(used):
        table[b, :u] = order[at:at + u]
        at += u
    return table, pages


class Pair:
    """The same cache on both sides."""

    def __init__(self, rng, lens, Hkv, P, D, fmt, table=None, pages=None, fill=None):
        if table is None:
            table, pages = table_of(rng, lens, P)
        self.cpu = plain.Cache(pages, Hkv, P, D, fmt, table)
        self.gpu = dma.KVCache.empty(torch.from_numpy(table).cuda(), pages, Hkv, D, P, FMT[fmt])
        # what nothing has written: codes of every kind, NaN among them
        for mine, theirs in ((self.cpu.k, self.gpu.k_codes), (self.cpu.v, self.gpu.v_codes)):
            mine[...] = rng.integers(0, 256, mine.shape) if fill is None else fill
            theirs.copy_(torch.from_numpy(mine))
        self.gpu.k_scales.fill_(127)
        self.gpu.v_scales.fill_(127)

    def write(self, k, v, start, n=None):
        self.cpu.write(k.double().numpy(), v.double().numpy(), start, n)
        dma.dma_kv_write(self.gpu, k.cuda(), v.cuda(), i32(start), i32(n))

    def same(self):
        """Scales of all pages, codes of every place that is defined (zeros of either sign are the same)."""
        g, w = plain.grid(self.cpu.fmt), self.cpu.written
        for name, mine, theirs in (("k", self.cpu.k, self.gpu.k_codes.cpu().numpy()),
                                   ("v", self.cpu.v.transpose(0, 1, 3, 2), self.gpu.v_codes.cpu().numpy().transpose(0, 1, 3, 2))):
            mine, theirs = (g[x.transpose(0, 2, 1, 3)[w]] for x in (mine, theirs))
            np.testing.assert_array_equal(theirs, mine, err_msg=name)
        used = w.any(1)
        np.testing.assert_array_equal(self.gpu.k_scales.cpu().numpy()[used], self.cpu.ks[used])
        np.testing.assert_array_equal(self.gpu.v_scales.cpu().numpy()[used], self.cpu.vs[used])

    def attn(self, q, start, n=None, window=0, sinks=0, out=None, **kw):
        got = dma.dma_cache_attn(q.cuda() if not q.is_cuda else q, self.gpu, i32(start), i32(n), window=window, sink_tokens=sinks, out=out, **kw)
        want, bound = self.cpu.attn(q.double().cpu().numpy(), start, n, window, sinks)
        rows = np.isfinite(want)
        assert rows.any() or not (np.asarray(start) >= 0).any() or got.numel() == 0 or (n is not None and not np.asarray(n).any())
        off = np.abs(got.double().cpu().numpy() - want)[rows]
        assert not np.isnan(off).any()
        worst = (off - bound[rows]).max(initial=-1)
        assert worst <= 0, (worst, off.max(), (off / bound[rows]).max())
        return got, rows


def i32(x):
    return None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


# ------------------------------------------------------------------------------------------------------ write and read
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("P", [16, 32, 64, 128, 256])
def test_write_and_read_back(fmt, D, P):
    """A prompt of odd lengths, then pieces of one and more tokens behind it: inside a page, across borders, up to one."""
    rng = np.random.default_rng(P + D)
    B, Hkv = 4, 3
    pieces = [np.array([P + 5, 1, 2 * P, P - 1]), np.array([1, 0, 1, 1]), np.array([P - 6, 7, 3, 2 * P + 1])]
    pair = Pair(rng, sum(pieces), Hkv, P, D, fmt)
    start = np.zeros(B, int)
    for n in pieces:
        N = int(n.max()) + 2                                    # a padded batch
        pair.write(bf16(rng, B, Hkv, N, D) * 2.0 ** rng.integers(-6, 7), bf16(rng, B, Hkv, N, D) * 2.0 ** rng.integers(-6, 7), start, n)
        start = start + n
        pair.same()
    # read from the middle, with rows behind the last that stay
    first, N = start // 3, int((start - start // 3).max()) + 3
    out = [torch.full((B, Hkv, N, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    dma.dma_kv_read(pair.gpu, i32(first), n_tokens=i32(start - first), out=out)
    for b in range(B):
        k, v, there = pair.cpu.values(b, int(start[b]))
        assert there.all()
        m = int(start[b] - first[b])
        for x, o in ((k, out[0]), (v, out[1])):
            np.testing.assert_array_equal(o[b, :, :m].double().cpu().numpy(), x[:, first[b]:])
            assert (o[b, :, m:] == 7).all()


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_scale_grows_token_by_token(fmt):
    """Single tokens whose magnitudes rise and fall over 40 binades: the scale of the page grows, earlier codes are rounded
    to it, down to subnormal codes and zeros; the next page starts anew; a page written again from its start forgets."""
    rng = np.random.default_rng(8)
    P, D, Hkv = 16, 64, 2
    pair = Pair(rng, [40, 40], Hkv, P, D, fmt)
    for t, e in enumerate([0, 3, -4, 1, 9, 9, 20, -20, 21, 2, 0, 33, -60, 5, 0, 40, -10, -3, 0, 1, 30]):
        pair.write(bf16(rng, 2, Hkv, 1, D) * 2.0 ** e, bf16(rng, 2, Hkv, 1, D) * 2.0 ** -e, [t, t + 3])
        pair.same()
    pair.write(bf16(rng, 2, Hkv, 2, D), bf16(rng, 2, Hkv, 2, D), [0, 16])
    pair.same()


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_every_magnitude(fmt):
    """All bf16 magnitudes of a binade around every power of two, from subnormal to the largest, as pages of their own."""
    rng = np.random.default_rng(1)
    P, D = 16, 64
    exps = np.arange(-133, 128, 3)
    x = (1 + rng.integers(0, 128, (len(exps), 1, P, D)) / 128) * 2.0 ** exps[:, None, None, None] * rng.choice([-1, 1], (len(exps), 1, P, D))
    x = torch.from_numpy(x).to(torch.bfloat16)
    x[torch.isinf(x)] = 3.3895e38
    pair = Pair(rng, [P] * len(exps), 1, P, D, fmt)
    pair.write(x, x.flip(0), [0] * len(exps))
    pair.same()
    k, v = dma.dma_kv_read(pair.gpu, i32([0] * len(exps)), P)
    for b in range(len(exps)):
        np.testing.assert_array_equal(k[b].double().cpu().numpy(), pair.cpu.values(b, P)[0])
        np.testing.assert_array_equal(v[b].double().cpu().numpy(), pair.cpu.values(b, P)[1])


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_infinities_and_nan(fmt):
    rng = np.random.default_rng(2)
    P, D = 32, 128
    pair = Pair(rng, [P, P, P], 1, P, D, fmt)
    k, v = bf16(rng, 3, 1, P, D), bf16(rng, 3, 1, P, D)
    k[0, 0, 3, 5], k[0, 0, 4, 6], v[0, 0, 31, 127] = float("inf"), float("-inf"), float("inf")
    k[1, 0, 0, 0], v[1, 0, 7, 9] = float("nan"), float("nan")
    k[2], v[2] = 0, float("inf")
    pair.write(k, v, [0, 0, 0])
    pair.same()
    kk, _ = dma.dma_kv_read(pair.gpu, i32([0, 0, 0]), P)
    top = 1.75 * 2.0 ** (plain.E_MAX[fmt] + int(pair.cpu.ks[pair.cpu.table[0, 0], 0]) - 127)
    assert kk[0, 0, 3, 5] == top and kk[0, 0, 4, 6] == -top and torch.isnan(kk[1, 0, 0, 0]) and not kk[2].any()


def test_places_that_do_not_exist():
    """Entries without a page, positions past the table, negative starts, counts outside [0, N]: dropped, or left as they were."""
    rng = np.random.default_rng(4)
    P, D, Hkv, N = 16, 64, 2, 40
    table = np.array([[3, -1, 5], [9, 2, 1 << 30], [0, 1, 4], [6, 7, -(1 << 31)], [8, 10, 11]], np.int32)
    pair = Pair(rng, None, Hkv, P, D, "e4m3", table, 12)
    before = [t.clone() for t in (pair.gpu.k_codes, pair.gpu.v_codes)]
    start, n = [0, 20, -1, 10, (1 << 31) - 1], [99, 40, 40, -3, 40]
    pair.write(bf16(rng, 5, Hkv, N, D), bf16(rng, 5, Hkv, N, D), start, n)
    pair.same()
    kept = ~pair.cpu.written.any(1)
    assert kept.sum() == 9
    for t, was in zip((pair.gpu.k_codes, pair.gpu.v_codes), before):
        assert torch.equal(t[torch.from_numpy(kept).cuda()], was[torch.from_numpy(kept).cuda()])
    out = [torch.full((5, Hkv, N, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    dma.dma_kv_read(pair.gpu, i32(start), n_tokens=i32(n), out=out)
    for o, which in zip(out, (0, 1)):
        want = np.full((5, Hkv, N, D), 7.0)
        want[0, :, :16] = pair.cpu.values(0, 16)[which]
        want[0, :, 32:] = pair.cpu.values(0, 40)[which][:, 32:]
        want[1, :, :12] = pair.cpu.values(1, 32)[which][:, 20:]
        np.testing.assert_array_equal(o.double().cpu().numpy(), want)


# ----------------------------------------------------------------------------------------------------------- attention
def filled(rng, lens, Hkv, P, D, fmt):
    pair = Pair(rng, lens, Hkv, P, D, fmt)
    N = max(lens)
    pair.write(bf16(rng, len(lens), Hkv, N, D), bf16(rng, len(lens), Hkv, N, D), [0] * len(lens), lens)
    return pair


@pytest.mark.parametrize("fmt,D,P,Hkv,G", [("e4m3", 128, 64, 2, 4), ("e5m2", 128, 16, 1, 1), ("e4m3", 64, 32, 3, 5), ("e5m2", 64, 256, 2, 8),
                                          ("e4m3", 128, 128, 1, 16), ("e4m3", 128, 32, 1, 24)])
@pytest.mark.parametrize("lens", [[1, 2, 63, 64, 65], [200, 16, 129, 777, 1500]])
def test_single_tokens(fmt, D, P, Hkv, G, lens):
    rng = np.random.default_rng(sum(lens) + D + P)
    pair = filled(rng, lens, Hkv, P, D, fmt)
    pair.attn(bf16(rng, len(lens), Hkv * G, 1, D), np.array(lens) - 1)


@pytest.mark.parametrize("fmt,D,P,Hkv,G,N", [("e4m3", 128, 64, 2, 4, 3), ("e4m3", 64, 16, 1, 1, 17), ("e5m2", 128, 128, 2, 5, 7), ("e4m3", 128, 32, 1, 4, 33),
                                            ("e4m3", 128, 256, 1, 3, 100), ("e5m2", 64, 64, 1, 8, 65), ("e4m3", 128, 16, 2, 1, 130)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (50, 0), (40, 4), (300, 70)])
def test_several_tokens(fmt, D, P, Hkv, G, N, window, sinks):
    """Pieces of a prompt: the first (positions 0 ..), one behind a long context, padded ones, under windows too."""
    rng = np.random.default_rng(N + window + sinks)
    n = np.array([N, max(1, N - 2), 1, 0, N])
    start = np.array([0, 5, 333, 7, 401])
    pair = filled(rng, list(start + n), Hkv, P, D, fmt)
    out = torch.full((5, Hkv * G, N, D), 7.0, dtype=torch.bfloat16, device="cuda")
    got, rows = pair.attn(bf16(rng, 5, Hkv * G, N, D), start, n, window, sinks, out=out)
    behind = got.float().cpu().numpy()[~rows]
    assert got is out and behind.size and (behind == 7).all()


@pytest.mark.parametrize("window,sinks", [(1, 0), (64, 4), (1000, 0), (128, 128), (100, 5000), (1 << 30, 3), ((1 << 31) - 1, (1 << 31) - 1)])
def test_windows_of_single_tokens(window, sinks):
    rng = np.random.default_rng(window % 1000 + sinks % 7)
    lens = [1, 64, 100, 1129, 2000]
    pair = filled(rng, lens, 2, 64, 128, "e4m3")
    pair.attn(bf16(rng, 5, 8, 1, 128), np.array(lens) - 1, None, window, sinks)


@pytest.mark.parametrize("fmt,D,P,G,N", [("e4m3", 128, 64, 2, 100), ("e5m2", 128, 16, 5, 70), ("e4m3", 64, 256, 1, 257), ("e5m2", 64, 32, 4, 33)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (60, 0), (33, 70)])
def test_many_rows(fmt, D, P, G, N, window, sinks):
    """Many sequences with pieces of prompts: enough rows for the chip."""
    rng = np.random.default_rng(N + window)
    B, Hkv = 18, 4
    n = rng.integers(0, N + 1, B)
    n[:3] = N, 1, 0
    start = rng.integers(0, 200, B)
    start[:2] = 0
    start[4] = 700
    pair = filled(rng, list(start + n), Hkv, P, D, fmt)
    out = torch.full((B, Hkv * G, N, D), 7.0, dtype=torch.bfloat16, device="cuda")
    got, rows = pair.attn(bf16(rng, B, Hkv * G, N, D), start, n, window, sinks, out=out)
    assert (got.float().cpu().numpy()[~rows] == 7).all()


@pytest.mark.parametrize("fmt,D,N,G", [("e4m3", 128, 16, 2), ("e4m3", 128, 33, 1), ("e5m2", 64, 16, 4), ("e4m3", 64, 5, 13)])
@pytest.mark.parametrize("B", [9, 66])
def test_between_few_and_many_rows(B, fmt, D, N, G):
    """32, 33, 64 and 65 rows per kv head, for few and for many sequences."""
    rng = np.random.default_rng(N * G + B)
    n = rng.integers(1, N + 1, B)
    n[:2] = N
    start = rng.integers(0, 150, B)
    pair = filled(rng, list(start + n), 4, 32, D, fmt)
    pair.attn(bf16(rng, B, 4 * G, N, D), start, n)


@pytest.mark.parametrize("N,G,D,window", [(1, 4, 128, 0), (3, 4, 64, 0), (7, 8, 128, 0), (1, 16, 64, 1500), (9, 2, 128, 2000)])
def test_long_and_short_sequences_together(N, G, D, window):
    """More sequences than a workgroup has threads, a few long ones among them: shares that hold many sequences, sequences that
    take many shares, and some without tokens."""
    rng = np.random.default_rng(N + G)
    B = 300
    start = rng.integers(0, 60, B)
    start[[0, 7, 150, 299]] = 2900, 1500, 2047, 2500
    n = np.full(B, N)
    n[[3, 4, 5, 298]] = 0
    pair = filled(rng, list(start + n), 1, 64, D, "e4m3")
    pair.attn(bf16(rng, B, G, N, D), start, n, window, 3)
    pair.attn(bf16(rng, B, G, N, D), start, np.zeros(B, int), window, 3)       # nothing at all


@pytest.mark.parametrize("N", [1, 9])
def test_table_of_the_largest_capacity(N):
    """2^30 - 256 positions per sequence, more than 2^31 steps of work by the sizes alone: short sequences among -1 entries."""
    rng = np.random.default_rng(N)
    B, Hkv, P, D, wide = 64, 4, 256, 64, (1 << 22) - 1
    lens = rng.integers(N, 700, B)
    table, pages = table_of(rng, lens, P, spare=0)
    pair = Pair(rng, None, Hkv, P, D, "e4m3", table, pages)
    big = torch.full((B, wide), -1, dtype=torch.int32, device="cuda")
    big[:, :table.shape[1]] = pair.gpu.page_table
    pair.gpu = dma.KVCache(pair.gpu.k_codes, pair.gpu.v_codes, pair.gpu.k_scales, pair.gpu.v_scales, big)
    n = int(max(lens))
    pair.write(bf16(rng, B, Hkv, n, D), bf16(rng, B, Hkv, n, D), [0] * B, lens)
    pair.same()
    pair.attn(bf16(rng, B, Hkv * 2, N, D), lens - N)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("B,Hkv,G,N", [(2, 1, 4, 3), (2, 1, 2, 20), (17, 4, 2, 100)])
def test_nan_reaches_only_who_sees_it(fmt, B, Hkv, G, N):
    """A NaN key or value: NaN for the queries behind it, nothing for those before it or whose window has passed it."""
    rng = np.random.default_rng(40 + N)
    D, S = 128, 150
    pair = Pair(rng, [S] * B, Hkv, 64, D, fmt)
    k, v = bf16(rng, B, Hkv, S, D), bf16(rng, B, Hkv, S, D)
    v[0, 0, S - N + N // 2, 5] = v[0, 0, S - N + N // 2, 77] = v[1, 0, S - N, 127] = float("nan")
    k[1, 0, S - 1, 3] = float("nan")
    pair.write(k, v, [0] * B)
    pair.same()
    for window in (0, 2, 70):
        q = bf16(rng, B, Hkv * G, N, D)
        got = dma.dma_cache_attn(q.cuda(), pair.gpu, i32([S - N] * B), window=window).double().cpu().numpy()
        with np.errstate(invalid="ignore"):
            want, bound = pair.cpu.attn(q.double().numpy(), [S - N] * B, None, window)
        np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
        assert np.isnan(want).any() and not np.isnan(want).all()
        fine = ~np.isnan(want)
        assert (np.abs(got - want) <= bound)[fine].all()


def test_nothing_to_see():
    """Rows whose keys have no page give zeros; sequences without tokens keep their rows."""
    rng = np.random.default_rng(6)
    table = np.array([[-1, -1], [-1, 1], [0, -1], [2, 3]], np.int32)
    pair = Pair(rng, None, 1, 32, 64, "e4m3", table, 4)
    pair.write(bf16(rng, 4, 1, 64, 64), bf16(rng, 4, 1, 64, 64), [0] * 4)
    for N, start, window in ((1, [40, 31, 63, -1], 0), (20, [0, 20, 40, 44], 0), (20, [0, 20, 40, 44], 3), (1, [10, 33, 63, 5], 20)):
        out = torch.full((4, 4, N, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        got, rows = pair.attn(bf16(rng, 4, 4, N, 64), start, None, window, 0, out=out)
        assert not got[0].any() and (got[3] == 7).all() == (start[3] < 0)


def test_queries_past_the_table():
    """Positions that the table has no place for: the query still sees what there is."""
    rng = np.random.default_rng(16)
    table, pages = table_of(rng, [64, 64], 16, spare=0)
    pair = Pair(rng, None, 2, 16, 64, "e4m3", table, pages)
    pair.write(bf16(rng, 2, 2, 64, 64), bf16(rng, 2, 2, 64, 64), [0, 0])
    for start, window, sinks in (([63, 64], 0, 0), ([100, 70], 20, 2), ([(1 << 31) - 1, (1 << 31) - 3], 0, 0), ([(1 << 31) - 1, 1 << 30], 50, 3)):
        pair.attn(bf16(rng, 2, 4, 5, 64), start, None, window, sinks)


def test_large_and_small_scores():
    """Scores over hundreds of units in both directions, all-equal keys, zero queries."""
    rng = np.random.default_rng(12)
    pair = Pair(rng, [300, 300, 300], 1, 64, 128, "e4m3")
    k, v = bf16(rng, 3, 1, 300, 128), bf16(rng, 3, 1, 300, 128)
    k[0] *= 16
    k[1] = k[1, :, :1]
    pair.write(k, v, [0, 0, 0])
    q = bf16(rng, 3, 4, 2, 128)
    q[0] *= 8
    q[2] = 0
    pair.attn(q, [298, 298, 298])


def test_strides():
    """Views of a projection that holds q, k and v side by side, token by token; outputs of the same kind."""
    rng = np.random.default_rng(21)
    B, N, Hq, Hkv, D = 3, 37, 4, 2, 64
    pair = Pair(rng, [N] * B, Hkv, 16, D, "e4m3")
    proj = bf16(rng, B, N, Hq + 2 * Hkv, D)
    q, k, v = (t.transpose(1, 2) for t in proj.cuda().split([Hq, Hkv, Hkv], 2))
    pair.cpu.write(k.double().cpu().numpy(), v.double().cpu().numpy(), [0] * B)
    dma.dma_kv_write(pair.gpu, k, v, i32([0] * B))
    pair.same()
    out = torch.zeros((B, N, 2 * Hq, D), dtype=torch.bfloat16, device="cuda")
    pair.attn(q, [0] * B, out=out[:, :, :Hq].transpose(1, 2))
    assert not out[:, :, Hq:].any() and out[:, :, :Hq].any()
    # tokens in front of heads, batch innermost of the outer dimensions, a broadcast query
    pair.attn(bf16(rng, N, B, Hq, D).cuda().permute(1, 2, 0, 3), [0] * B)
    pair.attn(bf16(rng, 1, 1, 1, D).cuda().expand(B, Hq, 3, D), [N - 3] * B)
    back = torch.zeros((N, Hkv, B, 2, D), dtype=torch.bfloat16, device="cuda").permute(3, 2, 1, 0, 4)
    dma.dma_kv_read(pair.gpu, i32([0] * B), out=(back[0], back[1]))
    for b in range(B):
        np.testing.assert_array_equal(back[0, b].double().cpu().numpy(), pair.cpu.values(b, N)[0])
        np.testing.assert_array_equal(back[1, b].double().cpu().numpy(), pair.cpu.values(b, N)[1])


def test_offsets_past_32_bits():
    """Pages that lie more than 4 GiB into the cache."""
    rng = np.random.default_rng(31)
    P, D, Hkv = 256, 128, 8
    pages = (5 << 30) // (P * D * Hkv)
    table = np.array([[pages - 1, 0], [pages - 2, pages // 2]], np.int32)
    gpu = dma.KVCache.empty(torch.from_numpy(table).cuda(), pages, Hkv, D, P)
    small = np.array([[0, 1], [2, 3]], np.int32)
    pair = Pair(rng, None, Hkv, P, D, "e4m3", small, 4)
    k, v = bf16(rng, 2, Hkv, 300, D), bf16(rng, 2, Hkv, 300, D)
    pair.write(k, v, [0, 0])
    dma.dma_kv_write(gpu, k.cuda(), v.cuda(), i32([0, 0]))
    for a, b in zip(dma.dma_kv_read(gpu, i32([0, 0]), 300), dma.dma_kv_read(pair.gpu, i32([0, 0]), 300)):
        assert torch.equal(a, b)
    pair.gpu = gpu
    pair.attn(bf16(rng, 2, 16, 1, D), [299, 290])
    pair.attn(bf16(rng, 2, 16, 50, D), [250, 250])


def test_empty_calls():
    table = torch.zeros((0, 3), dtype=torch.int32, device="cuda")
    cache = dma.KVCache.empty(table, 2, 2, 64, 16)
    none = torch.empty((0, 2, 4, 64), dtype=torch.bfloat16, device="cuda")
    dma.dma_kv_write(cache, none, none, i32(np.zeros(0)))
    assert dma.dma_cache_attn(none, cache, i32(np.zeros(0))).shape == none.shape
    cache = dma.KVCache.empty(torch.zeros((2, 0), dtype=torch.int32, device="cuda"), 0, 2, 64, 16)      # no page at all
    x = torch.ones((2, 2, 4, 64), dtype=torch.bfloat16, device="cuda")
    dma.dma_kv_write(cache, x, x, i32([0, 0]))
    assert not dma.dma_cache_attn(x, cache, i32([0, 0])).any()
    assert not dma.dma_kv_read(cache, i32([0, 0]), 4)[0].any()
    empty = x[:, :, :0]
    dma.dma_kv_write(cache, empty, empty, i32([0, 0]))
    assert dma.dma_cache_attn(empty, cache, i32([0, 0])).numel() == 0


# ------------------------------------------------------------------------------------------------------------ together
def test_prompt_then_tokens():
    """As a server uses it: the prompt's attention from its own keys and values (every tile unquantized), its keys and values
    written, then token after token written and attended to; and the prompt's last piece through the cache as well."""
    rng = np.random.default_rng(77)
    B, Hq, Hkv, S, D, P = 2, 8, 2, 200, 128, 64
    pair = Pair(rng, [S + 6] * B, Hkv, P, D, "e4m3")
    k, v, q = bf16(rng, B, Hkv, S + 6, D), bf16(rng, B, Hkv, S + 6, D), bf16(rng, B, Hq, S + 6, D)
    prompt = dma.dma_attn_fwd(q[:, :, :S].contiguous().cuda(), k[:, :, :S].contiguous().cuda(), v[:, :, :S].contiguous().cuda(),
                              diag_band_tiles=0, hi_fmt=dma.FMT_BF16, lo_fmt=dma.FMT_BF16)
    pair.write(k[:, :, :S], v[:, :, :S], [0] * B)
    piece, _ = pair.attn(q[:, :, S - 30:S], [S - 30] * B)
    # the prompt's attention saw the same keys before their rounding to 4 significant bits: near, and not the same
    a, b = prompt[:, :, S - 30:].double(), piece.double()
    assert 1e-4 < float((a - b).norm() / a.norm()) < 0.2
    for t in range(S, S + 6):
        pair.write(k[:, :, t:t + 1], v[:, :, t:t + 1], [t] * B)
        pair.attn(q[:, :, t:t + 1], [t] * B)
    pair.same()


@pytest.mark.parametrize("fmt,P", [("e4m3", 16), ("e5m2", 64)])
def test_drafts_taken_back(fmt, P):
    """Drafted tokens are written and attended to; the next ones stand from the first refused position on, inside the same page or
    before its border, with larger and smaller elements than those they replace."""
    rng = np.random.default_rng(P)
    B, Hkv, G, D, N = 3, 2, 4, 128, 7
    start = np.array([3, P - 2, 2 * P + 5])
    table, pages = table_of(rng, [int(s) + 40 for s in start], P)
    pair = Pair(rng, None, Hkv, P, D, fmt, table, pages)
    pair.write(bf16(rng, B, Hkv, 2 * P + 5, D), bf16(rng, B, Hkv, 2 * P + 5, D), [0] * B, start)
    at = start
    for step, size in enumerate([1.0, 30.0, 0.01, 200.0]):
        pair.write(bf16(rng, B, Hkv, N, D) * size, bf16(rng, B, Hkv, N, D) * size, at)
        pair.same()
        pair.attn(bf16(rng, B, Hkv * G, N, D), at)
        at = at + np.array([0, 2, 7]) if step % 2 == 0 else at + np.array([4, 1, 3])


@pytest.mark.parametrize("N", [1, 5, 40])
def test_shared_first_pages(N):
    """Sequences that begin alike hold the same pages at the front of their table; each goes on in pages of its own."""
    rng = np.random.default_rng(N)
    B, Hkv, G, D, P = 5, 2, 4, 64, 32
    own = 3
    table = np.concatenate([np.tile(np.array([[4, 0, 7]]), (B, 1)), 8 + rng.permutation(B * own).reshape(B, own)], 1).astype(np.int32)
    pair = Pair(rng, None, Hkv, P, D, "e4m3", table, 8 + B * own)
    pair.write(bf16(rng, B, Hkv, 3 * P, D), bf16(rng, B, Hkv, 3 * P, D), [0] * B, [3 * P] + [0] * (B - 1))
    n = np.array([50, 41, 96, 40, 77])
    pair.write(bf16(rng, B, Hkv, 96, D), bf16(rng, B, Hkv, 96, D), [3 * P] * B, n)
    pair.same()
    pair.attn(bf16(rng, B, Hkv * G, N, D), 3 * P + n - N)
    pair.attn(bf16(rng, B, Hkv * G, N, D), 3 * P + n - N, None, 70, 5)


def test_graph_follows_start():
    """One decoding step (write and attention) in a graph, replayed with other tokens and positions, eager work in between."""
    rng = np.random.default_rng(5)
    B, Hq, Hkv, D, P = 3, 8, 2, 64, 16
    lens = [70, 33, 500]
    pair = filled(rng, [n + 8 for n in lens], Hkv, P, D, "e4m3")
    state = np.random.default_rng(6)
    other = Pair(state, None, Hkv, P, D, "e4m3", pair.cpu.table, pair.cpu.pages)
    for a, b in ((pair.gpu.k_codes, other.gpu.k_codes), (pair.gpu.v_codes, other.gpu.v_codes), (pair.gpu.k_scales, other.gpu.k_scales), (pair.gpu.v_scales, other.gpu.v_scales)):
        b.copy_(a)
    kv = [torch.zeros((B, Hkv, 1, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    q, start = torch.zeros((B, Hq, 1, D), dtype=torch.bfloat16, device="cuda"), i32(lens)
    out = torch.zeros_like(q)

    def step():
        dma.dma_kv_write(pair.gpu, kv[0], kv[1], start)
        dma.dma_cache_attn(q, pair.gpu, start, window=48, sink_tokens=4, out=out)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for r in range(6):
        for t in (*kv, q):
            t.copy_(bf16(rng, *t.shape) * 2.0 ** r)
        start.copy_(i32([n + r for n in lens]))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        dma.dma_kv_write(other.gpu, kv[0], kv[1], start)
        eager = dma.dma_cache_attn(q, other.gpu, start, window=48, sink_tokens=4)
        torch.cuda.synchronize()
        assert torch.equal(out, eager), r
        assert torch.equal(dma.dma_kv_read(pair.gpu, start, 1)[0], dma.dma_kv_read(other.gpu, start, 1)[0])


@pytest.mark.parametrize("N,Hq", [(1, 4), (6, 8), (40, 4)])
def test_two_graphs_with_one_workspace(N, Hq):
    """Calls whose pieces are joined by a second kernel, captured in two graphs that are given the same workspace, replayed in turn and
    with other lengths, eager calls with their own workspace in between."""
    rng = np.random.default_rng(N)
    B, Hkv, D, P = 3, 2, 128, 64
    pair = filled(rng, [3000, 1500, 100], Hkv, P, D, "e4m3")
    start = i32([2900, 1400, 50])
    need = dma.dma_cache_attn_workspace_bytes(pair.gpu, Hq, N)
    assert need > 0
    ws = torch.full((need,), 0xff, dtype=torch.uint8, device="cuda")
    qs = [bf16(rng, B, Hq, N, D).cuda() for _ in range(2)]
    outs, graphs, side = [torch.zeros_like(q) for q in qs], [], torch.cuda.Stream()
    for q, o in zip(qs, outs):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            dma.dma_cache_attn(q, pair.gpu, start, out=o, workspace=ws)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            dma.dma_cache_attn(q, pair.gpu, start, out=o, workspace=ws)
    for lens in ([2900, 1400, 50], [10, 1400, 60], [2960, 0, 0], [700, 701, 55]):
        start.copy_(i32(lens))
        for _ in range(2):
            for g, q, o in zip(graphs, qs, outs):
                o.zero_()
                torch.cuda.synchronize()
                g.replay()
                eager = dma.dma_cache_attn(q, pair.gpu, start)
                torch.cuda.synchronize()
                assert torch.equal(o, eager), lens
    pair.attn(qs[0], lens)


def test_no_page_at_all():
    """A cache without pages under a table of thousands: nothing is read, rows are zeros."""
    empty = lambda *s: torch.empty(s, dtype=torch.uint8, device="cuda")
    cache = dma.KVCache(empty(0, 2, 64, 128), empty(0, 2, 128, 64), empty(0, 2), empty(0, 2), torch.full((3, 5000), 7, dtype=torch.int32, device="cuda"))
    for N in (1, 8, 70):
        x = torch.ones((3, 4, N, 128), dtype=torch.bfloat16, device="cuda")
        out = torch.ones_like(x)
        assert not dma.dma_cache_attn(x, cache, i32([300000, 5, 0]), out=out).any()
        dma.dma_kv_write(cache, x[:, :2], x[:, 2:], i32([300000, 5, 0]))
        assert (dma.dma_kv_read(cache, i32([300000, 5, 0]), out=(out[:, :2], x[:, :2]))[1] == 1).all()


def test_equal_calls_give_equal_bits_on_any_stream():
    rng = np.random.default_rng(9)
    pair = filled(rng, [1900, 3, 700], 2, 32, 128, "e4m3")
    q, start = bf16(rng, 3, 8, 2, 128).cuda(), i32([1898, 1, 698])
    first = dma.dma_cache_attn(q, pair.gpu, start)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = []
    for s in streams * 3:
        with torch.cuda.stream(s):
            outs.append(dma.dma_cache_attn(q, pair.gpu, start))
    torch.cuda.synchronize()
    assert all(torch.equal(first, o) for o in outs)
