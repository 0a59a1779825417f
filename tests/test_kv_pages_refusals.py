"""What the calls on shared pages refuse, and what they do without a launch.  No GPU: the pointers are never followed."""
import pytest

import kv_pages_plain as plain
from paper_2604_03950_amd import binding as dma
from test_kv_cache_refusals import FAKE, INVALID, OK, UNSUPPORTED, cache, handle, lib, on_gpu, rows  # noqa: F401


def fork(lib, c=None, refs=FAKE, B=2, src=FAKE, length=FAKE):
    return lib.dma_kv_fork(cache() if c is None else c, refs, B, src, length, None)


def reserve(lib, c=None, refs=FAKE, B=2, N=3, start=FAKE, n=None, missing=FAKE, ws=FAKE, size=1 << 40):
    return lib.dma_kv_reserve(cache() if c is None else c, refs, B, N, start, n, missing, ws, size, None)


def compact(lib, c=None, refs=FAKE, B=2, used=FAKE, moved=FAKE, ws=FAKE, size=1 << 40):
    return lib.dma_kv_compact(cache() if c is None else c, refs, B, used, moved, ws, size, None)


def shared(lib, c=None, r=None, o=None, B=2, Hq=4, N=1, start=FAKE, n=None, groups=1, first=FAKE, common=FAKE, window=0, sinks=0, ws=FAKE, size=1 << 40):
    r = rows() if r is None else r
    return lib.dma_cache_attn_shared(cache() if c is None else c, r, r if o is None else o, B, Hq, N, start, n, groups, first, common, window, sinks, ws, size, None)


@pytest.mark.parametrize("fields,code", [
    (dict(k_codes=None), INVALID), (dict(v_codes=None), INVALID), (dict(k_scales=None), INVALID), (dict(v_scales=None), INVALID), (dict(page_table=None), INVALID),
    (dict(k_codes=FAKE + 8), INVALID), (dict(page_table=FAKE + 2), INVALID), (dict(num_pages=-1), INVALID), (dict(max_pages=-1), INVALID), (dict(Hkv=0), INVALID),
    (dict(page_tokens=48), UNSUPPORTED), (dict(D=96), UNSUPPORTED), (dict(fmt=7), INVALID), (dict(fmt=dma.FMT_MXFP4_E2M1), UNSUPPORTED),
    (dict(max_pages=1 << 24), UNSUPPORTED), (dict(num_pages=1 << 27), UNSUPPORTED)])
def test_caches(lib, fields, code):
    assert [f(lib, cache(**fields)) for f in (fork, reserve, compact, shared)] == [code] * 4


def test_other_arguments(lib):
    for kw in (dict(refs=None), dict(refs=FAKE + 2), dict(src=None), dict(src=FAKE + 1), dict(length=FAKE + 2), dict(B=-1)):
        assert fork(lib, **kw) == INVALID, kw
    assert fork(lib, B=8193) == UNSUPPORTED
    for kw in (dict(refs=None), dict(refs=FAKE + 2), dict(start=None), dict(start=FAKE + 2), dict(n=FAKE + 1), dict(missing=None), dict(missing=FAKE + 2), dict(B=-1), dict(N=-1),
               dict(ws=None), dict(ws=FAKE + 2), dict(size=15)):
        assert reserve(lib, **kw) == INVALID, kw
    assert reserve(lib, N=1 << 30) == UNSUPPORTED and reserve(lib, cache(max_pages=1 << 20), B=1 << 20, N=1 << 26) == UNSUPPORTED
    for kw in (dict(refs=None), dict(refs=FAKE + 2), dict(used=None), dict(used=FAKE + 2), dict(moved=None), dict(moved=FAKE + 2), dict(ws=None), dict(ws=FAKE + 4), dict(size=47), dict(B=-1)):
        assert compact(lib, **kw) == INVALID, kw
    for kw in (dict(r=rows(None)), dict(r=rows(sh=12)), dict(r=rows(sb=-8)), dict(o=rows(sb=0)), dict(o=rows(sh=0)), dict(start=None), dict(n=FAKE + 2), dict(B=-1), dict(N=-1), dict(Hq=3),
               dict(Hq=0), dict(window=-1), dict(sinks=-1), dict(groups=-1), dict(first=None), dict(first=FAKE + 2), dict(common=None), dict(common=FAKE + 1)):
        assert shared(lib, **kw) == INVALID, kw
    assert shared(lib, groups=(1 << 24) + 1) == UNSUPPORTED == shared(lib, cache(max_pages=0), B=1 << 20, N=1 << 10) == shared(lib, N=1 << 30)


def test_nothing_to_do(lib):
    """No sequences or no tokens: the tensors are not looked at."""
    c = cache(k_codes=None, v_codes=None, k_scales=None, v_scales=None, page_table=None)
    assert fork(lib, c, None, 0, None, None) == OK == compact(lib, c, None, 0, None, None, None, 0)
    for kw in (dict(B=0), dict(N=0)):
        assert reserve(lib, c, None, start=None, missing=None, ws=None, size=0, **kw) == OK
        assert shared(lib, c, rows(None), start=None, first=None, common=None, ws=None, size=0, **kw) == OK
    # a table without columns has nothing to take over
    assert fork(lib, cache(max_pages=0, page_table=None)) == OK


def test_workspaces(lib):
    f = lib.dma_kv_reserve_workspace_bytes
    assert f(cache(), 2, 3) == 2 * 2 * 4 and f(cache(), 5, 64) == 5 * 2 * 4 and f(cache(), 5, 1000) == 5 * 4 * 4 and f(cache(), 7, 1) == 7 * 4
    assert f(cache(), 0, 3) == f(cache(), 3, 0) == f(None, 1, 1) == f(cache(D=96), 1, 1) == f(cache(max_pages=0), 1, 1) == 0
    g = lib.dma_kv_compact_workspace_bytes
    assert g(cache()) == 48 and g(cache(num_pages=0)) == 8 and g(None) == 0
    h = lib.dma_cache_attn_shared_workspace_bytes
    long = cache(max_pages=1000)
    need = h(long, 4, 8, 1, 1, 0, 0)
    if need:
        for ws, size in ((None, 0), (FAKE, need - 1), (FAKE + 8, need), (None, need)):
            assert shared(lib, long, B=4, Hq=8, ws=ws, size=size) == INVALID
    for args in ((None, 1, 4, 3, 1, 0, 0), (long, 0, 4, 3, 1, 0, 0), (long, 1, 3, 3, 1, 0, 0), (long, 1, 4, 0, 1, 0, 0), (long, 1, 4, 3, -1, 0, 0), (long, 1, 4, 3, 1, -1, 0),
                 (long, 1, 4, 3, 1, 0, -1), (cache(D=96), 1, 4, 3, 1, 0, 0), (long, 1 << 20, 4, 1 << 10, 1, 0, 0), (long, 1, 4, 3, (1 << 24) + 1, 0, 0)):
        assert h(*args) == 0


def test_binding_checks_shapes(handle, monkeypatch):  # noqa: F811
    import torch
    i32 = lambda *s: on_gpu(*s, dtype=torch.int32)  # noqa: E731
    refs, three, q = i32(4), i32(3), on_gpu(3, 8, 4, 64)
    for bad in (i32(5), on_gpu(4, dtype=torch.int64), torch.zeros(4, dtype=torch.int32), i32(8)[::2]):
        for call in (lambda: dma.dma_kv_fork(handle, bad, three), lambda: dma.dma_kv_reserve(handle, bad, three, 1), lambda: dma.dma_kv_compact(handle, bad)):
            with pytest.raises(ValueError):
                call()
    for bad in (i32(2), on_gpu(3, dtype=torch.int64), torch.zeros(3, dtype=torch.int32), i32(3, 1)):
        for call in (lambda: dma.dma_kv_fork(handle, refs, bad), lambda: dma.dma_kv_fork(handle, refs, three, bad), lambda: dma.dma_kv_reserve(handle, refs, bad, 1),
                     lambda: dma.dma_kv_reserve(handle, refs, three, 1, bad), lambda: dma.dma_kv_reserve(handle, refs, three, 1, missing=bad),
                     lambda: dma.dma_cache_attn_shared(q, handle, bad, i32(2), i32(1)), lambda: dma.dma_cache_attn_shared(q, handle, three, i32(2), i32(1), bad)):
            with pytest.raises(ValueError):
                call()
    for call in (lambda: dma.dma_kv_compact(handle, refs, used=i32(2), moved=i32(4)), lambda: dma.dma_kv_compact(handle, refs, used=i32(1), moved=i32(3)),
                 lambda: dma.dma_kv_reserve(handle, refs, three, 1 << 31, missing=three),
                 lambda: dma.dma_kv_reserve(handle, refs, three, 1, missing=three, workspace=torch.zeros(64, dtype=torch.uint8)),
                 lambda: dma.dma_kv_reserve(handle, refs, three, 1, missing=three, workspace=on_gpu(64, dtype=torch.int32))):
        with pytest.raises(ValueError):
            call()
    for args, kw in (((i32(2), i32(2)), {}), ((i32(3), i32(1)), {}), ((i32(2), i32(1, 1)), {}), ((on_gpu(2, dtype=torch.int64), i32(1)), {}),
                     ((torch.zeros(2, dtype=torch.int32), i32(1)), {}), ((i32(2), i32(1)), dict(window=-1)), ((i32(2), i32(1)), dict(window=1 << 31)),
                     ((i32(2), i32(1)), dict(sink_tokens=1 << 31)), ((i32(2), i32(1)), dict(out=on_gpu(3, 8, 5, 64))),
                     ((i32(2), i32(1)), dict(workspace=torch.zeros(9, dtype=torch.uint8)))):
        with pytest.raises(ValueError):
            dma.dma_cache_attn_shared(q, handle, three, *args, **{"out": q, **kw})
    for bad in (on_gpu(3, 8, 64), on_gpu(3, 8, 4, 128), on_gpu(2, 8, 4, 64), torch.zeros((3, 8, 4, 64), dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            dma.dma_cache_attn_shared(bad, handle, three, i32(2), i32(1), out=q)
    empty = dma.KVCache(handle.k_codes, handle.v_codes, handle.k_scales, handle.v_scales, i32(0, 5))
    with pytest.raises(ValueError):
        dma.dma_kv_compact(empty, refs, used=i32(1), moved=i32(4))
    monkeypatch.setattr(dma, "_current_device", lambda: 1)     # another device is the current one
    for call in (lambda: dma.dma_kv_fork(handle, refs, three), lambda: dma.dma_kv_reserve(handle, refs, three, 1), lambda: dma.dma_kv_compact(handle, refs),
                 lambda: dma.dma_cache_attn_shared(q, handle, three, i32(2), i32(1))):
        with pytest.raises(ValueError):
            call()


def test_the_definition():
    """kv_pages_plain by hand."""
    assert plain.fork([[1, 2, -1], [3, -1, -1]], 5, 16, [1, 0], [20, 17]) == [[3, -1, -1], [1, 2, -1]]
    assert plain.fork([[1, 2, 7], [3, 4, 0]], 5, 16, [0, 0], [48, 16]) == [[1, 2, -1], [1, -1, -1]]
    assert plain.fork([[1, 2], [3, 4]], 5, 16, [-1, 2]) == [[-1, -1], [-1, -1]]
    table, refs = [[2, -1], [2, -1], [4, -1]], [0, 0, 2, 0, 1]
    assert plain.reserve(table, refs, 16, [5, 16, 3], [1, 1, 1]) == ([0, 0, 0], [(2, 0)], [1])
    assert table == [[0, -1], [2, 1], [4, -1]] and refs == [1, 1, 1, 0, 1]
    assert plain.reserve(table, refs, 16, [16, 0, 16], [99, 0, 1]) == ([0, 0, 1], [], [3])
    table, refs = [[5, 1], [5, -1]], [0, 1, 0, 0, 0, 2]
    assert plain.compact(table, refs) == (2, [-1, 1, -1, -1, -1, 0], [(5, 0)]) and table == [[0, 1], [0, -1]] and refs == [2, 1, 0, 0, 0, 0]
