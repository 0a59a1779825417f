"""Where the calls on the 8-bit key / value cache end: sizes beyond a launch, results that would lie on one another.  No GPU: every call here ends in its checks."""
import pytest

from test_kv_cache_refusals import FAKE, INVALID, UNSUPPORTED, cache, calls, lib, rows  # noqa: F401


@pytest.mark.parametrize("pages,B,Hq,N", [(1, 1 << 23, 2, 1), (1 << 10, 1 << 21, 2, 1), (1 << 10, 1 << 20, 2, 5), (1 << 10, 1 << 18, 64, 1)])
def test_more_items_than_a_launch_holds(lib, pages, B, Hq, N):  # noqa: F811
    """Refused before anything is enqueued, and no workspace is asked for."""
    c = cache(max_pages=pages)
    assert calls(lib, c, B=B, Hq=Hq, N=N)[2] == UNSUPPORTED
    assert lib.dma_cache_attn_workspace_bytes(c, B, Hq, N, 0, 0) == 0
    # one less than the limit that the header names is not refused for its size: the missing workspace is what is looked at
    tiles = -(-N * (Hq // 2) // 32)
    assert lib.dma_cache_attn_workspace_bytes(cache(max_pages=1 << 10), ((1 << 19) - 1) // (2 * tiles), Hq, N, 0, 0) > 0


@pytest.mark.parametrize("strides,alone", [(dict(sb=0), dict(B=1, Hkv=2, Hq=8, N=1 << 29)), (dict(sh=0), dict(B=1 << 30, Hkv=1, Hq=1, N=2)),
                                           (dict(sn=0), dict(B=1 << 30, Hkv=2, Hq=4, N=1))])
def test_results_in_one_place(lib, strides, alone):  # noqa: F811
    """Rows that are written have places of their own."""
    out = rows(**strides)
    assert lib.dma_kv_read(cache(), rows(), out, 2, 3, FAKE, None, None) == INVALID
    assert lib.dma_kv_read(cache(), out, rows(), 2, 3, FAKE, None, None) == INVALID
    assert lib.dma_cache_attn(cache(), rows(), out, 2, 4, 3, FAKE, None, 0, 0, FAKE, 1 << 40, None) == INVALID
    # a stride says nothing where there is one row to step over: these sizes are refused by what is checked after the rows
    assert lib.dma_cache_attn(cache(Hkv=alone["Hkv"]), rows(), out, alone["B"], alone["Hq"], alone["N"], FAKE, None, 0, 0, FAKE, 1 << 40, None) == UNSUPPORTED
