"""Where the calls on the 8-bit key / value cache end: sizes beyond a launch.  No GPU: every call here ends in its checks."""
import pytest

from test_kv_cache_refusals import FAKE, UNSUPPORTED, cache, calls, lib  # noqa: F401


@pytest.mark.parametrize("pages,B,Hq,N", [(1, 1 << 23, 2, 1), (1 << 10, 1 << 21, 2, 1), (1 << 10, 1 << 20, 2, 5), (1 << 10, 1 << 18, 64, 1)])
def test_more_items_than_a_launch_holds(lib, pages, B, Hq, N):  # noqa: F811
    """Refused before anything is enqueued, and no workspace is asked for."""
    c = cache(max_pages=pages)
    assert calls(lib, c, B=B, Hq=Hq, N=N)[2] == UNSUPPORTED
    assert lib.dma_cache_attn_workspace_bytes(c, B, Hq, N, 0, 0) == 0
    # one less than the limit that the header names is not refused for its size: the missing workspace is what is looked at
    rows = -(-N * (Hq // 2) // 32)
    assert lib.dma_cache_attn_workspace_bytes(cache(max_pages=1 << 10), ((1 << 19) - 1) // (2 * rows), Hq, N, 0, 0) > 0
