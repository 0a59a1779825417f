"""Which kernels serve attention behind shared prefixes, by the workspace that a call asks for.  No GPU: the sizes decide."""
import pytest

from test_kv_cache_refusals import cache, lib  # noqa: F401


def together(lib, B, groups, positions, Hkv, G, N=1, D=128, window=0, sinks=0):  # noqa: F811
    c = cache(Hkv=Hkv, D=D, page_tokens=64, max_pages=positions // 64, num_pages=1000)
    return lib.dma_cache_attn_shared_workspace_bytes(c, B, Hkv * G, N, groups, window, sinks) != lib.dma_cache_attn_workspace_bytes(c, B, Hkv * G, N, window, sinks)


# us together and by the other kernels
@pytest.mark.parametrize("B,groups,positions,Hkv,G,N,D,want", [
    (64, 1, 8704, 8, 4, 1, 128, True), (256, 1, 33536, 8, 4, 1, 128, True), (256, 64, 2176, 8, 4, 1, 128, True),       # 34, 102; 204, 1845; 106, 117
    (4096, 1, 576, 8, 4, 1, 128, True), (16384, 1, 2176, 8, 4, 1, 128, True), (16384, 1, 576, 32, 1, 1, 128, True),    # 515, 980; 4180, 6465; 5399, 15005
    (4096, 256, 2176, 8, 4, 1, 128, True), (1024, 64, 640, 8, 4, 1, 128, True),                                        # 1850, 2084; 192, 240
    (1024, 256, 640, 8, 4, 1, 128, False), (4096, 1024, 640, 8, 4, 1, 128, False), (8192, 2048, 2176, 8, 4, 1, 128, False),      # 416, 254; 5902, 1007; 24764, 6090
    (2048, 512, 2176, 1, 8, 1, 128, False), (8192, 512, 2112, 2, 4, 4, 128, False), (16384, 1, 1088, 2, 4, 8, 128, False),      # 397, 179; 3536, 1673; 7200, 1680
    (16384, 1, 2048, 1, 8, 1, 64, False), (4096, 256, 2112, 1, 8, 1, 128, False)])                                     # 1350, 534; 576, 247
def test_large_batches_and_many_groups(lib, B, groups, positions, Hkv, G, N, D, want):  # noqa: F811
    """Finding its part costs every workgroup a way through the batch and the groups: many small groups of a large batch are served as by
    dma_cache_attn, long prefixes of large groups together."""
    assert together(lib, B, groups, positions, Hkv, G, N, D) == want


def test_a_workspace_is_for_its_call(lib):  # noqa: F811
    """More groups, tokens or sequences may need less."""
    c = cache(Hkv=8, D=128, page_tokens=64, max_pages=34, num_pages=1000)
    size = lambda B=1024, N=1, groups=1: lib.dma_cache_attn_shared_workspace_bytes(c, B, 32, N, groups, 0, 0)  # noqa: E731
    assert size(groups=1024) < size(groups=1) > size(N=17) and size(B=4096, groups=1024) < size(B=256)
