"""What the calls on the 8-bit key / value cache refuse, and what they do without a launch.  No GPU: the pointers are never
followed, every call here ends in its checks."""
import ctypes
import os

import pytest
import torch

from paper_2604_03950_amd import binding as dma

FAKE = 0x1000
OK, INVALID, UNSUPPORTED = 0, -1, -2


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(dma.lib_path()):
        from paper_2604_03950_amd import build
        build.build()
    return dma.load()


def cache(**kw):
    f = dict(k_codes=FAKE, v_codes=FAKE, k_scales=FAKE, v_scales=FAKE, page_table=FAKE, num_pages=10, max_pages=4, page_tokens=64, Hkv=2,
             D=128, fmt=dma.FMT_MXFP8_E4M3)
    f.update(kw)
    return ctypes.byref(dma._Cache(**f))


def rows(data=FAKE, sb=8192, sh=4096, sn=128):
    return ctypes.byref(dma._Rows(data, sb, sh, sn))


def calls(lib, c=None, r=None, B=1, N=3, start=FAKE, n_tokens=None, Hq=4, window=0, sinks=0, ws=FAKE, ws_bytes=1 << 40):
    """The codes of the three calls."""
    c = cache() if c is None else c
    r = rows() if r is None else r
    return (lib.dma_kv_write(c, r, r, B, N, start, n_tokens, None), lib.dma_kv_read(c, r, r, B, N, start, n_tokens, None),
            lib.dma_cache_attn(c, r, r, B, Hq, N, start, n_tokens, window, sinks, ws, ws_bytes, None))


@pytest.mark.parametrize("fields,code", [
    (dict(k_codes=None), INVALID), (dict(v_codes=None), INVALID), (dict(k_scales=None), INVALID), (dict(v_scales=None), INVALID),
    (dict(page_table=None), INVALID), (dict(k_codes=FAKE + 8), INVALID), (dict(v_codes=FAKE + 4), INVALID), (dict(page_table=FAKE + 2), INVALID),
    (dict(num_pages=-1), INVALID), (dict(max_pages=-1), INVALID), (dict(page_tokens=0), INVALID), (dict(Hkv=0), INVALID), (dict(D=-64), INVALID),
    (dict(page_tokens=8), UNSUPPORTED), (dict(page_tokens=48), UNSUPPORTED), (dict(page_tokens=512), UNSUPPORTED), (dict(D=96), UNSUPPORTED),
    (dict(fmt=7), INVALID), (dict(fmt=dma.FMT_BF16), UNSUPPORTED), (dict(fmt=dma.FMT_MXFP4_E2M1), UNSUPPORTED),
    (dict(max_pages=1 << 24), UNSUPPORTED), (dict(num_pages=1 << 27), UNSUPPORTED),
])
def test_caches(lib, fields, code):
    assert calls(lib, cache(**fields)) == (code,) * 3


def test_other_arguments(lib):
    assert lib.dma_kv_write(None, rows(), rows(), 1, 1, FAKE, None, None) == INVALID
    assert lib.dma_kv_read(cache(), rows(), None, 1, 1, FAKE, None, None) == INVALID
    assert lib.dma_cache_attn(cache(), None, rows(), 1, 4, 1, FAKE, None, 0, 0, FAKE, 1 << 40, None) == INVALID
    for kw in (dict(r=rows(None)), dict(r=rows(FAKE + 8)), dict(r=rows(sb=-8)), dict(r=rows(sh=12)), dict(r=rows(sn=132)), dict(start=None),
               dict(start=FAKE + 1), dict(n_tokens=FAKE + 2), dict(B=-1), dict(N=-1)):
        assert calls(lib, **kw) == (INVALID,) * 3, kw
    assert calls(lib, N=1 << 30) == (UNSUPPORTED,) * 3
    assert calls(lib, B=(1 << 31) - 1, N=1 << 29)[:2] == (UNSUPPORTED,) * 2
    for kw in (dict(Hq=3), dict(Hq=0), dict(window=-1), dict(sinks=-1)):
        assert calls(lib, B=0, **kw) == (OK, OK, INVALID), kw
    # more query rows than are counted in 32 bits
    assert calls(lib, B=1 << 20, N=1 << 10, Hq=4, c=cache(max_pages=0))[2] == UNSUPPORTED


def test_nothing_to_do(lib):
    """No sequences or no tokens: the tensors are not looked at."""
    for kw in (dict(B=0), dict(N=0)):
        c = cache(k_codes=None, v_codes=None, k_scales=None, v_scales=None, page_table=None)
        assert calls(lib, c, rows(None), start=None, ws=None, ws_bytes=0, **kw) == (OK,) * 3
    # a table without pages: nothing can be written or read
    assert calls(lib, cache(max_pages=0, page_table=None))[:2] == (OK, OK)


def test_workspace(lib):
    f = lib.dma_cache_attn_workspace_bytes
    long = cache(max_pages=1000)
    for n in (3, 70):
        need = f(long, 1, 4, n, 0, 0)
        assert need > 0
        for ws, size in ((None, 0), (FAKE, need - 1), (FAKE + 8, need), (None, need)):
            assert calls(lib, long, N=n, ws=ws, ws_bytes=size)[2] == INVALID
    assert f(cache(max_pages=1000, k_codes=None, v_codes=None, k_scales=None, v_scales=None, page_table=None), 1, 4, 3, 0, 0) == f(long, 1, 4, 3, 0, 0)
    # nothing to join where no query can see much
    assert f(cache(), 1, 4, 3, 0, 0) == 0 == f(long, 1, 4, 3, 100, 4) and f(long, 1, 4, 3, 100, (1 << 31) - 1) == need_of(f, long)
    for args in ((None, 1, 4, 3, 0, 0), (long, 0, 4, 3, 0, 0), (long, 1, 3, 3, 0, 0), (long, 1, 4, 0, 0, 0), (long, 1, 4, 3, -1, 0), (long, 1, 4, 3, 0, -1),
                 (cache(D=96), 1, 4, 3, 0, 0), (cache(fmt=0), 1, 4, 3, 0, 0), (long, 1 << 20, 4, 1 << 10, 0, 0)):
        assert f(*args) == 0


def need_of(f, c):
    return f(c, 1, 4, 3, 0, 0)


def test_binding_takes_gpu_tensors_only():
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)
    table = torch.zeros((2, 3), dtype=torch.int32)
    with pytest.raises(ValueError):
        dma.KVCache(u8(4, 2, 16, 64), u8(4, 2, 64, 16), u8(4, 2), u8(4, 2), table)
    with pytest.raises(ValueError):
        dma.KVCache.empty(table, 4, 2, 64, 16)


class Cuda(torch.Tensor):
    """A tensor on the CPU that says it is on a GPU, for the checks that come before any call."""
    is_cuda = True
    device = torch.device("cuda", 0)

    def get_device(self):
        return 0


def on_gpu(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype).as_subclass(Cuda)


@pytest.fixture
def handle(monkeypatch):
    monkeypatch.setattr(dma, "_current_device", lambda: 0)
    monkeypatch.setattr(dma, "_raw_stream", lambda index: 0x1000 + index)

    class Never:
        def __getattr__(self, name):
            raise AssertionError("the library was called")
    u8 = lambda *s: on_gpu(*s, dtype=torch.uint8)
    c = dma.KVCache(u8(4, 2, 16, 64), u8(4, 2, 64, 16), u8(4, 2), u8(4, 2), on_gpu(3, 5, dtype=torch.int32))
    monkeypatch.setattr(dma, "load", lambda: Never())
    return c


def test_binding_checks_shapes(handle, monkeypatch):
    u8, start, kv, q = (lambda *s: on_gpu(*s, dtype=torch.uint8)), on_gpu(3, dtype=torch.int32), on_gpu(3, 2, 4, 64), on_gpu(3, 8, 4, 64)
    for args in ((u8(4, 2, 16, 64), u8(4, 2, 16, 64), u8(4, 2), u8(4, 2)), (u8(4, 2, 16, 64), u8(4, 2, 64, 16), u8(4), u8(4, 2)),
                 (u8(4, 2, 16, 64), u8(4, 2, 64, 16), u8(4, 2), u8(3, 2)), (u8(4, 2, 64), u8(4, 2, 64, 16), u8(4, 2), u8(4, 2))):
        with pytest.raises(ValueError):
            dma.KVCache(*args, on_gpu(3, 5, dtype=torch.int32))
    for bad in (on_gpu(3, 5, dtype=torch.int64), on_gpu(3, dtype=torch.int32)):
        with pytest.raises(ValueError):
            dma.KVCache(u8(4, 2, 16, 64), u8(4, 2, 64, 16), u8(4, 2), u8(4, 2), bad)
    for k, s, n in ((on_gpu(3, 1, 4, 64), start, None), (on_gpu(2, 2, 4, 64), start, None), (on_gpu(3, 2, 4, 128), start, None), (on_gpu(3, 2, 64), start, None),
                    (on_gpu(3, 2, 4, 64, dtype=torch.float32), start, None), (on_gpu(3, 2, 64, 4).transpose(2, 3), start, None),
                    (kv, on_gpu(4, dtype=torch.int32), None), (kv, on_gpu(3, dtype=torch.int64), None), (kv, start, on_gpu(2, dtype=torch.int32)),
                    (kv, start, on_gpu(3, dtype=torch.int64)), (kv, torch.zeros(3, dtype=torch.int32), None), (kv, start, torch.zeros(3, dtype=torch.int32))):
        with pytest.raises(ValueError):
            dma.dma_kv_write(handle, k, k, s, n)
        with pytest.raises(ValueError):
            dma.dma_kv_read(handle, s, n_tokens=n, out=(k, k))
    with pytest.raises(ValueError):
        dma.dma_kv_write(handle, kv, on_gpu(3, 2, 5, 64), start)
    with pytest.raises(ValueError):
        dma.dma_kv_read(handle, start)
    with pytest.raises(ValueError):
        dma.dma_kv_read(handle, start, 5, out=(kv, kv))
    for args, kw in (((on_gpu(3, 8, 64),), {}), ((on_gpu(3, 8, 4, 128),), {}), ((q,), dict(out=on_gpu(3, 8, 5, 64))), ((q,), dict(out=on_gpu(3, 8, 4, 64, dtype=torch.float32))),
                     ((q,), dict(out=on_gpu(3, 8, 4, 128)[..., ::2])), ((q,), dict(out=q, workspace=torch.zeros(9, dtype=torch.uint8))),
                     ((q,), dict(out=q, window=-1)), ((q,), dict(out=q, window=1 << 31)), ((q,), dict(out=q, sink_tokens=(1 << 32) + 1)),
                     ((torch.zeros((3, 8, 4, 64), dtype=torch.bfloat16),), {})):
        with pytest.raises(ValueError):
            dma.dma_cache_attn(*args, handle, start, **kw)
    # another device is the current one
    monkeypatch.setattr(dma, "_current_device", lambda: 1)
    for call in (lambda: dma.dma_kv_write(handle, kv, kv, start), lambda: dma.dma_kv_read(handle, start, 4), lambda: dma.dma_cache_attn(q, handle, start)):
        with pytest.raises(ValueError):
            call()
