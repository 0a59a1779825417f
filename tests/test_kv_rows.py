"""The definition of the attention over the cache, all rows of a sequence at once, against the one that goes row by row (CPU)."""
import numpy as np
import pytest

import kv_plain as plain
import kv_rows


@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 0), (9, 30)])
@pytest.mark.parametrize("fmt,P,D,Hkv,G,N", [("e4m3", 16, 64, 2, 3, 4), ("e5m2", 32, 64, 1, 1, 1)])
def test_same_as_row_by_row(fmt, P, D, Hkv, G, N, window, sinks):
    rng = np.random.default_rng(P + N + window)
    lens = [90, 40, 7, 100, 33]
    table = rng.permutation(5 * 8).reshape(5, 8).astype(np.int32)
    table[0, 2], table[3, 1], table[4] = -1, 99, -1
    cache = plain.Cache(40, Hkv, P, D, fmt, table)
    cache.write(rng.standard_normal((5, Hkv, 100, D)), rng.standard_normal((5, Hkv, 100, D)), [0] * 5, lens)
    cache.v[table[1, 0], 0, 5, 3] = cache.k[table[3, 2 if P == 16 else 0], Hkv - 1, 4, 9] = 0x7f
    q = rng.standard_normal((5, Hkv * G, N, D))
    start, n = np.array(lens) - N, np.array([N, N, max(N - 1, 1), N, N])
    start[2] = -1
    with np.errstate(invalid="ignore"):
        want, bound = cache.attn(q, start, n, window, sinks)
    got, mine, exists = kv_rows.attn(cache, q, start, n, window, sinks)
    assert np.isnan(want).any() and not exists[2].any() and exists[4, :n[4]].all()
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
    np.testing.assert_allclose(got, want, rtol=1e-12, atol=1e-14)
    fine = ~np.isnan(want)
    np.testing.assert_allclose(mine[fine], bound[fine], rtol=1e-9)
