"""The counting of kv_counts finds a key too few or too many wherever a kernel could lose one (on the CPU, the mistake planted in
what is counted)."""
import numpy as np
import pytest
import torch

from kv_counts import counts, wrong


def bf16(x):
    return torch.from_numpy(x).to(torch.bfloat16).double().numpy()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("p,window,sinks", [(999, 0, 0), (1300, 0, 0), (4000, 0, 0), (3000, 700, 70), (4000, 1300, 5), (4000, 4001, 3)])
def test_one_key_shows(D, p, window, sinks):
    count, n = counts(D, p, window, sinks)
    assert not wrong(bf16(count / n), count, n).any()
    t = np.arange(p + 1)
    seen = (t > p - window) | (t < sinks) if window else np.ones(p + 1, bool)
    edges = {0, 63, 64, 65, 127, 128, 511, 512, p - 1, p, sinks - 1, sinks, p - window, p - window + 1}
    for at in (e for e in edges if 0 <= e <= p):
        other = seen.copy()
        other[at] = not other[at]                              # dropped, or seen too much
        bad, m = counts(D, p, seen=other)
        assert wrong(bf16(bad / m), count, n).any(1).all(), at
        if seen[at]:                                           # twice
            assert wrong(bf16((2 * count - bad) / (n + 1)), count, n).any(1).all(), at
            if at + D <= p and seen[at + D]:                   # in the place of another: in one pattern at least
                without = counts(D, p, seen=np.where(t == at + D, ~seen, seen))[0]
                assert wrong(bf16((without + count - bad) / n), count, n).any(), at
