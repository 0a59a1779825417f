"""Attention as counting.  With queries of zeros every key that is seen weighs the same, and with values of one in a single channel
of each position, channel d of the result is the number of keys seen there over the number of all: a key that is left out or
taken twice shows by one in a count of a few dozen, at any length."""
import numpy as np


def channel(t, D, odd):
    """The channel of position t's value: t % D, or one that moves on with every D positions, so that a key taken in the place of one D
    positions away shows in the other of the two."""
    return (t + t // D * odd) % D


def counts(D, p, window=0, sinks=0, seen=None):
    """For the query at position p: the keys seen in every channel, [2, D] for both patterns, and all of them.  seen: which of the positions
    0 .. p, in the place of the definition."""
    t = np.arange(p + 1)
    if seen is None:
        seen = (t > p - window) | (t < sinks) if window else np.ones(p + 1, bool)
    return np.stack([np.bincount(channel(t[seen], D, odd), minlength=D) for odd in (0, 1)]), int(seen.sum())


def wrong(got, count, n):
    """Where got (bf16 as float64, [2, D]) is not count / n.  Zero scores give probabilities of one, and sums of ones are exact
    in binary32; what is rounded is the quotient: 1 / n and its product with the sum, 2^-22 of it, and the result to bf16, half
    a step of 2^-8 of itself."""
    want = count / n
    return np.abs(got - want) > want * (2.0 ** -8 + 2.0 ** -22)
