"""The paged 8-bit key / value cache and its attention from their definition, in 64 bits on the CPU (numpy).

Pages hold code numbers (uint8) and E8M0 bytes as the library's do; nothing here shares code with it."""
import math

import numpy as np

E_MAX = {"e4m3": 8, "e5m2": 15}
MANT = {"e4m3": 3, "e5m2": 2}
SCALE_MIN = 17
NONE = -1


def grid(fmt):
    """The value of every code; NaN where the code is none or an infinity."""
    mant = MANT[fmt]
    bias = (1 << (6 - mant)) - 1
    out = np.empty(256)
    for code in range(256):
        e, m = (code & 127) >> mant, code & ((1 << mant) - 1)
        x = m * 2.0 ** (1 - bias - mant) if e == 0 else ((1 << mant) + m) * 2.0 ** (e - bias - mant)
        if (code & 127) > (0x7e if fmt == "e4m3" else 0x7b):
            x = math.nan
        out[code] = -x if code & 128 else x
    return out


def encode(x, fmt):
    """Nearest code of every |x| <= 1.75 * 2^e_max, ties to the even one; NaN -> 0x7f."""
    g = grid(fmt)
    pos = g[:128][np.isfinite(g[:128])]
    a = np.where(np.isnan(x), 0.0, np.abs(x))
    assert a.max(initial=0) <= pos[-1]
    up = np.clip(np.searchsorted(pos, a, side="left"), 1, len(pos) - 1)
    below, above = a - pos[up - 1], pos[up] - a
    code = np.where((above < below) | ((above == below) & (up % 2 == 0)), up, up - 1)
    code = np.where(np.isnan(x), 0x7f, code)
    return (code | (np.signbit(x) * 128)).astype(np.uint8)


def needed(amax, fmt):
    """Smallest scale byte that holds amax, found by trying them."""
    top = 254 - E_MAX[fmt]
    for s in range(SCALE_MIN, top):
        if amax <= 1.75 * 2.0 ** (E_MAX[fmt] + s - 127):
            return s
    return top


class Cache:
    def __init__(self, pages, Hkv, P, D, fmt, table, fill=0):
        self.k = np.full((pages, Hkv, P, D), fill, np.uint8)
        self.v = np.full((pages, Hkv, D, P), fill, np.uint8)
        self.ks = np.full((pages, Hkv), 127, np.uint8)
        self.vs = np.full((pages, Hkv), 127, np.uint8)
        self.table, self.fmt, self.P, self.Hkv, self.pages = np.asarray(table), fmt, P, Hkv, pages
        self.written = np.zeros((pages, P), bool)            # places whose content is defined

    def place(self, b, pos):
        j = pos // self.P
        if pos < 0 or j >= self.table.shape[1] or not 0 <= self.table[b, j] < self.pages:
            return None
        return self.table[b, j], pos % self.P

    def write(self, k, v, start, n_tokens=None):
        """k, v: float64 [B, Hkv, N, D]."""
        B, _, N, _ = k.shape
        for b in range(B):
            n = N if n_tokens is None else min(max(int(n_tokens[b]), 0), N)
            if start[b] < 0 or n == 0:
                continue
            for j in range(int(start[b]) // self.P, (int(start[b]) + n - 1) // self.P + 1):
                at = self.place(b, j * self.P)
                if at is None:
                    continue
                page = at[0]
                lo, hi = max(int(start[b]) - j * self.P, 0), min(int(start[b]) + n - j * self.P, self.P)
                i0 = j * self.P + lo - int(start[b])
                for h in range(self.Hkv):
                    for x, codes, scales in ((k, self.k[page, h], self.ks), (v, self.v[page, h].T, self.vs)):
                        new = x[b, h, i0:i0 + hi - lo]
                        fin = np.abs(new[np.isfinite(new)])
                        s = needed(fin.max(initial=0), self.fmt)
                        if lo:
                            old = int(scales[page, h])
                            if s > old:
                                g = grid(self.fmt)[codes[:lo]]
                                codes[:lo] = encode(g * 2.0 ** (old - s), self.fmt)
                            s = max(s, old)
                        top = 1.75 * 2.0 ** E_MAX[self.fmt]
                        codes[lo:hi] = encode(np.clip(new * 2.0 ** (127 - s), -top, top), self.fmt)
                        scales[page, h] = s
                self.written[page, lo:hi] = True
                self.written[page, hi:] = False

    def values(self, b, n):
        """k, v float64 [Hkv, n, D] and whether each position exists, of positions 0 .. n - 1."""
        g, D = grid(self.fmt), self.k.shape[3]
        k, v, there = np.zeros((self.Hkv, n, D)), np.zeros((self.Hkv, n, D)), np.zeros(n, bool)
        for t in range(n):
            at = self.place(b, t)
            if at is None:
                continue
            page, u = at
            there[t] = True
            k[:, t] = g[self.k[page, :, u]] * 2.0 ** (self.ks[page].astype(float) - 127)[:, None]
            v[:, t] = g[self.v[page, :, :, u]] * 2.0 ** (self.vs[page].astype(float) - 127)[:, None]
        return k, v, there

    def attn(self, q, start, n_tokens=None, window=0, sinks=0):
        """q: float64 [B, Hq, N, D] -> (out, bound): out NaN in rows that do not exist, and how far a bf16 result may be off.

        The bound counts: the result's rounding to bf16, half a step of 2^-8 of itself; the probabilities' rounding to bf16, half
        a step |d_t| <= 2^-8 each.  The sum that divides adds the rounded ones, so sum p_t (1 + d_t) v_t / sum p_t (1 + d_t) - o =
        sum p_t d_t (v_t - o) / sum p_t (1 + d_t), at most 2^-8 (1 + 2^-8) of the probability-weighted mean of |v| plus |o|; the binary32 scores, whose sums of D products are off by at
        most (D + 4) * 2^-24 of the sum of magnitudes (products of bf16 are exact; the factor log2(e) / sqrt(D), the subtraction of the
        maximum and their rounding are the 4), twice, as the row's sum divides; and the binary32 sums over n keys, exp2 and the
        division, at most (n + 32) * 2^-24 of that mean, twice.  Differences between hardware exp2 and the exact one (2 units of
        2^-23) are within the 32.  Below 2^-126 numbers may become zero: a result, 2^-126; and an exp2, of a probability or of the
        factor that brings sums of them (each at most 2^11, against a maximum that may lag by as much) to another maximum, where the
        largest weighs 1 at least: 2^-126 * 2^11 of every |v|."""
        B, Hq, N, D = q.shape
        out, bound = np.full(q.shape, np.nan), np.zeros(q.shape)
        for b in range(B):
            n = N if n_tokens is None else min(max(int(n_tokens[b]), 0), N)
            if start[b] < 0 or n == 0:
                continue
            L = min(int(start[b]) + n, self.table.shape[1] * self.P)
            k, v, there = self.values(b, L)
            t = np.arange(L)
            for i in range(n):
                p = int(start[b]) + i
                seen = there & (t <= p)
                if window:
                    seen &= (t > p - window) | (t < sinks)
                for h in range(Hq):
                    if not seen.any():
                        out[b, h, i] = 0
                        continue
                    kk, vv = k[h // (Hq // self.Hkv)][seen], v[h // (Hq // self.Hkv)][seen]
                    x = kk @ q[b, h, i] / math.sqrt(D)
                    mag = (np.abs(kk) @ np.abs(q[b, h, i]) / math.sqrt(D)).max()
                    w = np.exp(x - x.max())
                    w /= w.sum()
                    out[b, h, i] = w @ vv
                    mean = w @ np.abs(vv)
                    bound[b, h, i] = (2 ** -8 * (2 + 2 ** -8) * np.abs(out[b, h, i]) + mean * (2 ** -8 * (1 + 2 ** -8) + 2 * (D + 4) * 2 ** -24 * mag
                                      + 2 * (seen.sum() + 32) * 2 ** -24) + 2.0 ** -126 + 2.0 ** -115 * np.abs(vv).sum(0))
        return out, bound
