"""Attention over the cache from its definition in 64 bits, all rows of a sequence at once: what kv_plain.Cache.attn computes row by row, for
batches that would take it minutes.  Its bound too, whose derivation stands there."""
import math

import numpy as np
import torch

import kv_plain as plain


def sequence(cache, b, n):
    """k, v float64 [Hkv, n, D] and whether each position exists, of positions 0 .. n - 1 of sequence b of a kv_plain.Cache."""
    t = np.arange(n)
    j = t // cache.P
    page = np.where(j < cache.table.shape[1], cache.table[b, np.minimum(j, cache.table.shape[1] - 1)], -1)
    there = (page >= 0) & (page < cache.pages)
    page, g = np.where(there, page, 0), plain.grid(cache.fmt)
    k = g[cache.k[page, :, t % cache.P]] * 2.0 ** (cache.ks[page].astype(float) - 127)[:, :, None]
    v = g[cache.v[page, :, :, t % cache.P]] * 2.0 ** (cache.vs[page].astype(float) - 127)[:, :, None]
    k[~there], v[~there] = 0, 0
    return k.transpose(1, 0, 2), v.transpose(1, 0, 2), there


def attn(cache, q, start, n_tokens=None, window=0, sinks=0):
    """q: float64 [B, Hq, N, D] -> (out, bound, exists): out and bound as kv_plain's, and which rows exist, [B, N]."""
    B, Hq, N, D = q.shape
    G = Hq // cache.Hkv
    out, bound, exists = np.full(q.shape, np.nan), np.zeros(q.shape), np.zeros((B, N), bool)
    for b in range(B):
        n = N if n_tokens is None else min(max(int(n_tokens[b]), 0), N)
        if start[b] < 0 or n == 0:
            continue
        exists[b, :n] = True
        L = min(int(start[b]) + n, cache.table.shape[1] * cache.P)
        k, v, there = (torch.from_numpy(np.ascontiguousarray(x)) for x in sequence(cache, b, L))
        p, t = int(start[b]) + torch.arange(n)[:, None], torch.arange(L)[None]
        seen = there & (t <= p)
        if window:
            seen &= (t > p - window) | (t < sinks)
        seen = seen.repeat(G, 1)                                   # [G * n, L], rows head by head
        rows = torch.from_numpy(np.ascontiguousarray(q[b, :, :n])).reshape(cache.Hkv, G * n, D)
        # a NaN of a key goes to the scores of its position alone, one of a value is put back below
        bad_k, bad_v = torch.isnan(k).any(-1), torch.isnan(v)
        x = rows @ torch.nan_to_num(k).transpose(1, 2).contiguous() / math.sqrt(D)
        mag = (rows.abs() @ torch.nan_to_num(k).abs().transpose(1, 2).contiguous() / math.sqrt(D)).masked_fill(~seen, 0).amax(-1, keepdim=True)
        some = seen.any(-1)[None, :, None]
        w = torch.exp(x.masked_fill(~seen, -math.inf) - x.masked_fill(~seen, -math.inf).amax(-1, keepdim=True))
        w = torch.where(some, w / w.sum(-1, keepdim=True), torch.zeros(()).double())
        clean = torch.nan_to_num(v)
        o, mean = w @ clean, w @ clean.abs()
        hit = (seen.double() @ bad_v.double() > 0) | (seen[None] & bad_k[:, None]).any(-1, keepdim=True)
        o = o.masked_fill(hit, math.nan)
        count = seen.sum(-1)[None, :, None]
        e = (2 ** -8 * (2 + 2 ** -8) * o.abs() + mean * (2 ** -8 * (1 + 2 ** -8) + 2 * (D + 4) * 2 ** -24 * mag + 2 * (count + 32) * 2 ** -24) + 2.0 ** -126
             + 2.0 ** -115 * (seen.double() @ clean.abs()))
        out[b, :, :n] = o.reshape(Hq, n, D).numpy()
        bound[b, :, :n] = torch.where(some, e, torch.zeros(()).double()).reshape(Hq, n, D).numpy()
    return out, bound, exists
