"""Operators for sequences that share pages of the paged 8-bit cache: calls of real use over their range, in plain torch and
through the library.

The cache is that of ``perf/operators.py``: codes of keys [pages, Hkv, P, D] and of values [pages, Hkv, D, P], a power-of-two scale
per page and kv head for each, and a page table [B, max_pages] that names the pages of sequence b in order of position (-1: none).
Rows of the table may name the same page; refs [pages] counts the entries that do, and a page of which it says 0 is free.

  fork     row b of the table becomes the entries of row src[b] for its first length[b] positions, and nothing behind them:
           beams in their new order, samples of one prompt, drafts taken back, sequences that ended.
  reserve  the pages of positions [start[b], start[b] + n[b]) become the sequence's own, so that they can be written.  Where it has
           none, or one that others name too, it gets a free one: the r-th of all these entries, sequence by sequence, the r-th
           free page.  What the sequence holds in a shared page before start[b] is copied.  missing[b]: entries for which none was left.
  compact  the pages in use come to lie in the first places: the i-th used page behind them goes to the i-th free one among them.
  attn     q [B, Hq, N, D] bf16, token i of sequence b at position start[b] + i -> softmax(q k^T / sqrt(D)) v over the keys at and
           before its own position (window > 0: the last `window` of them and the first `sinks` positions), bf16.  The sequences of
           a group, groups[g] .. groups[g + 1] - 1, have the same pages for their first shared[g] positions.
"""
import math

import torch

own = False

FORMATS = {"e4m3": (1, torch.float8_e4m3fn, 8, 3, 7, 246), "e5m2": (3, torch.float8_e5m2, 15, 2, 15, 239)}   # id, type, e_max, mantissa bits, bias, largest scale
SCALE_MIN = 17


# ---------------------------------------------------------------------------------------------------------------- cases
def _attn_case(name, B, groups, Hq, Hkv, D, page, fmt, N, prefix, behind, ragged=False, window=0, sinks=0):
    """behind: the most positions of a sequence behind the prefix, its N new tokens among them."""
    return {"name": name, "op": "attn", "B": B, "groups": groups, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page, "fmt": fmt, "N": N, "prefix": prefix,
            "behind": behind, "ragged": ragged, "window": window, "sinks": sinks}


def _fork_case(name, B, page, context, mode):
    """mode: "beams" (every row continues one of the first half), "samples" (every group of eight rows continues its first), "ended"
    (a third of the rows end, a third lose their last 5 tokens)."""
    return {"name": name, "op": "fork", "B": B, "page": page, "context": context, "mode": mode}


def _reserve_case(name, B, Hkv, D, page, fmt, N, context, family, spare):
    """family: that many neighbouring sequences hold the same pages.  spare: free pages beyond what is asked for (below 0: too few)."""
    return {"name": name, "op": "reserve", "B": B, "Hkv": Hkv, "D": D, "page": page, "fmt": fmt, "N": N, "context": context, "family": family, "spare": spare}


def _compact_case(name, B, Hkv, D, page, fmt, pages, used, moves):
    return {"name": name, "op": "compact", "B": B, "Hkv": Hkv, "D": D, "page": page, "fmt": fmt, "pages": pages, "used": used, "moves": moves}


def listed():
    return [
        # four answers to one short prompt, sampled together: the smallest attention, latency
        _attn_case("attn_samples_4", 4, 1, 32, 8, 128, 64, "e4m3", 1, 1001, 24),
        # a serving batch behind one long instruction, its sequences of all lengths
        _attn_case("attn_batch_64", 64, 1, 32, 8, 128, 64, "e4m3", 1, 8192, 512, ragged=True),
        # drafted tokens of the sequences of several prompts, small heads, pages smaller than a tile
        _attn_case("attn_drafts_5_groups", 40, 5, 10, 5, 64, 16, "e5m2", 5, 4001, 300, ragged=True),
        # layers that look back a window and at the first tokens: the window's far end lies in the prefix for most
        _attn_case("attn_window_32", 32, 2, 40, 8, 128, 32, "e4m3", 1, 6000, 1500, ragged=True, window=4096, sinks=4),
        # a large batch behind a context of 32k
        _attn_case("attn_256_behind_32k", 256, 1, 32, 8, 128, 128, "e4m3", 1, 32768, 700, ragged=True),
        # the beams of one search put in their new order: the smallest call
        _fork_case("fork_beams_8", 8, 64, 1001, "beams"),
        # samples of many long prompts, small pages: the widest table
        _fork_case("fork_samples_256", 256, 16, 32768, "samples"),
        # a token of each of a batch: a few are at a border, eight are samples that have not parted yet
        _reserve_case("reserve_token_64", 64, 8, 128, 64, "e4m3", 1, 1500, 8, 1000),
        # prompts, page by page, from a large pool
        _reserve_case("reserve_prompts", 13, 5, 64, 32, "e5m2", 4100, 5000, 1, 40000),
        # many samples of one prompt part: each copies the page it is in
        _reserve_case("reserve_part_256", 256, 8, 128, 256, "e4m3", 1, 900, 256, 100),
        # a small cache, few moves
        _compact_case("compact_300", 9, 5, 64, 16, "e5m2", 300, 150, 40),
        # a cache of half a gigabyte and more that is to be handed on in one piece
        _compact_case("compact_4k", 64, 8, 128, 64, "e4m3", 4096, 2300, 1000),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "attn", "attn", "fork", "reserve", "reserve", "compact"])
    D = rng.choice([64, 128, 128])
    Hkv = rng.choice([1, 2, 5, 8, 32])
    page = rng.choice([16, 32, 64, 128, 256])
    fmt = rng.choice(["e4m3", "e4m3", "e5m2"])
    if op == "fork":
        c = _fork_case("", _log_int(rng, 1, 256), page, _log_int(rng, 1, 32768), rng.choice(["beams", "samples", "ended"]))
    elif op == "reserve":
        while True:
            B, N, context = _log_int(rng, 1, 256), 1 if rng.random() < 0.5 else _log_int(rng, 1, 4100), _log_int(rng, 1, 5000)
            family = rng.choice([1, 2, 8, B])
            if _reserve_pages(B, page, N, context, family) * Hkv * page * D <= 1.5e8:
                break
        c = _reserve_case("", B, Hkv, D, page, fmt, N, context, family, rng.choice([0, 5, 700, 9000, -3]))
    elif op == "compact":
        most = int(4096 * 64 * 8 * 128 / (page * Hkv * D))
        pages = _log_int(rng, 4, min(most, 30000))
        used = int(rng.uniform(0.05, 0.9) * pages) + 1
        c = _compact_case("", _log_int(rng, 1, 64), Hkv, D, page, fmt, pages, used, int(rng.random() * min(used, pages - used, 1 + pages // 4)))
    else:
        Hq = Hkv * rng.choice([1, 2, 4, 5, 8])
        while True:
            N = 1 if rng.random() < 0.6 else _log_int(rng, 1, 256)
            prefix, behind, B = _log_int(rng, 1, 32768), N + _log_int(rng, 1, 2048) - 1, _log_int(rng, 1, 256)
            if B * Hq * N * (prefix + behind) <= 2.8e8 and (prefix * 8 + B * behind) * Hkv * D <= 3e8 and prefix + behind <= 33000:
                break
        window = _log_int(rng, 1, 8192) if rng.random() < 0.3 else 0
        c = _attn_case("", B, min(rng.choice([1, 1, 2, 5, 8]), B), Hq, Hkv, D, page, fmt, N, prefix, behind, rng.random() < 0.7, window, rng.choice([0, 1, 4, 100]) if window else 0)
    del c["name"]
    return c


def _spans(case):
    """Of an attention: (start, n_tokens) of every sequence, (groups, shared).  Ragged: lengths spread by the golden ratio."""
    B, n_groups, N, P = (case[k] for k in ("B", "groups", "N", "page"))
    part = lambda i, r: (r * (i + 1)) % 1 if case["ragged"] else 1.0  # noqa: E731
    groups = [B * g // n_groups for g in range(n_groups + 1)]
    if case["ragged"] and n_groups > 1:
        groups = [0] + sorted(int(B * part(g, 0.618034)) for g in range(n_groups - 1)) + [B]
    prefix = [max(1, int(case["prefix"] * (0.3 + 0.7 * part(g, 0.754878) if n_groups > 1 else 1))) for g in range(n_groups)]
    start, tokens = [], []
    for g in range(n_groups):
        for b in range(groups[g], groups[g + 1]):
            n = max(1, int(math.ceil(N * (0.1 + 0.9 * part(b, 0.414214)))))
            behind = max(n, int(case["behind"] * (0.1 + 0.9 * part(b, 0.618034))))
            start.append(prefix[g] + behind - n)
            tokens.append(n)
    # whole pages are shared; where the prefix ends inside one, each sequence has its own copy of that
    return start, tokens, groups, [p // P * P for p in prefix]


def _reserve_spans(B, page, N, context, family):
    """(start, n_tokens) and how many leading pages of each sequence are the same for its family."""
    start, tokens, same = [], [], []
    for b in range(B):
        first = b // family * family
        length = int(context * (0.2 + 0.8 * ((0.618034 * (first + 1)) % 1)))
        alone = min(first + family, B) - first == 1
        start.append(length)
        tokens.append(max(1, int(N * (0.1 + 0.9 * ((0.414214 * (b + 1)) % 1)))) if N > 1 else 1)
        same.append(0 if alone else (length + page - 1) // page)
    return start, tokens, same


def _reserve_pages(B, page, N, context, family):
    """The most pages that the cache of a reserve case has in use behind the call."""
    start, tokens, _ = _reserve_spans(B, page, N, context, family)
    return sum((start[b] + page - 1) // page for b in range(0, B, family)) + sum(n // page + 2 for n in tokens)


def _visible(case):
    """(pairs of query and key, keys of the groups' shared parts, keys of the sequences' own parts) for one head."""
    start, tokens, groups, shared = _spans(case)
    W, K = case["window"], case["sinks"]
    pairs = common = alone = 0
    for g, S in enumerate(shared):
        seen_from = S
        for b in range(groups[g], groups[g + 1]):
            s, n = start[b], tokens[b]
            first = max(0, s - W + 1) if W else 0
            seen_from = min(seen_from, first)
            alone += s + n - max(first, S) + max(min(K, first) - S, 0)
            for p in range(s, s + n):
                lo = max(0, p - W + 1) if W else 0
                pairs += p + 1 - lo + min(K, lo)
        if groups[g + 1] > groups[g]:
            common += S - seen_from + min(K, seen_from)
    return pairs, common, alone


def work(case):
    B, P = case["B"], case["page"]
    if case["op"] == "fork":
        wide = (case["context"] + P - 1) // P + 1
        return {"bytes": 4 * (2 * B * wide + 2 * B), "flops": 0}
    Hkv, D = case["Hkv"], case["D"]
    page = 2 * Hkv * (P * D + 1)                  # bytes of one
    if case["op"] == "reserve":
        start, tokens, same = _reserve_spans(B, P, case["N"], case["context"], case["family"])
        entries = sum((s + n - 1) // P - s // P + 1 for s, n in zip(start, tokens))
        copies = sum(s % P > 0 and k > 0 for s, k in zip(start, same))
        return {"bytes": 2 * page * copies + 4 * (3 * B + 4 * entries), "flops": 0}
    if case["op"] == "compact":
        return {"bytes": 2 * page * case["moves"] + 4 * (3 * case["pages"] + 2 * case["used"]), "flops": 0}
    pairs, common, alone = _visible(case)
    _, tokens, _, _ = _spans(case)
    return {"bytes": 2 * Hkv * (common + alone) * (D + 1 / P) + 4 * sum(tokens) * case["Hq"] * D, "flops": 4 * D * case["Hq"] * pairs}


# --------------------------------------------------------------------------------------------------------------- inputs
def _needed(amax, fmt):
    """The smallest scale byte with amax <= 1.75 * 2^e_max * 2^(byte - 127), within the bytes that are used."""
    m, e = torch.frexp(amax)                                                            # amax = m * 2^e, 1/2 <= m < 1
    return (e + 126 + (m > 0.875).int() - fmt[2]).clamp(SCALE_MIN, fmt[5])


def _encode(x, scale, fmt):
    x = torch.ldexp(x, (127 - scale).float()).clamp(-1.75 * 2.0 ** fmt[2], 1.75 * 2.0 ** fmt[2])
    return x.to(fmt[1]).view(torch.uint8)


def _decode(codes, scale, fmt):
    return torch.ldexp(codes.view(fmt[1]).float(), (scale.int() - 127).float())


def _fill(s, g, pages):
    """Codes and scales of all pages."""
    c, fmt = s["case"], s["fmt"]
    Hkv, P, D = c["Hkv"], c["page"], c["D"]
    # keys have a few channels of large values, as projections of real models do
    loud = torch.where(torch.rand((Hkv, 1, D), generator=g, device="cuda") < 0.02, 14.0, 1.0)
    for name in ("k", "v"):
        x = torch.randn((pages, Hkv, P, D), generator=g, device="cuda")
        x = (x * loud if name == "k" else x.transpose(-1, -2).contiguous()).to(torch.bfloat16).float()
        scale = _needed(x.abs().amax((-1, -2)), fmt)
        s[name + "_codes"] = _encode(x, scale[..., None, None], fmt)
        s[name + "_scales"] = scale.to(torch.uint8)
        del x


def _books(s, table, refs):
    """The page table and the counts lie side by side, so that a pass that changes them begins with one copy of what they were."""
    s["book0"] = torch.cat([table.flatten(), refs]).to(torch.int32)
    s["book"] = s["book0"].clone()
    s["page_table"], s["refs"] = s["book"][:table.numel()].view(table.shape), s["book"][table.numel():]


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _count(table, pages):
    """How many entries of the table name each page."""
    named = table[table >= 0].long()
    return torch.zeros(pages, dtype=torch.int32, device="cuda").index_add_(0, named, torch.ones_like(named, dtype=torch.int32))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": dict(case), "fmt": FORMATS[case.get("fmt", "e4m3")]}
    {"attn": _prepare_attn, "fork": _prepare_fork, "reserve": _prepare_reserve, "compact": _prepare_compact}[case["op"]](s, g)
    if own:                                       # the handle of the tensors above
        from paper_2604_03950_amd import binding
        s["cache"] = binding.KVCache(s["k_codes"], s["v_codes"], s["k_scales"], s["v_scales"], s["page_table"], s["fmt"][0])
    return s


def _shuffled(pages, g):
    """The pages lie in no order, as after many sequences came and went."""
    return torch.randperm(pages, generator=g, device="cuda").to(torch.int32)


def _prepare_attn(s, g):
    c = s["case"]
    B, Hq, D, P, N = (c[k] for k in ("B", "Hq", "D", "page", "N"))
    start, tokens, groups, shared = _spans(c)
    used = [(a + n + P - 1) // P for a, n in zip(start, tokens)]
    table = torch.full((B, max(used) + 1), -1, dtype=torch.int32, device="cuda")
    pages = sum(S // P for S in shared) + sum(used) + 3
    order, at = _shuffled(pages, g), 0
    for i, S in enumerate(shared):
        table[groups[i]:groups[i + 1], :S // P] = order[at:at + S // P]
        at += S // P
        for b in range(groups[i], groups[i + 1]):
            n = used[b] - S // P
            table[b, S // P:used[b]] = order[at:at + n]
            at += n
    s.update(page_table=table, start=_i32(start), n_tokens=_i32(tokens) if c["ragged"] else None, groups=_i32(groups), shared=_i32(shared))
    _fill(s, g, pages)
    s["q"] = torch.randn((B, N, Hq, D), generator=g, device="cuda").to(torch.bfloat16).transpose(1, 2)
    s["out"] = torch.zeros((B, Hq, N, D), dtype=torch.bfloat16, device="cuda")


def _prepare_fork(s, g):
    c = s["case"]
    B, P, n = c["B"], c["page"], c["context"]
    lengths = torch.tensor([max(1, int(n * (0.5 + 0.5 * ((0.618034 * (b + 1)) % 1)))) for b in range(B)], device="cuda")
    wide = (n + P - 1) // P + 1
    used = (lengths + P - 1) // P
    pages = int(used.sum()) + 7
    filled = torch.arange(wide, device="cuda") < used[:, None]
    table = torch.full((B, wide), -1, dtype=torch.int32, device="cuda")
    table[filled] = _shuffled(pages, g)[:int(used.sum())]
    b = torch.arange(B, device="cuda")
    if c["mode"] == "beams":
        src = torch.randint(0, (B + 1) // 2, (B,), generator=g, device="cuda")
        length = lengths[src]
    elif c["mode"] == "samples":
        src = b // 8 * 8
        length = lengths[src]
    else:
        src = torch.where(b % 3 == 0, -1, b)
        length = torch.where(b % 3 == 1, (lengths - 5).clamp(min=0), lengths)
    s.update(src=src.to(torch.int32), length=length.to(torch.int32))
    _books(s, table, _count(table, pages))
    # no page is looked into: the smallest that the cache's form allows
    for name, shape in (("k", (pages, 1, P, 64)), ("v", (pages, 1, 64, P))):
        s[name + "_codes"] = torch.zeros(shape, dtype=torch.uint8, device="cuda")
        s[name + "_scales"] = torch.full((pages, 1), 127, dtype=torch.uint8, device="cuda")


def _prepare_reserve(s, g):
    c = s["case"]
    B, P, N = c["B"], c["page"], c["N"]
    start, tokens, same = _reserve_spans(B, P, N, c["context"], c["family"])
    wide = max(a + n + P - 1 for a, n in zip(start, tokens)) // P + 1
    held = [(a + P - 1) // P for a in start]
    named = sum(held[b] if not same[b] or b % c["family"] == 0 else 0 for b in range(B))
    asked = sum((a + n - 1) // P - a // P + 1 for a, n in zip(start, tokens)) - sum(a % P > 0 and not k for a, k in zip(start, same))
    pages = named + max(asked + c["spare"], 0)
    order, at = _shuffled(pages, g), 0
    table = torch.full((B, wide), -1, dtype=torch.int32, device="cuda")
    for b in range(B):
        if same[b] and b % c["family"]:
            table[b] = table[b - 1]
        else:
            table[b, :held[b]] = order[at:at + held[b]]
            at += held[b]
    s.update(start=_i32(start), n_tokens=_i32(tokens) if N > 1 else None, missing=torch.zeros(B, dtype=torch.int32, device="cuda"))
    _books(s, table, _count(table, pages))
    _fill(s, g, pages)


def _prepare_compact(s, g):
    c = s["case"]
    B, pages, used, moves = c["B"], c["pages"], c["used"], c["moves"]
    front = torch.randperm(used, generator=g, device="cuda")[:used - moves]
    back = used + torch.randperm(pages - used, generator=g, device="cuda")[:moves]
    names = torch.cat([front, back])[torch.randperm(used, generator=g, device="cuda")].to(torch.int32)
    # the pages of all sequences; where a few of them share a first page, it is named several times
    wide = (used + B - 1) // B + 2
    table = torch.full((B * (wide - 2),), -1, dtype=torch.int32, device="cuda")
    table[:used] = names
    table = torch.nn.functional.pad(table.view(B, wide - 2), (1, 1), value=-1)
    table[:(B + 1) // 2, 0] = names[0]
    table = table.contiguous()
    s.update(used=torch.zeros(1, dtype=torch.int32, device="cuda"), moved=torch.zeros(pages, dtype=torch.int32, device="cuda"))
    _books(s, table, _count(table, pages))
    _fill(s, g, pages)


# ---------------------------------------------------------------------------------------------------------- plain forms
def _cache_values(s):
    return {"page_table": s["page_table"], "refs": s["refs"], "k": s["k_codes"].view(s["fmt"][1]), "v": s["v_codes"].view(s["fmt"][1]),
            "k_scales": s["k_scales"], "v_scales": s["v_scales"]}


def _fork(s):
    table, refs, src, P = s["page_table"], s["refs"], s["src"].long(), s["case"]["page"]
    B, wide = table.shape
    keep = (torch.arange(wide, device=table.device) < ((s["length"] + P - 1) // P)[:, None]) & ((src >= 0) & (src < B))[:, None]
    new = torch.where(keep, table[src.clamp(0, B - 1)], -1)
    # counted in a place behind the pages where there is none
    change = torch.zeros(refs.numel() + 1, dtype=torch.int32, device=table.device)
    for t, by in ((new, 1), (table, -1)):
        at = torch.where((t >= 0) & (t < refs.numel()), t, refs.numel()).flatten().long()
        change.index_add_(0, at, torch.full_like(at, by, dtype=torch.int32))
    refs += change[:-1]
    table.copy_(new)
    return {"page_table": table, "refs": refs}


def _reserve(s):
    c, P, refs, table = s["case"], s["case"]["page"], s["refs"], s["page_table"]
    start = s["start"].long()
    n = torch.full_like(start, c["N"]) if s["n_tokens"] is None else s["n_tokens"].long().clamp(0, c["N"])
    j = torch.arange(table.shape[1], device=table.device)
    written = (j >= (start // P)[:, None]) & (j * P < (start + n)[:, None]) & (n > 0)[:, None]
    held = (table >= 0) & (table < refs.numel())
    count = refs[table.clamp(0, refs.numel() - 1).long()]
    b, j = torch.nonzero(written & (~held | (count > 1)), as_tuple=True)                # in order of sequence and position
    free = torch.nonzero(refs == 0)[:, 0]
    m = min(len(b), len(free))
    s["missing"].zero_().index_add_(0, b[m:], torch.ones_like(b[m:], dtype=torch.int32))
    b, j, new = b[:m], j[:m], free[:m]
    old, shared = table[b, j].long(), held[b, j]
    copy = shared & (j == start[b] // P) & (start[b] % P > 0)
    for x in (s["k_scales"], s["v_scales"]):
        x[new] = 255
    for x in (s["k_codes"], s["v_codes"], s["k_scales"], s["v_scales"]):
        x[new[copy]] = x[old[copy]]
    table[b, j] = new.to(torch.int32)
    refs[new] = 1
    refs.index_add_(0, old[shared], torch.full_like(old[shared], -1, dtype=torch.int32))
    return {"missing": s["missing"], **_cache_values(s)}


def _compact(s):
    refs, table = s["refs"], s["page_table"]
    used = refs > 0
    total = used.sum()
    place = torch.arange(refs.numel(), device=refs.device)
    from_, to = torch.nonzero(used & (place >= total))[:, 0], torch.nonzero(~used & (place < total))[:, 0]
    moved = torch.where(used, place, -1)
    moved[from_] = to
    s["moved"].copy_(moved)
    s["used"].copy_(total)
    for x in (s["k_codes"], s["v_codes"], s["k_scales"], s["v_scales"]):
        x[to] = x[from_]
    refs[to] = refs[from_]
    refs[from_] = 0
    held = (table >= 0) & (table < refs.numel())
    table.copy_(torch.where(held, moved[table.clamp(0, refs.numel() - 1).long()], table))
    return {"used": s["used"], "moved": s["moved"], **_cache_values(s)}


def _values(s, pages):
    """What pages [n, m] of the cache hold, by position: k, v [n, Hkv, m * P, D] in 32 bits."""
    page, fmt = pages.clamp(min=0).long(), s["fmt"]
    k = _decode(s["k_codes"][page], s["k_scales"][page][..., None, None], fmt).transpose(1, 2).flatten(2, 3)
    v = _decode(s["v_codes"][page], s["v_scales"][page][..., None, None], fmt).transpose(-1, -2).transpose(1, 2).flatten(2, 3)
    return k, v


def _attn(s):
    c = s["case"]
    Hq, Hkv, D, N, P, W = (c[k] for k in ("Hq", "Hkv", "D", "N", "page", "window"))
    start, tokens, groups, shared = _spans(c)
    i = torch.arange(N, device="cuda")
    count = torch.full_like(s["start"], N) if s["n_tokens"] is None else s["n_tokens"].clamp(0, N)
    for g, S in enumerate(shared):
        lo, hi = groups[g], groups[g + 1]
        if lo == hi:
            continue
        end = max(a + n for a, n in zip(start[lo:hi], tokens[lo:hi]))
        at = (s["start"][lo:hi, None] + i)[:, None, None, :, None]                      # [n, 1, 1, N, 1]
        q = s["q"][lo:hi].float().reshape(hi - lo, Hkv, -1, D)                          # rows by head and token

        def masked(x, first):
            t = torch.arange(first, first + x.shape[-1], device="cuda")
            seen = t <= at
            if W:
                seen = seen & ((t > at - W) | (t < c["sinks"]))
            return (x / math.sqrt(D)).view(hi - lo, Hkv, Hq // Hkv, N, -1).masked_fill_(~seen, -math.inf).flatten(2, 3)

        k1, v1 = _values(s, s["page_table"][lo:hi, S // P:(end + P - 1) // P])
        x1 = masked(q @ k1.transpose(-1, -2), S)
        top = x1.amax(-1, keepdim=True)
        if S:
            # the prefix: its keys and values once, for the rows of all sequences
            k0, v0 = _values(s, s["page_table"][lo:lo + 1, :S // P])
            x0 = q.transpose(0, 1).reshape(1, Hkv, -1, D) @ k0.transpose(-1, -2)
            x0 = masked(x0.view(Hkv, hi - lo, -1, S).transpose(0, 1).contiguous(), 0)
            top = torch.maximum(top, x0.amax(-1, keepdim=True))
        x1 = x1.sub_(top).exp_()
        o, total = x1 @ v1, x1.sum(-1, keepdim=True)
        if S:
            x0 = x0.sub_(top).exp_()
            o += (x0.transpose(0, 1).reshape(1, Hkv, -1, S) @ v0).view(Hkv, hi - lo, -1, D).transpose(0, 1)
            total += x0.sum(-1, keepdim=True)
        o = (o / total).view(hi - lo, Hq, N, D)
        exists = (i < count[lo:hi, None])[:, None, :, None]
        s["out"][lo:hi] = torch.where(exists, o.to(torch.bfloat16), s["out"][lo:hi])
    return s["out"]


def run(s):
    c = s["case"]
    if c["op"] != "attn":
        s["book"].copy_(s["book0"])
    if not own:
        return {"attn": _attn, "fork": _fork, "reserve": _reserve, "compact": _compact}[c["op"]](s)
    from paper_2604_03950_amd import binding
    if c["op"] == "fork":
        binding.dma_kv_fork(s["cache"], s["refs"], s["src"], s["length"])
        return {"page_table": s["page_table"], "refs": s["refs"]}
    if c["op"] == "reserve":
        binding.dma_kv_reserve(s["cache"], s["refs"], s["start"], c["N"], n_tokens=s["n_tokens"], missing=s["missing"])
        return {"missing": s["missing"], **_cache_values(s)}
    if c["op"] == "compact":
        binding.dma_kv_compact(s["cache"], s["refs"], used=s["used"], moved=s["moved"])
        return {"used": s["used"], "moved": s["moved"], **_cache_values(s)}
    return binding.dma_cache_attn_shared(s["q"], s["cache"], s["start"], s["groups"], s["shared"], n_tokens=s["n_tokens"], window=c["window"],
                                         sink_tokens=c["sinks"], out=s["out"])


# ------------------------------------------------------------------------------------------------------- in 64 bits
def _grid(fmt):
    """The 256 numbers of an 8-bit format, from its definition."""
    _, _, _, mant, bias, _ = fmt
    values = []
    for code in range(256):
        e, m = (code & 127) >> mant, code & ((1 << mant) - 1)
        x = math.ldexp(m, 1 - bias - mant) if e == 0 else math.ldexp((1 << mant) + m, e - bias - mant)
        if (fmt[1] is torch.float8_e5m2 and e == 31) or (fmt[1] is torch.float8_e4m3fn and code & 127 == 127):
            x = math.nan                                # never written by the operators
        values.append(-x if code & 128 else x)
    return torch.tensor(values, dtype=torch.float64, device="cuda")


def _held(s, moves, wiped=()):
    """The whole cache in 64 bits behind moves (from, to) of pages, and with the scales of pages set to "holds nothing"."""
    grid = _grid(s["fmt"])
    out = {}
    for name in ("k", "v"):
        codes, scales = s[name + "_codes"].clone(), s[name + "_scales"].clone()
        for p in wiped:
            scales[p] = 255
        for a, b in moves:
            codes[b] = s[name + "_codes"][a]
            scales[b] = s[name + "_scales"][a]
        out[name], out[name + "_scales"] = grid[codes.long()], scales
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "attn":
        return _exact_attn(s)
    table, refs, P = s["page_table"].tolist(), s["refs"].tolist(), case["page"]
    B, wide, pages = len(table), len(table[0]), len(refs)
    if case["op"] == "fork":
        src, length = s["src"].tolist(), s["length"].tolist()
        new = []
        for b in range(B):
            n = min(-(-max(length[b], 0) // P), wide) if 0 <= src[b] < B else 0
            new.append(table[src[b]][:n] + [-1] * (wide - n))
        refs = [0] * pages
        for row in new:
            for p in row:
                if p >= 0:
                    refs[p] += 1
        return {"page_table": _i32(new), "refs": _i32(refs)}
    if case["op"] == "reserve":
        start, tokens, _ = _reserve_spans(B, P, case["N"], case["context"], case["family"])
        free = [p for p in range(pages) if refs[p] == 0]
        before = list(refs)
        missing, moves, wiped, given = [0] * B, [], [], 0
        for b in range(B):
            for j in range(start[b] // P, (start[b] + tokens[b] - 1) // P + 1):
                p = table[b][j]
                if p >= 0 and before[p] <= 1:
                    continue
                if given == len(free):
                    missing[b] += 1
                    continue
                new = free[given]
                given += 1
                if p >= 0:
                    refs[p] -= 1
                if p >= 0 and j * P < start[b]:
                    moves.append((p, new))
                else:
                    wiped.append(new)
                refs[new] = 1
                table[b][j] = new
        return {"missing": _i32(missing), "page_table": _i32(table), "refs": _i32(refs), **_held(s, moves, wiped)}
    used = sum(r > 0 for r in refs)
    holes = [p for p in range(used) if refs[p] == 0]
    moves = list(zip([p for p in range(used, pages) if refs[p] > 0], holes))
    moved = [p if refs[p] > 0 else -1 for p in range(pages)]
    for a, b in moves:
        moved[a] = b
        refs[b], refs[a] = refs[a], 0
    table = [[moved[p] if p >= 0 else p for p in row] for row in table]
    return {"used": _i32([used]), "moved": _i32(moved), "page_table": _i32(table), "refs": _i32(refs), **_held(s, moves)}


def _exact_attn(s):
    case = s["case"]
    P, grid = case["page"], _grid(s["fmt"])
    Hq, Hkv, D = (case[n] for n in ("Hq", "Hkv", "D"))
    start, tokens, _, _ = _spans(case)
    table = s["page_table"].tolist()

    def of(codes, scales, pages, n, turn):
        x = grid[codes[pages].long()] * torch.exp2(scales[pages].double() - 127)[..., None, None]
        return (x.transpose(-1, -2) if turn else x).transpose(0, 1).flatten(1, 2)[:, :n]     # [Hkv, n, D]

    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    for b, (first, n) in enumerate(zip(start, tokens)):
        pages = table[b][:(first + n + P - 1) // P]
        kb = of(s["k_codes"], s["k_scales"], pages, first + n, False)
        vb = of(s["v_codes"], s["v_scales"], pages, first + n, True)
        at = torch.arange(first, first + n, device="cuda")[:, None]
        t = torch.arange(first + n, device="cuda")[None]
        hidden = t > at
        if case["window"]:
            hidden = hidden | ((at - t >= case["window"]) & (t >= case["sinks"]))
        for h in range(Hkv):
            G = Hq // Hkv
            q = s["q"][b, h * G:(h + 1) * G, :n].double()
            x = torch.matmul(q, kb[h].T.contiguous()) * D ** -0.5
            x = torch.softmax(x.masked_fill(hidden, -math.inf), -1)
            out[b, h * G:(h + 1) * G, :n] = torch.matmul(x, vb[h])
    return out
