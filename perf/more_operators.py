"""The operators of a cache held in 8 bits, and of pages that requests share, as cases to be timed and compared, with their plain forms.

A case is one pass; "op" names it:

  "append"   new keys and values into a cache held in 8 bits, and the values that their blocks then hold (`cache.sagebwd_cache_append`, `..._read`)
  "attend"   attention of ragged queries over it (`cache.sagebwd_cache_attention`)
  "share"    a step of requests that share pages: done ones are freed (`cache.sagebwd_cache_free`), others go on from their parents
             (`..._fork`), and who is about to write into a shared page gets a copy (`..._own`)
  "compact"  the pages in use moved to the front of the pool (`cache.sagebwd_cache_compact`)

The cache held in 8 bits.  A pool of pages, uint8 [pages, H, bytes]; a page of a head holds `page` tokens as K's codes (page * d bytes), V's
codes (the same), and for every 32 tokens two float32, K's and V's largest magnitude a (of a block of 64 tokens the two pairs are alike), up to a
multiple of 16 bytes.  A value is code * (a / 127), codes -127 .. 127.

  K's codes     token t = 32 b + 8 o + 4 s + i, channel c = 64 j + 16 g + e: byte 32 d b + 2048 j + 1024 s + 256 g + 64 o + 16 i + e
  V's codes     token t = 32 b + 8 o + i, channel c = 32 j + 16 h + m: byte 32 d b + 1024 j + 256 o + 16 m + 8 h + i

Quantiser, per block of tokens and head, in 32 bits: x = float(k) - mean; a = max|x| over the block's new tokens, and over what it held if the
first of them is not its first token; code = rne(x * r), r = 127 / a; where a grew from b, codes held become rne(code * (b / a)).

Shared pages.  shares int32 [3, pages]: row 0 has the holders of a page beyond the first; the other rows are the calls' own.  A page that loses its
last holder goes on the stack of free pages; of those that one call frees the lowest ends on top.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_DEFAULTS = dict(op="attend", R=1, Hq=32, H=8, d=128, block=64, page=64, q=1, queries="same", len=1024, ragged=False, causal=True, mean=False,
                 W=4, beams=False, spare=1.5, pattern=0)


def _case(**kw):
    return {**_DEFAULTS, **kw}


def listed():
    return [
        # One new token of each of 48 requests goes into the cache, anywhere in its block.
        _case(name="append_decode", op="append", R=48, q=1, mean=True),
        # Prompts of odd lengths go into the cache, one of them a chunk that begins inside a block.
        _case(name="append_prompts", op="append", R=3, q=5001, queries="ragged", block=32),
        # The smallest attention: four short requests decode.
        _case(name="attend_short", R=4, len=500, ragged=True, Hq=16, H=4),
        # A decoding batch of ragged lengths, grouped queries.
        _case(name="attend_batch", R=64, len=8192, ragged=True, mean=True),
        # One request decodes against a long cache.
        _case(name="attend_long", R=1, len=131000, block=32, page=128),
        # Twelve drafted tokens of each request are verified at once, 48 query rows of a head.
        _case(name="attend_verify", R=24, q=12, queries="ragged", len=3000, ragged=True, Hq=16, H=4, page=32, block=32),
        # Cross attention: new tokens of each request against its encoder's states, of another and odd length, nothing masked.
        _case(name="attend_cross", R=16, q=100, queries="ragged", len=1500, ragged=True, Hq=16, H=16, d=64, causal=False),
        # Chunked prefill: the newest 2048 tokens against a cache of 10000.
        _case(name="attend_chunk", R=1, q=2048, len=10000),
        # Four answers to each of two short prompts begin: launch latency is all there is.
        _case(name="share_samples", op="share", R=8, W=4, len=1000, H=4),
        # A beam search over many prompts moves its beams.
        _case(name="share_beams", op="share", R=256, W=8, len=4000, ragged=True, H=2, beams=True),
        # A small pool, half empty, is compacted.
        _case(name="compact_small", op="compact", R=12, len=700, ragged=True, H=4, page=32, block=32, spare=2.0),
        # A large pool is compacted before its tail is given back.
        _case(name="compact_large", op="compact", R=100, len=6000, ragged=True, H=8, spare=1.6),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: 1 to 512 requests, 1 to 2048 new tokens of each, up to 131072 in the cache, 1 to 16 query heads for each of the
    cache's 1 to 16, 2 to 8 requests that share; at most the work of the largest listed cases."""
    while True:
        c = _case(op=rng.choice(["append", "attend", "attend", "attend", "share", "compact"]), pattern=rng.randrange(1 << 20))
        c["H"] = _log_int(rng, 1, 16)
        c["Hq"] = c["H"] * rng.choice([1, 1, 2, 3, 4, 5, 7, 8, 16])
        c["d"], c["block"] = rng.choice([64, 128, 128]), rng.choice([32, 64, 64])
        c["page"] = max(c["block"], rng.choice([32, 64, 64, 128, 256]))
        c["R"], c["len"], c["ragged"] = _log_int(rng, 1, 512), _log_int(rng, 1, 131072), rng.random() < 0.7
        c["queries"] = rng.choice(["same", "ragged", "mixed"])
        c["q"] = min(c["len"], rng.choice([1, 1, _log_int(rng, 2, 16), _log_int(rng, 16, 2048)]))
        c["causal"], c["mean"] = rng.random() < 0.7, rng.random() < 0.4
        if c["op"] == "append":
            if c["R"] * c["q"] * c["H"] * c["d"] > 16 * 1024 * 1024:
                continue
            return c
        if c["op"] in ("share", "compact"):
            c["W"], c["beams"], c["spare"] = rng.randint(2, 8), rng.random() < 0.5, rng.uniform(1.1, 3.0)
            c["R"] = -(-c["R"] // c["W"]) * c["W"] if c["op"] == "share" else c["R"]
            if _pool_pages(c) * _page_bytes(c) > 5e8 or (c["op"] == "share" and c["R"] > 256) or c["len"] * c["R"] > (1 << 20):
                continue
            return c
        lens, news = _lengths(c)
        # padded, in 32 bits, the plain form has to fit the card; operations and bytes stay below the largest listed case's
        if len(lens) * max(lens) * c["H"] * c["d"] > 1.1e9 or len(lens) * max(news) * c["Hq"] * max(lens) > 1.5e9:
            continue
        if work(c)["flops"] > 3e11 or work(c)["bytes"] > 6e8:
            continue
        return c


def _lengths(case):
    """Tokens of every request in the cache (the new ones among them), and new ones: the same for every seed."""
    c = {**_DEFAULTS, **case}
    rng = random.Random(1000003 * c["pattern"] + 7919 * c["R"] + c["len"])
    lens, news = [], []
    for r in range(c["R"]):
        n = c["q"]
        if c["queries"] == "ragged" and r > 0:
            n = rng.randint(1, c["q"])
        elif c["queries"] == "mixed" and r % 17 != 0:
            n = 1
        full = c["len"]
        if c["ragged"] and r > 0:
            full = _log_int(rng, max(1, c["len"] // 16), c["len"])
        lens.append(max(n, full))
        news.append(n)
    return lens, news


def _groups(c):
    """Of a "share" case: tokens of each request (the same in a group), and how many of its last pages each request has to itself."""
    rng = random.Random(1000003 * c["pattern"] + 7919 * c["R"] + c["len"])
    lens, alone = [], []
    for k in range(c["R"] // c["W"]):
        n = _log_int(rng, max(1, c["len"] // 8), c["len"]) if c["ragged"] and k > 0 else c["len"]
        last = 1 if n % c["page"] else 0
        pages = -(-n // c["page"])
        for _ in range(c["W"]):
            lens.append(n)
            alone.append(min(pages, rng.randint(last, 3) if c["beams"] else last))
    return lens, alone


def _head_bytes(c):
    return 2 * c["page"] * c["d"] + -(-c["page"] // 4 // 16) * 16


def _page_bytes(c):
    return c["H"] * _head_bytes(c)


def _pool_pages(c):
    if c["op"] == "share":
        lens, alone = _groups(c)
        used = sum(alone) + sum(max(-(-lens[r] // c["page"]) - a for r, a in enumerate(alone[k:k + c["W"]], k)) for k in range(0, c["R"], c["W"]))
        return used + 2 * c["R"] + 7
    used = sum(-(-n // c["page"]) for n in _lengths(c)[0])
    return math.ceil(used * c["spare"]) + 3


def _copies(c):
    """Pages that one pass of a "share" case copies: of the requests that share their last page all but one."""
    lens, _ = _groups(c)
    parents, total = _parents(c), 0
    for k in range(0, c["R"], c["W"]):
        if lens[k] % c["page"]:
            total += c["W"] - len(set(parents[k:k + c["W"]]))
    return total


def _parents(c):
    """Whom each request goes on from: its group's first (that is kept), or any of its group."""
    if not c["beams"]:
        return [r // c["W"] * c["W"] for r in range(c["R"])]
    rng = random.Random(7 * c["pattern"] + c["R"])
    return [r // c["W"] * c["W"] + rng.randrange(c["W"]) for r in range(c["R"])]


def _moved(c):
    """Pages that a "compact" case moves: those in use behind the first as many."""
    order, used = _scattered(c)
    return sum(1 for p in order[:sum(used)] if p >= sum(used))


def _scattered(c):
    pages = _pool_pages(c)
    order = list(range(pages))
    random.Random(13 * c["pattern"] + pages).shuffle(order)
    return order, [-(-n // c["page"]) for n in _lengths(c)[0]]


def work(case):
    c = {**_DEFAULTS, **case}
    lens, news = _lengths(c)
    row = 2 * c["d"]
    if c["op"] == "append":
        # (read in bf16, written as codes; those read again, and the values that they stand for written)
        T = sum(news)
        return {"bytes": T * c["H"] * (4 * c["d"] + 2 * row + 4 * c["d"]) + 8 * T, "flops": 8 * T * c["H"] * c["d"]}
    if c["op"] == "share":
        lens, _ = _groups(c)
        entries = sum(-(-lens[r] // c["page"]) for r, p in enumerate(_parents(c)) if p != r)
        # (a forked request's entries read and written, what they and the ones before counted up and down, pages copied)
        return {"bytes": entries * (8 + 16) + 2 * _copies(c) * _page_bytes(c) + 24 * c["R"], "flops": 0}
    if c["op"] == "compact":
        entries = sum(-(-n // c["page"]) for n in lens)
        return {"bytes": 8 * entries + 8 * _pool_pages(c) + 2 * _moved(c) * _page_bytes(c), "flops": 0}
    pairs = sum((n * (a - n) + n * (n + 1) // 2) if c["causal"] else n * a for a, n in zip(lens, news))
    rows = sum(news) * c["Hq"]
    return {"bytes": sum(lens) * c["H"] * row + 8 * c["H"] * sum(-(-a // 32) for a in lens) + rows * (4 * c["d"] + 4) + 4 * sum(-(-a // c["page"]) for a in lens),
            "flops": 4 * pairs * c["Hq"] * c["d"]}


# ---- inputs ---------------------------------------------------------------------------------------------------------------------

def _pool(pages, c, g):
    """Codes as normal values of a block whose largest is about four times their deviation have them."""
    H, d, page = c["H"], c["d"], c["page"]
    at = (torch.arange(256, dtype=torch.float64, device="cuda") + 0.5) / 256
    table = (32 * torch.special.ndtri(at)).round().clamp(-127, 127).to(torch.int8).view(torch.uint8)
    codes = table[torch.randint(0, 256, (pages, H, 2 * page * d), generator=g, device="cuda", dtype=torch.int32)]
    n = page // c["block"]
    a = 3 + 2 * torch.rand((pages, H, n, 1, 2), generator=g, device="cuda")
    a = a.expand(pages, H, n, c["block"] // 32, 2).reshape(pages, H, -1).contiguous().view(torch.uint8)
    pad = torch.zeros((pages, H, _head_bytes(c) - 2 * page * d - a.shape[2]), dtype=torch.uint8, device="cuda")
    return torch.cat([codes, a, pad], dim=2)


def _normal(shape, g, scale=1.0):
    return (scale * torch.randn(shape, generator=g, device="cuda")).to(torch.bfloat16)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    c = {**_DEFAULTS, **case}
    g = torch.Generator(device="cuda").manual_seed(seed)
    state = {"case": c}
    make = {"append": _prepare_append, "attend": _prepare_attend, "share": _prepare_share, "compact": _prepare_compact}
    make[c["op"]](state, c, g)
    return state


def _prepare_append(state, c, g):
    Hq, H, d, page, block = c["Hq"], c["H"], c["d"], c["page"], c["block"]
    _, news = _lengths(c)
    places = random.Random(c["pattern"] + len(news))
    held = [places.randrange(page) for _ in news]        # tokens that a request's first page here holds
    counts = [-(-(h + n) // page) for h, n in zip(held, news)]
    pages = sum(counts) + 3
    order = torch.randperm(pages, generator=g, device="cuda")
    slots, blocks, first = [], [], 0
    for h, n, k in zip(held, news, counts):
        t = torch.arange(h, h + n, device="cuda")
        slots.append(order[first + t // page] * page + t % page)
        t = torch.arange(h // block * block, h + n, device="cuda")
        blocks.append(order[first + t // page] * page + t % page)
        first += k
    T = sum(news)
    # K and V are views of one projection's output, as a model hands them over
    qkv = _normal((T, Hq + 2 * H, d), g)
    state.update(K=qkv[:, Hq:Hq + H], V=qkv[:, Hq + H:], pool=_pool(pages, c, g), slots=torch.cat(slots), blocks=torch.cat(blocks))
    if c["mean"]:
        state["k_mean"] = 0.5 * torch.randn((H, d), generator=g, device="cuda")
        state["v_mean"] = 0.1 * torch.randn((H, d), generator=g, device="cuda")


def _prepare_attend(state, c, g):
    lens, news = _lengths(c)
    columns = -(-max(lens) // c["page"]) + 1
    used = [-(-a // c["page"]) for a in lens]
    order = torch.randperm(sum(used) + 2, generator=g, device="cuda").to(torch.int32)
    begin = [0]
    for n in news:
        begin.append(begin[-1] + n)
    state.update(pool=_pool(sum(used) + 2, c, g), table=_table(order, used, columns), lengths=_int32(lens), cu=_int32(begin), max_q=max(news),
                 max_len=max(lens), Q=_normal((begin[-1], c["Hq"], c["d"]), g))
    if c["mean"]:
        state["v_mean"] = 0.1 * torch.randn((c["H"], c["d"]), generator=g, device="cuda")


def _prepare_share(state, c, g):
    lens, alone = _groups(c)
    pages, page, W, R = _pool_pages(c), c["page"], c["W"], c["R"]
    order = torch.randperm(pages, generator=g, device="cuda").tolist()
    columns = -(-max(lens) // page) + 2
    table, shares = [], [0] * pages
    for k in range(0, R, W):
        n = -(-lens[k] // page)
        common = [order.pop() for _ in range(n - min(alone[k:k + W]))]
        for r in range(k, k + W):
            mine = common[:n - alone[r]] + [order.pop() for _ in range(alone[r])]
            for p in common[:n - alone[r]]:
                shares[p] += 1
            table.append(mine + [-1] * (columns - n))
        left = [p for p in common if shares[p] == 0]
        order.extend(left)
    shares = [max(0, n - 1) for n in shares]
    parents = _parents(c)
    keep = [n if c["beams"] or r % W == 0 else 0 for r, n in enumerate(lens)]
    state.update(pool=_pool(pages, c, g), table=_int32(table), lengths=_int32(lens), keep=_int32(keep), parents=_int32(parents), added=_int32([1] * R),
                 shares=torch.zeros((3, pages), dtype=torch.int32, device="cuda"), free_count=_int32([len(order)]),
                 free_pages=_int32(order + [0] * (pages - len(order))))
    state["shares"][0] = _int32(shares)


def _prepare_compact(state, c, g):
    order, used = _scattered(c)
    pages = len(order)
    columns = max(used) + 2
    state.update(pool=_pool(pages, c, g), table=_table(_int32(order), used, columns), lengths=_int32(_lengths(c)[0]))
    # what a program that compacts now and then keeps for the results
    i32 = dict(dtype=torch.int32, device="cuda")
    state["out"] = (torch.empty((c["R"], columns), **i32), torch.empty(pages, **i32), torch.empty(1, **i32), torch.zeros((3, pages), **i32),
                    torch.empty(1, **i32))


def _table(order, used, columns):
    """Block table: request r has used[r] pages, taken from `order`; the other entries are -1."""
    n = torch.tensor(used, device="cuda")
    column = torch.arange(columns, device="cuda")
    at = (n.cumsum(0) - n)[:, None] + column
    return torch.where(column < n[:, None], order[at.clamp(max=order.numel() - 1)], -1).to(torch.int32).contiguous()


# ---- one pass -------------------------------------------------------------------------------------------------------------------

def run(state):
    return {"append": _append, "attend": _attend, "share": _share, "compact": _compact}[state["case"]["op"]](state)


def _params(c):
    from paper_2603_02170_amd import cache
    return cache.CacheParams(H=c["H"], d=c["d"], page=c["page"], block=c["block"])


def _codes(pages, c):
    """K's and V's codes, float32 [n, H, page, d], and magnitudes, float32 [n, H, page / 32] each, of pages [n, H, bytes]."""
    d, page = c["d"], c["page"]
    both = pages[..., :2 * page * d].contiguous().view(torch.int8).float().unflatten(-1, (2, page // 32, 32 * d))
    k = both[:, :, 0].unflatten(-1, (d // 64, 2, 4, 4, 4, 16))             # j, s, g, o, i, e
    k = k.permute(0, 1, 2, 6, 4, 7, 3, 5, 8).flatten(6).flatten(2, 5)
    v = both[:, :, 1].unflatten(-1, (d // 32, 4, 16, 2, 8))                # j, o, m, h, i
    v = v.permute(0, 1, 2, 4, 7, 3, 6, 5).flatten(5).flatten(2, 4)
    a = pages[..., 2 * page * d:2 * page * d + page // 4].contiguous().view(torch.float32).unflatten(-1, (-1, 2))
    return k, v, a[..., 0], a[..., 1]


def _bytes(k, v, ka, va, c):
    """The inverse: pages [n, H, bytes] but for what fills them up."""
    d, page = c["d"], c["page"]
    k = k.unflatten(-1, (d // 64, 4, 16)).unflatten(2, (page // 32, 4, 2, 4))      # b, o, s, i, j, g, e
    k = k.permute(0, 1, 2, 6, 4, 7, 3, 5, 8).flatten(2)
    v = v.unflatten(-1, (d // 32, 2, 16)).unflatten(2, (page // 32, 4, 8))         # b, o, i, j, h, m
    v = v.permute(0, 1, 2, 5, 3, 7, 6, 4).flatten(2)
    a = torch.stack([ka, va], dim=-1).flatten(2).contiguous().view(torch.uint8)
    return torch.cat([k.to(torch.int8).view(torch.uint8), v.to(torch.int8).view(torch.uint8), a], dim=2)


def _by(a, number):
    return a / torch.full_like(a, number)        # (a division by a number is a product with its reciprocal, an ulp off)


def _stored(x, mean, code, a, ids, at, c):
    """New tokens x [T, H, d] of blocks `ids` at places `at` into the blocks' codes [n, H, block, d] and magnitudes [n, H]."""
    x = x.float() if mean is None else x.float() - mean
    n = code.shape[0]
    first = torch.full((n,), c["block"], device=x.device, dtype=torch.long).scatter_reduce_(0, ids, at, "amin")
    top = torch.zeros_like(a).scatter_reduce_(0, ids[:, None].expand(-1, c["H"]), x.abs().amax(-1), "amax")
    to = torch.where(first[:, None] > 0, torch.maximum(top, a), top)
    code = torch.where((to > a)[..., None, None], (code * (a / to)[..., None, None]).round(), code)
    r = torch.full_like(to, 127.0) / to
    code[ids, :, at] = (x * r[ids][..., None]).round()
    return code, to


def _append(s):
    c = s["case"]
    if own:
        from paper_2603_02170_amd import cache
        p = _params(c)
        cache.sagebwd_cache_append(s["K"], s["V"], s["slots"], s["pool"], p, k_mean=s.get("k_mean"), v_mean=s.get("v_mean"))
        return cache.sagebwd_cache_read(s["blocks"], s["pool"], p)
    page, block, H, d = c["page"], c["block"], c["H"], c["d"]
    touched, ids = torch.unique_consecutive(s["slots"] // block, return_inverse=True)      # blocks
    numbers, place = torch.unique_consecutive(touched * block // page, return_inverse=True)
    per = page // block
    k, v, ka, va = _codes(s["pool"][numbers], c)
    at = (place, touched % per)
    out = []
    for x, mean, code, a in ((s["K"], s.get("k_mean"), k, ka), (s["V"], s.get("v_mean"), v, va)):
        blocks = code.unflatten(2, (per, block))
        many = a.unflatten(2, (per, block // 32))
        new, to = _stored(x, mean, blocks[at[0], :, at[1]], many[at[0], :, at[1], 0], ids, s["slots"] % block, c)
        blocks[at[0], :, at[1]] = new
        many[at[0], :, at[1]] = to[..., None]
    s["pool"][numbers, :, :2 * page * d + page // 4] = _bytes(k, v, ka, va, c)
    order = numbers.argsort()
    row, t = order[torch.searchsorted(numbers[order], s["blocks"] // page)], s["blocks"] % page
    for code, a in ((k, ka), (v, va)):
        out.append((code[row, :, t] * _by(a, 127.0)[row, :, t // 32][..., None]).to(torch.bfloat16))
    return tuple(out)


def _attend(s):
    c = s["case"]
    if own:
        from paper_2603_02170_amd import cache
        return cache.sagebwd_cache_attention(s["Q"], s["pool"], s["table"], s["lengths"], s["cu"], _params(c), s["max_q"], causal=c["causal"],
                                             v_mean=s.get("v_mean"))
    Q, G, d, H = s["Q"], c["Hq"] // c["H"], c["d"], c["H"]
    T, R, q, length = Q.shape[0], c["R"], s["max_q"], s["max_len"]
    n_pages = -(-length // c["page"])
    k, v, ka, va = _codes(s["pool"][s["table"][:, :n_pages].long().clamp(min=0).flatten()], c)

    def values(code, a):
        x = (code.unflatten(2, (-1, 32)) * _by(a, 127.0)[..., None, None]).flatten(2, 3)
        return x.unflatten(0, (R, n_pages)).transpose(1, 2).flatten(2, 3)[:, :, :length]       # [R, H, length, d]

    k, v = values(k, ka), values(v, va)
    begin, L = s["cu"][:-1].long(), s["lengths"].long()
    n = s["cu"][1:].long() - begin
    i, j = torch.arange(q, device=Q.device), torch.arange(length, device=Q.device)
    rows = (begin[:, None] + i).clamp(max=T - 1)
    x = Q[rows].float().unflatten(2, (H, G)).permute(0, 2, 3, 1, 4).flatten(2, 3)        # [R, H, G q, d]
    last = L[:, None] - n[:, None] + i if c["causal"] else (L[:, None] - 1).expand(R, q)
    seen = (j <= last[..., None]) & (j < L[:, None, None])                               # [R, q, length]
    logits = (x @ k.transpose(2, 3)).mul_(d ** -0.5).unflatten(2, (G, q)).masked_fill_(~seen[:, None, None], -math.inf)
    lse = logits.logsumexp(-1)
    out = (logits.sub_(lse[..., None]).exp_().flatten(2, 3) @ v).unflatten(2, (G, q))
    if c["mean"]:
        out = out + s["v_mean"][:, None, None]
    of = torch.searchsorted(s["cu"][1:].long(), torch.arange(T, device=Q.device), right=True)
    at = torch.arange(T, device=Q.device) - begin[of]
    return out[of, :, :, at].flatten(1, 2).to(torch.bfloat16), lse[of, :, :, at].flatten(1, 2).T.contiguous()


def _pages_of(lengths, page, columns):
    return ((lengths.long() + page - 1) // page).clamp(max=columns)


def _settle(s, change):
    """Holders gained and lost, int64 [pages]: pages of no holder go on the stack, the lowest on top."""
    shares = s["shares"][0]
    now = shares + change
    freed = (change < 0) & (now < 0)
    shares.copy_(now.clamp(min=0))
    k = freed.sum()
    at = s["free_count"].long() + k - freed.long().cumsum(0)
    n = s["free_pages"].numel()
    wider = torch.cat([s["free_pages"], s["free_pages"].new_zeros(1)])
    wider[torch.where(freed, at, n)] = torch.arange(n, device=at.device, dtype=torch.int32)
    s["free_pages"].copy_(wider[:n])
    s["free_count"].add_(k)


def _plain_free(s):
    page, table = s["case"]["page"], s["table"]
    R, columns = table.shape
    keep, lengths = s["keep"].long(), s["lengths"].long()
    valid = (keep >= 0) & (keep <= lengths)
    column = torch.arange(columns, device=table.device)
    lost = valid[:, None] & (column >= _pages_of(keep, page, columns)[:, None]) & (column < _pages_of(lengths, page, columns)[:, None])
    change = torch.zeros(s["shares"].shape[1], dtype=torch.long, device=table.device)
    change.index_add_(0, table.clamp(min=0).flatten(), -(lost & (table >= 0)).flatten().long())
    table.copy_(torch.where(lost, -1, table))
    s["lengths"].copy_(torch.where(valid, keep, lengths))
    _settle(s, change)


def _plain_fork(s):
    page, table = s["case"]["page"], s["table"]
    R, columns = table.shape
    parents, lengths = s["parents"].long(), s["lengths"].long()
    r = torch.arange(R, device=table.device)
    forked = (parents >= 0) & (parents < R) & (parents != r)
    of = torch.where(forked, parents, r)
    held = _pages_of(lengths, page, columns)
    column = torch.arange(columns, device=table.device)
    new = torch.where(column < held[of][:, None], table[of], -1)
    change = torch.zeros(s["shares"].shape[1], dtype=torch.long, device=table.device)
    change.index_add_(0, new.clamp(min=0).flatten(), (forked[:, None] & (new >= 0)).flatten().long())
    lost = forked[:, None] & (column < held[:, None]) & (table >= 0)
    change.index_add_(0, table.clamp(min=0).flatten(), -lost.flatten().long())
    table.copy_(torch.where(forked[:, None], new, table))
    s["lengths"].copy_(lengths[of])
    _settle(s, change)


def _plain_own(s):
    page, table = s["case"]["page"], s["table"]
    R, columns = table.shape
    shares, lengths = s["shares"][0], s["lengths"].long()
    r = torch.arange(R, device=table.device)
    column = (lengths // page).clamp(max=columns - 1)
    entry = table[r, column].long()
    wants = (s["added"] > 0) & (lengths % page > 0) & (entry >= 0)
    e = entry.clamp(min=0)
    wants &= shares[e] > 0
    asked = torch.zeros(shares.numel(), dtype=torch.long, device=table.device).index_add_(0, e, wants.long())
    last = torch.full((shares.numel(),), -1, dtype=torch.long, device=table.device).scatter_reduce_(0, e, torch.where(wants, r, -1), "amax")
    copies = wants & ~((asked[e] == shares[e] + 1) & (last[e] == r))
    needs = copies.long().cumsum(0)
    count = s["free_count"].long()
    granted = ~wants | (needs <= count)
    copies &= granted
    to = s["free_pages"][(count - needs).clamp(min=0)].long()
    shares.index_add_(0, e, -copies.int())
    table[r, column] = torch.where(copies, to, entry).int()
    s["free_count"].sub_(copies.sum())
    s["pool"][to[copies]] = s["pool"][e[copies]]
    return torch.where(granted, s["added"], 0)


def _share(s):
    if own:
        from paper_2603_02170_amd import cache
        p, pages = _params(s["case"]), (s["lengths"], s["table"], s["free_pages"], s["free_count"], s["shares"])
        cache.sagebwd_cache_free(s["keep"], *pages, p)
        cache.sagebwd_cache_fork(s["parents"], *pages, p)
        added = cache.sagebwd_cache_own(s["added"], *pages, s["pool"], p)
    else:
        _plain_free(s)
        _plain_fork(s)
        added = _plain_own(s)
    return s["lengths"], s["table"], s["free_pages"], s["free_count"], s["shares"], added, s["pool"]


def _compact(s):
    c = s["case"]
    if own:
        from paper_2603_02170_amd import cache
        return tuple(cache.sagebwd_cache_compact(s["lengths"], s["table"], s["pool"], _params(c), out=s["out"])) + (s["pool"],)
    table, pool = s["table"], s["pool"]
    pages, columns = pool.shape[0], table.shape[1]
    held = torch.arange(columns, device=table.device) < _pages_of(s["lengths"], c["page"], columns)[:, None]
    holders = torch.zeros(pages, dtype=torch.long, device=table.device)
    holders.index_add_(0, table.clamp(min=0).flatten(), (held & (table >= 0)).flatten().long())
    used, page = holders > 0, torch.arange(pages, device=table.device)
    n = used.sum()
    moves = (used & (page >= n)).nonzero()[:, 0]
    to = (~used & (page < n)).nonzero()[:, 0]
    where = page.clone()
    where[moves] = to
    pool[to] = pool[moves]
    new = torch.where(held & (table >= 0), where[table.clamp(min=0).long()], -1).int()
    shares = torch.zeros((3, pages), dtype=torch.long, device=table.device)
    shares[0, where[used]] = holders[used] - 1
    free = torch.where(page < pages - n, pages - 1 - page, -1)
    return new, free.int(), (pages - n).int()[None], shares.int(), n.int()[None], pool


# ---- the definitions in 64 bits, byte by byte, request by request ---------------------------------------------------------------

def exact(case, seed):
    c = {**_DEFAULTS, **case}
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "share": _exact_share, "compact": _exact_compact}[c["op"]](c, s)


def _places(c):
    """Byte of every (token, channel) of K and of V, and of a token's magnitudes, in a page of a head."""
    d, page = c["d"], c["page"]
    t, ch = torch.arange(page, device="cuda")[:, None], torch.arange(d, device="cuda")[None]
    base, u = t // 32 * (32 * d), t % 32
    k = base + ch // 64 * 2048 + u // 4 % 2 * 1024 + ch // 16 % 4 * 256 + u // 8 * 64 + u % 4 * 16 + ch % 16
    v = page * d + base + ch // 32 * 1024 + u // 8 * 256 + ch % 16 * 16 + ch // 16 % 2 * 8 + u % 8
    return k, v, 2 * page * d + t[:, 0] // 32 * 8


def _word(pages, at):
    """float32 at byte `at`, as float64"""
    bits = sum(pages[..., at + i].int() << 8 * i for i in range(4))
    return bits.view(torch.float32).double()


def _number(bytes_):
    return (bytes_.int() - 256 * (bytes_ > 127).int()).double()


def _exact_append(c, s):
    page, block, H, d = c["page"], c["block"], c["H"], c["d"]
    k_at, v_at, a_at = _places(c)
    to32 = lambda x: x.float().double()  # noqa: E731  (the definition's decisions are in 32 bits)
    slots = s["slots"].tolist()
    runs, begin = [], 0
    for i in range(1, len(slots) + 1):
        if i == len(slots) or slots[i] // block != slots[begin] // block:
            runs.append((begin, i))
            begin = i
    if len(runs) > 4000:
        return None
    values = {}
    for b, e in runs:
        number, first = divmod(slots[b], page)
        o, base = first % block, first // block * block
        part = s["pool"][number]
        for which, x, mean, at, add in ((0, s["K"], s.get("k_mean"), k_at, 0), (1, s["V"], s.get("v_mean"), v_at, 4)):
            y = x[b:e].double()
            if mean is not None:
                y = to32(y - mean.double())
            old = _word(part, (a_at + add)[base])
            a = y.abs().amax(dim=(0, 2))
            if o > 0:
                a = torch.maximum(a, old)
            held = _number(part[:, at[base:base + o]])                                   # [H, o, d]
            if o > 0:
                f = to32(old / a)[:, None, None]
                held = torch.where((a > old)[:, None, None], torch.round(to32(held * f)), held)
            code = torch.round(to32(y * to32(127 / a)[:, None])).transpose(0, 1)
            values[slots[b] // block, which] = (torch.cat([held, code], dim=1) * (a / 127)[:, None, None]).transpose(0, 1)
    order = []
    for x in s["blocks"].tolist():
        if not order or order[-1] != x // block:
            order.append(x // block)
    return tuple(torch.cat([values[b, which] for b in order]) for which in (0, 1))


def _exact_attend(c, s):
    d, page, H, G = c["d"], c["page"], c["H"], c["Hq"] // c["H"]
    if work(c)["flops"] > 1e12:
        return None
    k_at, v_at, a_at = _places(c)
    out = torch.empty(s["Q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty((c["Hq"], s["Q"].shape[0]), dtype=torch.float64, device="cuda")
    cu = s["cu"].tolist()
    for r, L in enumerate(s["lengths"].tolist()):
        a, b = cu[r], cu[r + 1]
        pages = s["pool"][s["table"][r, :-(-L // page)].long()]
        k = (_number(pages[:, :, k_at]) * (_word(pages, a_at) / 127)[..., None]).transpose(0, 1).flatten(1, 2)[:, :L]
        v = (_number(pages[:, :, v_at]) * (_word(pages, a_at + 4) / 127)[..., None]).transpose(0, 1).flatten(1, 2)[:, :L]
        hidden = torch.ones((b - a, L), dtype=torch.bool, device="cuda").triu(L - (b - a) + 1) if c["causal"] else None
        for h in range(c["Hq"]):
            z = s["Q"][a:b, h].double() @ k[h // G].T / math.sqrt(d)
            if hidden is not None:
                z = z.masked_fill(hidden, -math.inf)
            top = z.max(dim=1, keepdim=True)[0]
            w = (z - top).exp()
            total = w.sum(dim=1, keepdim=True)
            out[a:b, h] = w @ v[h // G] / total
            if c["mean"]:
                out[a:b, h] += s["v_mean"][h // G].double()
            lse[h, a:b] = (top + total.log())[:, 0]
    return out, lse


def _exact_share(c, s):
    """Request after request, holders counted in a list of sets."""
    page, R = c["page"], c["R"]
    table, lengths, stack = s["table"].tolist(), s["lengths"].tolist(), s["free_pages"].tolist()
    pool, left = s["pool"].clone(), int(s["free_count"])
    holders = {}
    for r in range(R):
        for p in table[r]:
            if p >= 0:
                holders.setdefault(p, set()).add(r)

    def gone(before):
        nonlocal left
        for p in sorted((p for p in before if not holders.get(p)), reverse=True):
            stack[left] = p
            left += 1
            holders.pop(p, None)

    before = list(holders)
    for r, n in enumerate(s["keep"].tolist()):
        for k in range(-(-n // page), len(table[r])):
            if table[r][k] >= 0:
                holders[table[r][k]].discard(r)
                table[r][k] = -1
        lengths[r] = n
    gone(before)
    before = list(holders)
    parents = s["parents"].tolist()
    rows, sizes = [list(x) for x in table], list(lengths)
    for r, p in enumerate(parents):
        if p != r:
            for x in rows[r]:
                if x >= 0:
                    holders[x].discard(r)
            for x in rows[p]:
                if x >= 0:
                    holders[x].add(r)
            table[r], lengths[r] = list(rows[p]), sizes[p]
    gone(before)
    added = s["added"].tolist()
    for r in range(R):
        x = table[r][lengths[r] // page] if lengths[r] % page else -1
        if x >= 0 and len(holders[x]) > 1:
            if left == 0:
                return None
            left -= 1
            fresh = stack[left]
            holders[x].discard(r)
            holders[fresh] = {r}
            pool[fresh] = pool[x]
            table[r][lengths[r] // page] = fresh
    shares = torch.zeros_like(s["shares"])
    for p, who in holders.items():
        shares[0, p] = len(who) - 1
    return _int32(lengths), _int32(table), _int32(stack), _int32([left]), shares, _int32(added), pool


def _exact_compact(c, s):
    table, pool = s["table"].tolist(), s["pool"].clone()
    pages = pool.shape[0]
    used = sorted({p for row in table for p in row if p >= 0})
    n = len(used)
    holes = [p for p in range(n) if p not in set(used)]
    where = {p: p for p in used if p < n}
    for p, to in zip([p for p in used if p >= n], holes):
        where[p] = to
        pool[to] = s["pool"][p]
    new = [[where[p] if p >= 0 else -1 for p in row] for row in table]
    shares = torch.zeros((3, pages), dtype=torch.int32, device="cuda")
    for row in new:
        for p in row:
            if p >= 0:
                shares[0, p] += 1
    shares[0] = (shares[0] - 1).clamp(min=0)
    return _int32(new), _int32(list(range(pages - 1, n - 1, -1)) + [-1] * n), _int32([pages - n]), shares, _int32([n]), pool
