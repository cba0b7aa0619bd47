"""The operators of serving from a cache held in 4 bits, as cases to be timed and compared, with their plain forms.

A case is one pass through one operator; "op" names it:

  "plan"    pages, slots and positions of a step's new tokens, from the requests' lengths (`cache.sagebwd_cache_plan`)
  "rotary"  rotary positions of Q and K with one to three axes (`autograd.sage_rotary`); with "train" its gradients too
  "append"  new keys and values into the cache, and the values that it then holds (`cache.sagebwd_cache_append`, `..._read`)
  "attend"  attention of ragged queries over the cache (`cache.sagebwd_cache_attention`)

The cache.  A pool of pages, uint8 [pages, H, page * (d + 4 d / group)]; a page of a head holds `page` tokens as K's codes, V's codes,
K's scales, V's scales.  A value is (nibble - 8) * scale, with one bf16 scale per token, head and `group` channels whose last three
mantissa bits are zero, so that the product is a bf16 number.

  K's codes     token t, channel c = 32 j + 8 p + r:   nibble r // 2 + 4 (r % 2) of the word at byte t * d / 2 + p * d / 8 + 4 j
  V's codes     token t = 8 o + i, channel c = 64 h + 16 j + m:   nibble j of the half-word at byte o * 4 d + 256 h + 16 m + 2 i
  scales        token t = 8 o + i, group s:   bf16 at byte (o * d / group + s) * 16 + 2 i

Quantiser: x = float(k) - mean, a = max|x| over the group, scale = a / 7 rounded up to 5 significant bits, nibble = 8 + rne(x / scale).
"""
from __future__ import annotations

import math
import random

import torch

own = False

_DEFAULTS = dict(op="attend", R=1, T=1, Hq=32, H=8, d=128, group=64, page=64, q=1, queries="same", len=1024, ragged=False, causal=True,
                 mean=False, axes=1, rot=0, adjacent=False, train=False, far=1 << 15, pattern=0)


def _case(**kw):
    return {**_DEFAULTS, **kw}


def listed():
    return [
        # A decoding step's bookkeeping: every request of a small batch gets one token, one in `page` of them a page.
        _case(name="plan_decode", op="plan", R=32, q=1, len=4096),
        # A batch of prompts of ragged lengths arrives at once, beside requests that decode.
        _case(name="plan_prompts", op="plan", R=300, q=1024, queries="mixed", len=16384, ragged=True, page=32),
        # Rotary positions of a decoding step: far positions, one axis; launch latency is all there is.
        _case(name="rotary_decode", op="rotary", T=32, far=1 << 20),
        # A training batch of image and video tokens: three axes (time, height, width), forward and backward, d = 64, an odd length.
        _case(name="rotary_video_train", op="rotary", T=16381, Hq=16, H=16, axes=3, train=True),
        # One new token of each of 48 requests goes into the cache.
        _case(name="append_decode", op="append", T=48, mean=True),
        # A prompt of odd length goes into the cache.
        _case(name="append_prompt", op="append", T=8191, group=32),
        # The smallest attention: four short requests decode.
        _case(name="attend_short", R=4, len=500, ragged=True, Hq=16, H=4),
        # A decoding batch of ragged lengths, grouped queries.
        _case(name="attend_batch", R=64, len=8192, ragged=True, mean=True),
        # One request decodes against a long cache.
        _case(name="attend_long", R=1, len=131000, group=32),
        # Several drafted tokens of each request are verified at once; heads of 64, a query head for each of the cache.
        _case(name="attend_verify", R=24, q=5, queries="ragged", len=3000, ragged=True, Hq=12, H=12, d=64, page=32),
        # Chunked prefill: the newest 2048 tokens against a cache of 10000.
        _case(name="attend_chunk", R=1, q=2048, len=10000),
        # A step of mixed work: two requests bring chunks, the others decode.
        _case(name="attend_mixed", R=34, q=600, queries="mixed", len=6000, ragged=True, d=64, group=32, Hq=16, H=4),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: 1 to 512 requests, 1 to 2048 new tokens of each, up to 131072 in the cache, 1 to 16 query heads for each of the
    cache's 1 to 16, at most the work of the largest listed cases."""
    while True:
        c = _case(op=rng.choice(["plan", "rotary", "append", "attend", "attend", "attend"]), pattern=rng.randrange(1 << 20))
        c["H"] = _log_int(rng, 1, 16)
        c["Hq"] = c["H"] * rng.choice([1, 1, 2, 3, 4, 5, 7, 8, 16])
        c["d"], c["group"], c["page"] = rng.choice([64, 128, 128]), rng.choice([32, 64]), rng.choice([32, 64, 64, 128])
        c["R"], c["len"], c["ragged"] = _log_int(rng, 1, 512), _log_int(rng, 1, 131072), rng.random() < 0.7
        c["queries"] = rng.choice(["same", "ragged", "mixed"])
        c["q"] = min(c["len"], rng.choice([1, 1, _log_int(rng, 2, 16), _log_int(rng, 16, 2048)]))
        c["causal"], c["mean"] = rng.random() < 0.8, rng.random() < 0.4
        if c["op"] in ("rotary", "append"):
            c["T"] = _log_int(rng, 1, 16384)
            c["axes"], c["adjacent"], c["train"] = rng.choice([1, 2, 3]), rng.random() < 0.3, rng.random() < 0.4
            c["rot"], c["far"] = rng.choice([0, 0, c["d"] // 2]), _log_int(rng, 64, 1 << 20)
            if c["T"] * (c["Hq"] + c["H"]) * c["d"] > (1 << 26):
                continue
            return c
        lens, news = _lengths(c)
        if c["op"] == "plan":
            if sum(news) > 65536 or len(lens) * max(lens) > (1 << 25):
                continue
            return c
        # padded, in 32 bits, the plain form has to fit the card; operations and bytes stay below the largest listed case's
        if len(lens) * max(lens) * c["H"] * c["d"] > 1.1e9 or len(lens) * max(news) * c["Hq"] * max(lens) > 1.5e9:
            continue
        if work(c)["flops"] > 3.5e11 or work(c)["bytes"] > 4.5e8:
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


def _sections(c):
    half = (c["rot"] or c["d"]) // 2
    if c["axes"] == 1:
        return [half]
    if c["axes"] == 2:
        return [half // 2, half - half // 2]
    first = half // 4
    return [first, (half - first) // 2, half - first - (half - first) // 2]


def work(case):
    c = {**_DEFAULTS, **case}
    if c["op"] == "plan":
        lens, news = _lengths(c)
        pages = sum(-(-a // c["page"]) - -(-(a - n) // c["page"]) for a, n in zip(lens, news))
        return {"bytes": 24 * c["R"] + 8 * pages + 12 * sum(news), "flops": 0}
    if c["op"] == "rotary":
        values = c["T"] * (c["Hq"] + c["H"]) * c["d"]
        passes = 2 if c["train"] else 1
        return {"bytes": passes * (4 * values + 4 * c["T"] * c["axes"]), "flops": passes * 3 * values}
    row = c["d"] + 4 * c["d"] // c["group"]
    if c["op"] == "append":
        # (read in bf16, written as codes and scales; those read again, and the values that they stand for written)
        return {"bytes": c["T"] * c["H"] * (4 * c["d"] + 2 * row + 4 * c["d"]) + 8 * c["T"], "flops": 8 * c["T"] * c["H"] * c["d"]}
    lens, news = _lengths(c)
    pairs = sum((n * (a - n) + n * (n + 1) // 2) if c["causal"] else n * a for a, n in zip(lens, news))
    rows = sum(news) * c["Hq"]
    return {"bytes": sum(lens) * c["H"] * row + rows * (4 * c["d"] + 4) + 4 * sum(-(-a // c["page"]) for a in lens),
            "flops": 4 * pairs * c["Hq"] * c["d"]}


# ---- inputs ---------------------------------------------------------------------------------------------------------------------

def _codes(shape, g):
    """Bytes of two nibbles that are distributed as the codes of normal values are: 1 to 15, rarely at the ends."""
    at = [0.5 * (1 + math.erf((i - 8 + 0.5) / (2.6 * math.sqrt(2)))) for i in range(16)]
    nibble = [min(15, max(1, sum(1 for e in at if e <= (k + 0.5) / 16))) for k in range(16)]
    table = torch.tensor([nibble[b % 16] | nibble[b // 16] << 4 for b in range(256)], dtype=torch.uint8, device="cuda")
    return table[torch.randint(0, 256, shape, generator=g, device="cuda", dtype=torch.int32)]


def _pool(pages, c, g):
    H, d, page = c["H"], c["d"], c["page"]
    codes = _codes((pages, H, page * d), g)
    scales = torch.randint(0, 16, (pages, H, 2 * page * d // c["group"]), generator=g, device="cuda", dtype=torch.int32)
    scales = (0.25 * (1 + scales / 16)).to(torch.bfloat16)        # five significant bits, of groups whose largest value is 1.8 to 3.4
    return torch.cat([codes, scales.view(torch.uint8)], dim=2)


def _normal(shape, g, scale=1.0):
    return (scale * torch.randn(shape, generator=g, device="cuda")).to(torch.bfloat16)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    c = {**_DEFAULTS, **case}
    g = torch.Generator(device="cuda").manual_seed(seed)
    T, Hq, H, d, page = c["T"], c["Hq"], c["H"], c["d"], c["page"]
    state = {"case": c}
    if c["op"] == "rotary":
        # positions of text count up; of images and video the axes differ
        start = torch.randint(0, c["far"], (c["axes"], 1), generator=g, device="cuda")
        steps = torch.arange(T, device="cuda").repeat(c["axes"], 1) // _column([1, 7, 50][:c["axes"]])
        half = (c["rot"] or d) // 2
        state["positions"] = (start + steps).to(torch.int32)
        state["inv_freq"] = (10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)).float()
        # Q and K are views of one projection's output, as a model hands them over
        qkv = _normal((T, Hq + 2 * H, d), g)
        state["Q"], state["K"] = qkv[:, :Hq], qkv[:, Hq:Hq + H]
        if c["train"]:
            state["Q"], state["K"] = state["Q"].detach().requires_grad_(), state["K"].detach().requires_grad_()
            state["dQ"], state["dK"] = _normal((T, Hq, d), g), _normal((T, H, d), g)
        return state
    if c["op"] == "append":
        pages = -(-T // page) + 3
        qkv = _normal((T, Hq + 2 * H, d), g)
        state["K"], state["V"] = qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
        state["pool"] = _pool(pages, c, g)
        state["slots"] = torch.randperm(pages * page, generator=g, device="cuda")[:T].contiguous() if T < 256 else \
            (torch.randperm(pages, generator=g, device="cuda")[:, None] * page + torch.arange(page, device="cuda")).flatten()[:T].contiguous()
        if c["mean"]:
            state["k_mean"] = 0.5 * torch.randn((H, d), generator=g, device="cuda")
            state["v_mean"] = 0.1 * torch.randn((H, d), generator=g, device="cuda")
        return state
    lens, news = _lengths(c)
    columns = -(-max(lens) // page) + 1
    if c["op"] == "plan":
        held = [a - n for a, n in zip(lens, news)]
        used = sum(-(-a // page) for a in held)
        total = sum(-(-a // page) for a in lens) + 10007
        order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
        state.update(held=_int32(held), new=_int32(news), rows=sum(news), table=_table(order, [-(-a // page) for a in held], columns),
                     free_pages=order[used:].contiguous(), free_count=_int32([total - used]))
        return state
    used = [-(-a // page) for a in lens]
    order = torch.randperm(sum(used) + 2, generator=g, device="cuda").to(torch.int32)
    begin = [0]
    for n in news:
        begin.append(begin[-1] + n)
    state.update(pool=_pool(sum(used) + 2, c, g), table=_table(order, used, columns), lengths=_int32(lens), cu=_int32(begin), max_q=max(news),
                 max_len=max(lens), Q=_normal((begin[-1], Hq, d), g))
    if c["mean"]:
        state["v_mean"] = 0.1 * torch.randn((H, d), generator=g, device="cuda")
    return state


def _column(values):
    return torch.tensor(values, device="cuda")[:, None]


def _table(order, used, columns):
    """Block table: request r has used[r] pages, taken from `order`; the other entries are -1."""
    n = torch.tensor(used, device="cuda")
    column = torch.arange(columns, device="cuda")
    at = (n.cumsum(0) - n)[:, None] + column
    return torch.where(column < n[:, None], order[at.clamp(max=order.numel() - 1)], -1).to(torch.int32).contiguous()


# ---- one pass -------------------------------------------------------------------------------------------------------------------

def run(state):
    return {"plan": _plan, "rotary": _rotary, "append": _append, "attend": _attend}[state["case"]["op"]](state)


def _params(c):
    from paper_2603_02170_amd import cache
    return cache.CacheParams(H=c["H"], d=c["d"], page=c["page"], group=c["group"])


def _plan(s):
    c = s["case"]
    if own:
        from paper_2603_02170_amd import cache
        return tuple(cache.sagebwd_cache_plan(s["held"], s["new"], s["table"], s["free_pages"], s["free_count"], _params(c), s["rows"])) + (s["table"],)
    page, rows, table = c["page"], s["rows"], s["table"]
    held, new = s["held"].long(), s["new"].long()
    R, columns = table.shape
    sizes_fit = (held >= 0) & (new >= 0) & (held + new <= columns * page)
    new = torch.where(sizes_fit, new, 0)
    tokens = new.cumsum(0)
    first = (held + page - 1) // page                   # pages that the request has
    need = torch.where(sizes_fit, (held + new + page - 1) // page - first, 0)
    sums = need.cumsum(0)
    granted = sizes_fit & (tokens <= rows) & ((need == 0) | (sums <= s["free_count"].long()))
    column = torch.arange(columns, device=held.device)
    nth = column - first[:, None]                       # which of the request's new pages a column is
    fresh = granted[:, None] & (nth >= 0) & (nth < need[:, None])
    taken = torch.where(granted, need, 0).cumsum(0)
    at = s["free_count"].long() - 1 - (taken - torch.where(granted, need, 0))[:, None] - nth
    table.copy_(torch.where(fresh, s["free_pages"][at.clamp(0, s["free_pages"].numel() - 1)], table))
    row = torch.arange(rows, device=held.device)
    of = torch.searchsorted(tokens, row, right=True).clamp(max=R - 1)
    position = held[of] + row - (tokens - new)[of]
    used = (row < tokens[-1]) & granted[of]
    entry = table[of, (position // page).clamp(0, columns - 1)].long()
    slots = torch.where(used, entry * page + position % page, -1)
    cu = torch.cat([torch.zeros(1, dtype=torch.long, device=held.device), tokens]).clamp(max=rows)
    return (slots, torch.where(used, position, 0).int(), cu.int(), torch.where(granted, held + new, held).int(), granted.int(),
            (s["free_count"] - taken[-1]).int(), table)


def _rotated(x, cos, sin, rot, adjacent):
    x = x.float()
    y = x[..., :rot]
    cos, sin = cos[:, None], sin[:, None]
    if adjacent:
        a, b = y[..., 0::2], y[..., 1::2]
        z = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = y[..., :rot // 2], y[..., rot // 2:]
        z = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([z, x[..., rot:]], dim=-1).to(torch.bfloat16)


def _rotary(s):
    c = s["case"]
    rot = c["rot"] or c["d"]
    if own:
        from paper_2603_02170_amd.autograd import sage_rotary
        Q, K = sage_rotary(s["Q"], s["K"], s["positions"], s["inv_freq"], sections=_sections(c), adjacent=c["adjacent"])
        if not c["train"]:
            return Q, K
        return (Q.detach(), K.detach()) + torch.autograd.grad([Q, K], [s["Q"], s["K"]], [s["dQ"], s["dK"]])
    axis = torch.repeat_interleave(torch.arange(c["axes"], device="cuda"), _column(_sections(c))[:, 0])
    turn = s["positions"].double()[axis].T * s["inv_freq"].double()
    cos, sin = turn.cos().float(), turn.sin().float()
    out = tuple(_rotated(s[x].detach(), cos, sin, rot, c["adjacent"]) for x in ("Q", "K"))
    if c["train"]:
        out += tuple(_rotated(s[x], cos, -sin, rot, c["adjacent"]) for x in ("dQ", "dK"))
    return out


def _quantised(x, mean, group):
    """(codes 1 .. 15, scales as float32) of [T, H, d]."""
    x = x.float()
    if mean is not None:
        x = x - mean
    x = x.unflatten(-1, (-1, group))
    scale = x.abs().amax(-1, keepdim=True)
    scale = scale / torch.full_like(scale, 7.0)        # (a division by a number is a product with its reciprocal, an ulp off where 7 divides)
    scale = ((scale.view(torch.int32) + 0x7FFFF) & -0x80000).view(torch.float32)
    code = (x / torch.where(scale > 0, scale, 1.0)).round() + 8
    return code.flatten(-2).to(torch.uint8), scale.squeeze(-1)


def _k_order(d):
    """Channel of every nibble of a token's row of K, low nibbles first."""
    p, j, e = torch.meshgrid(torch.arange(4), torch.arange(d // 32), torch.arange(8), indexing="ij")
    return (32 * j + 8 * p + 2 * (e % 4) + e // 4).flatten().cuda()


def _append(s):
    c = s["case"]
    k_mean, v_mean = s.get("k_mean"), s.get("v_mean")
    if own:
        from paper_2603_02170_amd import cache
        p = _params(c)
        cache.sagebwd_cache_append(s["K"], s["V"], s["slots"], s["pool"], p, k_mean=k_mean, v_mean=v_mean)
        return cache.sagebwd_cache_read(s["slots"], s["pool"], p)
    T, H, d, page, group = c["T"], c["H"], c["d"], c["page"], c["group"]
    k, ks = _quantised(s["K"], k_mean, group)
    v, vs = _quantised(s["V"], v_mean, group)
    at, t = s["slots"] // page, s["slots"] % page
    o, i = t // 8, t % 8
    pool, n = s["pool"], d // group
    rows = pool[:, :, :page * d // 2].unflatten(2, (page, d // 2))
    k = k[:, :, _k_order(d)].unflatten(-1, (-1, 2))
    rows[at, :, t] = k[..., 0] | k[..., 1] << 4
    octets = pool[:, :, page * d // 2:page * d].unflatten(2, (page // 8, d // 64, 16, 8, 2))
    w = v.unflatten(-1, (d // 64, 2, 2, 16)).movedim(-1, -3)         # [T, H, half, m, byte, nibble]
    octets[at, :, o, :, :, i] = w[..., 0] | w[..., 1] << 4
    scales = pool[:, :, page * d:].unflatten(2, (2, page // 8, n, 8, 2))
    scales[at, :, 0, o, :, i] = ks.to(torch.bfloat16).view(torch.uint8).unflatten(-1, (n, 2))
    scales[at, :, 1, o, :, i] = vs.to(torch.bfloat16).view(torch.uint8).unflatten(-1, (n, 2))
    value = lambda q, x: ((q.float() - 8).unflatten(-1, (n, group)) * x[..., None]).flatten(-2).to(torch.bfloat16)  # noqa: E731
    k, _ = _quantised(s["K"], k_mean, group)
    return value(k, ks), value(v, vs)


def _values(blocks, c):
    """K and V, float32 [R, tokens, H, d], of pages [R, n, H, bytes]."""
    d, page, n = c["d"], c["page"], c["d"] // c["group"]
    nibbles = lambda b: torch.stack([b & 15, b >> 4], dim=-1).float() - 8  # noqa: E731
    k = nibbles(blocks[..., :page * d // 2].unflatten(-1, (page, d // 2))).flatten(-2)
    k = torch.empty_like(k).index_copy_(-1, _k_order(d), k)
    v = nibbles(blocks[..., page * d // 2:page * d].unflatten(-1, (page // 8, d // 64, 16, 8, 2)))
    v = v.flatten(-2).permute(0, 1, 2, 3, 6, 4, 7, 5).flatten(-3).flatten(3, 4)          # [R, n, H, page, d]
    x = blocks[..., page * d:].contiguous().view(torch.bfloat16).float().unflatten(-1, (2, page // 8, n, 8)).movedim(-1, -2).flatten(4, 5)
    k = (k.unflatten(-1, (n, -1)) * x[..., 0, :, :, None]).flatten(-2)
    v = (v.unflatten(-1, (n, -1)) * x[..., 1, :, :, None]).flatten(-2)
    return k.transpose(2, 3).flatten(1, 2), v.transpose(2, 3).flatten(1, 2)


def _attend(s):
    c = s["case"]
    if own:
        from paper_2603_02170_amd import cache
        return cache.sagebwd_cache_attention(s["Q"], s["pool"], s["table"], s["lengths"], s["cu"], _params(c), s["max_q"], causal=c["causal"],
                                             v_mean=s.get("v_mean"))
    Q, G, d = s["Q"], c["Hq"] // c["H"], c["d"]
    T, R, q, length = Q.shape[0], c["R"], s["max_q"], s["max_len"]
    pages = -(-length // c["page"])
    k, v = _values(s["pool"][s["table"][:, :pages].long().clamp(min=0)], c)
    k, v = k[:, :length].transpose(1, 2), v[:, :length].transpose(1, 2)                  # [R, H, length, d]
    begin, L = s["cu"][:-1].long(), s["lengths"].long()
    n = s["cu"][1:].long() - begin
    i, j = torch.arange(q, device=Q.device), torch.arange(length, device=Q.device)
    rows = (begin[:, None] + i).clamp(max=T - 1)
    x = Q[rows].float().unflatten(2, (c["H"], G)).permute(0, 2, 3, 1, 4).flatten(2, 3)   # [R, H, G q, d]
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


# ---- the definitions in 64 bits, byte by byte, request by request ---------------------------------------------------------------

def exact(case, seed):
    c = {**_DEFAULTS, **case}
    s = prepare(case, seed)
    return {"plan": _exact_plan, "rotary": _exact_rotary, "append": _exact_append, "attend": _exact_attend}[c["op"]](c, s)


def _exact_plan(c, s):
    page, table, stack = c["page"], s["table"].tolist(), s["free_pages"].tolist()[:int(s["free_count"])]
    slots, positions, cu, lengths, granted = [], [], [0], [], []
    need_so_far, at_first = 0, len(stack)
    for r, (a, n) in enumerate(zip(s["held"].tolist(), s["new"].tolist())):
        valid = a >= 0 and n >= 0 and a + n <= len(table[r]) * page
        n = n if valid else 0
        need = -(-(a + n) // page) - -(-a // page) if valid else 0
        need_so_far += need
        ok = valid and cu[-1] + n <= s["rows"] and (need == 0 or need_so_far <= at_first)
        for k in range(need if ok else 0):
            table[r][-(-a // page) + k] = stack.pop()
        for t in range(a, a + n):
            slots.append(table[r][t // page] * page + t % page if ok else -1)
            positions.append(t if ok else 0)
        cu.append(cu[-1] + n)
        lengths.append(a + n if ok else a)
        granted.append(int(ok))
    return (torch.tensor(slots, device="cuda"), _int32(positions), _int32(cu), _int32(lengths), _int32(granted), _int32([len(stack)]), _int32(table))


def _exact_rotary(c, s):
    rot, T = c["rot"] or c["d"], c["T"]
    angle = torch.zeros((T, rot // 2), dtype=torch.float64, device="cuda")
    begin = 0
    for axis, n in enumerate(_sections(c)):
        angle[:, begin:begin + n] = s["positions"][axis, :, None].double() * s["inv_freq"][begin:begin + n].double()
        begin += n

    def turned(x, sign):
        y = x.detach().double().clone()
        first = torch.arange(rot // 2, device="cuda") * (2 if c["adjacent"] else 1)
        second = first + (1 if c["adjacent"] else rot // 2)
        z = torch.complex(y[:, :, first], y[:, :, second]) * torch.polar(torch.ones_like(angle), sign * angle)[:, None]
        y[:, :, first], y[:, :, second] = z.real, z.imag
        return y

    out = (turned(s["Q"], 1), turned(s["K"], 1))
    return out + (turned(s["dQ"], -1), turned(s["dK"], -1)) if c["train"] else out


def _exact_append(c, s):
    out = []
    for x, mean in ((s["K"], s.get("k_mean")), (s["V"], s.get("v_mean"))):
        y = x.double() - (mean.double() if mean is not None else 0)
        y = y.reshape(y.shape[0], y.shape[1], -1, c["group"])
        step = y.abs().max(dim=-1, keepdim=True)[0] / 7
        m, e = torch.frexp(step)                                       # m in [1/2, 1): five significant bits are 32 m
        step = torch.ldexp(torch.ceil(32 * m) / 32, e)
        out.append((torch.round(y / step.clamp(min=1e-300)) * step).reshape(x.shape))
    return tuple(out)


def _exact_attend(c, s):
    d, page, group, H, G = c["d"], c["page"], c["group"], c["H"], c["Hq"] // c["H"]
    if work(c)["flops"] > 1e12:
        return None
    ch = torch.arange(d, device="cuda")
    t = torch.arange(page, device="cuda")[:, None]
    e = ch % 8 // 2 + 4 * (ch % 2)
    k_byte = t * (d // 2) + ch % 32 // 8 * (d // 8) + ch // 32 * 4 + e // 2
    k_shift = (e % 2 * 4).expand(page, d)
    v_byte = page * d // 2 + t // 8 * (4 * d) + ch // 64 * 256 + ch % 16 * 16 + t % 8 * 2 + ch % 64 // 32
    v_shift = (ch // 16 % 2 * 4).expand(page, d)
    x_byte = page * d + (t // 8 * (d // group) + ch // group) * 16 + t % 8 * 2

    def values(pages, byte, shift, scale):
        """[H, tokens, d] in 64 bits"""
        code = (pages[:, :, byte] >> shift & 15).double() - 8
        bits = pages[:, :, scale].int() << 16 | pages[:, :, scale + 1].int() << 24
        return (code * bits.view(torch.float32).double()).transpose(0, 1).flatten(1, 2)

    out = torch.empty(s["Q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty((c["Hq"], s["Q"].shape[0]), dtype=torch.float64, device="cuda")
    cu = s["cu"].tolist()
    for r, L in enumerate(s["lengths"].tolist()):
        a, b = cu[r], cu[r + 1]
        pages = s["pool"][s["table"][r, :-(-L // page)].long()]
        k = values(pages, k_byte, k_shift, x_byte)[:, :L]
        v = values(pages, v_byte, v_shift, x_byte + page * d // group * 2)[:, :L]
        hidden = torch.ones((b - a, L), dtype=torch.bool, device="cuda").triu(L - (b - a) + 1) if c["causal"] else None
        for h in range(c["Hq"]):
            z = s["Q"][a:b, h].double() @ k[h // G].T / math.sqrt(d)
            if hidden is not None:
                z = z.masked_fill(hidden, -math.inf)
            top = z.amax(-1, keepdim=True)
            w = (z - top).exp()
            out[a:b, h] = w @ v[h // G] / w.sum(-1, keepdim=True) + (s["v_mean"][h // G].double() if c["mean"] else 0)
            lse[h, a:b] = top[:, 0] + w.sum(-1).log()
    return out, lse
