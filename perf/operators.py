"""Cases of the operators on a Rollout's key/value cache, which follow a weight synchronisation: the cached keys and values of running
requests were computed with the old weights and are computed again with the new ones, or grow by single tokens.

A case names an operation (``op``):

* ``tables``     block tables, slots and positions of new tokens from request lengths, pages taken from a free list; then the pages go
                 back, so that every pass takes them again.  ``stale``: every token of every request is new and its pages are held.
* ``rope``       rotary positions on rows of heads; ``back``: the gradient of it, from the output's.
* ``write``      one step's queries and keys rotated, keys and values put into the pages of the cache.
* ``attention``  new tokens of several requests over the paged cache, with or without a window and first tokens that stay visible.

Heads and head sizes are those of the benchmark's weight sets (32 and 8 heads of 128, 32 and 4, 64 and 8) or generic ones.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
MOST_SCORES = 2 * 32 * 8192 * 8192      # query-key pairs over all heads of the largest case, padded
MOST_CACHE = 1 << 31                    # elements of keys and values in the cache


def listed():
    return [
        # a decoding step of a full batch: one token each, one request in sixteen needs a page
        {"name": "tables_step", "op": "tables", "requests": 128, "most": 1, "context": 8192, "page": 16, "stale": False},
        # all running requests re-encoded after a synchronisation: half a million slots, nothing to allocate
        {"name": "tables_reencode", "op": "tables", "requests": 256, "most": 1, "context": 4096, "page": 64, "stale": True},
        # queries and keys of a long packed batch in training
        {"name": "rope_train", "op": "rope", "tokens": 8192, "heads": 40, "d": 128, "rot": 128, "interleaved": False,
         "scaling": "none", "dtype": "bf16", "back": False, "far": 8192},
        # the gradient where half of the head turns, in pairs, at an odd number of tokens
        {"name": "rope_gradient", "op": "rope", "tokens": 4099, "heads": 24, "d": 96, "rot": 48, "interleaved": True,
         "scaling": "none", "dtype": "fp32", "back": True, "far": 4099},
        # a decoding step's rows into the cache
        {"name": "write_step", "op": "write", "tokens": 64, "hq": 32, "hkv": 8, "d": 128, "rot": 128, "interleaved": False,
         "scaling": "none", "dtype": "bf16", "page": 16, "far": 8192},
        # a prompt of a model whose positions are scaled by parts for long contexts
        {"name": "write_prompt", "op": "write", "tokens": 6001, "hq": 64, "hkv": 8, "d": 128, "rot": 128, "interleaved": False,
         "scaling": "parts", "dtype": "fp16", "page": 64, "far": 131072},
        # a few short requests decoding: latency
        {"name": "attn_step_short", "op": "attention", "requests": 8, "chunk": 1, "context": 1000, "hq": 32, "hkv": 4, "d": 128,
         "page": 16, "window": 0, "sinks": 0, "dtype": "bf16"},
        # a full batch decoding
        {"name": "attn_step_batch", "op": "attention", "requests": 128, "chunk": 1, "context": 8192, "hq": 32, "hkv": 8, "d": 128,
         "page": 16, "window": 0, "sinks": 0, "dtype": "bf16"},
        # two long contexts decoding: few rows, a long axis
        {"name": "attn_step_long", "op": "attention", "requests": 2, "chunk": 1, "context": 131072, "hq": 64, "hkv": 8, "d": 128,
         "page": 64, "window": 0, "sinks": 0, "dtype": "bf16"},
        # prompts in chunks beside decoding requests, small heads
        {"name": "attn_chunks_mixed", "op": "attention", "requests": 24, "chunk": 512, "context": 4096, "hq": 32, "hkv": 8, "d": 64,
         "page": 32, "window": 0, "sinks": 0, "dtype": "fp16"},
        # long contexts read through a window, the first tokens kept
        {"name": "attn_chunks_window", "op": "attention", "requests": 4, "chunk": 512, "context": 16384, "hq": 64, "hkv": 8, "d": 128,
         "page": 16, "window": 2048, "sinks": 4, "dtype": "bf16"},
        # two long requests re-encoded whole
        {"name": "attn_reencode", "op": "attention", "requests": 2, "chunk": 8192, "context": 0, "hq": 32, "hkv": 4, "d": 128,
         "page": 64, "window": 0, "sinks": 0, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tables", "rope", "write", "attention", "attention", "attention"])
    page = rng.choice([16, 32, 64, 128, 24])
    if op == "tables":
        stale = rng.random() < 0.5
        requests = _log(rng, 1, 512)
        return {"op": op, "requests": requests, "most": 1 if stale else rng.choice([1, 1, _log(rng, 2, 512)]),
                "context": _log(rng, 64, 1.0e6 / requests) if stale else _log(rng, 64, 16384), "page": page, "stale": stale}
    if op in ("rope", "write"):
        d = rng.choice([64, 80, 96, 128, 128, 128, 256])
        rot = rng.choice([d, d, d // 2])
        interleaved = rng.random() < 0.4
        case = {"op": op, "tokens": _log(rng, 1, 12000), "d": d, "rot": rot, "interleaved": interleaved,
                "scaling": rng.choice(["none", "none", "linear", "base", "parts"]), "dtype": rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                "far": _log(rng, 1024, 1.0e6)}
        if op == "rope":
            case.update(heads=_log(rng, 1, 64), back=rng.random() < 0.5)
        else:
            hkv = rng.choice([1, 2, 4, 8])
            case.update(hkv=hkv, hq=hkv * rng.choice([1, 4, 8]), page=page)
        return case
    hkv = rng.choice([1, 2, 4, 8])
    case = {"op": op, "requests": _log(rng, 1, 160), "chunk": rng.choice([1, 1, 1, _log(rng, 2, 16), _log(rng, 16, 4096)]),
            "context": rng.choice([0, _log(rng, 64, 131072), _log(rng, 64, 131072)]), "hkv": hkv, "hq": hkv * rng.choice([1, 2, 4, 8, 5]),
            "d": rng.choice([64, 128, 128, 128, 96, 256]), "page": page, "window": 0, "sinks": 0, "dtype": rng.choice(["bf16", "bf16", "fp16"])}
    if rng.random() < 0.35:
        case.update(window=_log(rng, 16, 4096), sinks=rng.choice([0, 1, 4, 16]))
    while case["requests"] > 1 and _too_large(case):
        case["requests"] -= 1
    while _too_large(case):
        case["context"], case["chunk"] = case["context"] * 7 // 8, max(1, case["chunk"] * 7 // 8)
    return case


def _too_large(case):
    keys = case["chunk"] + case["context"]
    return (case["requests"] * case["hq"] * case["chunk"] * keys > MOST_SCORES // 2
            or 2 * case["requests"] * case["hkv"] * case["d"] * keys > MOST_CACHE)


# ---- what a program has in hand ----------------------------------------------------------------------------------------

def _spread(low, high, n):
    """n whole numbers from low to high, evenly spread; high alone where n is 1."""
    return [high - (high - low) * i // max(1, n - 1) for i in range(n)]


def _lengths(case, seed):
    """start and count of every request, on the host: the scheduler knows them.  The seed says which request has which, so that the
    number of new tokens is the same for every seed."""
    g = torch.Generator().manual_seed(seed * 7919 + 17)
    R = case["requests"]

    def mixed(low, high):
        return torch.tensor(_spread(low, high, R))[torch.randperm(R, generator=g)]
    if case["op"] == "tables":
        start = mixed(max(1, case["context"] // 16), case["context"])
        if case["stale"]:
            return torch.zeros_like(start), start
        return start, mixed(1, case["most"])
    return mixed(case["context"] // 8, case["context"]), mixed(1, case["chunk"])


def _pages(have, wide, spare, g):
    """Block table, `wide` pages to a row, of requests that hold have[r] pages, scattered over a pool with `spare` more; what is left of
    the pool, and its size."""
    total = int(have.sum())
    pool = torch.randperm(total + spare, generator=g, device=DEV).to(torch.int32)
    table = torch.full((have.numel(), wide), -1, dtype=torch.int32, device=DEV)
    mine = torch.arange(wide, device=DEV)[None] < have.to(DEV)[:, None]
    table[mine] = pool[:total]
    return table, pool[total:].contiguous(), total + spare


def _frequencies(case):
    """Angle per position of each pair, and the factor on the result: what a model's configuration says, worked out once."""
    n, kind = case["rot"], case["scaling"]
    base = 1.0e6
    i = torch.arange(0, n, 2, dtype=torch.float64)
    if kind == "base":
        base *= 4.0 ** (n / max(1, n - 2))
    f = base ** (-i / n)
    if kind == "linear":
        f = f / 4.0
    if kind == "parts":
        # turns over the original context: many are left alone, few are slowed down four times, in between a mixture
        turns = f * 32768 / (2 * math.pi)
        left = ((turns - 1.0) / (32.0 - 1.0)).clamp(0, 1)
        f = f * (left + (1 - left) / 4.0)
    return f.to(DEV), 0.1 * math.log(4.0) + 1.0 if kind == "parts" else 1.0


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed * 1000003 + 5)
    op = case["op"]
    s = {"case": case}
    if op == "tables":
        start, count = _lengths(case, seed)
        page = case["page"]
        have = (torch.where(torch.tensor(case["stale"]), count, start) + page - 1) // page
        table, free, _ = _pages(have, (case["context"] + case["most"] + page - 1) // page + 1, case["requests"] * (case["most"] // page + 2), g)
        tokens = int(count.sum())
        s.update(start=start.int().to(DEV), count=count.int().to(DEV), held=have.int().to(DEV), keep=have.int().to(DEV), table=table,
                 free=free, free_count=torch.tensor([free.numel()], dtype=torch.int32, device=DEV),
                 token_begin=torch.empty(case["requests"] + 1, dtype=torch.int32, device=DEV),
                 slots=torch.empty(tokens, dtype=torch.int64, device=DEV), positions=torch.empty(tokens, dtype=torch.int32, device=DEV))
        return s
    dt = TYPES[case["dtype"]]
    if op in ("rope", "write"):
        T, d = case["tokens"], case["d"]
        s["inv_freq"], s["magnitude"] = _frequencies(case)
        s["positions"] = ((torch.arange(T, device=DEV) + int(torch.randint(0, case["far"], (1,), generator=g, device=DEV))) % case["far"]).int()
        if op == "rope":
            s["x"] = torch.randn(T, case["heads"], d, generator=g, device=DEV).to(dt)
            s["out"] = torch.empty_like(s["x"])
            return s
        # one row of the projection's output holds a token's queries, keys and values
        hq, hkv = case["hq"], case["hkv"]
        rows = torch.randn(T, hq + 2 * hkv, d, generator=g, device=DEV).to(dt)
        s["q"], s["k"], s["v"] = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
        s["q_out"] = torch.empty(T, hq, d, dtype=dt, device=DEV)
        pages = (T + case["page"] - 1) // case["page"] + 3
        s["slots"] = torch.randperm(pages * case["page"], generator=g, device=DEV)[:T] if T < 256 else (
            torch.randperm(pages, generator=g, device=DEV)[torch.arange(T, device=DEV) // case["page"]] * case["page"] + torch.arange(T, device=DEV) % case["page"])
        s["k_cache"] = torch.zeros(pages, case["page"], hkv, d, dtype=dt, device=DEV)
        s["v_cache"] = torch.zeros_like(s["k_cache"])
        return s
    start, count = _lengths(case, seed)
    page, d = case["page"], case["d"]
    table, _, pages = _pages((start + count + page - 1) // page, (case["context"] + case["chunk"] + page - 1) // page + 1, 7, g)
    T = int(count.sum())
    begin = torch.zeros(case["requests"] + 1, dtype=torch.int32)
    begin[1:] = count.cumsum(0)
    s.update(start=start.int().to(DEV), token_begin=begin.to(DEV), table=table, most_keys=int((start + count).max()), most_tokens=int(count.max()),
             q=torch.randn(T, case["hq"], d, generator=g, device=DEV).to(dt), scale=1.0 / math.sqrt(d))
    s["k_cache"] = torch.empty(pages, page, case["hkv"], d, dtype=dt, device=DEV).normal_(generator=g)
    s["v_cache"] = torch.empty_like(s["k_cache"]).normal_(generator=g)
    s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty(T, case["hq"], dtype=torch.float32, device=DEV)
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------------

_handle = None


def _context():
    """The library's handle on the device, one for the program."""
    global _handle
    if _handle is None:
        from paper_2605_07330_amd import srs
        _handle = srs.Context(0)
    return _handle


def _own(s):
    c, ctx = s["case"], _context()
    op = c["op"]
    if op == "tables":
        ctx.cache_tables(s["start"], s["count"], c["page"], s["held"], s["table"], s["free"], s["free_count"], s["token_begin"],
                         s["slots"], s["positions"])
        ctx.cache_release(s["keep"], s["held"], s["table"], s["free"], s["free_count"])
        return [s[n] for n in ("table", "held", "free", "free_count", "token_begin", "slots", "positions")]
    if op == "rope":
        ctx.rope(s["x"], s["out"], s["positions"], s["inv_freq"], interleaved=c["interleaved"], magnitude=s["magnitude"], transpose=c["back"])
        return [s["out"]]
    if op == "write":
        ctx.cache_write(s["k"], s["v"], s["k_cache"], s["v_cache"], s["slots"], q=s["q"], q_out=s["q_out"], positions=s["positions"],
                        inv_freq=s["inv_freq"], interleaved=c["interleaved"], magnitude=s["magnitude"])
        return [s["q_out"], s["k_cache"], s["v_cache"]]
    ctx.cache_attention(s["q"], s["out"], s["k_cache"], s["v_cache"], s["table"], s["token_begin"], s["start"], scale=s["scale"],
                        window=c["window"], sinks=c["sinks"], lse=s["lse"], most_tokens=s["most_tokens"], most_keys=s["most_keys"])
    return [s["out"], s["lse"]]


def run(s):
    if own:
        return _own(s)
    op = s["case"]["op"]
    return {"tables": _plain_tables, "rope": _plain_rope, "write": _plain_write, "attention": _plain_attention}[op](s)


def _plain_tables(s):
    page = s["case"]["page"]
    start, count, held, table, free, left = s["start"].long(), s["count"].long(), s["held"].long(), s["table"], s["free"], s["free_count"]
    wide = torch.arange(table.shape[1], device=DEV)[None]
    begin = torch.cat([torch.zeros(1, dtype=torch.long, device=DEV), count.cumsum(0)])
    want = ((start + count + page - 1) // page - held).clamp(min=0)
    before = want.cumsum(0) - want
    got = torch.minimum((left - before).clamp(min=0), want)
    fresh = (wide >= held[:, None]) & (wide < (held + got)[:, None])
    which = (left - 1 - before[:, None] - (wide - held[:, None])).clamp(0, max(0, free.numel() - 1))
    table.copy_(torch.where(fresh, free[which], table))
    r = torch.searchsorted(begin[1:], torch.arange(s["slots"].numel(), device=DEV), right=True)
    position = start[r] + torch.arange(s["slots"].numel(), device=DEV) - begin[r]
    s["positions"].copy_(position)
    s["slots"].copy_(table[r, position // page].long() * page + position % page)
    s["token_begin"].copy_(begin)
    # and the pages back: what was taken last goes first, so that the free list is what it was (its entries never moved)
    s["held"].copy_(torch.minimum(held + got, s["keep"].long()))
    return [s[n] for n in ("table", "held", "free", "free_count", "token_begin", "slots", "positions")]


def _turn(x, positions, inv_freq, interleaved, magnitude, sign):
    """Rotary positions on x [T, heads, d], in 32 bits; the angles, of far positions, in 64."""
    n = 2 * inv_freq.numel()
    angle = positions.double()[:, None] * inv_freq[None]
    c, si = (angle.cos() * magnitude).float()[:, None], (angle.sin() * magnitude * sign).float()[:, None]
    y = x.float()
    a, b = (y[..., 0:n:2], y[..., 1:n:2]) if interleaved else (y[..., :n // 2], y[..., n // 2:n])
    a, b = a * c - b * si, b * c + a * si
    turned = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([turned, y[..., n:]], -1).to(x.dtype)


def _plain_rope(s):
    c = s["case"]
    s["out"].copy_(_turn(s["x"], s["positions"], s["inv_freq"], c["interleaved"], s["magnitude"], -1.0 if c["back"] else 1.0))
    return [s["out"]]


def _plain_write(s):
    c = s["case"]
    s["q_out"].copy_(_turn(s["q"], s["positions"], s["inv_freq"], c["interleaved"], s["magnitude"], 1.0))
    k = _turn(s["k"], s["positions"], s["inv_freq"], c["interleaved"], s["magnitude"], 1.0)
    s["k_cache"].view(-1, c["hkv"], c["d"])[s["slots"]] = k
    s["v_cache"].view(-1, c["hkv"], c["d"])[s["slots"]] = s["v"]
    return [s["q_out"], s["k_cache"], s["v_cache"]]


def _plain_attention(s):
    c = s["case"]
    hq, hkv, d, page = c["hq"], c["hkv"], c["d"], c["page"]
    R, Q, L = c["requests"], s["most_tokens"], s["most_keys"]
    start, begin = s["start"].long(), s["token_begin"].long()
    count = begin[1:] - begin[:-1]
    j = torch.arange(L, device=DEV)
    rows = (s["table"].long()[:, j // page].clamp(min=0) * page + j % page).clamp(max=s["k_cache"].shape[0] * page - 1)   # [R, L]
    k = s["k_cache"].view(-1, hkv, d)[rows].float().permute(0, 2, 3, 1).contiguous()                                      # [R, hkv, d, L]
    v = s["v_cache"].view(-1, hkv, d)[rows].float().transpose(1, 2).contiguous()                                          # [R, hkv, L, d]
    i = torch.arange(Q, device=DEV)
    q = s["q"][(begin[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)].float()                                             # [R, Q, hq, d]
    q = q.view(R, Q, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(R, hkv, -1, d)
    score = (torch.matmul(q, k) * s["scale"]).view(R, hkv, hq // hkv, Q, L)
    at = (start[:, None] + i)[:, :, None]
    seen = (j <= at) & (i < count[:, None])[:, :, None]
    if c["window"]:
        seen = seen & ((at - j < c["window"]) | (j < c["sinks"]))
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=-1e30)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(R, hkv, -1, L), v).view(R, hkv, hq // hkv, Q, d) / total.clamp(min=1e-30)
    lse = (top + total.log()).squeeze(-1)
    # back to rows of tokens
    t = torch.arange(s["q"].shape[0], device=DEV)
    r = torch.searchsorted(begin[1:], t, right=True)
    s["out"].copy_(o.permute(0, 3, 1, 2, 4).reshape(R, Q, hq, d)[r, t - begin[r]])
    s["lse"].copy_(lse.permute(0, 3, 1, 2).reshape(R, Q, hq)[r, t - begin[r]])
    return [s["out"], s["lse"]]


# ---- what a pass cannot do without, and its result in 64 bits -------------------------------------------------------------

def _pairs(case):
    """Query-key pairs per query head, and keys read per key head, where lengths meet each other as in the mean over the seeds."""
    R, w = case["requests"], case["window"]
    mean = sum(_spread(case["context"] // 8, case["context"], R)) / R
    pairs = keys = 0.0
    for n in _spread(1, case["chunk"], R):
        seen, read = n * mean + n * (n + 1) / 2, mean + n
        if w:
            seen, read = min(seen, n * (w + case["sinks"])), min(read, n + w + case["sinks"])
        pairs, keys = pairs + seen, keys + read
    return pairs, keys


def work(case):
    op = case["op"]
    if op == "tables":
        tokens = sum(_spread(max(1, case["context"] // 16), case["context"], case["requests"]) if case["stale"] else _spread(1, case["most"], case["requests"]))
        return {"bytes": 12 * tokens + 24 * case["requests"] + 4 * max(case["requests"], tokens / case["page"]), "flops": 0}
    size = 4 if case["dtype"] == "fp32" else 2
    if op == "rope":
        n = case["tokens"] * case["heads"] * case["d"]
        return {"bytes": 2 * n * size + 4 * case["tokens"] + 4 * case["rot"], "flops": 3 * n}
    if op == "write":
        n = case["tokens"] * (case["hq"] + 2 * case["hkv"]) * case["d"]
        return {"bytes": 2 * n * size + 12 * case["tokens"] + 4 * case["rot"], "flops": 3 * n}
    pairs, keys = _pairs(case)
    tokens = sum(_spread(1, case["chunk"], case["requests"]))
    return {"bytes": 2 * keys * case["hkv"] * case["d"] * size + tokens * case["hq"] * (2 * case["d"] * size + 4) + 4 * keys / case["page"],
            "flops": 4 * pairs * case["hq"] * case["d"]}


def exact(case, seed):
    op = case["op"]
    if op == "tables":
        return None
    s = prepare(case, seed)
    if op in ("rope", "write"):
        phase = torch.polar(torch.full((1,), s["magnitude"], dtype=torch.float64, device=DEV),
                            torch.outer(s["positions"].to(torch.float64), s["inv_freq"]))          # magnitude * e^(i angle), [T, rot / 2]

        def turn(x, phase):
            n, y = case["rot"], x.to(torch.float64).clone()
            z = torch.complex(y[..., 0:n:2], y[..., 1:n:2]) if case["interleaved"] else torch.complex(y[..., 0:n // 2], y[..., n // 2:n])
            z = z * phase.unsqueeze(1)
            if case["interleaved"]:
                y[..., 0:n:2], y[..., 1:n:2] = z.real, z.imag
            else:
                y[..., 0:n // 2], y[..., n // 2:n] = z.real, z.imag
            return y
        if op == "rope":
            return [turn(s["x"], phase.conj() if case["back"] else phase)]
        caches = []
        for cache, rows in ((s["k_cache"], turn(s["k"], phase)), (s["v_cache"], s["v"].to(torch.float64))):
            full = torch.zeros(cache.shape, dtype=torch.float64, device=DEV)
            full[s["slots"] // case["page"], s["slots"] % case["page"]] = rows
            caches.append(full)
        return [turn(s["q"], phase)] + caches
    # attention: request by request, key head by key head
    begin, start, page, group = s["token_begin"].tolist(), s["start"].tolist(), case["page"], case["hq"] // case["hkv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device=DEV)
    for r in range(case["requests"]):
        a, b = begin[r], begin[r + 1]
        keys = start[r] + b - a
        pages = s["table"][r, : (keys + page - 1) // page].long()
        at = torch.arange(start[r], keys, device=DEV).unsqueeze(1)
        j = torch.arange(keys, device=DEV).unsqueeze(0)
        hidden = j > at
        if case["window"]:
            hidden = hidden | ((j <= at - case["window"]) & (j >= case["sinks"]))
        for h in range(case["hkv"]):
            k = s["k_cache"][pages, :, h].reshape(-1, case["d"])[:keys].to(torch.float64)
            v = s["v_cache"][pages, :, h].reshape(-1, case["d"])[:keys].to(torch.float64)
            for m in range(h * group, (h + 1) * group):
                x = (s["q"][a:b, m].to(torch.float64) @ k.t().contiguous()) * s["scale"]
                x.masked_fill_(hidden, -math.inf)
                lse[a:b, m] = torch.logsumexp(x, 1)
                out[a:b, m] = torch.softmax(x, 1) @ v
    return [out, lse]
