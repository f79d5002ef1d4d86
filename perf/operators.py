"""Timing cases of the paged 8-bit cache: what a session needs around its move.

A server holds the attention cache in blocks of tokens that its requests
share.  Four operators work on it: block tables and slot maps from request
lengths (``page_tables``), the store of new keys and values in 8 bits with a
scale for each block and head (``cache_append``), the attention that reads
them (``cache_attend``), and a session's blocks to and from the flat state
that the mover ships (``flatten_pages``, ``rehydrate_pages``).

Kinds of case:
  tables    a scheduler's step: requests grow, start, finish or step back
  append    the new tokens' keys and values into one layer's cache
  attend    the new tokens' attention over one layer's cache
  suspend   a session's blocks of every layer into the flat state
  resume    the flat state into other blocks of a pool

Cache of a layer: key codes [blocks, heads, block_tokens, dim], value codes
[blocks, heads, dim, block_tokens], scales [blocks, heads].  Keys and values
are N(0, 1) values scaled per channel by LogNormal(0, 0.5), 2% of the
channels another x20, as the mover's own stand-in states are.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda"
FP8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
LARGEST = {"e4m3": 448.0, "e5m2": 57344.0}
DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16}
SCALE_MIN = -100  # exponent of the smallest scale that a block is given


def _tables(name, **more):
    c = {"kind": "tables", "requests": 64, "old_lo": 1, "old_hi": 8192, "new_lo": 1, "new_hi": 1,
         "finish": 0.0, "back": 0.0, "block": 64}
    return {**c, **more, "name": name}


def _append(name, **more):
    c = {"kind": "append", "requests": 64, "old_lo": 1, "old_hi": 8192, "new_lo": 1, "new_hi": 1,
         "heads": 8, "dim": 128, "block": 64, "dtype": "bf16", "fmt": "e4m3"}
    return {**c, **more, "name": name}


def _attend(name, **more):
    c = {"kind": "attend", "requests": 64, "old_lo": 1, "old_hi": 8192, "new_lo": 1, "new_hi": 1,
         "heads": 8, "group": 4, "dim": 128, "block": 64, "dtype": "bf16", "fmt": "e4m3",
         "window": 0}
    return {**c, **more, "name": name}


def _pages(name, kind, **more):
    c = {"kind": kind, "layers": 28, "heads": 16, "dim": 128, "block": 64, "tokens": 7296,
         "fmt": "e4m3"}
    return {**c, **more, "name": name}


def listed():
    return [
        # The smallest scheduler's step: 64 requests, one token each, a few
        # of them done; one launch's latency.
        _tables("tables_step", finish=0.1, back=0.1),
        # A refill: a thousand prompts admitted at once, half of the older
        # requests leave; about a million slots.
        _tables("tables_admit", requests=1500, old_lo=0, old_hi=2048, new_lo=1, new_hi=8191,
                finish=0.3, block=16),
        # One token of 64 sessions into one layer: latency, and the blocks
        # whose scale a new token raises.
        _append("append_step"),
        # Prompts of ragged lengths into one layer of the production cache's
        # 16 heads, some of them continuing a session.
        _append("append_prompts", requests=24, old_lo=0, old_hi=512, new_lo=17, new_hi=7296,
                heads=16),
        # One session's token over a short cache of the tiny configuration
        # (8 heads x 512 tokens x 64): latency.
        _attend("attend_one", requests=1, old_lo=511, old_hi=511, group=1, dim=64),
        # A serving step: 64 sessions of 1 to 8192 tokens, grouped heads.
        _attend("attend_step"),
        # Eight sessions of the production cache (16 heads, 7296 tokens).
        _attend("attend_sessions", requests=8, old_lo=7295, old_hi=7295, heads=16, group=1),
        # The long-context state: 32 sessions of up to 32768 tokens, 8 heads.
        _attend("attend_long", requests=32, old_lo=24576, old_hi=32767, group=8),
        # Prompt chunks over what the sessions hold already.
        _attend("attend_prompts", requests=4, old_lo=1, old_hi=4096, new_lo=1500, new_hi=2048),
        # A chunk with a sliding window, half precision over 5-bit exponents.
        _attend("attend_window", requests=6, old_lo=1, old_hi=8192, new_lo=100, new_hi=1024,
                dim=64, dtype="fp16", fmt="e5m2", window=1024, block=32),
        # A short session leaves: a few blocks of 24 layers, ragged.
        _pages("suspend_short", "suspend", layers=24, heads=8, tokens=333),
        # The production cache arrives: 28 layers x 16 heads x 7296 tokens.
        _pages("resume_production", "resume"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["tables", "append", "attend", "attend", "suspend", "resume"])
    block = rng.choice([16, 32, 64, 128, 256])
    fmt = rng.choice(["e4m3", "e5m2"])
    dtype = rng.choice(["bf16", "fp16"])
    dim = rng.choice([64, 128, 192, 256])
    if kind == "tables":
        n = _log_int(rng, 1, 2000)
        return {"kind": kind, "requests": n, "old_lo": rng.choice([0, 1]),
                "old_hi": _log_int(rng, 1, 16384),
                "new_lo": 1, "new_hi": _log_int(rng, 1, max(2, min(8192, 1_000_000 // n))),
                "finish": rng.choice([0.0, 0.2, 0.5]), "back": rng.choice([0.0, 0.1, 0.3]),
                "block": block}
    if kind in ("suspend", "resume"):
        layers, heads = rng.randint(1, 32), rng.choice([1, 2, 5, 8, 16])
        most = 800_000_000 // (layers * heads * dim * 2)
        return {"kind": kind, "layers": layers, "heads": heads, "dim": dim, "block": block,
                "tokens": _log_int(rng, 1, min(32768, most)), "fmt": fmt}
    heads = rng.choice([1, 2, 4, 8, 16])
    if kind == "append":
        n = _log_int(rng, 1, 256)
        most = min(8192, 60_000_000 // (n * heads * dim))
        return {"kind": kind, "requests": n, "old_lo": rng.choice([0, 1]),
                "old_hi": _log_int(rng, 1, 2048), "new_lo": 1,
                "new_hi": _log_int(rng, 1, max(2, most)), "heads": heads, "dim": dim,
                "block": block, "dtype": dtype, "fmt": fmt}
    n = _log_int(rng, 1, 128)
    new = rng.choice([1, 1, 1, rng.randint(2, 8), _log_int(rng, 9, 1500)])
    group = rng.choice([1, 2, 3, 4, 7, 8, 16])
    new = min(new, max(1, 40_000_000 // (n * heads * group * dim)))
    # bounded by the size of the cache and by the number of scores
    most = min(32768, 500_000_000 // (n * heads * dim * 2),
               400_000_000 // (n * heads * group * new))
    old = _log_int(rng, 16, max(17, most))
    return {"kind": kind, "requests": n, "old_lo": rng.choice([0, 1, old // 2]), "old_hi": old,
            "new_lo": max(1, new // 2), "new_hi": new, "heads": heads, "group": group,
            "dim": dim, "block": block, "dtype": dtype, "fmt": fmt,
            "window": rng.choice([0, 0, 0, rng.randint(1, 2048)])}


# ---- inputs -----------------------------------------------------------------


def _spread(g, n, lo, hi):
    """n whole numbers of [lo, hi], even in their logarithm."""
    u = torch.rand(n, generator=g, dtype=torch.float64)
    a, b = math.log(lo + 0.5), math.log(hi + 1.0)
    return (a + (b - a) * u).exp().floor().clamp(lo, hi).to(torch.int64)


def _lengths(case, seed):
    """Each request's length before and after the step (host tensors): the
    same lengths for every seed, in another order."""
    g = torch.Generator().manual_seed(11)
    n = case["requests"]
    old = _spread(g, n, case["old_lo"], case["old_hi"])
    new = old + _spread(g, n, case["new_lo"], case["new_hi"])
    u = torch.rand(n, generator=g)
    finish, back = case.get("finish", 0.0), case.get("back", 0.0)
    steps = _spread(g, n, 1, 8)
    new = torch.where(u < finish, torch.zeros_like(new), new)
    new = torch.where((u >= finish) & (u < finish + back), (old - steps).clamp(min=0), new)
    order = torch.randperm(n, generator=g.manual_seed(seed))
    return old[order], new[order]


def _most_blocks(case):
    return -(-(case["old_hi"] + case["new_hi"]) // case["block"])


def _i32(t):
    return t.to(torch.int32).to(DEVICE)


def _pool_rows(case, g, lens):
    """A shuffled pool's block table for these lengths: (table, blocks)."""
    bt, width = case["block"], _most_blocks(case)
    need = (lens + bt - 1) // bt
    n_blocks = int(need.sum()) + int(need.sum()) // 8 + 4
    ids = torch.randperm(n_blocks, generator=g)
    start = torch.cumsum(need, 0) - need
    col = torch.arange(width)
    idx = (start[:, None] + col[None, :]).clamp(max=n_blocks - 1)
    table = torch.where(col[None, :] < need[:, None], ids[idx], torch.zeros_like(idx))
    return table, n_blocks, ids[int(need.sum()):]


def _channels(g, heads, dim):
    c = torch.exp(0.5 * torch.randn(heads, dim, generator=g, device=DEVICE))
    outlier = torch.rand(heads, dim, generator=g, device=DEVICE) < 0.02
    return torch.where(outlier, c * 20.0, c)


def _codes(g, shape, fmt):
    """Codes as a block's largest value leaves them: most of them well below
    the format's largest."""
    x = torch.randn(shape, generator=g, device=DEVICE, dtype=torch.bfloat16)
    return x.mul_(LARGEST[fmt] / 8.0).to(FP8[fmt])


def _cache(case, g, n_blocks, scale):
    h, bt, d, fmt = case["heads"], case["block"], case["dim"], case["fmt"]
    k = _codes(g, (n_blocks, h, bt, d), fmt)
    v = _codes(g, (n_blocks, h, d, bt), fmt)
    e = torch.randint(-1, 2, (2, n_blocks, h), generator=g, device=DEVICE).float()
    s = torch.exp2(e + math.floor(math.log2(scale * 8.0 / LARGEST[fmt])))
    return k, v, s[0].contiguous(), s[1].contiguous()


def prepare(case, seed):
    host = torch.Generator().manual_seed(seed)
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    s = {"case": case}
    if case["kind"] in ("suspend", "resume"):
        bt = case["block"]
        n = -(-case["tokens"] // bt)
        n_blocks = n + n // 2 + 2
        row = (case["layers"], 2, case["heads"])
        codes = _codes(g, (n_blocks, *row, bt * case["dim"]), case["fmt"]).view(torch.uint8)
        scales = torch.exp2(torch.randint(-9, -5, (n_blocks, *row), generator=g,
                                          device=DEVICE).float())
        s["pools"] = [codes, scales]
        s["pages"] = _i32(torch.randperm(n_blocks, generator=host)[:n])
        total = sum(-(-n * p[0].numel() * p.element_size() // 16) * 16 for p in s["pools"])
        s["flat"] = torch.zeros(total, dtype=torch.uint8, device=DEVICE)
        if case["kind"] == "resume":
            s["flat"].copy_(torch.randint(0, 256, (total,), generator=g, device=DEVICE,
                                          dtype=torch.uint8))
        s["verdict"] = torch.zeros(1, dtype=torch.int32, device=DEVICE)
        return s
    old, new = _lengths(case, seed)
    bt, width, n_req = case["block"], _most_blocks(case), case["requests"]
    if case["kind"] == "tables":
        table, n_blocks, rest = _pool_rows(case, host, old)
        need = int((((new + bt - 1) // bt) - ((old + bt - 1) // bt)).clamp(min=0).sum())
        extra = need + 17
        rest = torch.cat([rest, torch.arange(n_blocks, n_blocks + extra)])
        ring = torch.full((n_blocks + extra,), -1, dtype=torch.int64)
        head = int(torch.randint(0, ring.numel(), (1,), generator=host))
        ring[(head + torch.arange(rest.numel())) % ring.numel()] = rest
        tokens = int((new - old).clamp(min=0).sum())
        s.update(old=_i32(old), new=_i32(new), table=_i32(table), ring=_i32(ring),
                 pool_in=_i32(torch.tensor([head, rest.numel()])),
                 pool_out=_i32(torch.zeros(2)),
                 slots=torch.full((tokens + n_req,), -1, dtype=torch.int64, device=DEVICE),
                 q_start=_i32(torch.zeros(n_req + 1)), verdict=_i32(torch.zeros(1)))
        return s
    new_tokens = new - old
    q_start = torch.cat([torch.zeros(1, dtype=torch.int64), torch.cumsum(new_tokens, 0)])
    total = int(q_start[-1])
    table, n_blocks, _ = _pool_rows(case, host, new)
    h, d, dt = case["heads"], case["dim"], DTYPE[case["dtype"]]
    s.update(q_start=_i32(q_start), verdict=_i32(torch.zeros(1)))
    if case["kind"] == "append":
        s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"] = _cache(case, g, n_blocks, 6.0)
        req = torch.repeat_interleave(torch.arange(n_req), new_tokens)
        pos = old[req] + torch.arange(total) - q_start[req]
        s["slots"] = (table[req, pos // bt] * bt + pos % bt).to(DEVICE)
        # a projection's output: queries, keys and values of a token side by side
        qkv = torch.randn(total, 4 * h, d, generator=g, device=DEVICE, dtype=torch.float32)
        qkv.mul_(_channels(g, 4 * h, d))
        qkv = qkv.to(dt)
        s["k"], s["v"] = qkv[:, 2 * h:3 * h], qkv[:, 3 * h:]
        return s
    # logits of a trained model's spread: a few tokens carry most of the weight
    s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"] = _cache(case, g, n_blocks, 1.0)
    hq = h * case["group"]
    q = torch.randn(total, hq, d, generator=g, device=DEVICE, dtype=torch.float32) * 1.5
    s.update(q=q.to(dt), table=_i32(table), lens=_i32(new), max_len=int(new.max()),
             max_new=int(new_tokens.max()), scale=1.0 / math.sqrt(d),
             out=torch.zeros(total, hq, d, dtype=dt, device=DEVICE),
             lse=torch.zeros(total, hq, dtype=torch.float32, device=DEVICE))
    return s


# ---- the plain forms ----------------------------------------------------------


def _plain_tables(s):
    bt, old, new = s["case"]["block"], s["old"].long(), s["new"].long()
    table, ring, cap = s["table"], s["ring"], s["ring"].numel()
    width, n_slots = table.shape[1], s["slots"].numel()
    head, count = s["pool_in"][0].long(), s["pool_in"][1].long()
    zero = torch.zeros(1, dtype=torch.int64, device=old.device)
    q_start = torch.cat([zero, torch.cumsum((new - old).clamp(min=0), 0)])
    b, c = (old + bt - 1) // bt, (new + bt - 1) // bt
    need, give = (c - b).clamp(min=0), (b - c).clamp(min=0)
    p, q = torch.cumsum(need, 0) - need, torch.cumsum(give, 0) - give
    bad_len = ((old < 0) | (new < 0) | (old > width * bt) | (new > width * bt)).any()
    bad_pool = (need.sum() > count) | (count + give.sum() > cap)
    bad_slots = q_start[-1] > n_slots
    ok = ~(bad_len | bad_pool | bad_slots)
    col = torch.arange(width, device=old.device)[None, :]
    take = (col >= b[:, None]) & (col < c[:, None]) & ok
    got = ring[(head + p[:, None] + col - b[:, None]) % cap]
    table_new = torch.where(take, got, table)
    leave = (col >= c[:, None]) & (col < b[:, None]) & ok
    to = (head + count + q[:, None] + col - c[:, None]) % cap
    to = torch.where(leave, to, torch.full_like(to, cap))
    ring_new = torch.cat([ring, ring[:1]]).scatter_(0, to.reshape(-1), table.reshape(-1))[:cap]
    j = torch.arange(n_slots, device=old.device)
    r = (torch.searchsorted(q_start, j, right=True) - 1).clamp(max=old.numel() - 1)
    pos = old[r] + j - q_start[r]
    slot = table_new[r, (pos // bt).clamp(max=width - 1)].long() * bt + pos % bt
    slots = torch.where((j < q_start[-1]) & ok, slot, s["slots"])
    pool = torch.stack([(head + need.sum()) % cap, count - need.sum() + give.sum()])
    pool = torch.where(ok, pool, s["pool_in"].long())
    verdict = bad_len.int() + 2 * bad_pool.int() + 4 * bad_slots.int()
    q_start = torch.where(ok, q_start, s["q_start"].long())
    return {"table": table_new, "ring": ring_new, "pool": pool.int(), "slots": slots,
            "q_start": q_start.int(), "verdict": verdict.reshape(1)}


def _raise_scale(old_scale, amax, fresh, largest):
    """The scale that holds amax: a fresh block's own, or the older one times
    the smallest power of two that is enough."""
    base = torch.where(fresh, torch.ones_like(old_scale), old_scale).double()
    m, e = torch.frexp(amax.double())
    m0, e0 = torch.frexp(base * largest)
    k = e - e0 + (m > m0).int()
    k = torch.where(amax == 0, torch.full_like(k, -10000), k)
    low = torch.where(fresh, torch.full_like(k, SCALE_MIN), torch.zeros_like(k))
    return (base * torch.exp2(torch.maximum(k, low).double())).float()


def _to_codes(x, scale, fmt):
    y = x / scale
    y = torch.where(torch.isnan(y), y, y.clamp(-LARGEST[fmt], LARGEST[fmt]))
    return y.to(FP8[fmt])


def _plain_append(s):
    case = s["case"]
    bt, fmt, n_req = case["block"], case["fmt"], case["requests"]
    slots, q_start = s["slots"], s["q_start"].long()
    total = slots.numel()
    # the blocks that the new tokens touch: at most q/bt + 2 of a request,
    # so request r's begin at place q_start[r]/bt + 2r of a list; places that
    # are left over repeat the request's first block
    places = torch.arange(total // bt + 2 * n_req, device=slots.device)
    first = q_start // bt + 2 * torch.arange(n_req + 1, device=slots.device)
    r = (torch.searchsorted(first, places, right=True) - 1).clamp(max=n_req - 1)
    begin, end = q_start[r], q_start[r + 1]
    at = slots[begin] % bt
    nth = places - first[r]
    nth = torch.where(nth * bt < at + end - begin, nth, torch.zeros_like(nth))
    token = begin[:, None] + nth[:, None] * bt - at[:, None] + torch.arange(bt, device=slots.device)
    fresh_token = (token >= begin[:, None]) & (token < end[:, None])  # [places, bt]
    token = token.clamp(0, total - 1)
    page = slots[torch.maximum(begin, begin + nth * bt - at)] // bt
    fresh = ((nth > 0) | (at == 0))[:, None]

    def store(x, cache, scale, transposed):
        xs = x[token].float().transpose(1, 2)  # [places, heads, bt, dim]
        new = fresh_token[:, None, :, None]
        size = torch.where(new & torch.isfinite(xs), xs.abs(), torch.zeros_like(xs))
        amax = size.amax(dim=(2, 3))
        was = scale[page]
        now = _raise_scale(was, amax, fresh, LARGEST[fmt])
        codes = cache.view(torch.uint8)[page].view(FP8[fmt])
        codes = codes.transpose(2, 3) if transposed else codes
        moved = (codes.float() * (was / now)[:, :, None, None]).to(FP8[fmt]).view(torch.uint8)
        kept = torch.where(fresh[:, :, None, None], torch.zeros_like(moved), moved)
        put = _to_codes(xs, now[:, :, None, None], fmt).view(torch.uint8)
        page_new = torch.where(new, put, kept)
        page_new = page_new.transpose(2, 3) if transposed else page_new
        cache.view(torch.uint8)[page] = page_new
        scale[page] = now

    store(s["k"], s["k_cache"], s["k_scale"], False)
    store(s["v"], s["v_cache"], s["v_scale"], True)
    return {"k": s["k_cache"], "v": s["v_cache"], "k_scale": s["k_scale"],
            "v_scale": s["v_scale"], "verdict": s["verdict"]}


def _plain_attend(s):
    case = s["case"]
    n_req, h, g, d, bt = (case[x] for x in ("requests", "heads", "group", "dim", "block"))
    lens, q_start = s["lens"].long(), s["q_start"].long()
    n_new, total = s["max_new"], s["q"].shape[0]
    blocks = -(-s["max_len"] // bt)
    length = blocks * bt
    rows = s["table"][:, :blocks].long()

    def gather(cache, scale):
        x = cache.view(torch.uint8)[rows].view(cache.dtype).float()  # [requests, blocks, heads, ..]
        return x * scale[rows][..., None, None]

    k = gather(s["k_cache"], s["k_scale"]).permute(0, 2, 1, 3, 4).reshape(n_req, h, length, d)
    v = gather(s["v_cache"], s["v_scale"]).permute(0, 2, 1, 4, 3).reshape(n_req, h, length, d)
    i = torch.arange(n_new, device=lens.device)
    token = (q_start[:-1, None] + i).clamp(max=total - 1)
    q = s["q"][token].float().reshape(n_req, n_new, h, g, d).permute(0, 2, 1, 3, 4)
    scores = torch.matmul(q.reshape(n_req, h, n_new * g, d), k.transpose(2, 3)) * s["scale"]
    scores = scores.reshape(n_req, h, n_new, g, length)
    pos = (lens - (q_start[1:] - q_start[:-1]))[:, None] + i  # [requests, new]
    col = torch.arange(length, device=lens.device)
    seen = col <= pos[..., None]
    if case["window"]:
        seen = seen & (col > pos[..., None] - case["window"])
    scores = scores.masked_fill(~seen[:, None, :, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(torch.isfinite(top), top, torch.zeros_like(top)))
    den = p.sum(-1, keepdim=True)
    out = torch.matmul(p.reshape(n_req, h, n_new * g, length), v).reshape(n_req, h, n_new, g, d)
    out = out / torch.where(den > 0, den, torch.ones_like(den))
    lse = torch.log(den) + top
    t = torch.arange(total, device=lens.device)
    r = torch.searchsorted(q_start, t, right=True) - 1
    out = out[r, :, t - q_start[r]].reshape(total, h * g, d).to(s["q"].dtype)
    return {"out": out, "lse": lse[r, :, t - q_start[r]].reshape(total, h * g)}


def _plain_suspend(s):
    pages = s["pages"].long()
    at = 0
    for pool in s["pools"]:
        x = pool[pages].reshape(-1).view(torch.uint8)
        s["flat"][at:at + x.numel()] = x
        at += -(-x.numel() // 16) * 16
    return {"flat": s["flat"]}


def _plain_resume(s):
    pages = s["pages"].long()
    at = 0
    for pool in s["pools"]:
        size = pages.numel() * pool[0].numel() * pool.element_size()
        x = s["flat"][at:at + size].view(pool.dtype).reshape(pages.numel(), *pool.shape[1:])
        pool[pages] = x
        at += -(-size // 16) * 16
    return {"codes": s["pools"][0], "scales": s["pools"][1].view(torch.int32)}


def _own(s):
    from paper_2607_10389_amd import _cache as cache
    case = s["case"]
    kind = case["kind"]
    if kind == "tables":
        cache.page_tables(s["old"], s["new"], case["block"], s["table"], s["ring"], s["pool_in"],
                          s["pool_out"], s["slots"], s["q_start"], s["verdict"])
        return {"table": s["table"], "ring": s["ring"], "pool": s["pool_out"],
                "slots": s["slots"], "q_start": s["q_start"], "verdict": s["verdict"]}
    if kind == "append":
        cache.cache_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["k_scale"],
                           s["v_scale"], s["slots"], s["q_start"], s["verdict"])
        return {"k": s["k_cache"], "v": s["v_cache"], "k_scale": s["k_scale"],
                "v_scale": s["v_scale"], "verdict": s["verdict"]}
    if kind == "attend":
        if "ws" not in s:  # a server's own, kept from step to step
            n = cache.attend_ws_bytes(s["q"], s["k_cache"], s["lens"], s["max_len"])
            s["ws"] = torch.empty(n, dtype=torch.uint8, device=DEVICE)
        cache.cache_attend(s["q"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"],
                           s["table"], s["lens"], s["q_start"], s["out"], s["ws"],
                           max_len=s["max_len"], scale=s["scale"], window=case["window"],
                           lse=s["lse"], verdict=s["verdict"])
        return {"out": s["out"], "lse": s["lse"]}
    if "handle" not in s:  # the table of the pools' addresses, as for wm_flatten's leaves
        s["handle"] = cache.PoolTable(s["pools"])
    if kind == "suspend":
        cache.flatten_pages(s["handle"], s["pages"], s["flat"], s["verdict"])
        return {"flat": s["flat"]}
    cache.rehydrate_pages(s["flat"], s["handle"], s["pages"], s["verdict"])
    return {"codes": s["pools"][0], "scales": s["pools"][1].view(torch.int32)}


_PLAIN = {"tables": _plain_tables, "append": _plain_append, "attend": _plain_attend,
          "suspend": _plain_suspend, "resume": _plain_resume}


def run(state):
    if own:
        return _own(state)
    return _PLAIN[state["case"]["kind"]](state)


# ---- what a pass cannot do without -----------------------------------------------


def work(case):
    if case["kind"] in ("suspend", "resume"):
        n = -(-case["tokens"] // case["block"])
        page = case["layers"] * 2 * case["heads"] * (case["block"] * case["dim"] + 4)
        return {"bytes": 2 * n * page + 4 * n, "flops": 0}
    old, new = _lengths(case, 1)
    added = (new - old).clamp(min=0)
    bt, n_req, tokens = case["block"], case["requests"], int(added.sum())
    if case["kind"] == "tables":
        moved = int(((new + bt - 1) // bt - (old + bt - 1) // bt).abs().sum())
        return {"bytes": 8 * n_req + 4 * (n_req + 1) + 8 * moved + 8 * tokens + 20, "flops": 0}
    h, d = case["heads"], case["dim"]
    if case["kind"] == "append":
        blocks = int(((new + bt - 1) // bt - old // bt).sum())
        return {"bytes": tokens * (h * d * (2 * 2 + 2) + 8) + blocks * h * 16, "flops": 0}
    hq, window = h * case["group"], case["window"]
    lo = torch.zeros_like(old)
    if window:
        lo = (old + 1 - window).clamp(min=0)
    held = int((new - lo).sum())
    # sum of min(position + 1, window) over the new tokens
    if window:
        cut = new.clamp(max=window)
        start = old.clamp(max=window)
        seen = (cut * (cut + 1) - start * (start + 1)) // 2 + (new - cut - (old - start)) * window
    else:
        seen = (new * (new + 1) - old * (old + 1)) // 2
    size = held * 2 * h * d + (held // bt + n_req) * h * 8 + tokens * hq * (2 * 2 * d + 4)
    return {"bytes": size, "flops": 4 * d * hq * int(seen.sum())}


# ---- the definitions in 64 bits ----------------------------------------------------


def _grid(y, fmt):
    """y rounded to the nearest value of the format, ties to even."""
    bits, low = (3, -6) if fmt == "e4m3" else (2, -14)
    _, e = torch.frexp(y)
    step = torch.exp2((torch.clamp(e - 1, min=low) - bits).double())
    return torch.clamp(torch.round(y / step) * step, -LARGEST[fmt], LARGEST[fmt])


def _exact_append(case, s):
    bt, fmt = case["block"], case["fmt"]
    out = {}
    page, off = s["slots"] // bt, s["slots"] % bt
    n_blocks = s["k_cache"].shape[0]
    put = torch.zeros(n_blocks, bt, dtype=torch.bool, device=DEVICE)
    put[page, off] = True
    fresh, touched = put[:, 0], put.any(1)
    for x, name in ((s["k"], "k"), (s["v"], "v")):
        values = s[name + "_cache"].double()
        values = values.transpose(2, 3).contiguous() if name == "v" else values
        was = s[name + "_scale"].double()
        rows = torch.zeros_like(values)
        rows[page, :, off] = x.double()
        amax = rows.abs().amax(dim=(2, 3))
        # the least power of two that holds it: by logarithm, then put right
        base = torch.where(fresh[:, None], torch.ones_like(was), was) * LARGEST[fmt]
        k = torch.ceil(torch.log2(torch.where(amax > 0, amax, base * 1e-40) / base))
        k = torch.where(base * torch.exp2(k - 1) >= amax, k - 1, k)
        k = torch.where(base * torch.exp2(k) < amax, k + 1, k)
        k = torch.maximum(k, torch.where(fresh[:, None], SCALE_MIN, 0))
        now = base / LARGEST[fmt] * torch.exp2(k)
        now = torch.where(touched[:, None], now, was)
        values = torch.where(fresh[:, None, None, None], torch.zeros_like(values),
                             _grid(values * (was / now)[..., None, None], fmt))
        new = put[:, None, :, None]
        values = torch.where(new, _grid(rows / now[..., None, None], fmt), values)
        out[name] = values.transpose(2, 3).contiguous() if name == "v" else values
        out[name + "_scale"] = now
    return {**out, "verdict": None}


def exact(case, seed):
    if case["kind"] not in ("append", "attend"):
        return None  # whole numbers
    s = prepare(case, seed)
    if case["kind"] == "append":
        if s["k_cache"].numel() > 150_000_000:
            return None
        return _exact_append(case, s)
    bt, g, window = case["block"], case["group"], case["window"]
    out, lse = s["out"].double(), s["lse"].double()
    q_start, lens = s["q_start"].tolist(), s["lens"].tolist()
    for r, n in enumerate(lens):
        a, b = q_start[r], q_start[r + 1]
        pos = n - (b - a) + torch.arange(b - a, device=DEVICE)
        ids = s["table"][r, :-(-n // bt)].long()
        col = torch.arange(n, device=DEVICE)
        hidden = col[None, :] > pos[:, None]
        if window:
            hidden |= col[None, :] <= pos[:, None] - window
        hidden = hidden.repeat_interleave(g, 0)
        for head in range(case["heads"]):
            k = (s["k_cache"].view(torch.uint8)[ids, head].view(s["k_cache"].dtype).double()
                 * s["k_scale"][ids, head].double()[:, None, None])
            v = (s["v_cache"].view(torch.uint8)[ids, head].view(s["v_cache"].dtype).double()
                 * s["v_scale"][ids, head].double()[:, None, None])
            k = k.reshape(-1, case["dim"])[:n]
            v = v.transpose(1, 2).reshape(-1, case["dim"])[:n]
            q = s["q"][a:b, head * g:(head + 1) * g].double().reshape(-1, case["dim"])
            x = (q @ k.t() * s["scale"]).masked_fill_(hidden, -math.inf)
            z = torch.logsumexp(x, 1)
            y = torch.exp(x.sub_(z[:, None])) @ v
            out[a:b, head * g:(head + 1) * g] = y.reshape(b - a, g, -1)
            lse[a:b, head * g:(head + 1) * g] = z.reshape(b - a, g)
    return {"out": out, "lse": lse}
