"""Plain 64-bit (or whole-number) references of the paged cache's operators,
on host tensors, one request, block and head at a time."""
from __future__ import annotations

import math

import torch

LARGEST = {torch.float8_e4m3fn: 448.0, torch.float8_e5m2: 57344.0}


def decode(codes: torch.Tensor) -> torch.Tensor:
    return codes.to(torch.float32).double()


def tables(old, new, bt, table, ring, head, count, slots, q_start):
    """(table, ring, [head, count], slots, q_start, verdict); inputs are lists
    and copied."""
    table, ring, slots = [list(r) for r in table], list(ring), list(slots)
    width, cap = (len(table[0]) if table else 0), len(ring)
    up = [-(-n // bt) for n in old], [-(-n // bt) for n in new]
    need = sum(max(0, c - b) for b, c in zip(*up))
    give = sum(max(0, b - c) for b, c in zip(*up))
    tokens = [max(0, n - o) for o, n in zip(old, new)]
    verdict = 0
    if any(n < 0 or n > width * bt for n in list(old) + list(new)):
        return table, ring, [head, count], slots, list(q_start), 1
    if need > count or count + give > cap:
        verdict |= 2
    if sum(tokens) > len(slots):
        verdict |= 4
    if verdict:
        return table, ring, [head, count], slots, list(q_start), verdict
    take, put, at = head, head + count, 0
    starts = [0]
    for r, (b, c) in enumerate(zip(*up)):
        for j in range(b, c):
            table[r][j] = ring[take % cap]
            take += 1
        for j in range(c, b):
            ring[put % cap] = table[r][j]
            put += 1
        for i in range(tokens[r]):
            p = old[r] + i
            slots[at] = table[r][p // bt] * bt + p % bt
            at += 1
        starts.append(at)
    return table, ring, [(head + need) % cap, count - need + give], slots, starts, 0


def to_grid(y: torch.Tensor, dtype) -> torch.Tensor:
    """y (64 bits) at the nearest value of the 8-bit type, ties to even, kept
    within its largest; NaN stays."""
    bits, low = (3, -6) if dtype == torch.float8_e4m3fn else (2, -14)
    y = torch.where(torch.isinf(y), torch.sign(y) * LARGEST[dtype], y)
    _, e = torch.frexp(y)
    step = torch.exp2((torch.clamp(e - 1, min=low) - bits).double())
    r = torch.round(y / step) * step
    return torch.where(torch.isnan(y), y, r.clamp(-LARGEST[dtype], LARGEST[dtype]))


def raised(scale: float, amax: float, fresh: bool, largest: float) -> float:
    base, low = (1.0, -100) if fresh else (scale, 0)
    n = low
    while amax > largest * base * 2.0 ** n:
        n += 1
    return base * 2.0 ** n


def append(x, codes, scale, slots, q_start, transposed):
    """Values of the codes [blocks, heads, bt, dim] and the scales after x
    [tokens, heads, dim] is stored; codes as in the cache, host tensors."""
    dtype = codes.dtype
    vals = decode(codes)
    vals = vals.transpose(2, 3).contiguous() if transposed else vals.clone()
    scale = scale.double().clone()
    bt, heads = vals.shape[2], vals.shape[1]
    by_block: dict[int, list[tuple[int, int]]] = {}
    for a, b in zip(q_start[:-1], q_start[1:]):
        for i in range(a, b):
            if 0 <= slots[i] < vals.shape[0] * bt:
                by_block.setdefault(slots[i] // bt, []).append((slots[i] % bt, i))
    for blk, items in by_block.items():
        fresh = any(off == 0 for off, _ in items)
        for h in range(heads):
            rows = torch.stack([x[i, h].double() for _, i in items])
            fin = rows[torch.isfinite(rows)].abs()
            amax = float(fin.max()) if fin.numel() else 0.0
            was = float(scale[blk, h])
            now = raised(was, amax, fresh, LARGEST[dtype])
            if fresh:
                vals[blk, h] = 0.0
            elif now != was:
                vals[blk, h] = to_grid(vals[blk, h] * (was / now), dtype)
            scale[blk, h] = now
            for (off, _), row in zip(items, rows):
                # the division is rounded to 32 bits first where it is not exact
                y = (row.float() / torch.tensor(now, dtype=torch.float32)).double()
                vals[blk, h, off] = to_grid(y, dtype)
    return vals.transpose(2, 3).contiguous() if transposed else vals, scale


def attend(q, k_vals, v_vals, table, lens, q_start, bt, scale, window=0, hidden=None):
    """(out, lse, weight, spread) in 64 bits: k_vals and v_vals are scaled
    values [blocks, heads, bt, dim]; weight is sum of |w v| (what a relative
    error of the weights is relative to) and spread the largest
    scale * sum |q k| of a row.  hidden(r, j): tokens that count as unseen."""
    tokens, hq, dim = q.shape
    heads = k_vals.shape[1]
    group = hq // heads
    out = torch.zeros(tokens, hq, dim, dtype=torch.float64)
    lse = torch.full((tokens, hq), -math.inf, dtype=torch.float64)
    weight, spread = torch.zeros_like(out), torch.zeros_like(lse)
    for r, n in enumerate(lens):
        a, b = q_start[r], q_start[r + 1]
        for i in range(a, b):
            p = n - (b - a) + (i - a)
            lo = max(0, p - window + 1) if window else 0
            js = [j for j in range(lo, p + 1) if not (hidden and hidden(r, j))]
            if not js:
                continue
            jt = torch.tensor(js)
            blk = torch.tensor([table[r][j // bt] for j in js])
            off = jt % bt
            for h in range(heads):
                k, v = k_vals[blk, h, off], v_vals[blk, h, off]
                qs = q[i, h * group:(h + 1) * group].double()
                s = qs @ k.t() * scale
                z = torch.logsumexp(s, 1)
                w = torch.exp(s - z[:, None])
                out[i, h * group:(h + 1) * group] = w @ v
                weight[i, h * group:(h + 1) * group] = w @ v.abs()
                lse[i, h * group:(h + 1) * group] = z
                spread[i, h * group:(h + 1) * group] = (qs.abs() @ k.abs().t() * abs(scale)).amax(1)
    return out, lse, weight, spread


def attend_bound(dtype, out, lse, weight, spread, n_max, dim):
    """What an output and its lse may be off, element by element.

    A score is a sum of dim exact products in 32 bits and two more factors:
    off by at most (dim + 4) 2^-24 spread; as an exponent of base 2 it is
    rounded again at most at 2 spread and raised by 15 (3 half steps of
    2^-24 (2 spread + 16)), and exp2 is off by 2^-22.  So every weight has a
    relative error of at most
      d = (dim + 4) 2^-24 spread + 3 * 2^-24 (2 spread + 16) + 2^-22,
    twice that after the division by their sum; the sums of n_max terms add
    2 n_max 2^-24 in the worst order.  The weights are rounded to half
    precision for the second product: 2^-11 (bf16 results) or twice, 2^-22
    (half precision results).  The result's own rounding is half a step, and
    2^-24 absolute for half precision's subnormals."""
    eps = torch.finfo(dtype).eps / 2
    d = (dim + 4) * 2.0 ** -24 * spread + 3 * 2.0 ** -24 * (2 * spread + 16) + 2.0 ** -22
    p = 2.0 ** -11 if dtype == torch.bfloat16 else 2.0 ** -21
    rel = 2 * d + 2 * n_max * 2.0 ** -24 + p
    own = weight * rel[..., None]
    tiny = 2.0 ** -24 if dtype == torch.float16 else 2.0 ** -126
    bound_out = own + eps * (out.abs() + own) + tiny
    bound_lse = d + n_max * 2.0 ** -24 + 2.0 ** -22 * (1 + torch.nan_to_num(lse, neginf=0.0).abs())
    return bound_out, bound_lse
