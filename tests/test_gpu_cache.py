"""GPU parity of the paged 8-bit cache (include/wm_cache.h) against plain
whole-number and 64-bit references: block tables and slot maps, stored codes
and scales, attention, blocks to and from the flat state, and a session moved
with all of them."""
import math

import numpy as np
import pytest
import torch

import cache_reference as ref
from gpu_helpers import random_bytes, say

pytestmark = pytest.mark.gpu

E4, E5 = torch.float8_e4m3fn, torch.float8_e5m2
BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def wm():
    from paper_2607_10389_amd import _cache
    return _cache


def dev(x, dtype=torch.int32):
    return torch.as_tensor(x, dtype=dtype).cuda()


def word():
    return dev([0])


# ---- block tables and slot maps ----------------------------------------------


def run_tables(wm, old, new, bt, width, ring, head, count, slot_cap, seed=0, stride=None):
    g = np.random.default_rng(seed)
    n = len(old)
    stride = stride or width
    table = g.integers(0, 1 << 20, (n, stride)).tolist()
    slots = (-g.integers(1, 1000, slot_cap)).tolist()
    q0 = [-7] * (n + 1)
    want = ref.tables(old, new, bt, [r[:width] for r in table], ring, head, count, slots, q0)
    t = dev(table).reshape(n, stride)
    rg, pi, po = dev(ring), dev([head, count]), dev([-1, -1])
    sl, qs, v = dev(slots, torch.int64), dev(q0), dev([77])
    for _ in range(2):  # the same again: same inputs, same outputs
        wm.page_tables(dev(old), dev(new), bt, t[:, :width], rg, pi, po, sl, qs, v)
        torch.cuda.synchronize()
        assert int(v.item()) == want[5]
        got = t.cpu().tolist()
        assert [r[:width] for r in got] == want[0]
        assert [r[width:] for r in got] == [r[width:] for r in table]
        assert rg.cpu().tolist() == want[1]
        assert po.cpu().tolist() == want[2]
        assert sl.cpu().tolist() == want[3]
        assert qs.cpu().tolist() == want[4]
        assert pi.cpu().tolist() == [head, count]
    return want


@pytest.mark.parametrize("n,bt,most,seed", [(1, 16, 40, 0), (5, 64, 300, 1), (64, 32, 500, 2),
                                            (1024, 16, 90, 3), (1025, 128, 700, 4),
                                            (2500, 16, 40, 5)])
def test_tables_of_random_steps(wm, n, bt, most, seed):
    say(f"[tables] n={n} bt={bt} most={most}")
    g = np.random.default_rng(seed)
    old = g.integers(0, most + 1, n)
    new = np.where(g.random(n) < 0.3, g.integers(0, most + 1, n), old + 1)
    new = np.where(g.random(n) < 0.2, 0, new)
    width = -(-(most + 1) // bt)
    up = lambda x: -(-x // bt)  # noqa: E731
    need = int(np.maximum(0, up(new) - up(old)).sum())
    give = int(np.maximum(0, up(old) - up(new)).sum())
    count = need + 3
    cap = count + give + 5
    ring = g.permutation(cap * 2)[:cap].tolist()
    tokens = int(np.maximum(0, new - old).sum())
    run_tables(wm, old.tolist(), new.tolist(), bt, width, ring, cap - 2, count, tokens + 9, seed,
               stride=width + 3)


def test_tables_of_no_requests_and_of_no_change(wm):
    run_tables(wm, [5, 0, 64], [5, 0, 64], 64, 4, [1, 2, 3], 0, 3, 4)
    v, po, qs = dev([9]), dev([5, 5]), dev([3])
    e = dev([])
    wm.page_tables(e, e, 64, torch.zeros(0, 4, dtype=torch.int32, device="cuda"), dev([1, 2]),
                   dev([1, 2]), po, dev([], torch.int64), qs, v)
    assert v.item() == 0 and po.tolist() == [1, 2] and qs.tolist() == [0]


def test_tables_of_one_long_request(wm):
    # every workgroup writes slots of the same request
    run_tables(wm, [37, 3], [150_000, 4], 16, 9400, list(range(10_000)), 9_990, 9_800, 150_000)


@pytest.mark.parametrize("old,new,count,slots,verdict", [
    ([0, 10], [-1, 11], 9, 40, 1), ([0, -5], [3, 11], 9, 40, 1), ([0, 1], [3, 65], 9, 99, 1),
    ([65, 1], [0, 2], 9, 99, 1), ([0, 16], [33, 17], 3, 40, 2), ([0, 16], [33, 17], 4, 33, 4),
    ([0, 16], [33, 17], 4, 34, 0), ([64, 16], [0, 17], 9, 40, 2), ([0, 16], [33, 17], 3, 3, 6)])
def test_tables_that_are_refused_change_nothing(wm, old, new, count, slots, verdict):
    want = run_tables(wm, old, new, 16, 4, list(range(100, 112)), 7, count, slots)
    assert want[5] == verdict


# ---- stored codes ----------------------------------------------------------------


def make_cache(blocks, heads, bt, dim, fmt, seed, stride=0, spread=True):
    """Codes and scales in a pool whose blocks lie `stride` bytes further
    apart than they need to."""
    g = torch.Generator().manual_seed(seed)
    page = heads * bt * dim
    out = []
    for shape in ((heads, bt, dim), (heads, dim, bt)):
        x = (torch.randn(blocks, page, generator=g) * ref.LARGEST[fmt] / 8).to(fmt)
        pool = torch.zeros(blocks, page + stride, dtype=torch.uint8)
        pool[:, :page] = x.view(torch.uint8)
        out.append(pool.cuda()[:, :page].view(fmt).view(blocks, *shape))
    for _ in range(2):
        e = torch.randint(-9, -5, (blocks, heads), generator=g).float()
        s = torch.exp2(e)
        if spread:
            s = s * (1 + torch.rand(blocks, heads, generator=g))
        pool = torch.zeros(blocks, heads + stride // 16)
        pool[:, :heads] = s
        out.append(pool.cuda()[:, :heads])
    return out


def layout(lens, bt, seed, extra=3):
    """Block table rows of a shuffled pool for these lengths: (rows, blocks)."""
    g = np.random.default_rng(seed)
    need = [-(-n // bt) for n in lens]
    blocks = sum(need) + extra
    ids = g.permutation(blocks).tolist()
    width = max(need + [1])
    rows, at = [], 0
    for c in need:
        rows.append(ids[at:at + c] + [-5] * (width - c))
        at += c
    return rows, blocks


APPENDS = [
    # old lengths, new tokens, heads, bt, dim, type, format, block stride
    ([0], [1], 1, 16, 64, BF, E4, 0),
    ([5, 0, 31, 64], [1, 1, 1, 1], 2, 32, 128, BF, E4, 64),
    ([0, 17, 3], [130, 40, 0], 3, 64, 64, HF, E5, 0),
    ([1, 255, 0], [300, 2, 256], 2, 256, 192, BF, E5, 32),
    ([15, 16, 33], [1, 50, 16], 1, 16, 256, HF, E4, 0),
    ([0, 100], [129, 29], 2, 128, 128, HF, E4, 16),
]


@pytest.mark.parametrize("old,new,heads,bt,dim,dt,fmt,stride", APPENDS)
def test_stored_codes_and_scales(wm, old, new, heads, bt, dim, dt, fmt, stride):
    say(f"[append] old={old} new={new} heads={heads} bt={bt} dim={dim} {dt} {fmt}")
    rows, blocks = layout([o + n for o, n in zip(old, new)], bt, 1)
    k, v, ks, vs = make_cache(blocks, heads, bt, dim, fmt, 2, stride)
    starts = [0] + np.cumsum(new).tolist()
    slots = [rows[r][(o + i) // bt] * bt + (o + i) % bt
             for r, (o, n) in enumerate(zip(old, new)) for i in range(n)]
    g = torch.Generator().manual_seed(3)
    total = starts[-1]
    # a packed projection's rows, with magnitudes from far below the scales
    # to far above them, by token
    qkv = torch.randn(total + 2, 3 * heads + 1, dim, generator=g)
    qkv *= torch.exp2(torch.randint(-12, 7, (total + 2, 1, 1), generator=g).float())
    qkv[::5] = 0.0
    qkv = qkv.to(dt).cuda()
    kn, vn = qkv[:, heads:2 * heads], qkv[:, 2 * heads:3 * heads]
    want_k, want_ks = ref.append(kn.cpu(), k.cpu(), ks.cpu(), slots, starts, False)
    want_v, want_vs = ref.append(vn.cpu(), v.cpu(), vs.cpu(), slots, starts, True)
    verdict = word()
    for _ in range(2):  # storing the same again changes nothing
        wm.cache_append(kn, vn, k, v, ks, vs, dev(slots + [-1, -1], torch.int64), dev(starts),
                        verdict)
        torch.cuda.synchronize()
        assert verdict.item() == 0
        assert torch.equal(ks.cpu().double(), want_ks) and torch.equal(vs.cpu().double(), want_vs)
        assert torch.equal(ref.decode(k.cpu()), want_k)
        assert torch.equal(ref.decode(v.cpu()), want_v)


def test_stored_infinities_nan_and_extremes(wm):
    heads, bt, dim = 1, 16, 64
    for fmt in (E4, E5):
        k, v, ks, vs = make_cache(4, heads, bt, dim, fmt, 5)
        x = torch.zeros(6, heads, dim)
        x[0, 0, :4] = torch.tensor([math.inf, -math.inf, math.nan, 3.0])
        x[1] = 3.38e38        # the largest magnitudes of the type
        x[2] = 1e-38
        x[3] = -0.0
        x[4, 0, 0] = math.nan  # nothing finite but zeros
        x[5] = 448.0
        xb = x.to(BF).cuda()
        # tokens 0..3 fresh blocks of their own, 4 and 5 into a block in use
        slots, starts = [0, 16, 32, 48, 49, 50], [0, 1, 2, 3, 6]
        want_k, want_ks = ref.append(xb.cpu(), k.cpu(), ks.cpu(), slots, starts, False)
        want_v, want_vs = ref.append(xb.cpu(), v.cpu(), vs.cpu(), slots, starts, True)
        wm.cache_append(xb, xb, k, v, ks, vs, dev(slots, torch.int64), dev(starts))
        torch.cuda.synchronize()
        assert torch.equal(ks.cpu().double(), want_ks) and torch.equal(vs.cpu().double(), want_vs)
        for got, want in ((k, want_k), (v, want_v)):
            got = ref.decode(got.cpu())
            assert torch.equal(got.isnan(), want.isnan())
            assert torch.equal(got.nan_to_num(), want.nan_to_num())
        assert bool(torch.isfinite(ks).all())


def test_every_code_survives_the_store(wm):
    """Each finite code's value, stored, comes back as that code."""
    for fmt in (E4, E5):
        codes = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(fmt).float()
        codes = torch.where(torch.isfinite(codes), codes, torch.zeros_like(codes))
        x = torch.zeros(4, 1, 64)
        x.view(-1)[:] = codes
        # each row has the largest magnitude once, so the scale is 1
        x[:, 0, 0] = ref.LARGEST[fmt]
        k, v, ks, vs = make_cache(1, 1, 16, 64, fmt, 6)
        xb = x.to(BF).cuda()
        wm.cache_append(xb, xb, k, v, ks, vs, dev([0, 1, 2, 3], torch.int64), dev([0, 4]))
        assert ks.item() == 1.0 and vs.item() == 1.0
        assert torch.equal(k[0, 0, :4].float().cpu(), x[:, 0])
        assert torch.equal(v[0, 0, :, :4].float().cpu(), x[:, 0].t())
        assert not k[0, 0, 4:].float().any() and not v[0, 0, :, 4:].float().any()


def test_slots_outside_and_starts_beyond(wm):
    k, v, ks, vs = make_cache(3, 2, 16, 64, E4, 7)
    before = [t.clone() for t in (k.view(torch.uint8), v.view(torch.uint8), ks, vs)]
    x = torch.randn(4, 2, 64).to(BF).cuda()
    verdict = word()

    def same():
        torch.cuda.synchronize()
        now = (k.view(torch.uint8), v.view(torch.uint8), ks, vs)
        return all(torch.equal(a, b) for a, b in zip(now, before))
    # padding rows
    wm.cache_append(x, x, k, v, ks, vs, dev([-1] * 4, torch.int64), dev([0, 2, 4]), verdict)
    assert same() and verdict.item() == 0
    # beyond the pool
    wm.cache_append(x, x, k, v, ks, vs, dev([48, 1 << 40, 1 << 33, 99], torch.int64),
                    dev([0, 1, 2, 3, 4]), verdict)
    assert same() and verdict.item() == 8
    # starts beyond the rows: the rows that are there are stored
    verdict = word()
    want_k, _ = ref.append(x.cpu(), k.cpu(), ks.cpu(), [5, 6, 7, 8], [0, 4], False)
    wm.cache_append(x, x, k, v, ks, vs, dev([5, 6, 7, 8], torch.int64), dev([0, 30]), verdict)
    torch.cuda.synchronize()
    assert verdict.item() == 4
    assert torch.equal(ref.decode(k.cpu()), want_k)


# ---- attention ---------------------------------------------------------------------


def values(codes, scale, transposed):
    x = ref.decode(codes.cpu())
    x = x.transpose(2, 3) if transposed else x
    return (x * scale.cpu().double()[:, :, None, None]).contiguous()


def check_attend(wm, lens, new, heads, group, bt, dim, dt, fmt, window=0, seed=0, stride=0,
                 pad=2, max_len=None, packed=True, tail=None, scale=None, spread=1.5):
    say(f"[attend] lens={lens} new={new} heads={heads}x{group} bt={bt} dim={dim} {dt} {fmt} "
        f"window={window}")
    rows, blocks = layout(lens, bt, seed)
    k, v, ks, vs = make_cache(blocks, heads, bt, dim, fmt, seed + 1, stride)
    starts = [0] + np.cumsum(new).tolist()
    total, hq = starts[-1], heads * group
    g = torch.Generator().manual_seed(seed + 2)
    scale = scale if scale is not None else 1 / math.sqrt(dim)
    wide = torch.randn(total + pad, hq + (3 if packed else 0), dim, generator=g) * spread
    q = wide.to(dt).cuda()[:, :hq]
    if tail is not None:
        tail(k, v, ks, vs, rows)
    out = torch.full((total + pad, hq, dim + 8), 7.0, dtype=dt, device="cuda")[..., :dim]
    lse = torch.full((total + pad, hq), 7.0, device="cuda")
    verdict = word()
    table, most = dev(rows), max_len if max_len is not None else max(lens)
    n = wm.attend_ws_bytes(q, k, dev(lens), most)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    wm.cache_attend(q, k, v, ks, vs, table, dev(lens), dev(starts), out, ws, max_len=most,
                    scale=scale, window=window, lse=lse, verdict=verdict)
    torch.cuda.synchronize()
    assert verdict.item() == 0
    want, z, weight, sp = ref.attend(q.cpu(), values(k, ks, False), values(v, vs, True), rows,
                                     lens, starts, bt, scale, window)
    bo, bl = ref.attend_bound(dt, want, z, weight, sp, max(lens + [1]), dim)
    got, got_z = out[:total].cpu().double(), lse[:total].cpu().double()
    assert bool((out[total:].cpu() == 7.0).all()) and bool((lse[total:].cpu() == 7.0).all())
    empty = torch.isinf(z[:total])
    assert torch.equal(empty, torch.isneginf(got_z))
    assert not got[empty].any()
    off = (got - want[:total]).abs()
    assert bool((off <= bo[:total]).all()), float((off / bo[:total]).max())
    zoff = torch.where(empty, torch.zeros_like(z[:total]), (got_z - z[:total]).abs())
    assert bool((zoff <= bl[:total]).all()), float((zoff / bl[:total]).max())
    # the same bits again
    again = torch.full_like(out, 7.0)
    wm.cache_attend(q, k, v, ks, vs, table, dev(lens), dev(starts), again, ws, max_len=most,
                    scale=scale, window=window)
    assert torch.equal(again, out)


ATTENDS = [
    # lengths, new tokens, heads, group, bt, dim, type, format, more
    ([1], [1], 1, 1, 16, 64, BF, E4, {}),
    ([1, 2, 15, 16, 17, 63, 64, 65, 127], [1] * 9, 2, 4, 16, 64, BF, E4, {}),
    ([512], [1], 8, 1, 64, 64, BF, E4, {}),
    ([130, 64, 200], [1, 1, 1], 2, 8, 64, 128, HF, E5, {}),
    ([33, 300], [1, 1], 1, 16, 32, 192, BF, E5, {}),
    ([77, 513], [1, 1], 2, 3, 128, 256, HF, E4, dict(stride=48)),
    ([260, 5], [1, 2], 1, 32, 256, 128, BF, E4, dict(stride=16)),
    # prompts and chunks: rows that see different lengths
    ([5, 37, 64], [5, 20, 1], 2, 4, 16, 64, BF, E4, {}),
    ([100, 201], [100, 65], 1, 2, 64, 128, BF, E4, {}),
    ([90, 33], [70, 33], 2, 1, 32, 128, HF, E5, {}),
    ([64, 130], [33, 64], 1, 5, 16, 256, HF, E4, {}),
    ([150], [150], 1, 7, 128, 192, BF, E5, {}),
    # windows: shorter than a step, across blocks, longer than the sequence
    ([200, 90, 65], [1, 1, 1], 2, 2, 16, 64, BF, E4, dict(window=1)),
    ([200, 90, 300], [40, 90, 1], 1, 4, 32, 128, BF, E4, dict(window=37)),
    ([100, 40], [30, 40], 1, 2, 64, 64, HF, E5, dict(window=1000)),
    # requests without tokens, without queries, and queries before the start
    ([0, 50, 0, 7], [1, 0, 0, 1], 2, 2, 16, 64, BF, E4, {}),
    ([3, 0, 64], [5, 2, 1], 1, 3, 16, 128, HF, E4, {}),
    # split sequences, of very different lengths
    ([2000, 1, 700, 3333], [1, 1, 1, 1], 1, 4, 64, 128, BF, E4, {}),
    ([4097, 0, 130], [1, 1, 1], 2, 1, 16, 64, HF, E5, dict(window=1500)),
    ([2500, 40], [9, 3], 1, 2, 32, 256, BF, E5, {}),
    # a longest length that the caller put too low
    ([3000, 500], [1, 1], 1, 2, 64, 64, BF, E4, dict(max_len=600)),
    ([900], [1], 1, 1, 64, 64, BF, E4, dict(max_len=1)),
    # sharp and flat softmax, negative scale
    ([600, 333], [1, 1], 2, 4, 64, 128, BF, E4, dict(spread=20.0)),
    ([600, 333], [1, 5], 2, 4, 64, 128, HF, E4, dict(spread=0.01)),
    ([300], [2], 1, 4, 64, 64, BF, E4, dict(scale=-0.3)),
]


@pytest.mark.parametrize("lens,new,heads,group,bt,dim,dt,fmt,more", ATTENDS)
def test_attention(wm, lens, new, heads, group, bt, dim, dt, fmt, more):
    check_attend(wm, lens, new, heads, group, bt, dim, dt, fmt, **more)


@pytest.mark.parametrize("fmt", [E4, E5])
@pytest.mark.parametrize("window", [0, 40])
def test_what_is_not_seen_does_not_count(wm, fmt, window):
    """NaN (and infinite) codes behind the last token and before the window,
    NaN scales of blocks that no row sees."""
    bt, lens, new = 16, [37, 130, 64], [5, 1, 3]

    def poison(k, v, ks, vs, rows):
        bad = 0x7F if fmt == E4 else 0x7C
        used = {rows[r][j] for r, n in enumerate(lens) for j in range(-(-n // bt))}
        for t in (ks, vs):
            for b in range(t.shape[0]):
                if b not in used:
                    t[b] = math.nan
        for r, n in enumerate(lens):
            blk, off = rows[r][(n - 1) // bt], (n - 1) % bt + 1
            k.view(torch.uint8)[blk, :, off:] = bad
            v.view(torch.uint8)[blk, :, :, off:] = bad
            if window:
                p = n - new[r]  # the first row's position: nothing sees p - window
                for j in range(0, max(0, p - window + 1)):
                    k.view(torch.uint8)[rows[r][j // bt], :, j % bt] = 0xFF
                    v.view(torch.uint8)[rows[r][j // bt], :, :, j % bt] = 0xFF
    check_attend(wm, lens, new, 2, 2, bt, 64, BF, fmt, window=window, tail=poison)


def test_special_values_reach_the_rows_that_see_them(wm):
    """A NaN value at token 9 and an infinity at token 12: earlier rows of the
    same tile are untouched."""
    bt, lens, new, dim = 16, [20], [20], 64
    rows, blocks = layout(lens, bt, 3)
    k, v, ks, vs = make_cache(blocks, 1, bt, dim, E5, 4)
    v.view(torch.uint8)[rows[0][0], 0, 5, 9] = 0x7F
    v.view(torch.uint8)[rows[0][0], 0, 6, 12] = 0x7C
    v.view(torch.uint8)[rows[0][0], 0, 7, 12] = 0xFC
    v.view(torch.uint8)[rows[0][0], 0, 8, 12] = 0x7C
    v.view(torch.uint8)[rows[0][0], 0, 8, 13] = 0xFC
    k.view(torch.uint8)[rows[0][1], 0, 1, 3] = 0x7F  # a NaN key: token 17
    q = torch.randn(20, 2, dim).to(BF).cuda()
    out = torch.zeros_like(q)
    wm.cache_attend(q, k, v, ks, vs, dev(rows), dev(lens), dev([0, 20]), out, max_len=20,
                    scale=0.1)
    o = out.float().cpu()
    assert bool(torch.isfinite(o[:9]).all())
    assert bool(o[9:, :, 5].isnan().all())
    assert bool(torch.isfinite(o[9:12][..., [0, 6, 7, 8]]).all())
    assert bool((o[12:17, :, 6] == math.inf).all()) and bool((o[12:17, :, 7] == -math.inf).all())
    assert bool((o[12, :, 8] == math.inf).all()) and bool(o[13:17, :, 8].isnan().all())
    assert bool(torch.isfinite(o[12:17][..., 9:]).all())
    assert bool(o[17:].isnan().all())


def test_blocks_outside_the_pool_count_as_unseen(wm):
    bt, lens, new = 16, [90, 40], [1, 3]
    rows, blocks = layout(lens, bt, 5)
    k, v, ks, vs = make_cache(blocks, 2, bt, 64, E4, 6)
    q = torch.randn(4, 2, 64).to(BF).cuda()
    rows[0][2], rows[1][0] = blocks, -1
    lse, out, verdict = torch.zeros(4, 2, device="cuda"), torch.zeros_like(q), word()
    wm.cache_attend(q, k, v, ks, vs, dev(rows), dev(lens), dev([0, 1, 4]), out, max_len=90,
                    scale=0.2, lse=lse, verdict=verdict)
    assert verdict.item() == 8
    hidden = lambda r, j: (r, j // bt) in ((0, 2), (1, 0))  # noqa: E731
    want, z, weight, sp = ref.attend(q.cpu(), values(k, ks, False), values(v, vs, True), rows,
                                     lens, [0, 1, 4], bt, 0.2, hidden=hidden)
    bo, bl = ref.attend_bound(BF, want, z, weight, sp, 90, 64)
    assert bool(((out.cpu().double() - want).abs() <= bo).all())
    assert bool(((lse.cpu().double() - z).abs() <= bl).all())


def test_lengths_beyond_the_table(wm):
    bt = 16
    rows, blocks = layout([64], bt, 7)
    k, v, ks, vs = make_cache(blocks, 1, bt, 64, E4, 8)
    q = torch.randn(1, 1, 64).to(BF).cuda()
    a, b, verdict = torch.zeros_like(q), torch.zeros_like(q), word()
    wm.cache_attend(q, k, v, ks, vs, dev(rows), dev([64]), dev([0, 1]), a, max_len=64, scale=0.2)
    wm.cache_attend(q, k, v, ks, vs, dev(rows), dev([1 << 30]), dev([0, 1]), b, max_len=64,
                    scale=0.2, verdict=verdict)
    assert verdict.item() == 1 and torch.equal(a, b)


def test_answers_do_not_depend_on_the_blocks(wm):
    bt, n, heads, dim = 16, 1900, 2, 64
    need = -(-n // bt)
    k, v, ks, vs = make_cache(2 * need, heads, bt, dim, E4, 9)
    q = torch.randn(1, 8, dim).to(BF).cuda()
    first = torch.randperm(2 * need)[:need]
    second = torch.tensor([b for b in range(2 * need) if b not in set(first.tolist())][:need])
    for t in (k.view(torch.uint8), v.view(torch.uint8), ks, vs):
        t[second.flip(0).cuda()] = t[first.cuda()].clone()
    outs = []
    for ids in (first, second.flip(0)):
        out = torch.zeros_like(q)
        ws = torch.empty(wm.attend_ws_bytes(q, k, dev([n]), n), dtype=torch.uint8, device="cuda")
        wm.cache_attend(q, k, v, ks, vs, dev(ids)[None], dev([n]), dev([0, 1]), out, ws,
                        max_len=n, scale=0.125)
        outs.append(out)
    assert torch.equal(*outs) and bool(outs[0].any())


def test_unaligned_queries_and_outputs(wm):
    bt, lens = 16, [70]
    rows, blocks = layout(lens, bt, 11)
    k, v, ks, vs = make_cache(blocks, 1, bt, 64, E4, 12)
    flat = torch.randn(2 * 67 + 1).to(BF).cuda()
    q = flat[1:].as_strided((1, 2, 64), (134, 67, 1))
    aligned, odd = torch.zeros(1, 2, 64, dtype=BF, device="cuda"), torch.zeros(140, dtype=BF,
                                                                              device="cuda")
    view = odd[1:].as_strided((1, 2, 64), (134, 67, 1))
    args = (k, v, ks, vs, dev(rows), dev(lens), dev([0, 1]))
    wm.cache_attend(q.contiguous(), *args, aligned, max_len=70, scale=0.2)
    wm.cache_attend(q, *args, view, max_len=70, scale=0.2)
    assert torch.equal(view, aligned) and bool(aligned.any())
    odd[1:].as_strided((2, 64), (67, 1)).zero_()
    assert not odd.any()


# ---- blocks and the flat state -----------------------------------------------------


def pools_of(shapes, seed):
    """Pools [blocks, stride bytes] of which each page's first bytes count."""
    out = []
    for i, (blocks, page, stride) in enumerate(shapes):
        out.append(random_bytes(blocks * stride, seed + i).view(blocks, stride)[:, :page])
    return out


POOLS = [
    ([(5, 4, 4)], 3), ([(9, 4096, 4096), (11, 20, 36)], 7), ([(4, 16384 * 3 + 16, 60000)], 4),
    ([(40, 3584, 3584), (40, 65536, 65552), (44, 100, 100)], 33),
    ([(6, 48, 64)] * 70 + [(8, 12, 16)] * 61, 5), ([(3, 8, 8)], 1),
]


@pytest.mark.parametrize("shapes,n", POOLS)
def test_pages_out_and_in(wm, shapes, n):
    say(f"[pages] {shapes[:3]} x{len(shapes)} n={n}")
    pools = pools_of(shapes, 1)
    blocks = min(s[0] for s in shapes)
    pages = torch.randperm(blocks, generator=torch.Generator().manual_seed(2))[:min(n, blocks)]
    want = []
    for p in pools:
        b = p[pages.cuda()].reshape(-1)
        want += [b, torch.zeros(-b.numel() % 16, dtype=torch.uint8, device="cuda")]
    want = torch.cat(want)
    total = wm.flat_pages_bytes(pools, pages.numel())
    assert total == want.numel()
    flat = torch.full((total + 64,), 0xEE, dtype=torch.uint8, device="cuda")
    verdict = word()
    wm.flatten_pages(pools, dev(pages), flat, verdict)
    assert verdict.item() == 0
    assert torch.equal(flat[:total], want) and bool((flat[total:] == 0xEE).all())
    # into other pools' other pages; everything else stays
    dest = pools_of(shapes, 100)
    expect = [p.clone() for p in dest]
    to = pages.flip(0)
    at = 0
    for p, e in zip(pools, expect):
        e[to.cuda()] = p[pages.cuda()]
        at += p.shape[1]
    full = [d.as_strided((d.shape[0], d.stride(0)), (d.stride(0), 1)) for d in dest]
    gaps = [f[:, d.shape[1]:].clone() for f, d in zip(full, dest)]
    wm.rehydrate_pages(flat, dest, dev(to), verdict)
    assert verdict.item() == 0
    for d, e, f, gp in zip(dest, expect, full, gaps):
        assert torch.equal(d, e) and torch.equal(f[:, d.shape[1]:], gp)


def test_pages_move_only_on_a_zero_verdict_and_good_blocks(wm):
    pools = pools_of([(6, 64, 64), (5, 32, 32)], 3)
    before = [p.clone() for p in pools]
    flat = torch.full((1024,), 0x11, dtype=torch.uint8, device="cuda")
    for pages, v0, v1 in (([0, 1], 4, 4), ([0, 5], 0, 8), ([-1, 1], 0, 8), ([3, 1 << 30], 2, 10)):
        verdict = dev([v0])
        wm.rehydrate_pages(flat, pools, dev(pages), verdict)
        assert verdict.item() == v1
        verdict = dev([v0])
        wm.flatten_pages(pools, dev(pages), flat, verdict)
        assert verdict.item() == v1
        assert bool((flat == 0x11).all())
    assert all(torch.equal(a, b) for a, b in zip(pools, before))
    many = dev([0] * 5000 + [5])
    big = torch.full((wm.flat_pages_bytes(pools, 5001),), 0x11, dtype=torch.uint8, device="cuda")
    verdict = word()
    wm.flatten_pages(pools, many, big, verdict)
    assert verdict.item() == 8 and bool((big == 0x11).all())


# ---- together -----------------------------------------------------------------------


def feed(cache, tokens, group, g):
    """One step's random keys, values and queries through every layer."""
    outs = []
    for n in range(cache.layers):
        k, v = (torch.randn(tokens, cache.heads, cache.dim, generator=g, device="cuda").to(BF)
                for _ in range(2))
        q = torch.randn(tokens, cache.heads * group, cache.dim, generator=g,
                        device="cuda").to(BF)
        cache.append(n, k, v)
        outs.append(cache.attend(n, q, 1 / math.sqrt(cache.dim)))
    return outs


def test_a_session_moves_and_answers_the_same():
    """Prompts, steps, a session's move through the mover (encode, decode,
    verify, install) into another cache, and the next token there: the same
    bits as the next token here."""
    from paper_2607_10389_amd import WM_OK, Mover, PagedCache
    args = dict(layers=3, heads=2, dim=64, block_tokens=16, max_requests=4)
    src, dst = PagedCache(blocks=40, **args), PagedCache(blocks=50, **args)
    g = torch.Generator(device="cuda").manual_seed(1)
    feed(src, src.step({0: 37, 1: 100, 3: 5}), 4, g)
    for i in range(20):
        feed(src, src.step({0: 38 + i, 3: 6 + i}), 4, g)
    feed(src, src.step({1: 0, 0: 58}), 4, g)  # one leaves, its blocks are reused
    feed(dst, dst.step({2: 77, 0: 3}), 4, g)  # the destination serves others
    n = src.lengths[0]
    flat = src.suspend(0)
    m = Mover(flat.numel())
    m.encode_step(flat, None)
    m.decode()
    dst.resume(1, n, m.staging, m.verdict)
    assert m.commit(None, scatter=False) == WM_OK
    assert int(m.verdict.item()) == 0
    assert torch.equal(dst.suspend(1), flat)
    a, b = (torch.Generator(device="cuda").manual_seed(5) for _ in range(2))
    here = feed(src, src.step({0: n + 1}), 4, a)
    there = feed(dst, dst.step({1: n + 1}), 4, b)
    assert all(torch.equal(x, y) and bool(x.any()) for x, y in zip(here, there))
    # a verdict that is not zero installs nothing
    dst.step({1: 0})
    before = dst.codes.clone()
    dst.resume(1, n, m.staging, dev([4]))
    assert torch.equal(dst.codes, before)


def test_a_step_that_does_not_fit_changes_nothing():
    from paper_2607_10389_amd import PagedCache, WmError
    c = PagedCache(layers=1, blocks=4, heads=1, dim=64, block_tokens=16, max_requests=3)
    c.step({0: 20, 1: 3})
    before = [t.clone() for t in (c.block_table, c.ring, c.pool, c.lens)]
    with pytest.raises(WmError):
        c.step({0: 40, 2: 16})
    assert all(torch.equal(a, b) for a, b in zip(before, (c.block_table, c.ring, c.pool, c.lens)))
    assert c.step({0: 0, 1: 16}) == 13 and c.step({2: 48}) == 48
    with pytest.raises(ValueError):
        c.resume(2, 5, torch.zeros(1 << 16, dtype=torch.uint8, device="cuda"))


def test_captured_step_replays(wm):
    """Tables, store and attention of a decoding step in one graph, replayed
    with new lengths and inputs and checked against the eager calls each
    time; the calls are also made on a stream of their own."""
    heads, group, bt, dim, n = 2, 4, 16, 64, 3
    rows, blocks = layout([200] * n, bt, 1, extra=50)
    free = sorted(set(range(blocks)) - {b for r in rows for b in r})
    k, v, ks, vs = make_cache(blocks, heads, bt, dim, E4, 2)
    eager = [t.clone() for t in (k.view(torch.uint8), v.view(torch.uint8), ks, vs)]
    ek, ev, eks, evs = eager[0].view(E4), eager[1].view(E4), eager[2], eager[3]
    lens, nxt = dev([30, 64, 111]), dev([31, 65, 112])
    table, ring = dev([r + [0] * 4 for r in rows]), dev(free)
    pi, po, sl, qs, vd = dev([3, 50]), dev([0, 0]), dev([0] * n, torch.int64), dev([0] * 4), word()
    x = torch.zeros(n, heads * (group + 2), dim, dtype=BF, device="cuda")
    q, kn, vn = x[:, :heads * group], x[:, heads * group:heads * (group + 1)], \
        x[:, heads * (group + 1):]
    out, lse = torch.zeros(n, heads * group, dim, dtype=BF, device="cuda"), \
        torch.zeros(n, heads * group, device="cuda")
    ws = torch.empty(wm.attend_ws_bytes(q, k, nxt, 4000), dtype=torch.uint8, device="cuda")

    def step(kc, vc, s0, s1, o, z, stream=None):
        wm.page_tables(lens, nxt, bt, table, ring, pi, po, sl, qs, vd, stream)
        wm.cache_append(kn, vn, kc, vc, s0, s1, sl, qs, None, stream)
        wm.cache_attend(q, kc, vc, s0, s1, table, nxt, qs, o, ws, max_len=4000, scale=0.125,
                        lse=z, stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(ek, ev, eks, evs, torch.zeros_like(out), torch.zeros_like(lse), side)
    side.synchronize()
    for a, b in zip(eager, (k.view(torch.uint8), v.view(torch.uint8), ks, vs)):
        a.copy_(b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(k, v, ks, vs, out, lse)
    g = torch.Generator(device="cuda").manual_seed(3)
    for i in range(6):
        x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        graph.replay()
        want, z = torch.zeros_like(out), torch.zeros_like(lse)
        step(ek, ev, eks, evs, want, z)
        torch.cuda.synchronize()
        assert vd.item() == 0
        assert torch.equal(out, want) and torch.equal(lse, z) and bool(out.any()), i
        assert torch.equal(k.view(torch.uint8), eager[0])
        assert torch.equal(v.view(torch.uint8), eager[1])
        lens.copy_(nxt)
        nxt.add_(1)
        pi.copy_(po)


# ---- ranges ------------------------------------------------------------------------


@pytest.mark.parametrize("dim", [64, 128, 192, 256])
@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("fmt", [E4, E5])
def test_prompts_of_every_size_and_type(wm, dim, dt, fmt):
    """Tiles with steps that every row sees whole, with masked ones, and with
    both ends of a window."""
    bt = {64: 16, 128: 64, 192: 32, 256: 128}[dim]
    check_attend(wm, [300, 77], [40, 60], 1, 4, bt, dim, dt, fmt, seed=dim)
    check_attend(wm, [400], [70], 1, 3, bt, dim, dt, fmt, seed=dim + 1, window=150)


@pytest.mark.parametrize("lens,new,heads,group,dim,more", [
    # rows without anything to see among prompts
    ([0, 20, 200], [40, 50, 40], 1, 2, 64, {}),
    # few tiles over long sequences: parts, joined
    ([5000], [40], 1, 2, 64, {}),
    ([2600, 70, 0], [33, 33, 40], 1, 1, 128, dict(window=1100)),
    ([4000, 900], [50, 45], 2, 1, 256, dict(max_len=1000)),
    # a mix of a prompt and single tokens
    ([130, 500, 64, 1], [100, 1, 1, 1], 2, 4, 64, {})])
def test_prompts_at_the_edges(wm, lens, new, heads, group, dim, more):
    check_attend(wm, lens, new, heads, group, 32, dim, BF, E4, **more)


def test_many_requests(wm):
    """More requests than a wave counts at once: single tokens of 300, short
    prompts of 150 and of 600 (whose items are found by their place)."""
    g = np.random.default_rng(1)
    check_attend(wm, g.integers(0, 700, 300).tolist(), [1] * 300, 1, 2, 16, 64, BF, E4)
    for n in (150, 600):
        new = g.integers(0, 20, n)
        lens = new + g.integers(0, 40, n)
        check_attend(wm, lens.tolist(), new.tolist(), 1, 5, 16, 64, BF, E4)


def test_a_token_is_answered_the_same_in_any_batch(wm):
    bt, heads, group, dim = 16, 2, 4, 128
    lens = [1900, 3, 5000, 700]
    rows, blocks = layout(lens, bt, 21)
    k, v, ks, vs = make_cache(blocks, heads, bt, dim, E4, 22)
    q = torch.randn(4, heads * group, dim).to(BF).cuda()

    def ask(ids, most):
        out = torch.zeros(len(ids), heads * group, dim, dtype=BF, device="cuda")
        ln = dev([lens[i] for i in ids])
        ws = torch.empty(wm.attend_ws_bytes(out, k, ln, most), dtype=torch.uint8, device="cuda")
        wm.cache_attend(q[ids].contiguous(), k, v, ks, vs, dev([rows[i] for i in ids]), ln,
                        dev(list(range(len(ids) + 1))), out, ws, max_len=most, scale=0.09)
        return out
    every = ask([0, 1, 2, 3], 5000)
    for i in range(4):
        assert torch.equal(ask([i], lens[i])[0], every[i]), i
        assert torch.equal(ask([3, i], 100_000)[1], every[i]), i


def far_pool(blocks, page, step=1 << 30):
    """Pages a GiB apart: offsets beyond 32 bits with few blocks."""
    buf = torch.empty((blocks - 1) * step + page, dtype=torch.uint8, device="cuda")
    return buf.as_strided((blocks, page), (step, 1))


def test_offsets_beyond_32_bits(wm):
    heads, bt, dim, blocks = 1, 16, 64, 6
    page = heads * bt * dim
    near = make_cache(blocks, heads, bt, dim, E4, 31)
    far_k, far_v = far_pool(blocks, page), far_pool(blocks, page)
    k = far_k.view(E4).view(blocks, heads, bt, dim)
    v = far_v.view(E4).view(blocks, heads, dim, bt)
    k.view(torch.uint8).copy_(near[0].view(torch.uint8))
    v.view(torch.uint8).copy_(near[1].view(torch.uint8))
    far = [k, v, near[2].clone(), near[3].clone()]
    rows, lens = [[5, 4], [3, 0]], [20, 32]
    x = torch.randn(4, heads, dim).to(BF).cuda()
    slots = dev([5 * 16 + 15, 4 * 16, 4 * 16 + 1, 0], torch.int64)
    q, outs = torch.randn(2, 2, dim).to(BF).cuda(), []
    for c in (near, far):
        verdict = word()
        wm.cache_append(x, x, *c, slots, dev([0, 3, 4]), verdict)
        out = torch.zeros_like(q)
        wm.cache_attend(q, *c, dev(rows), dev(lens), dev([0, 1, 2]), out, max_len=32, scale=0.1,
                        verdict=verdict)
        assert verdict.item() == 0
        outs.append(out)
    assert torch.equal(*outs) and bool(outs[0].any())
    assert torch.equal(far[0].view(torch.uint8), near[0].view(torch.uint8))
    assert torch.equal(far[1].view(torch.uint8), near[1].view(torch.uint8))
    flat, verdict = torch.zeros(3 * page, dtype=torch.uint8, device="cuda"), word()
    wm.flatten_pages([far_k], dev([5, 1, 4]), flat, verdict)
    assert torch.equal(flat.view(3, page), far_k[[5, 1, 4]])
    wm.rehydrate_pages(flat, [far_v], dev([4, 0, 5]), verdict)
    assert torch.equal(far_v[[4, 0, 5]], flat.view(3, page)) and verdict.item() == 0


def test_blocks_without_a_usable_scale_count_as_fresh(wm):
    for bad in (0.0, -1.0, math.nan, math.inf, 1e-42):
        k, v, ks, vs = make_cache(2, 1, 16, 64, E4, 41)
        ks[1, 0] = vs[1, 0] = bad
        x = torch.randn(2, 1, 64).to(BF).cuda()
        wm.cache_append(x, x, k, v, ks, vs, dev([21, 22], torch.int64), dev([0, 2]))
        want, scale = ref.append(x.cpu(), torch.zeros_like(k.cpu().view(torch.uint8)).view(E4),
                                 torch.ones(2, 1), [16, 17], [0, 2], False)
        assert ks[1, 0].item() == scale[1, 0].item() == vs[1, 0].item()
        got = ref.decode(k.cpu())[1, 0]
        assert torch.equal(got[5:7], want[1, 0, :2]) and not got[:5].any() and not got[7:].any()
        got = ref.decode(v.cpu())[1, 0].t()
        assert torch.equal(got[5:7], want[1, 0, :2]) and not got[:5].any() and not got[7:].any()


def test_calls_on_two_streams_at_once(wm):
    bt, lens = 64, [3000, 2500]
    rows, blocks = layout(lens, bt, 51)
    k, v, ks, vs = make_cache(blocks, 2, bt, 128, E4, 52)
    args = (k, v, ks, vs, dev(rows), dev(lens), dev([0, 1, 2]))
    qs = [torch.randn(2, 8, 128).to(BF).cuda() for _ in range(2)]
    n = wm.attend_ws_bytes(qs[0], k, dev(lens), 3000)
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(2)]
    want = []
    for q in qs:
        want.append(torch.zeros_like(q))
        wm.cache_attend(q, *args, want[-1], ws[0], max_len=3000, scale=0.1)
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], [torch.zeros_like(q) for q in qs]
    torch.cuda.synchronize()
    for _ in range(20):
        for q, o, w, s in zip(qs, outs, ws, streams):
            wm.cache_attend(q, *args, o, w, max_len=3000, scale=0.1, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])


@pytest.mark.parametrize("n", [100, 200, 600])
def test_every_request_of_prompts_tells_of_its_length(wm, n):
    bt, each = 16, 40
    k, v, ks, vs = make_cache(4, 1, bt, 64, E4, 50)
    q = torch.randn(n * each, 1, 64).to(BF).cuda()
    table = dev([[0, 1, 2, 3]] * n)
    starts = dev([each * i for i in range(n + 1)])
    for last, want in ((64, 0), (65, 1)):
        say(f"[attend] the last of {n} requests has {last} tokens")
        out, verdict = torch.zeros_like(q), word()
        wm.cache_attend(q, k, v, ks, vs, table, dev([each] * (n - 1) + [last]), starts, out,
                        max_len=64, scale=0.2, verdict=verdict)
        assert verdict.item() == want


@pytest.mark.parametrize("lens,new,heads,group,bt,dim,dt,fmt,window,low", [
    ([500, 300], [500, 300], 1, 1, 64, 128, BF, E4, 32, -40),
    ([400], [400], 2, 2, 64, 64, HF, E5, 40, -60),
    ([600], [200], 1, 1, 128, 192, BF, E4, 50, -60),
    ([520], [300], 1, 1, 256, 256, HF, E4, 50, -20),
    ([300], [300], 1, 1, 16, 64, BF, E4, 10, -12),
    ([700, 90, 210], [1, 1, 1], 2, 4, 64, 128, HF, E4, 20, -40),
    ([700, 333], [3, 9], 1, 1, 64, 64, BF, E5, 20, -60),
    ([300, 129], [20, 9], 1, 1, 128, 256, BF, E4, 20, -60),
    ([256, 200], [8, 1], 1, 2, 32, 128, HF, E4, 0, -40),
])
def test_values_of_very_different_scales(wm, lens, new, heads, group, bt, dim, dt, fmt, window,
                                         low):
    """Every other block's values are 2^low times smaller: rows whose window
    lies in such a block are as precise as the others."""
    def tail(k, v, ks, vs, rows):
        for row in rows:
            for b in row[1::2]:
                if b >= 0:
                    vs[b] *= 2.0 ** low

    check_attend(wm, lens, new, heads, group, bt, dim, dt, fmt, window=window, seed=60, tail=tail)


def test_a_resume_of_too_small_a_state_changes_nothing():
    from paper_2607_10389_amd.paged import PagedCache
    c = PagedCache(1, 8, 1, 64, 16, max_requests=2)
    c.step({0: 20})
    flat = c.suspend(0)
    with pytest.raises(ValueError):
        c.resume(1, 33, flat)
    assert c.lengths == [20, 0] and c.pool.tolist()[1] == 6
    c.resume(1, 20, flat)
    assert c.lengths == [20, 20] and c.lens.tolist() == [20, 20]


@pytest.mark.parametrize("n", [8, 260])
def test_tables_of_sums_beyond_32_bits(wm, n):
    """Tokens and blocks in all that no 32-bit sum holds: refused."""
    bt, width = 256, (2 ** 31 - 1) // 256
    say(f"[tables] n={n} of 2^31 - 256 tokens each")
    table = torch.empty(n, width, dtype=torch.int32, device="cuda")
    ring, pool, po = dev([5, 6, 7]), dev([1, 2]), dev([-1, -1])
    slots, starts, v = dev([-9] * 10, torch.int64), dev([-3] * (n + 1)), dev([77])
    most = dev([width * bt] * n)
    wm.page_tables(dev([0] * n), most, bt, table, ring, pool, po, slots, starts, v)
    assert v.item() == 6 and po.tolist() == [1, 2]
    wm.page_tables(most, dev([0] * n), bt, table, ring, pool, po, slots, starts, v)
    assert v.item() == 2 and po.tolist() == [1, 2]
    assert ring.tolist() == [5, 6, 7] and slots.tolist() == [-9] * 10
    assert starts.tolist() == [-3] * (n + 1)


@pytest.mark.parametrize("first", [0, 1, 2])
@pytest.mark.parametrize("n", [300, 2050])
def test_tables_of_lengths_at_any_place(wm, n, first):
    """Lengths that begin at no 16-byte address, and slots in runs."""
    g = np.random.default_rng(70 + n)
    bt, old = 32, g.integers(0, 200, n)
    new = np.where(g.random(n) < 0.5, old, old + g.integers(0, 120, n))
    new[n // 2] = 9000
    up = lambda x: -(-x // bt)  # noqa: E731
    need = int(np.maximum(0, up(new) - up(old)).sum())
    width, tokens = up(9000) + 1, int(np.maximum(0, new - old).sum())
    ring = g.permutation(need + 5).tolist()
    table = g.integers(0, 1 << 20, (n, width)).tolist()
    want = ref.tables(old.tolist(), new.tolist(), bt, table, ring, 3, need + 2,
                      [-1] * (tokens + 4), [-7] * (n + 1))
    pad = lambda x: dev([9] * first + x.tolist())[first:]  # noqa: E731
    t, rg, po = dev(table), dev(ring), dev([-1, -1])
    sl, qs, v = dev([-1] * (tokens + 4), torch.int64), dev([-7] * (n + 1)), word()
    wm.page_tables(pad(old), pad(new), bt, t, rg, dev([3, need + 2]), po, sl, qs, v)
    assert v.item() == want[5] == 0
    assert t.tolist() == want[0] and rg.tolist() == want[1] and po.tolist() == want[2]
    assert sl.tolist() == want[3] and qs.tolist() == want[4]


@pytest.mark.parametrize("lens,new,heads,group,dim,more", [
    # parts and windows of tiles of 128 rows, a request without a token
    ([2600, 70, 0], [70, 70, 80], 1, 1, 128, dict(window=1100)),
    ([4000, 900], [80, 75], 2, 1, 256, dict(max_len=1000)),
    # 33 to 64 rows a request: few of them, and many
    ([700, 90], [20, 12], 2, 2, 128, {}),
    ([90, 40, 130, 64] * 10, [12, 9, 10, 11] * 10, 4, 4, 64, {})])
def test_prompts_of_either_tile(wm, lens, new, heads, group, dim, more):
    check_attend(wm, lens, new, heads, group, 32, dim, BF, E4, seed=80, **more)


@pytest.mark.parametrize("lens,starts,rows,dim,window", [
    ([40], [0, 12], 5, 64, 0),                     # few rows: the reading kernel
    ([40], [0, 12], 5, 64, 9),
    ([300, 20], [0, 200, 210], 150, 128, 0),       # prompts
    ([300, 20], [0, 200, 210], 150, 128, 70),
    ([2000], [0, 12], 4, 64, 0),                   # parts, joined
    ([40, 30, 50], [0, 3, 3, 9], 3, 64, 0),        # a request that begins behind the rows
    ([40, 50, 60], [0, 90, 90, 99], 90, 64, 0),
    ([300, 50, 60], [0, 200, 200, 209], 200, 64, 0),
    ([40], [-3, 4], 4, 64, 0),                     # rows before the first
    ([200], [-30, 100], 100, 64, 33),
    ([5], [0, 2 ** 31 - 1], 3, 64, 2 ** 31 - 1),   # every row before the sequence
])
def test_starts_beyond_the_rows(wm, lens, starts, rows, dim, window):
    """Rows that are there keep the positions that the starts give them."""
    say(f"[attend] lens={lens} starts={starts} rows={rows} dim={dim} window={window}")
    bt, hq = 16, 2
    table, blocks = layout(lens, bt, 90)
    k, v, ks, vs = make_cache(blocks, 1, bt, dim, E4, 91)
    q = torch.randn(rows, hq, dim, generator=torch.Generator().manual_seed(92)).to(BF)
    out, lse, verdict = torch.zeros(rows, hq, dim, dtype=BF, device="cuda"), \
        torch.zeros(rows, hq, device="cuda"), word()
    ws = torch.empty(wm.attend_ws_bytes(q, k, dev(lens), max(lens)), dtype=torch.uint8,
                     device="cuda")
    wm.cache_attend(q.cuda(), k, v, ks, vs, dev(table), dev(lens), dev(starts), out, ws,
                    max_len=max(lens), scale=0.2, window=window, lse=lse, verdict=verdict)
    assert verdict.item() == 4
    want, z = torch.zeros(rows, hq, dim, dtype=torch.float64), \
        torch.full((rows, hq), -math.inf, dtype=torch.float64)
    weight, sp = torch.zeros_like(want), torch.zeros_like(z)
    kv, vv = values(k, ks, False), values(v, vs, True)
    for r, n in enumerate(lens):
        a, b = max(0, starts[r]), min(rows, starts[r + 1])
        if a >= b:
            continue
        last = n - (starts[r + 1] - b)  # one behind the last row's position
        if last <= 0:
            continue
        got = ref.attend(q[a:b], kv, vv, [table[r]], [last], [0, b - a], bt, 0.2, window)
        for x, y in zip((want, z, weight, sp), got):
            x[a:b] = y
    bo, bl = ref.attend_bound(BF, want, z, weight, sp, max(lens), dim)
    assert bool(((out.cpu().double() - want).abs() <= bo).all())
    seen = torch.isfinite(z)
    assert torch.equal(torch.isneginf(lse.cpu()), ~seen)
    assert bool(((lse.cpu().double() - z).abs()[seen] <= bl[seen]).all())


def test_a_captured_step_outlives_larger_ones():
    """A decoding step of a PagedCache, captured, replayed before and after a
    prompt that needs a larger workspace and more slots: each replay against
    the eager step of a second cache."""
    from paper_2607_10389_amd import PagedCache
    args = dict(layers=1, blocks=420, heads=2, dim=64, block_tokens=16, max_requests=3)
    c, twin = PagedCache(**args), PagedCache(**args)
    g = torch.Generator(device="cuda").manual_seed(7)

    def inputs(n):
        return torch.randn(n, 12, 64, generator=g, device="cuda").to(BF)

    def calls(cache, x, out=None):
        cache.append(0, x[:, 8:10], x[:, 10:])
        return cache.attend(0, x[:, :8], 0.125, out=out)

    def both(lengths):
        n = c.step(lengths)
        assert twin.step(lengths) == n
        return n

    x = inputs(both({0: 600, 1: 30}))
    calls(c, x), calls(twin, x)
    x = inputs(both({0: 601, 1: 31}))
    out = torch.zeros(2, 8, 64, dtype=BF, device="cuda")
    calls(c, x, out), calls(twin, x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(c, x, out)
    junk = []
    for i in range(8):
        if i == 3:
            y = inputs(both({2: 5000}))
            a, b = calls(c, y), calls(twin, y)
            assert torch.equal(a, b)
            # (a freed buffer would be given out here)
            junk = [torch.full((1 << k,), 0x55, dtype=torch.uint8, device="cuda")
                    for k in range(6, 24) for _ in range(4)]
        both({0: 602 + i, 1: 32 + i})
        x.copy_(inputs(2))
        out.zero_()
        graph.replay()
        want = calls(twin, x)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and bool(out.any()), i
        assert torch.equal(c.codes, twin.codes) and torch.equal(c.scales, twin.scales), i
        assert c.verdict.item() == 0
        assert all(bool((t == 0x55).all()) for t in junk), i


def test_findings_of_a_cache_reach_its_next_step():
    """A captured append of fewer rows than a later step has tokens: the step
    after it raises, and the one after that goes on."""
    from paper_2607_10389_amd import PagedCache, WmError
    c = PagedCache(layers=1, blocks=20, heads=1, dim=64, block_tokens=16, max_requests=3)
    x = torch.randn(4, 1, 64, device="cuda").to(BF)
    c.step({0: 1})
    c.append(0, x[:1], x[:1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.append(0, x[:1], x[:1])
    c.step({0: 2, 1: 3})
    with pytest.raises(ValueError):
        c.append(0, x[:3], x[:3])
    graph.replay()
    flat = c.suspend(0)
    assert c.verdict.item() == 4
    before = [t.clone() for t in (c.block_table, c.ring, c.pool, c.lens, c.q_start)]
    with pytest.raises(WmError):
        c.step({0: 3})
    after = (c.block_table, c.ring, c.pool, c.lens, c.q_start)
    assert all(torch.equal(a, b) for a, b in zip(before, after)) and c.lengths == [2, 3, 0]
    assert c.step({0: 3}) == 1
    c.resume(2, 2, flat)
    assert c.verdict.item() == 0 and torch.equal(c.suspend(2), flat)


def test_a_resume_from_the_host_takes_no_blocks():
    from paper_2607_10389_amd import PagedCache
    c = PagedCache(layers=1, blocks=8, heads=1, dim=64, block_tokens=16, max_requests=2)
    c.step({0: 20})
    flat = c.suspend(0)
    state = c.lengths, c.lens.tolist(), c.pool.tolist(), c.q_start.tolist()
    for f, v in ((flat.cpu(), None), (flat, torch.zeros(1, dtype=torch.int32))):
        with pytest.raises(ValueError):
            c.resume(1, 20, f, v)
        assert state == (c.lengths, c.lens.tolist(), c.pool.tolist(), c.q_start.tolist())
    # a verdict that is not zero: blocks, nothing in them, and they go back
    before = c.codes.clone()
    c.resume(1, 20, flat, dev([1]))
    assert c.lengths == [20, 20] and torch.equal(c.codes, before)
    c.step({1: 0})
    assert c.pool.tolist()[1] == 6


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("lens,new,heads,group,bt,dim,window", [
    ([300, 520], [1, 1], 1, 16, 16, 64, 0),      # the reading kernel, rows that see all
    ([300], [1], 2, 4, 64, 128, 0),
    ([1200], [1], 1, 16, 32, 64, 0),             # in parts
    ([700], [1], 1, 16, 16, 256, 400),
    ([400], [80], 1, 2, 16, 64, 0),              # prompts
    ([400], [80], 1, 2, 64, 128, 0),
    ([500], [90], 1, 2, 32, 192, 320),
    ([400], [80], 1, 2, 128, 256, 0),
])
def test_infinite_values_that_every_row_sees(wm, dt, lens, new, heads, group, bt, dim, window):
    """An infinity stays one whatever its weight, if no other sign meets it."""
    say(f"[attend] {dt} lens={lens} new={new} {heads}x{group} bt={bt} dim={dim} window={window}")
    rows, blocks = layout(lens, bt, 95)
    k, v, ks, vs = make_cache(blocks, heads, bt, dim, E5, 96)
    for r, n in enumerate(lens):
        for off, d, code in ((70, 3, 0x7C), (130, 4, 0xFC), (75, 5, 0x7C), (140, 5, 0xFC)):
            j = n - new[r] - off  # every row sees it
            v.view(torch.uint8)[rows[r][j // bt], :, d, j % bt] = code
    starts = [0] + np.cumsum(new).tolist()
    q = (torch.randn(starts[-1], heads * group, dim,
                     generator=torch.Generator().manual_seed(97)) * 8).to(dt).cuda()
    out = torch.zeros_like(q)
    ws = torch.empty(wm.attend_ws_bytes(q, k, dev(lens), max(lens)), dtype=torch.uint8,
                     device="cuda")
    wm.cache_attend(q, k, v, ks, vs, dev(rows), dev(lens), dev(starts), out, ws,
                    max_len=max(lens), scale=0.5, window=window)
    o = out.float().cpu()
    assert bool((o[..., 3] == math.inf).all())
    assert bool((o[..., 4] == -math.inf).all())
    assert bool(o[..., 5].isnan().all())
    assert bool(torch.isfinite(o[..., [0, 1, 2]]).all()) and bool(torch.isfinite(o[..., 6:]).all())


@pytest.mark.parametrize("lens,new,heads,group,bt,dim,dt,fmt,window,first,factor", [
    # causal: rows of the first block see nothing of the ones after it
    ([64], [64], 1, 1, 16, 64, BF, E4, 0, 0, 40),
    ([64], [64], 1, 2, 16, 128, BF, E5, 0, 0, 60),     # 128 rows: prompts
    ([100, 64], [100, 64], 1, 2, 32, 64, BF, E4, 0, 0, 90),
    ([80], [80], 2, 2, 16, 192, BF, E4, 0, 0, 40),
    ([90], [90], 1, 1, 32, 256, BF, E4, 0, 0, 40),
    ([64], [40], 1, 2, 32, 64, HF, E4, 0, -10, 20),
    ([50], [30], 1, 1, 32, 256, HF, E4, 0, -10, 20),
    # behind a window: later rows see nothing of the blocks before it
    ([64], [64], 1, 1, 16, 64, BF, E4, 9, 60, -50),
    ([400], [200], 1, 1, 64, 128, BF, E4, 20, 50, -20),
    ([300], [9], 1, 1, 32, 64, BF, E4, 12, 100, -100),
])
def test_scales_of_what_is_not_seen_do_not_count(wm, lens, new, heads, group, bt, dim, dt, fmt,
                                                 window, first, factor):
    """Block j's values are scaled by 2^(first + factor j), up to 2^100: a row
    is as precise as what it sees allows."""
    def tail(k, v, ks, vs, rows):
        for row in rows:
            for j, b in enumerate(row):
                if b >= 0:
                    vs[b] *= 2.0 ** max(-100, min(100, first + factor * j))

    check_attend(wm, lens, new, heads, group, bt, dim, dt, fmt, window=window, seed=98, tail=tail,
                 spread=0.5)


@pytest.mark.parametrize("slots", [
    [-1] * 3 + list(range(23, 43)),          # padding at the start of a request
    list(range(16, 32)) + list(range(35, 42)),  # a gap behind a block's last place
    list(range(16, 31)) + list(range(32, 40)),  # a gap before it
])
@pytest.mark.parametrize("requests", [1, 8])  # a workgroup and a wave for a block
def test_slots_that_do_not_follow_each_other(wm, slots, requests):
    """Tokens of a later block are not stored at places that they do not have."""
    bt, n = 16, 23
    k, v, ks, vs = make_cache(6, 2, bt, 64, E4, 101)
    before = [t.clone() for t in (k.view(torch.uint8), v.view(torch.uint8), ks, vs)]
    x = torch.randn(n, 2, 64).to(BF).cuda()
    starts = dev([0] + [n] * requests)
    verdict = word()
    wm.cache_append(x, x, k, v, ks, vs, dev(slots, torch.int64), starts, verdict)
    assert verdict.item() == 8
    after = (k.view(torch.uint8), v.view(torch.uint8), ks, vs)
    # a request's first block is stored if its slots are sound
    same = [torch.equal(a[2:], b[2:]) for a, b in zip(after, before)]
    assert all(same) and all(torch.equal(a[0], b[0]) for a, b in zip(after, before))
    first = all(torch.equal(a[1], b[1]) for a, b in zip(after, before))
    assert first == (slots[:16] != list(range(16, 32)))


@pytest.mark.parametrize("new", [[1, 1, 1], [90, 80, 70]])  # single tokens, prompts
def test_lengths_below_zero_are_told(wm, new):
    bt, lens = 16, [100, -5, 80]
    rows, blocks = layout([100, 0, 80], bt, 103)
    k, v, ks, vs = make_cache(blocks, 1, bt, 64, E4, 104)
    starts = [0] + np.cumsum(new).tolist()
    q = torch.randn(starts[-1], 2, 64).to(BF).cuda()
    outs = []
    for ln, want in ((lens, 1), ([100, 0, 80], 0), ([100, 90, -(1 << 31)], 1)):
        out, lse, verdict = torch.full_like(q, 7.0), torch.zeros(starts[-1], 2, device="cuda"), word()
        table = dev([rows[0], rows[0], rows[2]])
        ws = torch.empty(wm.attend_ws_bytes(q, k, dev(ln), 100), dtype=torch.uint8, device="cuda")
        wm.cache_attend(q, k, v, ks, vs, table, dev(ln), dev(starts), out, ws, max_len=100,
                        scale=0.2, lse=lse, verdict=verdict)
        assert verdict.item() == want
        outs.append(out)
    assert torch.equal(outs[0], outs[1]) and bool(outs[0].any())
    assert not outs[2][starts[2]:].any()


def test_more_workgroups_than_an_axis_of_a_grid_holds(wm):
    """440 million query vectors in requests of 33 tokens: 17 million tiles.
    Queries and outputs are one token's, again and again, and every row sees
    one of a block's equal tokens: one answer for all, an lse for each."""
    n, each, heads, dim, bt = 840_000, 33, 16, 64, 64
    g = torch.Generator().manual_seed(105)
    k = torch.randn(1, heads, 1, dim, generator=g).expand(1, heads, bt, dim).to(E4).contiguous()
    v = torch.randn(1, heads, dim, 1, generator=g).expand(1, heads, dim, bt).to(E4).contiguous()
    one = torch.ones(1, heads, device="cuda")
    q1 = torch.randn(1, heads, dim, generator=g).to(BF)
    q, out = q1.cuda().expand(n * each, heads, dim), torch.zeros(1, heads, dim, dtype=BF,
                                                                 device="cuda")
    lse = torch.full((n * each, heads), 7.0, device="cuda")
    lens = torch.full((n,), bt, dtype=torch.int32, device="cuda")
    starts = torch.arange(n + 1, dtype=torch.int32, device="cuda") * each
    table, verdict = torch.zeros(n, 1, dtype=torch.int32, device="cuda"), word()
    say(f"[attend] {n} requests of {each} tokens and {heads} heads")
    wm.cache_attend(q, k.cuda(), v.cuda(), one, one, table, lens, starts,
                    out.expand(n * each, heads, dim), max_len=bt, scale=0.125, window=1, lse=lse,
                    verdict=verdict)
    torch.cuda.synchronize()
    assert verdict.item() == 0
    assert torch.equal(out.float().cpu()[0], v.float()[0, :, :, 0])
    qk = q1.double()[0] * k.double()[0, :, 0] * 0.125
    spread, z = qk.abs().sum(-1), qk.sum(-1)
    zero = torch.zeros(heads, dim, dtype=torch.float64)
    _, bound = ref.attend_bound(BF, zero, z, zero, spread, 1, dim)
    assert bool(((lse[0].cpu().double() - z).abs() <= bound).all())
    assert bool((lse == lse[0]).all())


def test_tables_of_addresses_keep_their_tensors(wm):
    import weakref
    from paper_2607_10389_amd import _wm
    for make in (wm.PoolTable, _wm.LeafTable):
        t = torch.zeros(4, 16, dtype=torch.uint8, device="cuda")
        table, there = make([t]), weakref.ref(t)
        del t
        assert there() is not None and there().data_ptr() == table.t[0].ptr
        del table
        assert there() is None


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("lens,new,group,dim", [([200], [90], 2, 64), ([150, 90], [90, 80], 1, 128),
                                                ([140], [75], 1, 256), ([900], [9], 3, 64)])
def test_prompts_at_any_address(wm, dt, lens, new, group, dim):
    """Queries and outputs that begin at odd elements, with odd strides: the
    bits of aligned ones, and nothing between the vectors."""
    say(f"[attend] {dt} lens={lens} new={new} group={group} dim={dim}")
    bt, heads, total = 32, 2, sum(new)
    rows, blocks = layout(lens, bt, 115)
    k, v, ks, vs = make_cache(blocks, heads, bt, dim, E4, 116)
    hq, starts = heads * group, [0] + np.cumsum(new).tolist()
    shape, step = (total, hq, dim), (hq * (dim + 3) + 2, dim + 3, 1)
    flat = torch.randn(total * step[0] + 1, generator=torch.Generator().manual_seed(117)).to(dt)
    q = flat.cuda()[1:].as_strided(shape, step)
    aligned, odd = torch.zeros(shape, dtype=dt, device="cuda"), torch.zeros_like(flat.cuda())
    args = (k, v, ks, vs, dev(rows), dev(lens), dev(starts))
    ws = torch.empty(wm.attend_ws_bytes(aligned, k, dev(lens), max(lens)), dtype=torch.uint8,
                     device="cuda")
    wm.cache_attend(q.contiguous(), *args, aligned, ws, max_len=max(lens), scale=0.1)
    view = odd[1:].as_strided(shape, step)
    wm.cache_attend(q, *args, view, ws, max_len=max(lens), scale=0.1)
    assert torch.equal(view, aligned) and bool(aligned.any())
    view.zero_()
    assert not odd.any()


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("fmt", [E4, E5])
@pytest.mark.parametrize("new,dim", [([1] * 9, 64), ([3, 1, 8], 128), ([40, 1, 77], 64),
                                     ([130, 20], 192)])
def test_rows_at_any_address_are_stored(wm, dt, fmt, new, dim):
    """Keys and values that begin at odd elements, with odd strides."""
    say(f"[append] {dt} {fmt} new={new} dim={dim}")
    bt, heads = 32, 2
    old = [5 * i for i in range(len(new))]
    rows, blocks = layout([o + n for o, n in zip(old, new)], bt, 111)
    k, v, ks, vs = make_cache(blocks, heads, bt, dim, fmt, 112)
    starts = [0] + np.cumsum(new).tolist()
    slots = [rows[r][(o + i) // bt] * bt + (o + i) % bt
             for r, (o, n) in enumerate(zip(old, new)) for i in range(n)]
    total, g = starts[-1], torch.Generator().manual_seed(113)
    row, head = heads * (dim + 3) + 4, dim + 3
    flat = (torch.randn(2 * total * row + 1, generator=g) * 3).to(dt)
    kn = flat[1:].as_strided((total, heads, dim), (row, head, 1))
    vn = flat[1 + total * row:].as_strided((total, heads, dim), (row, head, 1))
    want_k, want_ks = ref.append(kn, k.cpu(), ks.cpu(), slots, starts, False)
    want_v, want_vs = ref.append(vn, v.cpu(), vs.cpu(), slots, starts, True)
    there, verdict = flat.cuda(), word()
    wm.cache_append(there[1:].as_strided((total, heads, dim), (row, head, 1)),
                    there[1 + total * row:].as_strided((total, heads, dim), (row, head, 1)),
                    k, v, ks, vs, dev(slots, torch.int64), dev(starts), verdict)
    assert verdict.item() == 0
    assert torch.equal(ks.cpu().double(), want_ks) and torch.equal(vs.cpu().double(), want_vs)
    assert torch.equal(ref.decode(k.cpu()), want_k)
    assert torch.equal(ref.decode(v.cpu()), want_v)


@pytest.mark.parametrize("lens,new,heads,group,more", [
    # 17 to 32 rows a request at 64 dimensions, over several parts
    ([1500, 700], [5, 5], 2, 4, {}), ([2100, 30, 600], [1, 1, 1], 1, 32, {}),
    ([1700], [24], 1, 1, dict(window=900)), ([1300, 1200], [9, 7], 1, 3, dict(max_len=600))])
def test_tiles_of_32_rows_in_parts(wm, lens, new, heads, group, more):
    for dt, fmt in ((BF, E4), (HF, E5)):
        check_attend(wm, lens, new, heads, group, 16, 64, dt, fmt, seed=120, **more)


def test_a_prompt_in_a_mostly_empty_cache():
    """One session among 64 places for them, prompt and token: as good as in a
    cache of its own."""
    from paper_2607_10389_amd import PagedCache
    heads, dim, bt, n = 2, 64, 16, 150
    g = torch.Generator(device="cuda").manual_seed(8)
    x = [torch.randn(m, 8 * heads, dim, generator=g, device="cuda").to(BF) for m in (n, 1)]
    for places in (64, 1):
        c = PagedCache(layers=1, blocks=20, heads=heads, dim=dim, block_tokens=bt,
                       max_requests=places)
        for i, y in enumerate(x):
            assert c.step({places // 2: n + i}) == y.shape[0]
            c.append(0, y[:, 6 * heads:7 * heads], y[:, 7 * heads:])
            lse = torch.zeros(y.shape[0], 6 * heads, device="cuda")
            out = c.attend(0, y[:, :6 * heads], 0.125, lse=lse)
            k, v, ks, vs = c.layer(0)
            want, z, weight, sp = ref.attend(
                y[:, :6 * heads].cpu(), values(k, ks, False), values(v, vs, True),
                c.block_table[places // 2:places // 2 + 1].tolist(), [n + i], [0, y.shape[0]], bt,
                0.125)
            bo, bl = ref.attend_bound(BF, want, z, weight, sp, n + i, dim)
            assert bool(((out.cpu().double() - want).abs() <= bo).all())
            assert bool(((lse.cpu().double() - z).abs() <= bl).all())


def test_captured_prompts_and_pages_replay(wm):
    """A prompt in parts, and a session's blocks out of one pool and into
    another, captured and replayed with new inputs, each time as the eager
    calls."""
    bt, lens, new, dim = 32, [1900, 400], [40, 30], 128
    rows, blocks = layout(lens, bt, 121)
    k, v, ks, vs = make_cache(blocks, 1, bt, dim, E4, 122)
    args = (k, v, ks, vs, dev(rows), dev(lens), dev([0, 40, 70]))
    q = torch.zeros(70, 2, dim, dtype=BF, device="cuda")
    out, lse = torch.zeros_like(q), torch.zeros(70, 2, device="cuda")
    ws = torch.empty(wm.attend_ws_bytes(q, k, args[5], 1900), dtype=torch.uint8, device="cuda")
    assert ws.numel()
    pool, other = random_bytes(20 * 300, 1).view(20, 300), random_bytes(20 * 300, 2).view(20, 300)
    pages, to, verdict = dev([7, 7, 3, 19]), dev([0, 4, 8, 2]), word()
    flat = torch.zeros(wm.flat_pages_bytes([pool], 4), dtype=torch.uint8, device="cuda")
    tables = wm.PoolTable([pool]), wm.PoolTable([other])

    def calls(o, z):
        wm.cache_attend(q, *args, o, ws, max_len=1900, scale=0.1, lse=z)
        wm.flatten_pages(tables[0], pages, flat, verdict)
        wm.rehydrate_pages(flat, tables[1], to, verdict)

    calls(out, lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(out, lse)
    g = torch.Generator(device="cuda").manual_seed(123)
    for i in range(5):
        q.copy_(torch.randn(q.shape, generator=g, device="cuda"))
        pages.copy_(torch.randint(0, 20, (4,), generator=g, device="cuda"))
        pool.copy_(random_bytes(20 * 300, 10 + i).view(20, 300))
        expect = other.clone()
        expect[to.long()] = pool[pages.long()]
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(other, expect) and verdict.item() == 0, i
        want, z = torch.zeros_like(out), torch.zeros_like(lse)
        wm.cache_attend(q, *args, want, ws, max_len=1900, scale=0.1, lse=z)
        assert torch.equal(out, want) and torch.equal(lse, z) and bool(out.any()), i


def test_a_token_is_answered_the_same_among_empty_places(wm):
    """32 query heads per key head at 64 dimensions: tiles of 32 rows, and of 16
    where most requests have no token."""
    bt, group, dim, n = 16, 32, 64, 1400
    rows, blocks = layout([n], bt, 131)
    for dt, fmt in ((BF, E4), (HF, E4), (BF, E5)):
        k, v, ks, vs = make_cache(blocks, 1, bt, dim, fmt, 132)
        q = torch.randn(1, group, dim, generator=torch.Generator().manual_seed(133)).to(dt).cuda()
        outs = []
        for places in (1, 2, 5):
            lens, starts = dev([n] * places), dev([0] + [1] * places)
            out, lse = torch.zeros_like(q), torch.zeros(1, group, device="cuda")
            ws = torch.empty(wm.attend_ws_bytes(q, k, lens, n), dtype=torch.uint8, device="cuda")
            wm.cache_attend(q, k, v, ks, vs, dev(rows * places), lens, starts, out, ws, max_len=n,
                            scale=0.1 if fmt == E4 else 1e-3, lse=lse)
            outs.append((out, lse))
        for o, z in outs[1:]:
            assert torch.equal(o, outs[0][0]) and torch.equal(z, outs[0][1]) and bool(o.any())


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("order", ["up", "down", "mixed"])
@pytest.mark.parametrize("new,group,bt,dim,window", [
    (1, 16, 16, 64, 0), (1, 4, 64, 256, 50), (126, 2, 16, 64, 0), (100, 2, 64, 128, 0),
    (126, 1, 32, 192, 20), (120, 2, 128, 256, 0)])
@pytest.mark.parametrize("high", [2.0 ** 20, 2.0 ** 27, 2.0 ** 40])
def test_scores_beyond_the_bits_of_32(wm, dt, order, new, group, bt, dim, window, high):
    """Scores up to `high`: where a row's largest is 64 above the next (the others
    then weigh less than 126 e^-64 together), its answer is that token's value,
    whatever the scales; the rows of small scores by the bound of all tests."""
    n, scale = 126, high / 2.0 ** 14
    rows, blocks = layout([n], bt, 141)
    k, v, ks, vs = make_cache(blocks, 1, bt, dim, E4, 142, spread=False)
    codes = torch.arange(1, 127)
    if order != "up":
        codes = codes.flip(0) if order == "down" else codes[torch.randperm(
            126, generator=torch.Generator().manual_seed(143))]
    place = [(rows[0][j // bt], j % bt) for j in range(n)]
    kb = torch.zeros(blocks, 1, bt, dim, dtype=torch.uint8)
    for (b, t), c in zip(place, codes.tolist()):
        kb[b, 0, t, 0] = c
    k.view(torch.uint8).copy_(kb)
    ks.fill_(1.0)
    q = torch.zeros(new, group, dim, dtype=dt)
    q[..., 0] = 32.0
    out = torch.zeros(new, group, dim, dtype=dt, device="cuda")
    lse = torch.zeros(new, group, device="cuda")
    wm.cache_attend(q.cuda(), k, v, ks, vs, dev(rows), dev([n]), dev([0, new]), out, max_len=n,
                    scale=scale, window=window, lse=lse)
    vals = values(v, vs, True)
    score = torch.tensor([float(ref.decode(k.cpu())[b, 0, t, 0]) for b, t in place]) * 32 * scale
    o, z = out.cpu().double(), lse.cpu().double()
    for i in range(new):
        p = n - new + i
        lo = max(0, p - window + 1) if window else 0
        two = torch.cat([score[lo:p + 1], torch.tensor([-math.inf])]).topk(2).values
        j = lo + int(score[lo:p + 1].argmax())
        if two[0] - two[1] >= 64:
            want = vals[place[j][0], 0, place[j][1]].to(dt).double()
            assert torch.equal(o[i], want.expand(group, dim)), (i, j)
            # lse: the sum of the weights is near 2^11 or 2^15, its logarithm and
            # the two sums after it each off by up to 2^-21 of 1, the score by
            # 2^-23 of itself: within the bound of all tests
            zero = torch.zeros(1, 1, dtype=torch.float64)
            _, bl = ref.attend_bound(dt, zero[..., None], score[j].double() + zero,
                                     zero[..., None], score[j].double() + zero, n, dim)
            assert bool(((z[i] - score[j].double()).abs() <= bl).all()), (i, j)
            continue
        got = ref.attend(q[i:i + 1], values(k, ks, False), vals, rows, [p + 1], [0, 1], bt, scale,
                         window)
        bo, bl = ref.attend_bound(dt, *got, n, dim)
        assert bool(((o[i] - got[0][0]).abs() <= bo[0]).all()), (i, j)
        assert bool(((z[i] - got[1][0]).abs() <= bl[0]).all()), (i, j)
