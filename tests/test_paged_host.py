"""PagedCache's host logic without a GPU: its calls of the binding are replaced
by plain ones on host tensors."""
import os
import weakref

import pytest
import torch

import cache_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2607_10389_amd", "libwm.so")


class Calls(list):
    """(name, address of the slot map or the workspace) of each call."""


@pytest.fixture
def paged(monkeypatch):
    if not os.path.exists(LIB):
        pytest.skip("libwm.so is not built")
    from paper_2607_10389_amd import _cache, paged
    calls = Calls()

    def page_tables(old, new, bt, table, ring, pool_in, pool_out, slots, starts, verdict,
                    stream=None):
        head, count = pool_in.tolist()
        got = ref.tables(old.tolist(), new.tolist(), bt, table.tolist(), ring.tolist(), head,
                         count, slots.tolist(), starts.tolist())
        for t, x in zip((table, ring, pool_out, slots, starts), got):
            t.copy_(torch.tensor(x, dtype=t.dtype).reshape(t.shape))
        verdict.fill_(got[5])

    def cache_append(k, v, kc, vc, ks, vs, slots, starts, verdict=None, stream=None):
        calls.append(("append", slots.data_ptr()))

    def cache_attend(q, kc, vc, ks, vs, table, lens, starts, out, ws=None, **kw):
        calls.append(("attend", ws.data_ptr()))

    def flatten_pages(pools, pages, flat, verdict, stream=None):
        calls.append(("flatten", int(verdict.item())))
        verdict |= paged.found

    def rehydrate_pages(flat, pools, pages, verdict, stream=None):
        calls.append(("rehydrate", int(verdict.item())))
        verdict |= paged.found

    for f in (page_tables, cache_append, cache_attend, flatten_pages, rehydrate_pages):
        monkeypatch.setattr(_cache, f.__name__, f)
    monkeypatch.setattr(_cache, "PoolTable", lambda pools: pools)
    monkeypatch.setattr(_cache, "flat_pages_bytes", lambda pools, n: 1024 * n)
    monkeypatch.setattr(paged, "calls", calls, raising=False)
    monkeypatch.setattr(paged, "found", 0, raising=False)  # by the page calls
    return paged


def small(paged, **kw):
    args = dict(layers=1, blocks=400, heads=2, dim=64, block_tokens=16, max_requests=3,
                device="cpu")
    return paged.PagedCache(**{**args, **kw})


def rows(n, heads=2):
    return torch.zeros(n, heads, 64, dtype=torch.bfloat16)


def test_a_larger_step_leaves_the_buffers_of_captured_calls(paged):
    """What a captured append reads is what every later step writes, and what a
    captured attend writes belongs to nobody else."""
    c = small(paged)
    c.step({0: 600})
    c.step({0: 601})
    c.append(0, rows(1), rows(1))
    c.attend(0, rows(1, 8), 0.1)
    (_, slots), (_, ws) = paged.calls
    kept = weakref.ref(c._ws)
    n = c.step({1: 5000})  # more tokens, a longer sequence
    c.append(0, rows(n), rows(n))
    c.attend(0, rows(n, 8), 0.1)
    c.step({0: 602, 1: 5001})
    c.attend(0, rows(2, 8), 0.1)
    assert paged.calls[-1][1] != ws
    assert c.slot_map.data_ptr() == slots == paged.calls[2][1]
    want = [int(c.block_table[r, p // 16]) * 16 + p % 16 for r, p in ((0, 601), (1, 5000))]
    assert c.slot_map[:2].tolist() == want
    assert kept() is not None and kept().data_ptr() == ws


def test_the_slot_map_holds_the_largest_step(paged):
    c = small(paged, blocks=9, max_requests=4)
    assert c.step({0: 64, 1: 33, 2: 16, 3: 16}) == 129  # all nine blocks
    c.step({r: 0 for r in range(4)})
    assert c.step({1: 144}) == 144
    c = small(paged, blocks=100, max_requests=2, max_blocks=3)
    assert c.step({0: 48, 1: 48}) == 96
    from paper_2607_10389_amd import WmError
    with pytest.raises(WmError):
        c.step({0: 49})
    assert c.lengths == [48, 48]


def test_findings_stay_until_a_step_raises_for_them(paged):
    from paper_2607_10389_amd import WmError
    c = small(paged)
    c.step({0: 20})
    c.verdict.fill_(4)  # an append's, say
    flat = c.suspend(0)
    assert paged.calls[-1] == ("flatten", 0) and c.verdict.item() == 4
    state = c.lengths, c.lens.tolist(), c.pool.tolist(), c.q_start.tolist(), c.slot_map.tolist()
    with pytest.raises(WmError, match="verdict 4"):
        c.step({0: 21})
    assert state == (c.lengths, c.lens.tolist(), c.pool.tolist(), c.q_start.tolist(),
                     c.slot_map.tolist())
    assert c.step({0: 21}) == 1
    with pytest.raises(WmError, match="verdict 2"):
        c.step({0: 1 << 12, 1: 1 << 12})
    assert c.step({0: 22}) == 1  # a refused step leaves no finding
    paged.found = 8
    c.suspend(0)
    assert c.verdict.item() == 8
    with pytest.raises(WmError, match="verdict 8"):
        c.step({0: 23})
    c.resume(1, 20, flat)
    assert paged.calls[-1] == ("rehydrate", 0) and c.verdict.item() == 8


def test_fewer_rows_than_the_step_has_tokens_are_refused(paged):
    c = small(paged)
    n = c.step({0: 5, 2: 1})
    for short in (0, n - 1):
        with pytest.raises(ValueError):
            c.append(0, rows(short), rows(short))
        with pytest.raises(ValueError):
            c.attend(0, rows(short, 8), 0.1)
    assert not paged.calls
    c.append(0, rows(n + 2), rows(n + 2))  # padding
    c.attend(0, rows(n, 8), 0.1)
    c.step({0: 6})
    c.append(0, rows(1), rows(1))
    assert [x for x, _ in paged.calls] == ["append", "attend", "append"]


def test_a_resume_that_is_refused_takes_no_blocks(paged):
    c = small(paged)
    c.step({0: 20})
    buf = torch.zeros(1 << 14, dtype=torch.uint8)
    good = buf[-buf.data_ptr() % 16:][:4096]
    word = torch.zeros(1, dtype=torch.int32)
    state = c.lengths, c.lens.tolist(), c.pool.tolist(), c.q_start.tolist(), c.ring.tolist()
    for flat, verdict in ((good[1:], None), (good[8:], word), (good.view(2, 2048)[:, ::2], word),
                          (good.view(64, 64).t(), None), (good, word.long()),
                          (good, torch.zeros(0, dtype=torch.int32))):
        with pytest.raises(ValueError):
            c.resume(1, 20, flat, verdict)
    assert not paged.calls
    assert state == (c.lengths, c.lens.tolist(), c.pool.tolist(), c.q_start.tolist(),
                     c.ring.tolist())
    c.resume(1, 20, good, word)
    assert paged.calls == [("rehydrate", 0)] and c.lengths == [20, 20, 0]
