"""A paged 8-bit attention cache that owns its buffers, and its sessions' way
to and from the mover.

A ``PagedCache`` holds one pool of blocks for every layer, the block tables
and lengths of its requests, and the ring of free blocks.  ``step`` gives
requests room for their new tokens (or takes it back), ``append`` and
``attend`` are one layer's store and attention for those tokens, and
``suspend`` / ``resume`` are a session's way out and in: a flat state of every
layer's blocks, which a ``Mover`` ships like any other, into whichever blocks
the destination has free.  A token's answers after a move are the same bits as
before it, in any call of single tokens with up to 32 query heads per key head:
they do not depend on where its blocks lie or who else is asked.  (A call that
holds prompts too may take another kernel, whose results differ by roundings.
The kernel goes by the mean of new tokens per place for a request, empty ones
counted: long prompts are answered fastest in a cache without many of those,
or in a call of their own.)

``append`` and ``attend`` may be captured into a graph and replayed after any
later ``step`` of no more tokens: tables, lengths, slot map and row starts keep
their addresses, and a workspace that has become too small is kept as long as
the cache, for the graphs and streams that still use it.  (Calls on different
streams share it: they have to be ordered.)  What the calls find on the device
is ORed into ``verdict`` and stays there until the next ``step`` raises for it.
"""
from __future__ import annotations

import torch

from . import _cache, _wm


class PagedCache:
    def __init__(self, layers: int, blocks: int, heads: int, dim: int, block_tokens: int = 64,
                 dtype: torch.dtype = torch.float8_e4m3fn, max_requests: int = 64,
                 max_blocks: int | None = None, device: str | torch.device = "cuda"):
        self.layers, self.heads, self.dim, self.block_tokens = layers, heads, dim, block_tokens
        self.max_requests = max_requests
        i32 = dict(dtype=torch.int32, device=torch.device(device))
        # a block of all layers is one piece: a session moves in large copies
        self.codes = torch.zeros(blocks, layers, 2, heads * block_tokens * dim,
                                 dtype=torch.uint8, device=i32["device"])
        self.scales = torch.zeros(blocks, layers, 2, heads, dtype=torch.float32,
                                  device=i32["device"])
        self._layers = []
        for n in range(layers):
            k, v = (self.codes[:, n, i].view(dtype) for i in (0, 1))
            self._layers.append((k.view(blocks, heads, block_tokens, dim),
                                 v.view(blocks, heads, dim, block_tokens),
                                 self.scales[:, n, 0], self.scales[:, n, 1]))
        self.block_table = torch.zeros(max_requests, max_blocks or blocks, **i32)
        self.ring = torch.arange(blocks, **i32)
        self.pool = torch.tensor([0, blocks], **i32)
        self._pool_next = torch.zeros(2, **i32)
        self.lens = torch.zeros(max_requests, **i32)
        self.lengths = [0] * max_requests  # the same on the host
        self.q_start = torch.zeros(max_requests + 1, **i32)
        # no step has more new tokens than the blocks have places
        places = min(blocks, max_requests * self.block_table.shape[1]) * block_tokens
        self.slot_map = torch.zeros(min(places, 2 ** 31 - 1), dtype=torch.int64,
                                    device=i32["device"])
        self.verdict = torch.zeros(1, **i32)
        self._word = torch.zeros(1, **i32)  # a call's own verdict
        self._tokens = 0  # of the last step
        self._ws = torch.zeros(0, dtype=torch.uint8, device=i32["device"])
        self._outgrown = []  # smaller workspaces
        self.pools = _cache.PoolTable([self.codes, self.scales])

    def layer(self, n: int):
        """(key codes, value codes, key scales, value scales) of layer n."""
        return self._layers[n]

    def step(self, new_lengths: dict[int, int]) -> int:
        """Take requests to new lengths (0: done); the others stay.  Returns
        the number of new tokens, whose keys, values and queries append() and
        attend() expect ordered by request.  Waits for the verdict; raises
        WmError, and changes nothing, if the pool or the tables are too small,
        or (once) if a call since the last step has left a finding."""
        want = list(self.lengths)
        for r, n in new_lengths.items():
            want[r] = n
        found = int(self.verdict.item())
        if found:
            self.verdict.zero_()
            raise _wm.WmError(_wm.WM_ERR_INVALID_ARG, f"a call before step (verdict {found})")
        tokens = sum(max(0, n - o) for o, n in zip(self.lengths, want))
        new = torch.tensor(want, dtype=torch.int32).to(self.lens.device)
        _cache.page_tables(self.lens, new, self.block_tokens, self.block_table, self.ring,
                           self.pool, self._pool_next, self.slot_map[:tokens], self.q_start,
                           self._word)
        bits = int(self._word.item())
        if bits & _cache.C_POOL:
            bits &= ~_cache.C_SLOTS  # (the slot map is as large as the pool)
        if bits:
            raise _wm.WmError(_wm.WM_ERR_CAPACITY, f"step (verdict {bits})")
        self.pool, self._pool_next = self._pool_next, self.pool
        self.lens.copy_(new)  # (captured calls read it where it is)
        self.lengths, self._tokens = want, tokens
        return tokens

    def _rows(self, t: torch.Tensor) -> None:
        if t.shape[0] < self._tokens:
            raise ValueError(f"{t.shape[0]} rows for the step's {self._tokens} tokens")

    def append(self, layer: int, k: torch.Tensor, v: torch.Tensor) -> None:
        """Store the step's new keys and values [tokens, heads, dim] (rows
        behind the last token are padding)."""
        self._rows(k)
        _cache.cache_append(k, v, *self._layers[layer], self.slot_map, self.q_start,
                            self.verdict)

    def attend(self, layer: int, q: torch.Tensor, scale: float, window: int = 0,
               out: torch.Tensor | None = None, lse: torch.Tensor | None = None) -> torch.Tensor:
        """Attention of the step's new tokens [tokens, query heads, dim] (rows
        behind the last token are padding, and stay as they are in out)."""
        self._rows(q)
        c = self._layers[layer]
        most = max(self.lengths)
        need = _cache.attend_ws_bytes(q, c[0], self.lens, most)
        if self._ws.numel() < need:
            # at least twice as large: the smaller ones together are no larger
            self._outgrown.append(self._ws)
            self._ws = torch.empty(max(need, 2 * self._ws.numel()), dtype=torch.uint8,
                                   device=q.device)
        out = torch.empty_like(q) if out is None else out
        _cache.cache_attend(q, *c, self.block_table, self.lens, self.q_start, out, self._ws,
                            max_len=most, scale=scale, window=window, lse=lse,
                            verdict=self.verdict)
        return out

    # ---- a session's move
    def _blocks(self, length: int) -> int:
        return -(-length // self.block_tokens)

    def flat_bytes(self, length: int) -> int:
        """Bytes of the flat state of a session of this length."""
        return _cache.flat_pages_bytes(self.pools, self._blocks(length))

    def suspend(self, request: int, flat: torch.Tensor | None = None) -> torch.Tensor:
        """The request's blocks of every layer as one flat state; the request
        stays (step({request: 0}) frees its blocks)."""
        n = self._blocks(self.lengths[request])
        if flat is None:
            flat = torch.empty(self.flat_bytes(self.lengths[request]), dtype=torch.uint8,
                               device=self.codes.device)
        self._word.zero_()
        _cache.flatten_pages(self.pools, self.block_table[request, :n], flat, self._word)
        self.verdict |= self._word
        return flat

    def resume(self, request: int, length: int, flat: torch.Tensor,
               verdict: torch.Tensor | None = None) -> None:
        """Give an empty request blocks for a session of this length and
        install its flat state there, if the verdict word (wm_decode_verify's,
        say) is 0 on the device.  If it is not, the request has its blocks all
        the same, with nothing installed: step({request: 0}) frees them.  The
        next call is a step()."""
        if self.lengths[request]:
            raise ValueError(f"request {request} holds a session")
        if flat.numel() * flat.element_size() < self.flat_bytes(length):
            raise ValueError(f"flat is no state of {length} tokens")
        # (the copy's own checks come behind the step: too late to change nothing)
        dev = self.lens.get_device()
        if flat.get_device() != dev or not flat.is_contiguous() or flat.data_ptr() % 16:
            raise ValueError(f"flat is dense, 16-byte aligned and on device {dev}")
        if verdict is not None:
            _cache._word(verdict, dev)
        self.step({request: length})
        n = self._blocks(length)
        word = self._word.zero_() if verdict is None else verdict
        _cache.rehydrate_pages(flat, self.pools, self.block_table[request, :n], word)
        if verdict is None:
            self.verdict |= word
