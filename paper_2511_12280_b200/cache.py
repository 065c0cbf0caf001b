"""A K/V cache in pages for one layer, from prefix to response block:

    append (prefix, keys rotated)  ->  per step: append (block) -> attend -> evict or drop the block

``PagedCache`` owns the pools, hands out pages and keeps the host's copy of the lengths (all sizes are known on the host, as
everywhere in this package); every step of the path runs in the library's kernels.  Slots of a request are in no order that
matters to attention; ``token`` holds the number that the caller gave a slot's token.  All work, the small uploads of table
and lengths included, is enqueued on torch's current stream; calls of one cache share a context, so those on different
streams must not overlap.
"""
from __future__ import annotations

from typing import Optional, Sequence

import numpy as np
import torch

from . import binding as B_


class PagedCache:
    def __init__(self, batch: int, heads: int, kv_heads: int, head_dim: int, dtype: torch.dtype, pages: int, page_size: int,
                 max_rows: int, max_length: int, max_scored_rows: int = 1, device: int = 0):
        """max_rows: new rows per call over the batch; max_length: slots of a request; max_scored_rows: rows of a call that
        feeds the weights."""
        self.dev = torch.device("cuda", device)
        self.batch, self.heads, self.kv_heads, self.dh, self.dtype = batch, heads, kv_heads, head_dim, dtype
        self.page_size, self.max_length = page_size, max_length
        # the scratch of an eviction is counted in words of max_total_tokens rows
        tokens = max(max_rows, -(-batch * (max_length + 1) // (heads * head_dim)))
        self.ctx = B_.Context(tokens, batch, heads, head_dim, max(1, max_scored_rows), max(1, max_length), device)
        shape = (pages, page_size)
        kw = dict(device=self.dev)
        self.k = torch.zeros(*shape, kv_heads, head_dim, dtype=dtype, **kw)
        self.v = torch.zeros_like(self.k)
        self.weight = torch.zeros(shape, dtype=torch.float32, **kw)
        self.token = torch.zeros(shape, dtype=torch.int32, **kw)
        self.table_h = np.full((batch, -(-max_length // page_size)), -1, dtype=np.int32)
        self.table = torch.as_tensor(self.table_h, device=self.dev)
        self.length = torch.zeros(batch, dtype=torch.int32, **kw)
        self.cache = B_.Cache(self.k, self.v, self.weight, self.token, self.table, self.length)
        self.lengths_h = [0] * batch
        self.free = list(range(pages - 1, -1, -1))
        self.scale = 1.0 / float(np.sqrt(head_dim))

    def _of_requests(self, numbers: Sequence[int], least: Optional[int] = 0):
        """A number for every request, none below `least`."""
        if len(numbers) != self.batch or (least is not None and min(numbers) < least):
            raise ValueError("%d numbers are wanted, one for every request, not below %s: %s" % (self.batch, least, list(numbers)))
        return numbers

    def _resize(self, lengths: Sequence[int]):
        """Pages for the new lengths; table and lengths on the device follow in stream order.  Pages are given back in the
        reverse of the order they were taken in: a growth that is taken back leaves everything as it was."""
        need = [-(-n // self.page_size) for n in lengths]
        have = [-(-n // self.page_size) for n in self.lengths_h]
        if max(lengths) > self.max_length or sum(max(0, n - h) for n, h in zip(need, have)) > len(self.free):
            raise RuntimeError("the cache is full: %s slots asked for" % (list(lengths),))
        for b, (n, h) in reversed(list(enumerate(zip(need, have)))):
            for p in range(h - 1, n - 1, -1):
                self.free.append(int(self.table_h[b, p]))
                self.table_h[b, p] = -1
        for b, (n, h) in enumerate(zip(need, have)):
            for p in range(h, n):
                self.table_h[b, p] = self.free.pop()
        if need != have:
            self.table.copy_(torch.from_numpy(self.table_h.copy()))
        self.length.copy_(torch.tensor(list(lengths), dtype=torch.int32))
        self.lengths_h = [int(n) for n in lengths]

    def _cu(self, rows: Sequence[int]):
        return torch.as_tensor(np.concatenate([[0], np.cumsum(rows)]).astype(np.int32), device=self.dev)

    def append(self, rows: Sequence[int], k, v, tokens, q=None, q_out=None, spec: Optional[B_.RopeSpec] = None,
               positions=None, first_weight=None):
        """Writes rows[b] new rows of every request behind its slots; q rotated alike goes to q_out.  first_weight +inf
        keeps a row from being evicted.  A call that is refused leaves lengths and pages as they were."""
        before = self.lengths_h
        self._resize([n + r for n, r in zip(before, self._of_requests(rows))])
        try:
            self.ctx.d3tom_cache_append(self.cache, spec, q, k, v, positions, tokens, first_weight, self._cu(rows), self.batch,
                                        int(sum(rows)), q_out)
        except BaseException:
            self._resize(before)
            raise

    def attend(self, rows: Sequence[int], q, out, mode: int = B_.WEIGHT_NONE, row_weight=None):
        """Attention of rows[b] rows of every request over all of its slots."""
        self._of_requests(rows)
        self.ctx.d3tom_attn_cached(self.cache, q, self._cu(rows), self.batch, int(sum(rows)), max(rows), max(self.lengths_h),
                                   self.scale, mode, row_weight, out)

    def evict(self, budget: Sequence[int], protect_from=None):
        """Keeps the min(budget[b], length) heaviest slots of every request; frees the pages behind them."""
        want = torch.as_tensor(np.asarray(self._of_requests(budget, None), dtype=np.int32), device=self.dev)
        self.ctx.d3tom_cache_evict(self.cache, want, protect_from, self.batch, max(self.lengths_h), self.length)
        self._resize([min(max(int(x), 0), n) for x, n in zip(budget, self.lengths_h)])

    def drop_last(self, rows: Sequence[int]):
        """Gives up the last rows[b] slots of every request (a block that the next step writes again).  Before an eviction: that
        one moves kept slots, and the last ones are the block's no longer."""
        left = [n - r for n, r in zip(self.lengths_h, self._of_requests(rows))]
        self._resize(self._of_requests(left))
