"""Caches and batches for the tests of the paged 4-bit cache (test infrastructure only)."""
from __future__ import annotations

import numpy as np
import torch

from oracle import cache as oc


class Batch:
    """A cache filled with random 4-bit keys and values, and sequences over it: `rows`
    and `lengths` of each (lengths with their rows), pages dealt at random."""

    def __init__(self, rows, lengths, heads, d, page=64, seed=0, spare=1, width=0):
        rng = np.random.default_rng(seed)
        self.rows, self.lengths, self.heads, self.d, self.page = list(rows), list(lengths), heads, d, page
        need = [-(-n // page) for n in lengths]
        self.pages = sum(need) + spare
        deal = rng.permutation(self.pages)
        self.W = max(need + [1, width])
        self.page_table = np.full((len(need), self.W), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            self.page_table[b, :n] = deal[at:at + n]
            at += n
        self.starts = np.concatenate(([0], np.cumsum(self.rows))).astype(np.int32)
        self.T = int(self.starts[-1])
        chunks = page // oc.CHUNK
        def byte(*shape):
            return rng.integers(0, 256, (self.pages, heads) + shape).astype(np.uint8)

        def scale():   # 2^-2 to 2^2
            return rng.integers(125, 130, (self.pages, heads, chunks, d // oc.BLOCK, oc.CHUNK)).astype(np.uint8)
        self.cache = (byte(page, d // 2), byte(chunks, d // 2, oc.CHUNK), scale(), scale())

    def gpu(self, hcms):
        """(cache, page_table, lengths, starts) on the GPU."""
        k, v, ks, vs = (torch.from_numpy(x.copy()).cuda() for x in self.cache)
        cache = hcms.KvCache(k, v, ks.view(hcms.E8M0), vs.view(hcms.E8M0))
        return (cache, torch.from_numpy(self.page_table).cuda(),
                torch.tensor(self.lengths, dtype=torch.int32).cuda(), torch.from_numpy(self.starts).cuda())

    def read(self, b):
        return oc.read(self.cache, self.page_table[b], self.lengths[b])

    def places(self):
        """(sequence, place) of each row."""
        return [(b, n - r + i) for b, (r, n) in enumerate(zip(self.rows, self.lengths)) for i in range(r)]

    def store(self, k, v):
        """The rows k and v [T][heads][d] (float64, keys turned) into self.cache."""
        for t, (b, p) in enumerate(self.places()):
            if p < 0 or p >= self.W * self.page or not 0 <= self.page_table[b, p // self.page] < self.pages:
                continue
            for h in range(self.heads):
                oc.store(self.cache, self.page_table[b, p // self.page], p % self.page, h, k[t, h], v[t, h])


def numpy_of(cache):
    return [t.view(torch.uint8).cpu().numpy() for t in cache]


def same_values(got, want):
    """Bytes of two caches' values equal but for the sign of zeros."""
    def plain(x):
        lo, hi = x & 15, x >> 4
        return np.where(lo == 8, 0, lo) + 16 * np.where(hi == 8, 0, hi)
    return np.array_equal(plain(got), plain(want))
