"""Inputs of the tests of paged caches: packed chunks, tables of pages in no order, poison where nothing may be read."""

import numpy as np
import torch

from lowbit_common import cuda

POISON = float("nan")


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


class Cache:
    """Pages of sequences that hold `lens` tokens: the pool, the table, and poison in every token that no sequence holds."""

    def __init__(self, rng, lens, page, kv_heads, head_dim, spare=2, table_pages=None, amp=1.0, poison=True):
        used = [-(-max(0, n) // page) for n in lens]
        self.table_pages = table_pages or max(1, *used)
        self.pages = sum(used) + spare
        order = rng.permutation(self.pages)
        self.table = np.full((len(lens), self.table_pages), -1, dtype=np.int64)
        held = np.zeros((self.pages, page), dtype=bool)
        at = 0
        for b, (n, u) in enumerate(zip(lens, used)):
            self.table[b, :u] = order[at:at + u]
            at += u
            for c in range(max(0, n)):
                held[self.table[b, c // page], c % page] = True
        self.page = page
        shape = (self.pages, page, kv_heads, head_dim)
        self.k, self.v = rng.normal(size=shape) * amp, rng.normal(size=shape)
        if poison:
            self.k[~held] = self.v[~held] = POISON

    def device(self):
        self.dk, self.dv, self.dt = cuda(self.k, "bf16"), cuda(self.v, "bf16"), ints(self.table)
        self.k, self.v = (t.double().cpu().numpy() for t in (self.dk, self.dv))
        return self


def begins(lens, first=0):
    return np.concatenate(([first], first + np.cumsum(lens))).astype(np.int64)
