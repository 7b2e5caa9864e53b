"""Shared helpers of the tests of the cache in 4 bits."""
import numpy as np
import torch

from oracle import fp4 as F
from paged import np64, rows


def codes_of(cache):
    return F.unpack(cache.data.view(torch.uint8).cpu().numpy())


class Filled4:
    """A 4-bit cache on the device with sequences in pages of random order, and on the host what its codes stand for; used with paged.attend_and_check."""

    def __init__(self, keys, kv_heads, d, page, dtype, seed=0, change=None, spare=3):
        from paper_2505_21070_amd import binding as B
        gen = torch.Generator().manual_seed(seed)
        rng = np.random.RandomState(seed)
        need = [-(-n // page) for n in keys]
        n_pages = sum(need) + spare
        order = rng.permutation(n_pages).tolist()
        table = torch.full((len(keys), max(need + [1])), -7, dtype=torch.int32)        # what lies behind a sequence's pages is never looked at
        self.cache = B.KVCache.empty(n_pages, kv_heads, page, d, dtype, fp4=True)
        # what other sequences left in the pages: NaN
        self.cache.scales.fill_(255)
        self.k, self.v = [], []
        for b, n in enumerate(keys):
            own, order = order[: need[b]], order[need[b]:]
            table[b, : need[b]] = torch.tensor(own, dtype=torch.int32)
            k, v = rows(gen, n, kv_heads, d, dtype, 1.3), rows(gen, n, kv_heads, d, dtype)
            if change:
                change(b, k, v)
            slot = torch.tensor([own[i // page] * page + i % page for i in range(n)], dtype=torch.int32, device="cuda")
            self.cache.write(k.cuda(), v.cuda(), slot)
            self.k.append(F.rows(np64(k))[0] if n else np64(k))
            self.v.append(F.rows(np64(v))[0] if n else np64(v))
        self.table, self.keys, self.d, self.dtype = table.cuda(), list(keys), d, dtype
