"""Seeded cases of the 4-bit cache, shared by its CPU and GPU tests."""
import numpy as np
import torch

from oracle import cache_oracle as co


class CacheCase:
    """Sequences of the given lengths and new rows in a cache of shuffled pages; keys and values of all
    positions, the cache bytes with every position stored by the oracle."""

    def __init__(self, lens, news, heads, dim, group, page, seed=0, dtype="bf16", spare=2, scale_k=1.0):
        rng = np.random.default_rng(seed)
        self.lens, self.news, self.heads, self.dim, self.group, self.page, self.dtype = list(lens), list(news), heads, dim, group, page, dtype
        self.n_seqs = len(self.lens)
        need = [-(-n // page) for n in self.lens]
        self.n_pages = sum(need) + spare
        order = rng.permutation(self.n_pages)
        self.table = np.full((self.n_seqs, max(1, max(need, default=1))), -1, dtype=np.int32)
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = order[at:at + n]
            at += n
        self.k = [self.cast(rng.standard_normal((n, heads, dim)) * scale_k + rng.standard_normal((heads, dim))) for n in self.lens]
        self.v = [self.cast(rng.standard_normal((n, heads, dim))) for n in self.lens]
        ns = dim // group
        self.block = 16 * dim + 128 * ns
        self.garbage = rng.integers(0, 256, (self.n_pages, heads, page // 16, self.block), dtype=np.uint8)
        self.row_start = np.concatenate([[0], np.cumsum(self.news)]).astype(np.int32)
        self.rows = int(self.row_start[-1])

    def cast(self, x):
        x = x.astype(np.float32)
        return co.round_bf16(x) if self.dtype == "bf16" else x

    def full_pages(self):
        pages = self.garbage.copy()
        for s in range(self.n_seqs):
            if self.lens[s]:
                co.store(pages, self.page, self.group, self.table[s], self.lens[s], self.k[s], self.v[s])
        return pages

    def new(self, which):
        x = self.k if which == "k" else self.v
        parts = [x[s][self.lens[s] - n:] for s, n in enumerate(self.news)]
        return np.concatenate(parts).reshape(self.rows, self.heads * self.dim) if parts else np.zeros((0, self.heads * self.dim), np.float32)

    def held(self, s):
        return co.held(self.k[s], self.group), co.held(self.v[s], self.group)

    # device side
    def seqs(self, row_start=True):
        from paper_2607_28418_b200 import binding
        return binding.Sequences(torch.from_numpy(self.table).cuda(), torch.tensor(self.lens, dtype=torch.int32).cuda(),
                                 torch.from_numpy(self.row_start).cuda() if row_start else None)

    def cache(self, pages):
        from paper_2607_28418_b200 import binding
        return binding.Cache(torch.from_numpy(pages).cuda(), self.heads, self.dim, self.group, self.page)


def to_device(x, dtype="bf16"):
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda()
    return t.to(torch.bfloat16) if dtype == "bf16" else t


def pack_bits(on):
    """bool [T, n_groups] -> int32 words [T, ceil(n_groups / 32)]."""
    T, NG = on.shape
    words = np.zeros((T, (NG + 31) // 32), dtype=np.uint32)
    for g in range(NG):
        words[:, g // 32] |= on[:, g].astype(np.uint32) << np.uint32(g % 32)
    return words.view(np.int32)
