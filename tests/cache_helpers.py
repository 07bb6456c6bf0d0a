"""Inputs of the page cache's tests: pools with NaN wherever no key is, tables,
trees, all from a seed, on the host and on the GPU."""

from __future__ import annotations

import numpy as np

from gpu_helpers import device
from oracle import serve_oracle as S


class Batch:
    def __init__(self, lens, new, hq, hkv, d, dtype, page=64, gaps=False, moved=False, tree=None,
                 seed=0, extra_pages=1, fill=float("nan")):
        """lens, new: slots and new tokens of every sequence.  tree: None for a chain,
        else a function (rng, n) -> [n, n] booleans."""
        import torch
        rng = np.random.default_rng(seed)
        B = len(lens)
        pages = max(1, -(-max(lens) // page)) + extra_pages
        self.B, self.hq, self.hkv, self.d, self.page, self.max_pages = B, hq, hkv, d, page, pages
        self.slots = pages * page
        self.dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.max_rows = max(1, max(new))
        used = np.clip(np.asarray(lens)[:, None] - page * np.arange(pages)[None], 0, page)
        if gaps:
            cut = (rng.random(used.shape) < 0.4) & (used > 0)
            used = np.where(cut, rng.integers(0, np.maximum(used, 1)), used)
        self.page_lens = used.astype(np.int32) if gaps else None
        pool = B * pages + 2
        table = rng.permutation(pool)[:B * pages].reshape(B, pages).astype(np.int32)
        k = np.full((pool * page, hkv, d), fill, np.float32)
        v = k.copy()
        for b in range(B):
            for j in range(pages):
                n, a = int(used[b, j]), int(table[b, j]) * page
                k[a:a + n] = self.keys(rng, n)
                v[a:a + n] = rng.standard_normal((n, hkv, d))
        # entries past a sequence's pages may hold anything
        for b in range(B):
            table[b, -(-lens[b] // page):] = rng.integers(-5, pool + 5, pages - -(-lens[b] // page))
        rows = sum(new)
        self.rows = rows
        self.row_ptr = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        q = rng.standard_normal((rows, hq, d))
        k_new, v_new = self.keys(rng, rows), rng.standard_normal((rows, hkv, d))
        self.sees = None if tree is None else [np.asarray(tree(rng, n), bool) for n in new]
        self.key_pos = self.row_pos = None
        if moved:
            self.key_pos = np.stack([np.stack([rng.permutation(self.slots) for _ in range(hkv)])
                                     for _ in range(B)]).astype(np.int32)
            self.row_pos = (self.slots + rng.integers(0, 50, rows)).astype(np.int32)
        self.lens = np.asarray(lens, np.int32)
        self.table = table
        dev = device()
        up = lambda x: None if x is None else torch.from_numpy(np.ascontiguousarray(x)).to(dev)  # noqa: E731
        as_t = lambda x: torch.from_numpy(x.astype(np.float32)).to(dev).to(self.dtype)  # noqa: E731
        self.q, self.k_new, self.v_new = as_t(q), as_t(k_new), as_t(v_new)
        self.k, self.v = as_t(k), as_t(v)
        self.t = {n: up(getattr(self, n)) for n in ("table", "lens", "page_lens", "key_pos",
                                                    "row_ptr", "row_pos")}
        self.words = (self.max_rows + 63) // 64
        self.mask = None
        if self.sees is not None:
            bits = np.zeros((rows, self.words), np.uint64)
            for b, m in enumerate(self.sees):
                for i, j in zip(*np.nonzero(m)):
                    bits[self.row_ptr[b] + i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
            self.mask = up(bits.view(np.int64))

    def keys(self, rng, n):
        x = rng.standard_normal((n, self.hkv, self.d))
        return x * np.where(rng.random((n, self.hkv, 1)) < 0.05, 4.0, 1.0)

    def cache(self):
        from paper_2606_09441_amd import Cache
        return Cache(self.B, self.hq, self.hkv, self.d, page=self.page, max_pages=self.max_pages,
                     max_rows=self.max_rows)

    def pages(self):
        from paper_2606_09441_amd import CachePages
        return CachePages(self.k, self.v, self.t["table"], self.t["lens"],
                          page_lens=self.t["page_lens"], key_pos=self.t["key_pos"])

    def host(self):
        f = lambda x: x.float().cpu().numpy()  # noqa: E731
        return S.Pages(f(self.k), f(self.v), self.table, self.lens, self.page, self.page_lens,
                       self.key_pos)

    def oracle(self, **kw):
        f = lambda x: x.float().cpu().numpy()  # noqa: E731
        return S.cache_attention(f(self.q), f(self.k_new), f(self.v_new), self.host(), self.row_ptr,
                                 self.sees, self.row_pos, **kw)


def random_tree(rng, n):
    """Ancestors and self of a random tree's nodes."""
    m = np.eye(n, dtype=bool)
    for i in range(1, n):
        m[i] |= m[rng.integers(0, i)]
    return m


def some_empty(rng, n):
    """A random mask with rows that see nothing."""
    m = rng.random((n, n)) < 0.3
    m[rng.random(n) < 0.4] = False
    return m
