"""One layer's keys of a batch of prompts, from their prefill to the answers.

A RAG prompt's documents leave a cache far longer than an answer needs.  A
PromptCache runs the layer's attention over it: the prefill of the documents and
the query (sparse over the metadata bits, or dense with capped or biased scores),
the cut of the cache to the keys that the query's tokens attend to, and then the
answer, a token or a drafted tree at a time, with further cuts as it grows:

    cache = PromptCache(seg_offsets, prompt_seg_ptr, hq, hkv, d, room=256, max_rows=8)
    out = cache.prefill(q, k, v, la, ca)          # every token of the prompts
    cache.cut(budget=1024)                        # keys of a kv head that stay
    while ...:
        out, lse = cache.step(q, k_new, v_new, tree_mask=mask, row_pos=pos)
        cache.append(q, k_new, v_new, lse, accepted, row_pos=pos)

With a Rotary the keys and queries come as they are projected, and are turned here by
their places in the prompt; with held=torch.float8_e4m3fn the keys that the cut leaves
are held in 8 bits from then on, and not cut again.

`python -m paper_2606_09441_amd.serve` runs this on random tensors.
"""

from __future__ import annotations

from ._lib import Cache, CachePages, Plan, Rotary, SiftError, _torch, rotary_frequencies


def _dense(x):
    """x as the library reads it: contiguous, from a 16-byte boundary on."""
    x = x.contiguous()
    return x if x.data_ptr() % 16 == 0 else x.clone()


class PromptCache:
    """Every prompt's last segment is its query, the others its documents.  A page
    holds one key tile; room: slots beyond the prompt's, for the answer; max_rows:
    new tokens of a prompt in one step at most; rotary: the Rotary that turns q and k
    (None: they are turned already); held: the type of the keys after the first cut
    (None: as before it)."""

    def __init__(self, seg_offsets, prompt_seg_ptr, num_q_heads, num_kv_heads, head_dim, page=64,
                 room=0, max_rows=1, dtype=None, rotary=None, held=None):
        torch = _torch()
        dtype = torch.bfloat16 if dtype is None else dtype
        self._codes = held is torch.float8_e4m3fn
        if held not in (None, dtype) and not (self._codes and dtype is torch.bfloat16):
            raise SiftError("PromptCache", 4, f"keys of {dtype} held in {held}")
        self.rotary = rotary
        so, ps = [int(x) for x in seg_offsets], [int(x) for x in prompt_seg_ptr]
        self.plan = Plan(so, ps, num_q_heads, num_kv_heads, head_dim, page)
        seqs = len(ps) - 1
        tiles = [-(-(b - a) // page) for a, b in zip(so, so[1:])]
        most = max(sum(tiles[a:b]) for a, b in zip(ps, ps[1:]))
        max_pages = max(1, most + -(-room // page))
        sizes = (seqs, num_q_heads, num_kv_heads, head_dim, page, max_pages)
        self._room_asked = room
        self.longest = max(so[b] - so[b - 1] for b in ps[1:])  # query
        # of the queries' tokens, and of the answers'
        self._queries = Cache(*sizes, max(1, self.longest))
        self.cache = Cache(*sizes, max_rows)
        self.max_rows = max_rows

        table = [[b * max_pages + p for p in range(max_pages)] for b in range(seqs)]
        tile_page, slots, lens, page_lens, pos = [], [], [], [], []
        for b in range(seqs):
            at, ends, where = 0, [page] * max_pages, [0] * (max_pages * page)
            docs = 0
            for s in range(ps[b], ps[b + 1]):
                for j in range(so[s], so[s + 1], page):
                    n = min(page, so[s + 1] - j)
                    tile_page.append(table[b][at])
                    slots += range(at * page, at * page + n)
                    if s < ps[b + 1] - 1:
                        ends[at] = n
                        where[at * page:at * page + n] = range(j - so[ps[b]], j - so[ps[b]] + n)
                        docs = at * page + n
                    at += 1
            lens.append(docs)
            page_lens.append(ends)
            pos.append(where)
        dev = self.cache.device
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
        pool = (seqs * max_pages * page, num_kv_heads, head_dim)
        self._dtype = dtype
        k, v = (torch.zeros(pool, dtype=dtype, device=dev) for _ in range(2))
        key_pos = ints(pos)[:, None, :].expand(-1, num_kv_heads, -1).contiguous()
        self.pages = CachePages(k, v, ints(table), ints(lens), ints(page_lens), key_pos)
        longs = lambda x: torch.tensor(x, dtype=torch.int64, device=dev)  # noqa: E731
        self._tile_page, self._slots = ints(tile_page), ints(slots)
        self._token_ptr = ints([so[s] for s in ps])
        self._token_pos = ints([t - so[a] for a, z in zip(ps, ps[1:]) for t in range(so[a], so[z])])
        query = [t for b in range(seqs) for t in range(so[ps[b + 1] - 1], so[ps[b + 1]])]
        first = [0]
        for b in range(seqs):
            first.append(first[-1] + so[ps[b + 1]] - so[ps[b + 1] - 1])
        self._query, self._query_ptr = longs(query), ints(first)
        self._query_rows = first
        self._query_pos = ints([t - so[ps[b]] for b in range(seqs)
                                for t in range(so[ps[b + 1] - 1], so[ps[b + 1]])])
        self.next_pos = ints([so[b] - so[a] for a, b in zip(ps, ps[1:])])  # of the next token
        self.used = max(lens)  # slots of a prompt, at most
        self.weights = None
        self._score = {}
        self._pending = None

    def close(self):
        self.plan.close()
        self._queries.close()
        self.cache.close()

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def prefill(self, q, k, v, la=None, ca=None, mask="causal", scale=None, cap=0.0, slopes=None):
        """Attention of every token of the prompts: over the bits la and ca, or dense
        under `mask`; leaves the documents' keys in the pages, with the weights that
        the query's tokens give them, and the query's own (with those that they give
        each other) to be appended by cut."""
        torch = _torch()
        if self.weights is not None:
            raise SiftError("PromptCache.prefill", 6, "the prompts are prefilled already")
        if la is not None and (cap or slopes is not None):
            raise SiftError("PromptCache.prefill", 4, "the sparse prefill takes no cap and no bias")
        tokens = self._slots.shape[0]
        for name, x, heads in (("q", q, self.cache.hq), ("k", k, self.cache.hkv),
                               ("v", v, self.cache.hkv)):
            self._check("PromptCache.prefill", name, x, (tokens, heads, self.cache.d))
        self._score = dict(scale=scale, cap=cap, slopes=slopes)
        pages, turn = self.pages, self.rotary
        k, v = _dense(k), _dense(v)
        if turn is not None:
            # (the sparse prefill reads the keys in the pages, where they are turned on the way)
            q, turned = turn.rotate(q, k if la is None else None, self._token_pos)
            k, turn = (k, turn) if la is not None else (turned, None)
        self.cache.append(pages, k, v, row_ptr=self._token_ptr, row_pos=self._token_pos,
                          rotary=turn, slots=self._slots)
        qq, kq, vq = (t[self._query] for t in (q, k, v))
        if turn is not None:
            kq = turn.rotate(kq, None, self._query_pos)[0]
        if la is not None:
            out = self.plan.run_paged(q, pages.k_pages, pages.v_pages, self._tile_page, la, ca, scale)
            # the query attends to every document: its rows again, for their log sums
            lse = torch.empty(qq.shape[:2], dtype=torch.float32, device=q.device)
            self._queries.attention(qq, kq, vq, pages, row_ptr=self._query_ptr, lse=lse, scale=scale)
        else:
            lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
            out = self.plan.dense(q, k, v, mask, lse=lse, **self._score)
            lse = lse[self._query]
        self.weights = self._queries.accumulate(qq, lse, pages, row_ptr=self._query_ptr,
                                                row_pos=self._query_pos, **self._score)
        own = [self._drawn(qq[a:z], kq[a:z], lse[a:z], self._query_pos[a:z])
               for a, z in zip(self._query_rows, self._query_rows[1:])]
        self._pending = (kq, vq, torch.cat(own))
        return out

    def _check(self, fn, name, x, shape):
        """Before anything is written: what is indexed by a prompt's rows has to hold them."""
        if x.shape != shape or x.dtype != self._dtype:
            raise SiftError(fn, 2, f"{name} holds {tuple(x.shape)} {x.dtype}, has to be {shape} "
                                   f"{self._dtype}")
        if x.device != self.cache.device:
            raise SiftError(fn, 7, f"{name} is on {x.device}, the cache on {self.cache.device}")

    def cut(self, budget, sinks=4, recent=0):
        """Every kv head keeps `budget` keys: the first `sinks`, the last `recent` and
        those of the largest weights."""
        if self.weights is None:
            raise SiftError("PromptCache.cut", 6, "the prompts are not prefilled yet")
        if self.pages.k_scales is not None:
            raise SiftError("PromptCache.cut", 4, "keys held in 8 bits are not cut again")
        self.weights, key_pos, lens = self.cache.evict(self.pages, self.weights, budget, sinks,
                                                       recent, self.next_pos)
        self.pages = CachePages(self.pages.k_pages, self.pages.v_pages, self.pages.page_table, lens,
                                None, key_pos)
        self.used = min(self.used, budget)
        if self._codes:
            self._encode()
        if self._pending is not None:
            k, v, own = self._pending
            self._pending = None
            rows = _torch().arange(k.shape[0], device=k.device)
            seq, used = self._room("PromptCache.cut", k, v, rows, self._query_ptr, self.longest)
            self._store(k, v, seq, used, self._query_pos, own)

    def _encode(self):
        """The pages in e4m3, as many as the queries and the answers need."""
        torch = _torch()
        old, cache, was = self.pages, self.cache, self.cache.page
        seqs, hkv, d, dev = cache.num_seqs, cache.hkv, cache.d, cache.device
        most = -(-max(1, self.used + self.longest + self._room_asked) // was)
        codes, scales = ([f() for _ in range(2)] for f in (
            lambda: torch.zeros(seqs * most * was, hkv, d, dtype=torch.uint8, device=dev),
            lambda: torch.zeros(seqs * most, hkv, device=dev)))
        table = torch.arange(seqs * most, dtype=torch.int32, device=dev).view(seqs, most)
        n = old.lens.tolist()
        row = torch.cat([old.page_table[b].long().repeat_interleave(was)[:x] * was +
                         torch.arange(x, device=dev) % was for b, x in enumerate(n)])
        ptr = torch.nn.functional.pad(old.lens.cumsum(0, dtype=torch.int32), (1, 0))
        slots = min(most * was, cache.slots)
        key_pos = torch.zeros(seqs, hkv, most * was, dtype=torch.int32, device=dev)
        key_pos[:, :, :slots] = old.key_pos[:, :, :slots]
        self.weights = self.weights.new_zeros(seqs, hkv, most * was)
        self.cache = Cache(seqs, cache.hq, hkv, d, was, most, self.max_rows)
        e4m3 = [x.view(torch.float8_e4m3fn) for x in codes]
        empty = CachePages(*e4m3, table, torch.zeros_like(old.lens), k_scales=scales[0],
                           v_scales=scales[1])
        lens = self.cache.append(empty, old.k_pages[row], old.v_pages[row], row_ptr=ptr)
        self.pages = CachePages(*e4m3, table, lens, key_pos=key_pos, k_scales=scales[0],
                                v_scales=scales[1])
        cache.close()

    def step(self, q, k_new, v_new, row_ptr=None, tree_mask=None, row_pos=None):
        """(out, lse) of new tokens over the cache and each other; row_pos None: each
        follows the one before."""
        torch = _torch()
        if self.weights is None or self._pending is not None:
            raise SiftError("PromptCache.step", 6, "the prompts' caches are not cut yet")
        pos = self._positions(q.shape[0], row_ptr, row_pos)
        if self.rotary is not None:
            q, k_new = self.rotary.rotate(q, k_new, pos)
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
        out = self.cache.attention(q, k_new, v_new, self.pages, row_ptr=row_ptr, tree_mask=tree_mask,
                                   row_pos=pos, lse=lse, **self._score)
        return out, lse

    def append(self, q, k_new, v_new, lse, rows, row_ptr=None, row_pos=None, decay=1.0):
        """Takes a step's accepted rows (int64, ascending; those of a prompt follow each
        other in the answer) into the cache, with the weights that they give each other,
        and adds those that they give the cached keys."""
        torch = _torch()
        if self.weights is None or self._pending is not None:
            raise SiftError("PromptCache.append", 6, "the prompts' caches are not cut yet")
        ptr = self._pointers(q.shape[0], row_ptr)
        pos = self._positions(q.shape[0], row_ptr, row_pos)
        # whatever may be refused comes before the weights and the pages change
        for name, x in (("k_new", k_new), ("v_new", v_new), ("row_pos", pos),
                        ("lse", q if self._codes else lse)):
            if x.shape[0] < q.shape[0]:
                raise SiftError("PromptCache.append", 2, f"{name} holds {x.shape[0]} rows, q {q.shape[0]}")
        seq, used = self._room("PromptCache.append", k_new, v_new, rows, ptr, self.max_rows)
        if self._codes:   # not cut again: no weights
            added = self._store(k_new[rows], v_new[rows], seq, used, pos[rows], turn=self.rotary)
            self.next_pos = self.next_pos + added
            return
        if self.rotary is not None:
            q, k_new = self.rotary.rotate(q, k_new, pos)
        k, v, at = k_new[rows], v_new[rows], pos[rows]
        own = self._drawn(q[rows], k, lse[rows], at, seq)
        counts = torch.zeros(q.shape[0], device=q.device).index_fill_(0, rows, 1.0)
        self.cache.accumulate(q, lse, self.pages, self.weights, decay, row_ptr=row_ptr, row_pos=pos,
                              row_weight=counts, **self._score)
        added = self._store(k, v, seq, used, at, own)
        self.next_pos = self.next_pos + added

    def _pointers(self, rows, row_ptr):
        torch = _torch()
        if row_ptr is not None:
            return row_ptr
        seqs = self.cache.num_seqs
        return torch.arange(seqs + 1, dtype=torch.int32, device=self.cache.device) * (rows // seqs)

    def _positions(self, rows, row_ptr, row_pos):
        torch = _torch()
        if row_pos is not None:
            return row_pos
        ptr = self._pointers(rows, row_ptr)
        row = torch.arange(rows, dtype=torch.int32, device=ptr.device)
        seq = torch.searchsorted(ptr, row, right=True).clamp_(max=self.cache.num_seqs) - 1
        return (self.next_pos[seq] + row - ptr[seq]).int()

    def _room(self, fn, k, v, rows, row_ptr, most):
        """The prompts of rows of k and v, and how many slots one has with them at most."""
        torch = _torch()
        pages = self.pages
        for name, x in (("k", k), ("v", v)):
            if x.shape[1:] != pages.k_pages.shape[1:] or x.dtype != self._dtype:
                raise SiftError(fn, 2, f"{name} holds {tuple(x.shape)} {x.dtype}")
        seq = torch.searchsorted(row_ptr, rows.int(), right=True) - 1
        used = self.used + min(rows.shape[0], most)
        if used > self.cache.slots:
            # a bound that knows no prompt's own rows; the exact number, read from the device
            used = int((pages.lens + torch.bincount(seq, minlength=self.cache.num_seqs)).max())
            if used > self.cache.slots:
                raise SiftError(fn, 5, f"{used} slots, room for {self.cache.slots}")
        return seq, used

    def _drawn(self, q, k, lse, pos, seq=None):
        """The attention weight that each of these tokens, which the cache does not hold
        yet, draws from those that see it: itself and its prompt's later ones.  seq:
        the tokens' prompts (None: one).  [tokens, kv heads]"""
        torch = _torch()
        n, hq, d = q.shape
        hkv = k.shape[1]
        g = hq // hkv
        scale, cap, slopes = (self._score[x] for x in ("scale", "cap", "slopes"))
        scale = scale if scale is not None and 0 < scale < float("inf") else d ** -0.5
        qt = torch.empty(hkv, n, g, d, device=q.device).copy_(q.view(n, hkv, g, d).transpose(0, 1))
        kt = k.float().permute(1, 2, 0)
        if seq is None:
            seq = torch.zeros(n, dtype=torch.bool, device=q.device)
        some = max(1, (1 << 24) // max(1, hq * n))   # rows at a time: 64 MB of scores
        out = torch.zeros(n, hkv, device=q.device) if some < n or n == 0 else None
        for a in range(0, n, some):
            z = min(n, a + some)                     # (they see no key past their last)
            s = torch.matmul(qt[:, a:z].view(hkv, -1, d), kt[:, :, :z]).mul_(scale)
            if cap:
                s = s.div_(cap).tanh_().mul_(cap)
            s = s.view(hkv, z - a, g, z)
            if slopes is not None:
                far = (pos[a:z, None] - pos[:z]).abs_()
                s = s.sub_(slopes[:hq].view(hkv, 1, g, 1) * far[:, None])
            w = s.sub_(lse[a:z].view(z - a, hkv, g, 1).transpose(0, 1)).exp_()
            hidden = (seq[a:z, None] == seq[:z]).tril_(a).logical_not_()
            own = w.masked_fill_(hidden[:, None], 0.0).sum((1, 2)).t()
            if out is None:
                return own
            out[:z] += own
        return out

    def _store(self, k, v, seq, used, pos, own=None, turn=None):
        """Keys of prompts seq into the slots after their last, with the weights `own`;
        how many of each.  turn: the Rotary that turns them on the way."""
        torch = _torch()
        pages = self.pages
        self.used = used
        ptr = torch.searchsorted(seq, torch.arange(self.cache.num_seqs + 1, device=seq.device),
                                 out_int32=True)
        if own is not None:
            at = torch.arange(seq.shape[0], device=seq.device)
            self.weights[seq, :, pages.lens[seq] + at - ptr[seq]] = own
        self.cache.append(pages, k, v, row_ptr=ptr, row_pos=pos, rotary=turn, lens_out=pages.lens)
        return ptr.diff()


def main():
    """Two prompts of unlike documents, cut to 512 keys, and drafted trees of four: in
    bf16, cut again as the answers grow, and with the keys turned here and held in 8 bits."""
    torch = _torch()
    hq, hkv, d = 32, 8, 128
    lens = [[700, 1300, 64, 90], [2000, 311, 47]]
    so, ps = [0], [0]
    for prompt in lens:
        for n in prompt:
            so.append(so[-1] + n)
        ps.append(len(so) - 1)
    gen = torch.Generator("cuda").manual_seed(1)
    draw = lambda n, h: torch.randn(n, h, d, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    rotary = Rotary(rotary_frequencies(d, 500000.0)[0])
    for more in ({}, {"rotary": rotary, "held": torch.float8_e4m3fn}):
        with PromptCache(so, ps, hq, hkv, d, room=128, max_rows=4, **more) as cache:
            n = cache.plan.info
            bits = [torch.randint(0, 256, (n[x],), generator=gen, device="cuda", dtype=torch.uint8)
                    for x in ("la_bytes", "ca_bytes")]
            out = cache.prefill(draw(so[-1], hq), draw(so[-1], hkv), draw(so[-1], hkv), *bits)
            print(f"prefill: {tuple(out.shape)}; cached keys {cache.pages.lens.tolist()} and the queries'")
            cache.cut(512, recent=16)
            print(f"cut: {cache.pages.lens.tolist()} of {cache.pages.k_pages.dtype}")
            # each tree: 0, its children 1 and 2, and 3 a child of 1; 0, 1 and 3 are accepted
            mask = torch.tensor([1, 3, 5, 11] * 2, device="cuda").view(8, 1)
            depth = torch.tensor([0, 1, 1, 2] * 2, dtype=torch.int32, device="cuda")
            for _ in range(3):
                q, k, v = draw(8, hq), draw(8, hkv), draw(8, hkv)
                pos = (cache.next_pos.repeat_interleave(4) + depth).int()
                out, lse = cache.step(q, k, v, tree_mask=mask, row_pos=pos)
                cache.append(q, k, v, lse, torch.tensor([0, 1, 3, 4, 5, 7], device="cuda"), row_pos=pos)
                print(f"step: {tuple(out.shape)}; cached keys {cache.pages.lens.tolist()}")
            if not more:
                cache.cut(512, recent=16)
                print(f"cut: {cache.pages.lens.tolist()}; next positions {cache.next_pos.tolist()}")


if __name__ == "__main__":
    main()
