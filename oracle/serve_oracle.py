"""Plain fp64 CPU oracle of the dense attention with transformed scores and of
the page cache's operators.

TEST INFRASTRUCTURE ONLY: nothing in the product path imports it, and it shares
no code with the HIP library.  Every function takes numpy arrays and works from
the definition, one query row and head at a time:

    z = scale q.k;  s = cap tanh(z / cap) if cap else z;  s -= slope |distance|
    lse = log sum over the visible keys of e^s  (-inf where there is none)
    out = sum over the visible keys of e^(s - lse) v  (0 where there is none)

A key that is not visible has no influence, whatever its values.
"""

from __future__ import annotations

import numpy as np


def scores(q, k, scale, cap=0.0, slope=0.0, dist=None):
    """Scores of one query [D] on keys [n, D]."""
    z = np.asarray(k, np.float64) @ np.asarray(q, np.float64) * scale
    if cap:
        z = cap * np.tanh(z / cap)
    if slope:
        z = z - slope * np.abs(np.asarray(dist, np.float64))
    return z


def attend(q, k, v, scale, cap=0.0, slope=0.0, dist=None):
    """(out [D], lse) of one query over its visible keys."""
    if len(k) == 0:
        return np.zeros(q.shape[-1]), -np.inf
    s = scores(q, k, scale, cap, slope, dist)
    m = s.max()
    w = np.exp(s - m)
    return (w @ np.asarray(v, np.float64)) / w.sum(), m + np.log(w.sum())


def segment_of(seg_offsets, n):
    return np.searchsorted(np.asarray(seg_offsets)[1:], np.arange(n), side="right")


def dense_visible(seg_offsets, prompt_seg_ptr, mask):
    """[n, n] booleans: key j is visible to row i."""
    n = int(seg_offsets[-1])
    seg = segment_of(seg_offsets, n)
    prompt = np.searchsorted(np.asarray(prompt_seg_ptr)[1:], seg, side="right")
    query = np.asarray(prompt_seg_ptr)[prompt + 1] - 1 == seg
    i, j = np.arange(n)[:, None], np.arange(n)[None]
    same = prompt[:, None] == prompt[None]
    if mask == "document":
        return same & (j <= i) & (query[:, None] | (seg[:, None] == seg[None]))
    if mask == "prefix":
        return same & ((j <= i) | ~query[None])
    return same & (j <= i)


def dense(q, k, v, seg_offsets, prompt_seg_ptr, mask, scale=None, cap=0.0, slopes=None):
    """(out [n, Hq, D], lse [n, Hq]) of the dense attention, row by row."""
    n, hq, d = q.shape
    g = hq // k.shape[1]
    scale = d ** -0.5 if scale is None else scale
    sees = dense_visible(seg_offsets, prompt_seg_ptr, mask)
    out, lse = np.zeros((n, hq, d)), np.zeros((n, hq))
    for i in range(n):
        j = np.nonzero(sees[i])[0]
        for h in range(hq):
            out[i, h], lse[i, h] = attend(q[i, h], k[j, h // g], v[j, h // g], scale, cap,
                                          0.0 if slopes is None else slopes[h], i - j)
    return out, lse


def dense_by_head(q, k, v, seg_offsets, prompt_seg_ptr, mask, scale=None, cap=0.0, slopes=None):
    """The same, a head's whole score matrix at a time (finite inputs)."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    n, hq, d = q.shape
    g = hq // k.shape[1]
    scale = d ** -0.5 if scale is None else scale
    sees = dense_visible(seg_offsets, prompt_seg_ptr, mask)
    far = np.abs(np.arange(n)[:, None] - np.arange(n)[None])
    out, lse = np.zeros((n, hq, d)), np.zeros((n, hq))
    for h in range(hq):
        s = q[:, h] @ k[:, h // g].T * scale
        if cap:
            s = cap * np.tanh(s / cap)
        if slopes is not None:
            s = s - float(slopes[h]) * far
        s = np.where(sees, s, -np.inf)
        m = s.max(1, keepdims=True)
        w = np.exp(s - m)
        out[:, h] = w @ v[:, h // g] / w.sum(1, keepdims=True)
        lse[:, h] = m[:, 0] + np.log(w.sum(1))
    return out, lse


class Pages:
    """A page cache on the host: pools [pool rows, Hkv, D], page_table [B][pages],
    lens [B] slots, page_lens [B][pages] or None, key_pos [B][Hkv][slots] or None."""

    def __init__(self, k, v, page_table, lens, page, page_lens=None, key_pos=None):
        self.k, self.v, self.table, self.lens, self.page = k, v, page_table, lens, page
        self.page_lens, self.key_pos = page_lens, key_pos

    def slots(self, b):
        """Slots of sequence b that hold a key."""
        return np.array([i for i in range(int(self.lens[b]))
                         if self.page_lens is None
                         or i % self.page < self.page_lens[b][i // self.page]], np.int64)

    def rows(self, b, slots):
        return np.asarray(self.table[b], np.int64)[slots // self.page] * self.page \
            + slots % self.page

    def pos(self, b, h, slots):
        return slots if self.key_pos is None else np.asarray(self.key_pos[b, h], np.int64)[slots]


def chain(n):
    return np.tril(np.ones((n, n), bool))


def cache_attention(q, k_new, v_new, pages, row_ptr, sees=None, row_pos=None, scale=None, cap=0.0,
                    slopes=None):
    """(out, lse): sees[b] [n, n] booleans of the sequence's new tokens (None: each
    sees those up to itself)."""
    rows, hq, d = q.shape
    hkv = k_new.shape[1]
    g = hq // hkv
    scale = d ** -0.5 if scale is None else scale
    out, lse = np.zeros((rows, hq, d)), np.full((rows, hq), -np.inf)
    for b in range(len(row_ptr) - 1):
        a, n = int(row_ptr[b]), int(row_ptr[b + 1] - row_ptr[b])
        seen = chain(n) if sees is None else sees[b]
        slots = pages.slots(b)
        at = pages.rows(b, slots)
        rp = np.arange(n) + int(pages.lens[b]) if row_pos is None else row_pos[a:a + n]
        for i in range(n):
            new = a + np.nonzero(seen[i])[0]
            for h in range(hq):
                kv = h // g
                k = np.concatenate([pages.k[at, kv], k_new[new, kv]])
                v = np.concatenate([pages.v[at, kv], v_new[new, kv]])
                pos = np.concatenate([pages.pos(b, kv, slots), rp[new - a]])
                out[a + i, h], lse[a + i, h] = attend(
                    q[a + i, h], k, v, scale, cap, 0.0 if slopes is None else slopes[h],
                    rp[i] - pos)
    return out, lse


def accumulate(q, lse, pages, weights, decay, row_ptr, row_pos=None, row_weight=None, scale=None,
               cap=0.0, slopes=None):
    """New weights [B, Hkv, slots]: decay * weights + sum of e^(s - lse) over the
    sequence's rows and the kv head's query heads; 0 in the slots before the
    sequence's length that hold no key; unchanged past it (NaN here)."""
    rows, hq, d = q.shape
    hkv = pages.k.shape[1]
    g = hq // hkv
    scale = d ** -0.5 if scale is None else scale
    out = np.full(weights.shape, np.nan)
    for b in range(len(row_ptr) - 1):
        a, z = int(row_ptr[b]), int(row_ptr[b + 1])
        slots = pages.slots(b)
        at = pages.rows(b, slots)
        rp = np.arange(z - a) + int(pages.lens[b]) if row_pos is None else row_pos[a:z]
        for kv in range(hkv):
            w = decay * weights[b, kv, slots].astype(np.float64) if decay else np.zeros(len(slots))
            for r in range(a, z):
                f = 1.0 if row_weight is None else float(row_weight[r])
                if f == 0.0:
                    continue
                for h in range(kv * g, kv * g + g):
                    if lse[r, h] == -np.inf:
                        continue
                    s = scores(q[r, h], pages.k[at, kv], scale, cap,
                               0.0 if slopes is None else slopes[h],
                               rp[r - a] - pages.pos(b, kv, slots))
                    w = w + f * np.exp(s - lse[r, h])
            out[b, kv, :int(pages.lens[b])] = 0.0
            out[b, kv, slots] = w
    return out


def evict(pages, weights, budget, sinks=0, recent=0, next_pos=None):
    """(k, v, weights, pos, lens) after the eviction: copies of the pools with the
    kept keys in their sequence's first slots; weights 0 and positions -1 past
    them.  A NaN weight counts as less than every other."""
    k, v = pages.k.copy(), pages.v.copy()
    B, hkv, S = weights.shape
    w_out, p_out = np.zeros(weights.shape, weights.dtype), np.full(weights.shape, -1, np.int32)
    lens = np.zeros(B, np.int32)
    for b in range(B):
        slots = pages.slots(b)
        n = lens[b] = min(len(slots), budget)
        nxt = int(pages.lens[b] if next_pos is None else next_pos[b])
        for h in range(hkv):
            pos = pages.pos(b, h, slots)
            safe = (pos < sinks) | (pos >= nxt - recent)
            w = weights[b, h, slots]
            rank = sorted(range(len(slots)),
                          key=lambda i: (not safe[i], np.isnan(w[i]) and not safe[i],
                                         0.0 if safe[i] or np.isnan(w[i]) else -float(w[i]), i))
            kept = sorted(int(slots[i]) for i in rank[:n])
            source = {i: i for i in kept if i < n}
            for to, frm in zip([i for i in range(n) if i not in source],
                               [i for i in kept if i >= n]):
                source[to] = frm
            if not n:
                continue
            to = np.arange(n)
            frm = np.array([source[i] for i in range(n)])
            k[pages.rows(b, to), h] = pages.k[pages.rows(b, frm), h]
            v[pages.rows(b, to), h] = pages.v[pages.rows(b, frm), h]
            w_out[b, h, :n] = weights[b, h, frm]
            p_out[b, h, :n] = pages.pos(b, h, frm)
    return k, v, w_out, p_out, lens
