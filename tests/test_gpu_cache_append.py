"""GPU: sift_cache_append (Cache.append) against a plain computation in 64 bits.

Rows of the pools' own type: V is copied, K rounded once (bounds as of the rotation's own
tests).  e4m3: the scale is exact; a value x of a new row is off by the rounding, half a
step: |x| 2^-4 or, below the smallest normal code, scale 2^-10; a turned one also by the
cosine's and sine's errors, (|x| + |y|) m 2^-16, which may move it to the next code: a
whole step.  A held row whose scale grew is off by half a step of the smallest codes.
Everything that no new row enters keeps its bits.
"""

import math

import numpy as np
import pytest
import torch

from gpu_helpers import device, say

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}


class Case:
    """Sequences with keys held, and new ones; pools filled with codes or NaN."""

    def __init__(self, lens, new, hkv, d, page, pool, rot=0, interleaved=False, magnitude=1.0,
                 seed=0, extra=1, spread=0.0):
        rng = np.random.default_rng(seed)
        self.lens, self.new, self.hkv, self.d, self.page = lens, new, hkv, d, page
        self.rot, self.interleaved, self.magnitude = rot, interleaved, magnitude
        self.pool = pool
        B = len(lens)
        self.pages = max(1, max(-(-(a + n) // page) for a, n in zip(lens, new)) - 1 + extra)
        self.slots = self.pages * page
        num = B * self.pages + 2
        self.table = rng.permutation(num)[:B * self.pages].reshape(B, self.pages).astype(np.int32)
        self.row_ptr = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        rows = int(self.row_ptr[-1])
        self.rows = rows
        self.row_pos = rng.integers(0, 100000, rows).astype(np.int32)
        dev = device()
        up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(dev)  # noqa: E731
        dt = torch.float32 if pool == "f32" else torch.bfloat16
        size = np.exp(spread * rng.standard_normal((rows, hkv, 1)))
        self.k = up((rng.standard_normal((rows, hkv, d)) * size).astype(np.float32)).to(dt)
        self.v = up((rng.standard_normal((rows, hkv, d)) * size).astype(np.float32)).to(dt)
        self.k_scales = self.v_scales = None
        shape = (num * page, hkv, d)
        if pool == "e4m3":
            make = lambda: up(rng.uniform(-300, 300, shape).astype(np.float32)).to(DTYPES[pool])  # noqa: E731
            self.k_pages, self.v_pages = make(), make()
            sc = lambda: up(np.exp2(rng.integers(-12, -5, (num, hkv))).astype(np.float32))  # noqa: E731
            self.k_scales, self.v_scales = sc(), sc()
        else:
            self.k_pages, self.v_pages = (torch.full(shape, math.nan, dtype=dt, device=dev)
                                          for _ in range(2))
        self.key_pos = torch.full((B, hkv, self.slots), -7, dtype=torch.int32, device=dev)
        i = np.arange(rot // 2)
        self.inv_freq = (10000.0 ** (-2.0 * i / max(rot, 1))).astype(np.float32)
        self.t = {n: up(getattr(self, n)) for n in ("table", "row_ptr", "row_pos")}
        self.t["lens"] = up(np.asarray(lens, np.int32))

    def rotary(self):
        from paper_2606_09441_amd import Rotary
        return Rotary(self.inv_freq, self.interleaved, self.magnitude) if self.rot else None

    def cache(self):
        from paper_2606_09441_amd import Cache
        return Cache(len(self.lens), 2 * self.hkv, self.hkv, self.d, page=self.page,
                     max_pages=self.pages)

    def kv(self, key_pos=True):
        from paper_2606_09441_amd import CachePages
        return CachePages(self.k_pages, self.v_pages, self.t["table"], self.t["lens"],
                          key_pos=self.key_pos if key_pos else None, k_scales=self.k_scales,
                          v_scales=self.v_scales)

    def snapshot(self):
        raw = lambda x: x.view(torch.uint8).cpu().clone() if self.pool == "e4m3" else x.cpu().clone()  # noqa: E731
        s = {"k": raw(self.k_pages), "v": raw(self.v_pages), "pos": self.key_pos.cpu().clone()}
        if self.pool == "e4m3":
            s |= {"ks": self.k_scales.cpu().clone(), "vs": self.v_scales.cpu().clone()}
        return s

    def turned(self):
        """The new keys in 64 bits, and |x| + |y| of each dim's pair (0: it stays)."""
        x = self.k.double().cpu().numpy()
        out, size = x.copy(), np.zeros_like(x)
        if self.rot:
            half = self.rot // 2
            a = self.row_pos[:, None].astype(np.float64) * self.inv_freq.astype(np.float64)
            c, s = np.cos(a)[:, None], np.sin(a)[:, None]
            re, im = (slice(0, self.rot, 2), slice(1, self.rot, 2)) if self.interleaved else (
                slice(0, half), slice(half, self.rot))
            u, w, m = x[..., re], x[..., im], self.magnitude
            out[..., re], out[..., im] = m * (u * c - w * s), m * (w * c + u * s)
            size[..., re] = size[..., im] = m * (np.abs(u) + np.abs(w))
        return out, size

    def places(self, slots=None):
        """(row, sequence, slot, pool row) of every new row that has room."""
        for b, (a, n) in enumerate(zip(self.lens, self.new)):
            for i in range(n):
                r = int(self.row_ptr[b]) + i
                slot = a + i if slots is None else int(slots[r])
                if 0 <= slot < self.slots:
                    yield r, b, slot, int(self.table[b, slot // self.page]) * self.page + slot % self.page

    def verify(self, before, lens_out=None, slots=None, tag=""):
        torch.cuda.synchronize()
        after = self.snapshot()
        places = list(self.places(slots))
        if lens_out is not None:
            assert lens_out.tolist() == [min(a + n, self.slots) for a, n in zip(self.lens, self.new)]
        pos = before["pos"].clone()
        for r, b, slot, _ in places:
            pos[b, :, slot] = int(self.row_pos[r])
        assert torch.equal(pos, after["pos"])
        k, pair = self.turned()
        v = self.v.double().cpu().numpy()
        at = [p[3] for p in places]
        src = [p[0] for p in places]
        others = np.ones(before["k"].shape[0], bool)
        others[at] = False
        if self.pool != "e4m3":
            for name, ref in (("k", k), ("v", v)):
                was, now = before[name], after[name]
                assert torch.equal(was[others].isnan(), now[others].isnan())
                got = now[at].double().numpy()
                if name == "v" or not self.rot:
                    assert np.array_equal(got, ref[src])
                    continue
                step, angle = (2.0 ** -24, 2.0 ** -22) if self.pool == "f32" else (2.0 ** -8, 2.0 ** -16)
                bound = np.abs(ref[src]) * step + pair[src] * angle + 1e-40
                worst = float((np.abs(got - ref[src]) / bound).max()) if src else 0.0
                say(f"[append] {tag} {name}: {worst:.3f} of the bound")
                assert worst <= 1
            return
        # which pages new rows enter, and their first row in them
        first = {}
        for r, b, slot, p in places:
            q = p // self.page
            first[q] = min(first.get(q, self.page), p % self.page)
        for name, ref, off in (("k", k, pair), ("v", v, np.zeros_like(v))):
            raw = self.k if name == "k" else self.v
            raw = np.abs(raw.double().cpu().numpy())
            if name == "k" and self.rot:
                raw[..., :self.rot] *= float(np.float32(1.4142137)) * self.magnitude
            raw = np.where(np.isfinite(raw), raw, 0.0)
            was = before[name].view(DTYPES["e4m3"]).double().numpy()
            now = after[name].view(DTYPES["e4m3"]).double().numpy()
            ws, ns = (x[name + "s"].double().numpy() for x in (before, after))
            need = np.full(ws.shape, 2.0 ** -100)
            for r, b, slot, p in places:
                top = raw[r].max(-1)
                with np.errstate(divide="ignore"):
                    e = np.where(top > 0, np.exp2(np.ceil(np.log2(top / 448))), 0)
                need[p // self.page] = np.maximum(need[p // self.page], e)
            for q in range(ws.shape[0]):
                rows = slice(q * self.page, (q + 1) * self.page)
                if q not in first:
                    assert np.array_equal(ws[q], ns[q])
                    assert np.array_equal(before[name][rows], after[name][rows])
                    continue
                want = np.maximum(need[q], ws[q]) if first[q] > 0 else need[q]
                assert np.array_equal(ns[q], want), (tag, name, q)
                held = slice(q * self.page, q * self.page + first[q])
                x = was[held] * ws[q][:, None]
                err = np.abs(now[held] * ns[q][:, None] - x)
                grew = (ns[q] > ws[q])[:, None]
                assert (err <= np.where(grew, ns[q][:, None] * 2.0 ** -10, 0)).all()
                # rows behind the last new one
                end = max(p[3] % self.page for p in places if p[3] // self.page == q) + 1
                rest = slice(q * self.page + end, (q + 1) * self.page)
                assert np.array_equal(before[name][rest], after[name][rest])
            if src:
                sc = ns[np.asarray(at) // self.page][..., None]
                got, x = now[at] * sc, ref[src]
                bad = ~np.isfinite(x)
                assert np.array_equal(np.isnan(got), bad)
                half = np.maximum(np.abs(x) * 2.0 ** -4, sc * 2.0 ** -10)
                bound = np.where(off[src] > 0, 2 * half + off[src] * 2.0 ** -16, half)
                worst = float((np.abs(got - x) / bound)[~bad].max())
                say(f"[append] {tag} {name}: {worst:.3f} of the bound")
                assert worst <= 1
                # few are at a border where the cosine's error counts
                assert ((np.abs(got - x) > half * (1 + 2.0 ** -8))[~bad]).mean() < 0.01


SHAPES = [
    # lens, new, hkv, d, page
    ([0], [1], 1, 64, 16),
    ([5], [1], 8, 128, 64),
    ([0, 63, 64, 65], [1, 1, 1, 1], 2, 128, 64),
    ([0, 15, 16, 31], [40, 0, 1, 17], 3, 64, 16),
    ([100, 0, 7], [129, 300, 0], 8, 128, 128),
    ([1, 2, 3, 4, 5] * 15, [2, 0, 1, 3, 33] * 15, 2, 64, 32),   # more than 64 sequences
    ([130], [500], 1, 128, 32),
]


@pytest.mark.parametrize("pool", ["bf16", "f32", "e4m3"])
@pytest.mark.parametrize("rot", [(0, False), ("all", False), ("all", True), (32, False), (48, True),
                                 (20, False), (22, True)])
@pytest.mark.parametrize("shape", SHAPES)
def test_append(shape, rot, pool):
    lens, new, hkv, d, page = shape
    n, interleaved = rot
    c = Case(lens, new, hkv, d, page, pool, d if n == "all" else n, interleaved, seed=len(lens))
    before = c.snapshot()
    with c.cache() as cache:
        out = cache.append(c.kv(), c.k, c.v, row_ptr=c.t["row_ptr"], row_pos=c.t["row_pos"],
                           rotary=c.rotary())
        c.verify(before, out, tag=f"{pool} {rot}")
    assert c.t["lens"].tolist() == lens


@pytest.mark.parametrize("pool", ["bf16", "f32", "e4m3"])
def test_defaults_and_lens_in_place(pool):
    """As many rows of each, positions the slots, no table of positions; the lens written
    where they are read."""
    c = Case([3, 70, 0], [5, 5, 5], 2, 128, 64, pool, 64)
    c.row_pos = np.concatenate([np.arange(a, a + 5) for a in c.lens]).astype(np.int32)
    before = c.snapshot()
    with c.cache() as cache:
        out = cache.append(c.kv(key_pos=False), c.k, c.v, rotary=c.rotary(), lens_out=c.t["lens"])
        assert out is c.t["lens"]
        got = c.key_pos.clone()
        assert bool((got == -7).all())
        for _, b, slot, _ in c.places():
            before["pos"][b, :, slot] = -7
        after_pos = c.snapshot()["pos"]
        assert torch.equal(after_pos, before["pos"])
        for r, b, slot, _ in c.places():   # what verify expects of a call with the table
            c.key_pos[b, :, slot] = int(c.row_pos[r])
        c.verify(before, out, tag=pool)


@pytest.mark.parametrize("pool", ["bf16", "f32"])
def test_slots(pool):
    """Rows go where they are told; slots outside the cache take none."""
    c = Case([10, 20], [30, 9], 2, 64, 16, pool, 64, extra=3)
    rng = np.random.default_rng(1)
    slots = np.concatenate([rng.permutation(c.slots)[:30], rng.permutation(c.slots)[:9]]).astype(np.int32)
    slots[3], slots[35] = -1, c.slots
    before = c.snapshot()
    with c.cache() as cache:
        out = cache.append(c.kv(), c.k, c.v, row_ptr=c.t["row_ptr"], row_pos=c.t["row_pos"],
                           rotary=c.rotary(), slots=torch.from_numpy(slots).to(device()))
        assert out is None
        c.verify(before, slots=slots, tag=pool)


@pytest.mark.parametrize("pool", ["bf16", "f32", "e4m3"])
def test_rows_past_the_last_slot_are_left_out(pool):
    c = Case([120, 128, 0], [30, 4, 128], 2, 64, 32, pool, 32, extra=0)
    assert c.slots == 128 and c.lens[0] + c.new[0] > c.slots
    before = c.snapshot()
    with c.cache() as cache:
        out = cache.append(c.kv(), c.k, c.v, row_ptr=c.t["row_ptr"], row_pos=c.t["row_pos"],
                           rotary=c.rotary())
        c.verify(before, out, tag=pool)
        assert out.tolist() == [128, 128, 128]


@pytest.mark.parametrize("pool", ["bf16", "f32", "e4m3"])
def test_bad_tables_stay_inside(pool):
    """Pages, lengths and row pointers out of range: nothing outside the pools changes."""
    c = Case([5, 40, 9], [20, 20, 20], 2, 64, 16, pool, 64)
    dev = device()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
    pad = 64
    whole, views = [], []
    for t in (c.k_pages, c.v_pages):
        raw = t.view(torch.uint8).flatten()
        n = raw.numel()
        w = torch.full((n + 2 * pad * 16,), 0x5a, dtype=torch.uint8, device=dev)
        w[pad * 16:pad * 16 + n] = raw
        whole.append(w)
        views.append(w[pad * 16:pad * 16 + n].view(t.dtype).view(t.shape))
    c.k_pages, c.v_pages = views
    with c.cache() as cache:
        for lens, ptr in ((i32(-5, 1 << 30, 7), i32(0, 20, 40, 60)),
                          (i32(5, 40, 9), i32(-9, 1 << 30, -(1 << 31), 50)),
                          (i32(5, 40, 9), i32(60, 0, 60, 0)),
                          (i32(5, 40, 9), i32(0, 60, 0, 60))):
            c.t["lens"] = lens
            c.t["table"] = torch.randint(-(1 << 31), (1 << 31) - 1, c.table.shape, device=dev,
                                         dtype=torch.int64).int()
            out = cache.append(c.kv(), c.k, c.v, row_ptr=ptr, row_pos=c.t["row_pos"],
                               rotary=c.rotary())
            torch.cuda.synchronize()
            assert bool(((out >= 0) & (out <= c.slots)).all())
            for w in whole:
                assert bool((w[:pad * 16] == 0x5a).all()) and bool((w[-pad * 16:] == 0x5a).all())


@pytest.mark.parametrize("pool", ["bf16", "f32", "e4m3"])
def test_rows_of_no_page_are_left_out(pool):
    """A table's values out of range lead to nobody's page: neither the first nor the last
    of the pool, and no position, changes."""
    c = Case([5, 40, 9, 3], [20, 20, 20, 40], 2, 64, 16, pool, 64)
    num = c.k_pages.shape[0] // c.page
    c.table[0, 1], c.table[1], c.table[3, 0] = num, -1, -(1 << 31)
    c.t["table"] = torch.from_numpy(c.table).to(device())
    some = c.places
    c.places = lambda slots=None: (p for p in some(slots) if 0 <= p[3] < num * c.page)
    before = c.snapshot()
    with c.cache() as cache:
        out = cache.append(c.kv(), c.k, c.v, row_ptr=c.t["row_ptr"], row_pos=c.t["row_pos"],
                           pos_out=c.key_pos, rotary=c.rotary())
        c.verify(before, out, tag=pool)


def test_scales_of_unlike_and_odd_values():
    """Rows of sizes far apart, a page of zeros, of the smallest numbers, infinities and
    NaN: held as NaN, without a part in the scale."""
    c = Case([40, 0, 0, 3], [30, 64, 10, 2], 2, 128, 64, "e4m3", 128, spread=6.0, seed=4)
    rng = np.random.default_rng(0)
    lo, hi = int(c.row_ptr[2]), int(c.row_ptr[3])
    c.k[lo:hi] = 0
    c.v[lo:hi] = 1e-38
    c.k[2, 0, 5], c.k[9, 1, 70], c.v[4, 1, 3] = math.inf, math.nan, -math.inf
    c.k[12] = 3.38e38 * torch.from_numpy(rng.choice([-1, 1], (2, 128))).to(c.k)
    # a turned pair with one value that is not finite has two of them
    before = c.snapshot()
    with c.cache() as cache:
        out = cache.append(c.kv(), c.k, c.v, row_ptr=c.t["row_ptr"], row_pos=c.t["row_pos"],
                           rotary=c.rotary())
        torch.cuda.synchronize()
        k = c.k_pages.float()
        rows = {p[0]: p[3] for p in c.places()}
        for r, h, dims in ((2, 0, (5, 69)), (9, 1, (6, 70))):
            bad = k[rows[r], h].isnan().nonzero().flatten().tolist()
            assert bad == list(dims)
        assert c.v_pages.float()[rows[4], 1].isnan().nonzero().flatten().tolist() == [3]
        # a page of zeros, at the smallest scale
        assert not k[rows[lo]].any()
        page = rows[lo] // c.page
        assert (c.k_scales[page] == 2.0 ** -100).all() and (c.v_scales[page] == 2.0 ** -100).all()
        assert out.tolist() == [70, 64, 10, 5]
        # 3.38e38 sqrt(2) does not fit a float: the largest scale that one asks for
        assert (c.k_scales[rows[12] // c.page] == 2.0 ** 120).all()
        del before


def test_one_at_a_time_is_as_all_at_once_where_the_scale_never_grows():
    """A token a call, with the lens in place, in a captured graph that is replayed:
    the same as one call of all, for pages whose first row is the largest."""
    dev = device()
    c = Case([0, 0], [50, 50], 2, 128, 16, "e4m3", 128, seed=7)
    c.k[0::1] = c.k.clamp(-1, 1)
    c.v[0::1] = c.v.clamp(-1, 1)
    for b in range(2):
        for i in range(0, 50, 16):
            c.k[b * 50 + i] = 1.0
            c.v[b * 50 + i] = 1.0
    one = Case([0, 0], [50, 50], 2, 128, 16, "e4m3", 128, seed=7)
    rot = c.rotary()
    with c.cache() as cache:
        cache.append(c.kv(), c.k, c.v, row_ptr=c.t["row_ptr"], row_pos=c.t["row_pos"], rotary=rot)
        k, v = torch.empty_like(c.k[:2]), torch.empty_like(c.v[:2])
        pos = torch.empty(2, dtype=torch.int32, device=dev)
        kv = one.kv()
        graph = torch.cuda.CUDAGraph()
        warm = torch.zeros(1, device=dev)
        with torch.cuda.graph(graph):
            cache.append(kv, k, v, row_pos=pos, rotary=rot, lens_out=one.t["lens"])
        for i in range(50):
            for x, y in ((k, c.k), (v, c.v), (pos, c.t["row_pos"])):
                x.copy_(y[[i, 50 + i]])
            graph.replay()
            warm += 1
            torch.cuda.synchronize()
            assert one.t["lens"].tolist() == [i + 1, i + 1]
    assert torch.equal(c.key_pos, one.key_pos)
    rows = [p[3] for p in c.places()]
    for a, b in ((c.k_pages, one.k_pages), (c.v_pages, one.v_pages)):
        assert torch.equal(a.view(torch.uint8)[rows], b.view(torch.uint8)[rows])
    pages = sorted({r // 16 for r in rows})
    assert torch.equal(c.k_scales[pages], one.k_scales[pages])


def test_growing_scales_keep_what_is_held():
    """Rows that grow eightfold: the page's scale follows, and what it held stays to half a
    step of its smallest codes."""
    c = Case([0], [16], 1, 64, 16, "e4m3", 0)
    for i in range(16):
        c.k[i] = c.k[i].clamp(-2, 2) * 8.0 ** (i % 5)
    with c.cache() as cache:
        for i in range(16):
            c.t["lens"].fill_(i)
            cache.append(c.kv(), c.k[i:i + 1], c.v[i:i + 1])
    torch.cuda.synchronize()
    at = int(c.table[0, 0])
    got = c.k_pages[at * 16:at * 16 + 16].double().cpu() * c.k_scales[at].double().cpu()[:, None]
    x = c.k.double().cpu()
    s = float(c.k_scales[at, 0])
    # each of the few growths rounds the smallest again
    assert ((got - x).abs() <= torch.maximum(x.abs() * 2.0 ** -4, torch.tensor(4 * s * 2.0 ** -10))).all()


def test_pages_under_scales_that_are_no_powers():
    """Pages that another program filled: their scale becomes the next power of two, and
    what they hold is rounded again, by half a step."""
    c = Case([5, 20], [3, 2], 2, 64, 16, "e4m3", 32)
    for t in (c.k_scales, c.v_scales):
        t.mul_(1.37)
    before = c.snapshot()
    with c.cache() as cache:
        cache.append(c.kv(), c.k, c.v, row_ptr=c.t["row_ptr"], row_pos=c.t["row_pos"],
                     rotary=c.rotary())
    torch.cuda.synchronize()
    after = c.snapshot()
    for b, n in ((0, 5), (1, 4)):
        page = int(c.table[b, c.lens[b] // 16])
        for name in "kv":
            was, now = (x[name].view(DTYPES["e4m3"]).double()[page * 16:page * 16 + n] *
                        x[name + "s"].double()[page][:, None] for x in (before, after))
            s = after[name + "s"].double()[page]
            assert torch.equal(s.log2(), s.log2().round()) and (s >= before[name + "s"][page]).all()
            half = torch.maximum(was.abs() * 2.0 ** -4, s[:, None] * 2.0 ** -10)
            assert ((now - was).abs() <= half).all()


def test_another_stream():
    c = Case([5, 6], [70, 3], 2, 128, 64, "e4m3", 128)
    before = c.snapshot()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with c.cache() as cache:
        out = cache.append(c.kv(), c.k, c.v, row_ptr=c.t["row_ptr"], row_pos=c.t["row_pos"],
                           rotary=c.rotary(), stream=side)
        side.synchronize()
        c.verify(before, out)


def test_no_rows():
    c = Case([5, 6], [0, 0], 2, 128, 64, "bf16")
    before = c.snapshot()
    with c.cache() as cache:
        assert cache.append(c.kv(), c.k, c.v, row_ptr=c.t["row_ptr"]).tolist() == [5, 6]
        c.verify(before)


def test_offsets_past_32_bits():
    """Pools of more than 2^32 bytes, the sequence's page at their end."""
    from paper_2606_09441_amd import Cache, CachePages, Rotary
    dev = device()
    hkv, d, page = 8, 128, 128
    pages = (1 << 32) // (page * hkv * d) + 3
    for pool in ("e4m3", "bf16"):
        num = pages if pool == "e4m3" else pages // 2 + 2
        kp, vp = (torch.zeros(num * page, hkv, d, dtype=DTYPES[pool], device=dev) for _ in range(2))
        sc = [torch.ones(num, hkv, device=dev) for _ in range(2)] if pool == "e4m3" else [None] * 2
        table = torch.tensor([[num - 1, 0]], dtype=torch.int32, device=dev)
        lens = torch.tensor([7], dtype=torch.int32, device=dev)
        k, v = (torch.randn(5, hkv, d, device=dev).bfloat16() for _ in range(2))
        f = torch.ones(64, device=dev)
        with Cache(1, hkv, hkv, d, page=page, max_pages=2) as cache:
            cache.append(CachePages(kp, vp, table, lens, k_scales=sc[0], v_scales=sc[1]), k, v,
                         rotary=Rotary(f))
            torch.cuda.synchronize()
        got = vp[(num - 1) * page + 7:(num - 1) * page + 12].float()
        if pool == "e4m3":
            assert (got - v.float()).abs().max() <= 0.25   # half a step of a number under 4
        else:
            assert torch.equal(got, v.float())
        assert not vp[:(num - 1) * page].view(torch.uint8).any()
        del kp, vp
        torch.cuda.empty_cache()
