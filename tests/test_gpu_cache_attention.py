"""GPU tests of the attention over a paged cache (sift_cache_attention) against
the fp64 oracle, element by element.  Pool rows that hold no key are NaN."""

from __future__ import annotations

import numpy as np
import pytest

from cache_helpers import Batch, random_tree, some_empty
from gpu_helpers import max_abs, say

pytestmark = pytest.mark.gpu

# as in test_gpu_dense.py: the project's bars on N(0, 1) inputs; the log sum's
# error is that of the scores
TOL = {"f32": 1e-5, "bf16": 2e-2}
LSE_TOL = 1e-4


def check(x, cap=0.0, bias=False, scale=None, row_ptr=True, name=""):
    import torch
    slopes = (2.0 ** (-4.0 * np.arange(1, x.hq + 1) / x.hq)).astype(np.float32) if bias else None
    lse = torch.full((x.rows, x.hq), 7.0, device=x.q.device)
    out = torch.full_like(x.q, 7.0)
    with x.cache() as cache:
        cache.attention(x.q, x.k_new, x.v_new, x.pages(), row_ptr=x.t["row_ptr"] if row_ptr else None,
                        tree_mask=x.mask, row_pos=x.t["row_pos"], scale=scale, cap=cap,
                        slopes=None if slopes is None else torch.from_numpy(slopes).to(x.q.device),
                        out=out, lse=lse)
        torch.cuda.synchronize()
    ref, ref_lse = x.oracle(scale=scale, cap=cap, slopes=slopes)
    out, lse = out.float().cpu().numpy(), lse.cpu().numpy()
    none = np.isneginf(ref_lse)
    assert np.array_equal(none, np.isneginf(lse))
    assert not out[none].any()
    dt = "bf16" if x.q.dtype == torch.bfloat16 else "f32"
    e, el = max_abs(out, ref), max_abs(lse[~none], ref_lse[~none])
    say(f"{name} {dt}: {e:.2e}, lse {el:.2e}")
    assert e <= TOL[dt] and el <= LSE_TOL
    return out, lse


TYPES = [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)]
LENS = [0, 1, 15, 16, 17, 31, 33, 64, 127, 129, 300, 700]


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_single_tokens(dtype, d, page):
    check(Batch(LENS, [1] * len(LENS), 8, 2, d, dtype, page), row_ptr=False)
    check(Batch(LENS, [1] * len(LENS), 8, 2, d, dtype, page, gaps=True), cap=20.0)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("tree", [None, random_tree, some_empty])
def test_trees(dtype, d, tree):
    new = [5, 0, 1, 33, 3, 2, 64, 12, 0, 1, 20, 40]
    for gaps, moved, cap, bias in [(False, False, 0.0, False), (True, True, 0.0, True),
                                   (True, False, 30.0, False), (False, True, 20.0, True),
                                   (False, False, 0.0, True)]:
        check(Batch(LENS, new, 6, 2, d, dtype, 32, gaps, moved, tree, seed=3), cap, bias,
              name=f"gaps {gaps} moved {moved} cap {cap} bias {bias}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_new_tokens(dtype):
    """More than a mask word of them, and a chain longer than the cache."""
    check(Batch([40, 0, 513], [130, 65, 200], 4, 1, 128, dtype, tree=random_tree, seed=4))
    check(Batch([40, 0], [150, 90], 4, 4, 64, dtype, seed=5))


@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 8), (5, 1), (12, 3), (64, 1), (40, 1), (20, 1)])
def test_head_layouts(hq, hkv):
    check(Batch([200, 0, 77], [3, 1, 2], hq, hkv, 64, "bf16", seed=6))
    check(Batch([200, 0, 77], [3, 1, 2], hq, hkv, 128, "f32", seed=6), bias=True)


def test_many_sequences():
    """More sequences than a wavefront has lanes, many of them without work."""
    rng = np.random.default_rng(7)
    lens = rng.integers(0, 90, 150).tolist()
    new = [int(rng.integers(0, 3)) for _ in lens]
    check(Batch(lens, new, 4, 2, 64, "bf16", 16, seed=7))
    new = [int(rng.integers(0, 12)) for _ in lens]
    check(Batch(lens, new, 16, 2, 64, "bf16", 16, tree=random_tree, seed=7))   # wide units


def test_long_cache():
    """Every workgroup shares units with others."""
    for dtype in ("bf16", "f32"):
        check(Batch([20000, 7], [1, 1], 4, 1, 128, dtype, 128, seed=8))
        check(Batch([9000], [21], 8, 2, 64, dtype, 16, tree=random_tree, gaps=True, seed=9), cap=50.0)


def test_shared_pages():
    """Two sequences read the same pages."""
    x = Batch([100, 100], [2, 2], 4, 2, 128, "bf16", 64, seed=10)
    x.table[1] = x.table[0]
    x.t["table"][1] = x.t["table"][0]
    check(x)


def test_rows_left_out():
    """Rows that row_ptr does not name stay as they are."""
    import torch
    x = Batch([50, 60], [4, 4], 4, 2, 64, "bf16", seed=11)
    out = torch.full_like(x.q, 7.0)
    with x.cache() as cache:
        whole = cache.attention(x.q, x.k_new, x.v_new, x.pages(), row_ptr=x.t["row_ptr"])
        ptr = torch.tensor([0, 4, 6], dtype=torch.int32, device=x.q.device)
        cache.attention(x.q, x.k_new, x.v_new, x.pages(), row_ptr=ptr, out=out)
    assert torch.equal(out[:6], whole[:6]) and bool((out[6:] == 7).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("hq", [2, 4])
def test_unseen_new_tokens_do_not_matter(dtype, value, hq):
    """A drafted token with such values reaches the rows that see it and no other."""
    x = Batch([70, 0], [9, 40], hq, 2, 128, dtype, tree=random_tree, seed=12)
    for bad, b in ((3, 0), (9 + 20, 1)):
        x.v_new[bad, 1, 5:9] = value
    import torch
    with x.cache() as cache:
        out = cache.attention(x.q, x.k_new, x.v_new, x.pages(), row_ptr=x.t["row_ptr"],
                              tree_mask=x.mask).float().cpu().numpy()
        x.k_new[3], x.k_new[29] = value, value
        worse = cache.attention(x.q, x.k_new, x.v_new, x.pages(), row_ptr=x.t["row_ptr"],
                                tree_mask=x.mask).float().cpu().numpy()
    torch.cuda.synchronize()
    x.k_new[3], x.k_new[29] = 0, 0
    sees = np.concatenate([x.sees[0][:, 3], x.sees[1][:, 20]])
    with np.errstate(all="ignore"):
        ref, _ = x.oracle()
    assert max_abs(worse[~sees], ref[~sees]) <= TOL[dtype]
    ref_k = Batch([70, 0], [9, 40], hq, 2, 128, dtype, tree=random_tree, seed=12)
    ref_k.v_new.copy_(x.v_new)
    with np.errstate(all="ignore"):
        ref, _ = ref_k.oracle()
    fine = np.isfinite(ref)
    assert np.array_equal(fine, np.isfinite(out))
    assert max_abs(out[fine], ref[fine]) <= TOL[dtype]
    assert np.array_equal(np.isnan(out), np.isnan(ref))


def test_streams_and_repeats():
    """The same bits on another stream and in a captured graph; a replay follows the
    tables' present contents."""
    import torch
    x = Batch([300, 41], [7, 7], 8, 2, 128, "bf16", tree=random_tree, seed=13)
    args = (x.q, x.k_new, x.v_new, x.pages())
    with x.cache() as cache:
        kw = dict(row_ptr=x.t["row_ptr"], tree_mask=x.mask)
        first = cache.attention(*args, **kw)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        out = torch.zeros_like(first)
        with torch.cuda.stream(side):
            cache.attention(*args, out=out, **kw)
        side.synchronize()
        assert torch.equal(out, first)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cache.attention(*args, out=out, **kw)
        for n in (300, 200, 0, 300):
            x.t["lens"][0] = n
            out.zero_()
            graph.replay()
            got = out.clone()
            assert torch.equal(got, cache.attention(*args, **kw))
        assert torch.equal(got, first)


def test_offsets_beyond_32_bits():
    """Pages at the far end of pools of more than 2^31 elements, through all three
    calls: the same bits as from a small pool."""
    import torch
    from paper_2606_09441_amd import CachePages
    x = Batch([300, 41], [3, 3], 16, 8, 128, "bf16", 64, seed=15)
    page, rows = x.page, (1 << 31) // (8 * 128) + 64 * 32
    rows -= rows % page
    far = rows // page - 1 - torch.arange(x.B * x.max_pages, device=x.q.device).view(x.B, -1)
    k = torch.empty(rows, 8, 128, dtype=torch.bfloat16, device=x.q.device)
    v = torch.empty_like(k)
    near = x.t["table"].long().clamp(0, x.k.shape[0] // page - 1)
    at = lambda t: (t.long()[..., None] * page + torch.arange(page, device=t.device)).flatten()  # noqa: E731
    k[at(far)], v[at(far)] = x.k[at(near)], x.v[at(near)]
    small = x.pages()
    big = CachePages(k, v, far.int().contiguous(), x.t["lens"])
    with x.cache() as cache:
        res = []
        for kv in (small, big):
            lse = torch.empty(6, 16, device=x.q.device)
            out = cache.attention(x.q, x.k_new, x.v_new, kv, row_ptr=x.t["row_ptr"], lse=lse)
            w = cache.accumulate(x.q, lse, kv, row_ptr=x.t["row_ptr"])
            ev = cache.evict(kv, w, 100, 4, 8)
            after = CachePages(kv.k_pages, kv.v_pages, kv.page_table, ev[2], key_pos=ev[1])
            res.append((out, lse, w, *ev, cache.attention(x.q, x.k_new, x.v_new, after,
                                                          row_ptr=x.t["row_ptr"])))
        torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*res))


def test_refusals():
    import torch
    from paper_2606_09441_amd import Cache, CachePages, SiftError
    x = Batch([100, 30], [2, 2], 4, 2, 128, "bf16", seed=14)
    kv = x.pages()

    def refused(status, fn, *a, **kw):
        with pytest.raises(SiftError) as e:
            fn(*a, **kw)
        assert e.value.status == status

    for status, args in ((2, (0, 4, 2, 128)), (2, (2, 3, 2, 128)), (4, (2, 4, 2, 96)),
                         (5, (2, 4, 2, 128, 128, 1 << 24))):
        refused(status, Cache, *args)
    refused(4, Cache, 2, 4, 2, 128, page=48)
    refused(2, Cache, 2, 4, 2, 128, max_rows=0)
    with x.cache() as cache:
        f = cache.attention
        refused(2, f, x.q[:3], x.k_new[:3], x.v_new[:3], kv)          # not as many of each
        refused(2, f, x.q, x.k_new[:3], x.v_new, kv)
        refused(4, f, x.q, x.k_new, x.v_new.float(), kv)
        refused(4, f, x.q.float(), x.k_new.float(), x.v_new.float(), kv)
        refused(4, f, x.q, x.k_new, x.v_new, kv, cap=-2.0)
        refused(5, f, x.q, x.k_new, x.v_new, kv, row_ptr=x.t["row_ptr"][:2])
        refused(4, f, x.q, x.k_new, x.v_new, kv, row_ptr=x.t["row_ptr"].long())
        refused(5, f, x.q, x.k_new, x.v_new, kv, tree_mask=torch.zeros(3, 1, dtype=torch.int64,
                                                                       device=x.q.device))
        refused(5, f, x.q, x.k_new, x.v_new, kv, lse=torch.zeros(3, device=x.q.device))
        small = CachePages(x.k, x.v, x.t["table"][:1].contiguous(), x.t["lens"])
        refused(5, f, x.q, x.k_new, x.v_new, small)
        odd = CachePages(x.k[:-1], x.v[:-1], x.t["table"], x.t["lens"])
        refused(2, f, x.q, x.k_new, x.v_new, odd)
        other = CachePages(x.k, x.v[:-64], x.t["table"], x.t["lens"])
        refused(2, f, x.q, x.k_new, x.v_new, other)
    refused(4, CachePages, x.k, x.v, x.t["table"].long(), x.t["lens"])
    refused(1, CachePages, x.k, x.v, None, x.t["lens"])


def test_more_steps_than_the_split_counts():
    """Row pointers may give every sequence the most rows, whatever they add up to."""
    import torch
    from paper_2606_09441_amd import Cache, CachePages, SiftError
    dev = torch.device("cuda")
    seqs, pages, rows = 64, 8192, 2048
    pool = torch.zeros(128, 1, 64, dtype=torch.bfloat16, device=dev)
    ints = dict(dtype=torch.int32, device=dev)
    kv = CachePages(pool, pool.clone(), torch.zeros(seqs, pages, **ints), torch.zeros(seqs, **ints))
    new = torch.zeros(rows, 1, 64, dtype=torch.bfloat16, device=dev)
    with Cache(seqs, 64, 1, 64, page=128, max_pages=pages, max_rows=rows) as cache:
        with pytest.raises(SiftError) as e:
            cache.attention(new.expand(-1, 64, -1).contiguous(), new, new, kv,
                            row_ptr=torch.zeros(seqs + 1, **ints))
    assert e.value.status == 5


# so many rows times slots that bf16 goes by the units of 128 rows, and so many steps
# that a workgroup has runs of several, which end inside units
WIDE = ([9000, 300, 0], [100, 40, 3])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("tree,gaps,moved,cap,bias", [
    (None, False, False, 0.0, False), (random_tree, True, False, 0.0, False),
    (some_empty, False, False, 30.0, False), (random_tree, False, True, 0.0, True),
    (None, True, True, 20.0, True)])
def test_many_rows_over_long_caches(d, tree, gaps, moved, cap, bias):
    x = Batch(*WIDE, 8, 1, d, "bf16", 128, gaps, moved, tree, seed=16, extra_pages=16)
    assert x.max_rows * 8 * x.B * x.slots >= 24 << 20
    check(x, cap, bias)


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_unseen_new_tokens_of_many_rows(value):
    x = Batch(*WIDE, 8, 1, 64, "bf16", 128, tree=random_tree, seed=17, extra_pages=16)
    x.v_new[20, 0, 5:9] = value
    x.v_new[100 + 30, 0, 40] = value
    with x.cache() as cache:
        out = cache.attention(x.q, x.k_new, x.v_new, x.pages(), row_ptr=x.t["row_ptr"],
                              tree_mask=x.mask).float().cpu().numpy()
    with np.errstate(all="ignore"):
        ref, _ = x.oracle()
    fine = np.isfinite(ref)
    assert np.array_equal(fine, np.isfinite(out))
    assert max_abs(out[fine], ref[fine]) <= TOL["bf16"]


@pytest.mark.parametrize("end", [-2 ** 31, -1, 2 ** 31 - 1])
def test_row_pointers_out_of_range(end):
    """They give a sequence no rows that the buffers do not have: rows past the last
    are not written, the other sequence's are its own."""
    import torch
    x = Batch([50, 60], [0, 4], 4, 2, 64, "bf16", seed=23)
    out = torch.full((12, 4, 64), 7.0, dtype=x.dtype, device=x.q.device)
    lse = torch.full((12, 4), 7.0, device=x.q.device)
    ptr = torch.tensor([3, end, 4], dtype=torch.int32, device=x.q.device)
    with x.cache() as cache:
        want = cache.attention(x.q, x.k_new, x.v_new, x.pages(), row_ptr=x.t["row_ptr"])
        cache.attention(x.q, x.k_new, x.v_new, x.pages(), row_ptr=ptr, out=out[:4], lse=lse[:4])
        torch.cuda.synchronize()
        assert bool((out[4:] == 7).all()) and bool((lse[4:] == 7).all())
        if end < 0:      # (else row 3 is the first one's, and the second has none)
            assert torch.equal(out[:4], want)
        w = cache.accumulate(x.q, lse[:4], x.pages(), row_ptr=ptr)
        torch.cuda.synchronize()
        if end < 0:
            assert not bool(w[0].any())


def test_scales_and_caps_that_fp32_does_not_hold():
    import torch
    from paper_2606_09441_amd import SiftError
    x = Batch([100, 30], [2, 2], 4, 2, 128, "bf16", seed=14)
    lse = torch.zeros(4, 4, device=x.q.device)
    with x.cache() as cache:
        for kw in (dict(cap=2e-7), dict(cap=1e-20), dict(scale=3.4e38, cap=1.0), dict(scale=1e30, cap=1.0)):
            for call in (lambda: cache.attention(x.q, x.k_new, x.v_new, x.pages(), **kw),
                         lambda: cache.accumulate(x.q, lse, x.pages(), **kw)):
                with pytest.raises(SiftError) as e:
                    call()
                assert e.value.status == 4


def test_tables_of_longer_rows():
    """A table made for larger caches would be read as another one."""
    import torch
    from paper_2606_09441_amd import CachePages, SiftError
    x = Batch([100, 30], [2, 2], 4, 2, 128, "bf16", seed=24, moved=True)
    more = lambda t, n: torch.cat([t, torch.zeros_like(t[..., :n])], -1)  # noqa: E731
    t, lens, pos = x.t["table"], x.t["lens"], x.t["key_pos"]
    lse = torch.zeros(4, 4, device=x.q.device)
    w = torch.zeros(2, 2, x.slots, device=x.q.device)
    args = (x.q, x.k_new, x.v_new)
    with x.cache() as cache:
        want = cache.attention(*args, x.pages())
        rows = CachePages(x.k, x.v, torch.cat([t, t]), torch.cat([lens, lens]), key_pos=torch.cat([pos, pos]))
        assert torch.equal(want, cache.attention(*args, rows))
        for bad in (CachePages(x.k, x.v, more(t, 2), lens), CachePages(x.k, x.v, t, lens, page_lens=more(t, 1)),
                    CachePages(x.k, x.v, t, lens, key_pos=more(pos, 64))):
            for call in (lambda: cache.attention(*args, bad), lambda: cache.evict(bad, w, 8),
                         lambda: cache.accumulate(x.q, lse, bad)):
                with pytest.raises(SiftError) as e:
                    call()
                assert e.value.status == 2
        kv = x.pages()
        for call in (lambda: cache.evict(kv, more(w, 64), 8), lambda: cache.accumulate(x.q, lse, kv, more(w, 64)),
                     lambda: cache.accumulate(x.q, more(lse, 2), kv),
                     lambda: cache.attention(*args, kv, lse=more(lse, 2))):
            with pytest.raises(SiftError) as e:
                call()
            assert e.value.status == 2


def wide(x):
    """Whether bf16 goes by the units of 128 rows: 24 * 2^20 rows of a kv head times
    slots of all caches."""
    return x.max_rows * (x.hq // x.hkv) * x.B * x.hkv * x.slots >= 24 << 20


@pytest.mark.parametrize("hq,hkv", [(8, 2), (9, 3), (16, 8)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("tree,gaps,moved,cap,bias", [
    (None, False, False, 0.0, False), (random_tree, True, False, 0.0, False),
    (some_empty, False, False, 30.0, False), (random_tree, False, True, 0.0, True),
    (None, True, True, 20.0, True)])
def test_many_rows_of_several_kv_heads(hq, hkv, d, tree, gaps, moved, cap, bias):
    x = Batch([5000, 300, 0], WIDE[1], hq, hkv, d, "bf16", 128, gaps, moved, tree, seed=21, extra_pages=47)
    assert wide(x)
    check(x, cap, bias)


@pytest.mark.parametrize("gaps,moved,cap,bias", [(False, False, 0.0, False), (True, False, 0.0, False),
                                                 (False, True, 0.0, True), (False, False, 20.0, True)])
def test_many_rows_of_many_sequences(gaps, moved, cap, bias):
    """More sequences than a wavefront has lanes, some without rows or keys."""
    rng = np.random.default_rng(22)
    lens = rng.integers(0, 300, 70).tolist()
    new = rng.integers(0, 21, 70).tolist()
    lens[5], new[3], new[66] = 0, 20, 0
    x = Batch(lens, new, 8, 2, 64, "bf16", 128, gaps, moved, random_tree, seed=22, extra_pages=16)
    assert wide(x)
    check(x, cap, bias)


def test_units_by_rows_and_slots():
    """The same rows over the same keys by either unit: a handle with room for more
    slots goes by the wide ones."""
    import torch
    outs = []
    for extra, is_wide in ((1, False), (400, True)):
        x = Batch([500, 90], [40, 9], 16, 2, 128, "bf16", 128, tree=random_tree, seed=25, extra_pages=1)
        x.max_pages += extra - 1
        x.slots = x.max_pages * 128
        x.table = np.concatenate([x.table, np.zeros((2, extra - 1), np.int32)], 1)
        x.t["table"] = torch.from_numpy(x.table).to(x.q.device)
        assert wide(x) == is_wide
        outs.append(check(x))
    assert max_abs(outs[0][0], outs[1][0]) <= TOL["bf16"]
    assert max_abs(outs[0][1], outs[1][1]) <= LSE_TOL
