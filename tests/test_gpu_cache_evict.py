"""GPU tests of the eviction (sift_cache_evict) against the oracle: everything
exact, the pools' other rows untouched."""

from __future__ import annotations

import numpy as np
import pytest

from cache_helpers import Batch
from oracle import serve_oracle as S

pytestmark = pytest.mark.gpu

LENS = [0, 1, 15, 16, 17, 31, 33, 64, 127, 129, 300, 700]


def weights_of(x, kind, seed=0):
    rng = np.random.default_rng(seed)
    shape = (x.B, x.hkv, x.slots)
    if kind == "equal":
        return np.full(shape, 0.5, np.float32)
    if kind == "ties":
        return (rng.integers(0, 4, shape) / 4).astype(np.float32)
    w = rng.standard_normal(shape).astype(np.float32) * 10.0 ** rng.integers(-30, 30, shape)
    if kind == "odd":
        odd = rng.random(shape)
        w = np.select([odd < 0.1, odd < 0.2, odd < 0.3, odd < 0.4, odd < 0.5, odd < 0.55],
                      [np.nan, np.inf, -np.inf, 0.0, -0.0, 1e-40], w).astype(np.float32)
    return w.astype(np.float32)


def check(x, kind, budget, sinks=0, recent=0, own_next=False):
    import torch
    w = weights_of(x, kind)
    nxt = (x.lens + 3).astype(np.int32) if own_next else None
    if x.key_pos is not None:
        nxt = np.full(x.B, x.slots, np.int32)
    dev = x.q.device
    up = lambda a: None if a is None else torch.from_numpy(a).to(dev)  # noqa: E731
    # NaN marks the rows that hold no key; compare bits, as integers
    k0, v0 = x.k.clone(), x.v.clone()
    bits = lambda t: t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)  # noqa: E731
    host = S.Pages(bits(k0).cpu().numpy(), bits(v0).cpu().numpy(), x.table, x.lens, x.page,
                   x.page_lens, x.key_pos)
    with np.errstate(all="ignore"):
        k, v, wr, pr, lr = S.evict(host, w, budget, sinks, recent, nxt)
    with x.cache() as cache:
        wo, po, lo = cache.evict(x.pages(), up(w), budget, sinks, recent, up(nxt))
        torch.cuda.synchronize()
    assert np.array_equal(lo.cpu().numpy(), lr)
    assert np.array_equal(po.cpu().numpy(), pr)
    assert np.array_equal(wo.cpu().numpy().view(np.int32), wr.view(np.int32))
    assert np.array_equal(bits(x.k).cpu().numpy(), k)
    assert np.array_equal(bits(x.v).cpu().numpy(), v)


@pytest.mark.parametrize("kind", ["any", "equal", "ties", "odd"])
@pytest.mark.parametrize("budget", [1, 16, 40, 64, 128, 500, 5000])
def test_budgets(kind, budget):
    check(Batch(LENS, [0] * len(LENS), 4, 2, 64, "bf16", 32), kind, budget)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("page", [16, 64, 128])
def test_types_pages_and_positions(dtype, d, page):
    for gaps, moved in [(True, False), (False, True), (True, True)]:
        x = Batch(LENS, [0] * len(LENS), 3, 3, d, dtype, page, gaps, moved, seed=1)
        check(x, "any", 60, sinks=4, recent=16)


@pytest.mark.parametrize("sinks,recent", [(0, 0), (4, 0), (0, 30), (4, 26), (30, 0), (0, 29)])
def test_protected(sinks, recent):
    check(Batch(LENS, [0] * len(LENS), 2, 1, 64, "bf16", 16, seed=2), "odd", 30, sinks, recent)
    check(Batch(LENS, [0] * len(LENS), 2, 1, 64, "bf16", 16, seed=2), "equal", 30, sinks, recent,
          own_next=True)


@pytest.mark.parametrize("kind", ["any", "equal", "ties", "odd"])
@pytest.mark.parametrize("budget", [1, 700, 8192, 15000, 40000])
def test_long_caches(kind, budget):
    """Caches that several workgroups select from."""
    check(Batch([20000, 9000, 1, 0, 2048, 16385], [0] * 6, 2, 2, 64, "bf16", 16, budget % 2 == 0,
                budget > 8000, seed=7), kind, budget, min(4, budget), min(64, budget // 2))


def test_long():
    check(Batch([20000, 300], [0, 0], 2, 2, 64, "bf16", 128, gaps=True, seed=3), "any", 3000, 4, 64)
    check(Batch([20000], [0], 1, 1, 64, "bf16", 128, seed=3), "ties", 9999, 4, 64)


def test_twice_and_again():
    """The inputs stay: a second call gives the same; and its result can be evicted
    further, and attended over."""
    import torch
    from paper_2606_09441_amd import CachePages
    x = Batch([200, 90], [2, 2], 4, 2, 128, "bf16", 64, gaps=True, seed=4)
    w = torch.from_numpy(weights_of(x, "any")).to(x.q.device)
    with x.cache() as cache:
        a = [t.clone() for t in cache.evict(x.pages(), w, 80, 4, 8)]
        k = x.k.clone()
        b = cache.evict(x.pages(), w, 80, 4, 8)
        assert all(torch.equal(s, t) for s, t in zip(a, b))
        assert torch.equal(x.k.view(torch.int16), k.view(torch.int16))
        kv = CachePages(x.k, x.v, x.t["table"], a[2], key_pos=a[1])
        w2, p2, l2 = cache.evict(kv, a[0], 33, 4, 8, x.t["lens"])
        kv = CachePages(x.k, x.v, x.t["table"], l2, key_pos=p2)
        out = cache.attention(x.q, x.k_new, x.v_new, kv)
    x.lens, x.page_lens, x.key_pos = l2.cpu().numpy(), None, p2.cpu().numpy()
    assert x.lens.tolist() == [33, 33]
    ref, _ = x.oracle()
    assert np.abs(out.float().cpu().numpy() - ref).max() <= 2e-2


def test_graph():
    import torch
    x = Batch([200, 90], [0, 0], 4, 2, 128, "bf16", 64, seed=5)
    w = torch.from_numpy(weights_of(x, "any")).to(x.q.device)
    k0, v0 = x.k.clone(), x.v.clone()
    with x.cache() as cache:
        kv = x.pages()
        want = [t.clone() for t in cache.evict(kv, w, 50)]
        k1 = x.k.clone()
        out = [torch.zeros_like(t) for t in want]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cache.evict(kv, w, 50, weights_out=out[0], pos_out=out[1], lens_out=out[2])
        for _ in range(3):
            x.k.copy_(k0)
            x.v.copy_(v0)
            for t in out:
                t.zero_()
            graph.replay()
            assert all(torch.equal(s, t) for s, t in zip(want, out))
            assert torch.equal(x.k.view(torch.int16), k1.view(torch.int16))


def test_refusals():
    import torch
    from paper_2606_09441_amd import SiftError
    x = Batch([100, 30], [0, 0], 4, 2, 128, "bf16", moved=True, seed=6)
    w = torch.from_numpy(weights_of(x, "any")).to(x.q.device)
    kv = x.pages()
    with x.cache() as cache:
        def refused(status, *a, **kw):
            with pytest.raises(SiftError) as e:
                cache.evict(*a, **kw)
            assert e.value.status == status
        refused(2, kv, w, 0)
        refused(2, kv, w, 10, sinks=-1)
        refused(2, kv, w, 10, sinks=6, recent=5)
        refused(5, kv, w[:1].contiguous(), 10)
        refused(4, kv, w.double(), 10)
        refused(4, kv, w, 10, weights_out=w)
        refused(4, kv, w, 10, pos_out=kv.key_pos)
        refused(4, kv, w, 10, lens_out=kv.lens)
        refused(5, kv, w, 10, next_pos=kv.lens[:1])


def test_as_many_slots_as_a_cache_can_have():
    """Slots near 2^31, whose index a step of the clearing loop passes: all past the
    kept ones are cleared, and nothing outside."""
    import torch
    from paper_2606_09441_amd import Cache, CachePages
    dev = torch.device("cuda")
    max_pages, guard = (1 << 24) - 2, 1 << 20
    slots = max_pages * 128
    pool = torch.randn(8 * 128, 1, 64, device=dev).bfloat16()
    table = torch.zeros(1, max_pages, dtype=torch.int32, device=dev)
    table[0, :8] = torch.arange(8)
    kv = CachePages(pool, pool.clone(), table, torch.tensor([300], dtype=torch.int32, device=dev))
    w = torch.zeros(slots, device=dev)
    w[:300] = torch.arange(300, device=dev)
    weights = torch.full((slots + 2 * guard,), 7.0, device=dev)
    pos = torch.full((slots + 2 * guard,), 7, dtype=torch.int32, device=dev)
    inner = slice(guard, guard + slots)
    with Cache(1, 1, 1, 64, page=128, max_pages=max_pages) as cache:
        for budget, n in ((1 << 20, 300), (100, 100)):
            _, _, lens = cache.evict(kv, w, budget, weights_out=weights[inner], pos_out=pos[inner])
            torch.cuda.synchronize()
            assert lens.tolist() == [n]
            assert sorted(pos[inner][:n].tolist()) == list(range(300 - n, 300))
            for t, none in ((weights, 0), (pos, -1)):
                at = torch.cat([t[:guard], t[-guard:]])
                assert bool((at == 7).all())
                for a in range(n, slots, 1 << 28):
                    assert bool((t[inner][a:a + (1 << 28)] == none).all())
