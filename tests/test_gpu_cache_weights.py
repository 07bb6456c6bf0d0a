"""GPU tests of the accumulated attention weights (sift_cache_accumulate) against
the fp64 oracle."""

from __future__ import annotations

import numpy as np
import pytest

from cache_helpers import Batch, random_tree
from gpu_helpers import max_abs, say

pytestmark = pytest.mark.gpu

TYPES = [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)]
LENS = [0, 1, 15, 16, 17, 31, 33, 64, 127, 129, 300, 700]
NEW = [5, 0, 1, 33, 3, 2, 64, 12, 0, 1, 20, 40]

# A weight e^(s - lse) has the relative error of the absolute one of s - lse: at
# most 128 * 2^-24 * sum|q k| * scale in the worst case (about 1e-4 at |s| = 16),
# a hundredth of it for roundings that do not line up, and 2^-22 for the rest.
REL = 2e-5


def inputs(x, seed=0):
    """Log sums of the rows, with some without keys, weights of the rows and of the
    keys."""
    import torch
    rng = np.random.default_rng(seed)
    dev = x.q.device
    lse = rng.uniform(8.0, 20.0, (x.rows, x.hq)).astype(np.float32)
    lse[rng.random(lse.shape) < 0.05] = -np.inf
    rw = rng.uniform(0.25, 2.0, x.rows).astype(np.float32)
    rw[rng.random(x.rows) < 0.2] = 0.0
    w = rng.random((x.B, x.hkv, x.slots)).astype(np.float32)
    return [(a, torch.from_numpy(a).to(dev)) for a in (lse, rw, w)]


def check(x, cap=0.0, bias=False, decay=0.75, weighted=False, fresh=False, name=""):
    import torch
    slopes = (2.0 ** (-4.0 * np.arange(1, x.hq + 1) / x.hq)).astype(np.float32) if bias else None
    (lse, lse_d), (rw, rw_d), (w, w_d) = inputs(x)
    f = lambda t: t.float().cpu().numpy()  # noqa: E731
    ref = S().accumulate(f(x.q), lse, x.host(), np.zeros_like(w) if fresh else w, decay, x.row_ptr,
                         x.row_pos, rw if weighted else None, None, cap, slopes)
    out = torch.full_like(w_d, 9.0)
    with x.cache() as cache:
        cache.accumulate(x.q, lse_d, x.pages(), None if fresh else w_d, decay,
                         row_ptr=x.t["row_ptr"], row_pos=x.t["row_pos"],
                         row_weight=rw_d if weighted else None, cap=cap, out=out,
                         slopes=None if slopes is None else torch.from_numpy(slopes).to(x.q.device))
        torch.cuda.synchronize()
    got = out.cpu().numpy()
    past = np.isnan(ref)
    assert (got[past] == 9.0).all()
    err = np.abs(got[~past] - ref[~past]) / np.maximum(1e-3, np.abs(ref[~past]))
    say(f"{name} {x.q.dtype} {x.d}: {err.max() if err.size else 0:.2e}")
    assert not err.size or err.max() <= REL


def S():
    from oracle import serve_oracle
    return serve_oracle


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("page", [16, 128])
def test_against_the_oracle(dtype, d, page):
    for gaps, moved, cap, bias, weighted in [(False, False, 0.0, False, False),
                                             (True, True, 0.0, True, True),
                                             (True, False, 30.0, False, True),
                                             (False, True, 20.0, True, False),
                                             (False, False, 0.0, True, False)]:
        check(Batch(LENS, NEW, 6, 2, d, dtype, page, gaps, moved, seed=3), cap, bias,
              weighted=weighted, name=f"gaps {gaps} moved {moved} cap {cap} bias {bias}")


@pytest.mark.parametrize("dtype,d", TYPES)
def test_few_rows(dtype, d):
    """Rows of a block or two, whose keys come through LDS."""
    new = [2, 0, 1, 6, 3, 2, 9, 4, 0, 1, 5, 8]
    for gaps, moved, cap, bias, weighted in [(False, False, 0.0, False, True),
                                             (True, True, 20.0, True, True),
                                             (True, False, 30.0, False, False)]:
        check(Batch(LENS, new, 12, 2, d, dtype, 32, gaps, moved, seed=3), cap, bias,
              weighted=weighted, name=f"gaps {gaps} moved {moved} cap {cap} bias {bias}")


def test_many_sequences():
    rng = np.random.default_rng(11)
    lens = rng.integers(0, 90, 150).tolist()
    check(Batch(lens, [int(rng.integers(0, 3)) for _ in lens], 4, 2, 64, "bf16", 16, seed=11))


@pytest.mark.parametrize("dtype,d", TYPES)
def test_single_tokens(dtype, d):
    check(Batch(LENS, [1] * len(LENS), 8, 2, d, dtype, 64))
    check(Batch(LENS, [1] * len(LENS), 8, 1, d, dtype, 64), fresh=True)
    check(Batch(LENS, [1] * len(LENS), 3, 3, d, dtype, 64), decay=0.0)


@pytest.mark.parametrize("dtype,hq", [("bf16", 12), ("f32", 6)])
def test_more_rows_than_lds_holds(dtype, hq):
    check(Batch([90, 40], [100, 7], hq, 1, 128, dtype, 32, seed=4))


def test_long_cache():
    check(Batch([9000, 10], [3, 3], 8, 2, 64, "bf16", 64, seed=5))


def test_in_place_and_from_the_attention():
    """The weights of a row over cache and new tokens sum to the query heads' number
    less what the new tokens have: with none visible but itself, at most 1 a head."""
    import torch
    x = Batch([200, 50], [1, 1], 4, 2, 128, "bf16", seed=6)
    with x.cache() as cache:
        lse = torch.empty(2, 4, device=x.q.device)
        cache.attention(x.q, x.k_new, x.v_new, x.pages(), lse=lse)
        w = cache.accumulate(x.q, lse, x.pages())
        first = w.clone()
        again = cache.accumulate(x.q, lse, x.pages(), w, decay=1.0)
    assert again is w
    torch.cuda.synchronize()
    f = lambda t: t.float().cpu().numpy()  # noqa: E731
    self_w = np.stack([[np.exp(f(x.q)[b, h].astype(np.float64) @ f(x.k_new)[b, h // 2] / 128 ** 0.5
                               - float(lse[b, h])) for h in range(4)] for b in range(2)])
    want = 2.0 - self_w.reshape(2, 2, 2).sum(2)
    assert max_abs(first.sum(2).cpu().numpy(), want) <= 1e-4
    assert max_abs(w.cpu().numpy(), 2 * first.cpu().numpy()) <= 1e-5


def test_rows_left_out_do_not_matter():
    """A row of weight 0, or without a log sum, holding NaN."""
    import torch
    x = Batch([80], [4], 4, 2, 64, "bf16", tree=random_tree, seed=7)
    lse = torch.full((4, 4), 5.0, device=x.q.device)
    rw = torch.tensor([1.0, 0.0, 1.0, 1.0], device=x.q.device)
    with x.cache() as cache:
        lse[3] = -float("inf")
        want = cache.accumulate(x.q, lse, x.pages(), row_weight=rw).clone()
        x.q[1], x.q[3], lse[1] = float("nan"), float("inf"), float("nan")
        got = cache.accumulate(x.q, lse, x.pages(), row_weight=rw)
    assert bool(torch.isfinite(want).all()) and torch.equal(want, got)


def test_graph():
    import torch
    x = Batch([300, 41], [7, 7], 8, 2, 128, "bf16", seed=8)
    (_, lse), (_, rw), (_, w) = inputs(x)
    out = torch.zeros_like(w)
    with x.cache() as cache:
        kw = dict(row_ptr=x.t["row_ptr"], row_weight=rw)
        first = cache.accumulate(x.q, lse, x.pages(), w, out=torch.zeros_like(w), **kw)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        kv = x.pages()
        with torch.cuda.graph(graph):
            cache.accumulate(x.q, lse, kv, w, out=out, **kw)
        for _ in range(3):
            out.zero_()
            graph.replay()
            assert torch.equal(out, first)


def test_refusals():
    import torch
    from paper_2606_09441_amd import SiftError
    x = Batch([100, 30], [2, 2], 4, 2, 128, "bf16", seed=9)
    (_, lse), (_, rw), (_, w) = inputs(x)
    kv = x.pages()
    with x.cache() as cache:
        def refused(status, *a, **kw):
            with pytest.raises(SiftError) as e:
                cache.accumulate(*a, **kw)
            assert e.value.status == status
        refused(1, x.q, None, kv)
        refused(5, x.q, lse[:3], kv)
        refused(5, x.q, lse, kv, w[:1].contiguous())
        refused(4, x.q, lse, kv, w, decay=float("inf"))
        refused(4, x.q.float(), lse, kv, w)
        refused(5, x.q, lse, kv, w, row_weight=rw[:2])
        refused(4, x.q, lse, kv, w, out=w.int())
        refused(2, x.q[:3], lse, kv, w)
        refused(4, x.q, lse, kv, w, cap=-1.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 40, 300, 320])
def test_a_log_sum_that_is_no_number(dtype, rows):
    """Every weight it is part of is none either, however the rows are dealt out; where
    the row counts for nothing, none is."""
    import torch
    x = Batch([80, 50], [rows, 2], 2, 2, 64, dtype, seed=18)
    lse = torch.full((x.rows, 2), 5.0, device=x.q.device)
    lse[rows - 1] = float("nan")
    ones = torch.ones(x.rows, device=x.q.device)
    some = ones.clone()
    some[0] = 0.0 if rows > 1 else 1.0
    without = ones.clone()
    without[rows - 1] = 0.0
    with x.cache() as cache:
        for rw, number in ((None, False), (ones, False), (some, False), (without, True)):
            w = cache.accumulate(x.q, lse, x.pages(), row_ptr=x.t["row_ptr"], row_weight=rw)
            assert torch.isfinite(w[0, :, :80]).unique().tolist() == [number]
            assert bool(torch.isfinite(w[1, :, :50]).all())


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("rows", [1, 8, 300])
def test_scores_near_the_log_sum_keep_their_bits(dtype, d, rows):
    """Scores that fp32 holds exactly (one product each), all large and near the log
    sum of the one row that counts: their difference x is rounded once, its product
    with log2(e) once more and the exponential to its last bit, 2^-22 (1 + |x|) in
    all.  Rounding log sum or score in another unit would cost 2^-24 of 120."""
    import torch
    x = Batch([200], [rows], 4, 4, d, dtype, seed=19)
    rng = np.random.default_rng(20)
    x.q.zero_()
    x.k.zero_()
    x.q[:, :, 0] = 8.0
    s = 112.0 + 0.5 * rng.integers(0, 16, tuple(x.k.shape[:2]))
    x.k[:, :, 0] = torch.from_numpy(s).to(x.k)
    lse = np.full((rows, 4), 1e4, np.float32)        # weights of 0
    lse[rows // 2] = rng.uniform(119.0, 121.0, 4)
    with x.cache() as cache:
        w = cache.accumulate(x.q, torch.from_numpy(lse).to(x.q.device), x.pages(), scale=0.125)
    p = x.host()
    e = p.k[p.rows(0, np.arange(200)), :, 0].astype(np.float64).T - lse[rows // 2][:, None].astype(np.float64)
    rel = np.abs(w[0, :, :200].cpu().numpy() / np.exp(e) - 1)
    say(f"{dtype} {d} {rows}: {rel.max():.2e}, of the bound {(rel / (2.0 ** -22 * (1 + np.abs(e)))).max():.2f}")
    assert (rel <= 2.0 ** -22 * (1 + np.abs(e))).all()
