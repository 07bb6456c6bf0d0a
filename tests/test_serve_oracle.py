"""CPU checks of oracle/serve_oracle.py: closed forms and special cases, so that the
GPU tests compare with something that is itself fixed."""

from __future__ import annotations

import numpy as np
import pytest

from oracle import serve_oracle as S

SO, PS = [0, 5, 6, 9, 13, 13], [0, 3, 5]     # two prompts; the second's query is empty


def draw(n, hq, hkv, d, seed=0):
    rng = np.random.default_rng(seed)
    return (rng.standard_normal((n, hq, d)), rng.standard_normal((n, hkv, d)),
            rng.standard_normal((n, hkv, d)))


def test_visible_keys_hand_written():
    c, d, p = (S.dense_visible(SO, PS, m) for m in ("causal", "document", "prefix"))
    assert c[7].nonzero()[0].tolist() == [0, 1, 2, 3, 4, 5, 6, 7]
    assert c[10].nonzero()[0].tolist() == [9, 10]
    assert d[4].nonzero()[0].tolist() == [0, 1, 2, 3, 4]
    assert d[5].nonzero()[0].tolist() == [5]
    assert d[7].nonzero()[0].tolist() == [0, 1, 2, 3, 4, 5, 6, 7]
    assert p[0].nonzero()[0].tolist() == [0, 1, 2, 3, 4, 5]
    assert p[7].nonzero()[0].tolist() == [0, 1, 2, 3, 4, 5, 6, 7]
    assert p[9].nonzero()[0].tolist() == [9, 10, 11, 12]


@pytest.mark.parametrize("mask", ["causal", "document", "prefix"])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (3.0, False), (0.0, True), (3.0, True)])
def test_by_head_equals_by_row(mask, cap, bias):
    q, k, v = draw(13, 4, 2, 8)
    slopes = [0.5, 0.25, -0.1, 2.0] if bias else None
    a = S.dense(q, k, v, SO, PS, mask, None, cap, slopes)
    b = S.dense_by_head(q, k, v, SO, PS, mask, None, cap, slopes)
    assert np.allclose(a[0], b[0], atol=1e-13) and np.allclose(a[1], b[1], atol=1e-13)


def test_uniform_scores_give_the_mean():
    q, k, v = draw(13, 2, 1, 8)
    out, lse = S.dense(q * 0, k, v, SO, PS, "causal")
    assert np.allclose(out[7, 1], v[:8, 0].mean(0)) and np.allclose(lse[7], np.log(8))


def test_cap_and_bias_closed_forms():
    k = np.eye(4)
    s = S.scores([6.0, 0.0, -6.0, 1e9], k, 0.5, cap=2.0, slope=0.25, dist=[1, -2, 3, 4])
    want = 2 * np.tanh([1.5, 0.0, -1.5, 1e9]) - 0.25 * np.array([1, 2, 3, 4])
    assert np.allclose(s, want)


def test_no_visible_key():
    out, lse = S.attend(np.ones(4), np.zeros((0, 4)), np.zeros((0, 4)), 1.0)
    assert not out.any() and lse == -np.inf


def pages():
    """Two sequences of pages of 4: slots 0 .. 5 and 0 .. 2, the first page of the
    first ends early."""
    rng = np.random.default_rng(1)
    k, v = rng.standard_normal((24, 1, 8)), rng.standard_normal((24, 1, 8))
    table = np.array([[3, 1], [5, 0]])
    return S.Pages(k, v, table, np.array([6, 3]), 4, np.array([[2, 4], [4, 4]]))


def test_slots_and_rows():
    p = pages()
    assert p.slots(0).tolist() == [0, 1, 4, 5]
    assert p.rows(0, p.slots(0)).tolist() == [12, 13, 4, 5]
    assert p.slots(1).tolist() == [0, 1, 2]


def test_cache_attention_is_dense_attention_over_the_gathered_keys():
    p = pages()
    q, kn, vn = draw(3, 2, 1, 8, 2)
    out, lse = S.cache_attention(q, kn, vn, p, [0, 2, 3])
    k = np.concatenate([p.k[[12, 13, 4, 5], 0], kn[:2, 0]])
    v = np.concatenate([p.v[[12, 13, 4, 5], 0], vn[:2, 0]])
    want, wl = S.attend(q[1, 1], k, v, 8 ** -0.5)
    assert np.allclose(out[1, 1], want) and np.isclose(lse[1, 1], wl)
    want, _ = S.attend(q[0, 0], k[:5], v[:5], 8 ** -0.5)
    assert np.allclose(out[0, 0], want)


def test_accumulated_weights_sum_to_what_the_new_tokens_leave():
    p = pages()
    q, kn, vn = draw(2, 2, 1, 8, 3)
    _, lse = S.cache_attention(q, kn, vn, p, [0, 1, 2])
    w = S.accumulate(q, lse, p, np.zeros((2, 1, 8)), 1.0, [0, 1, 2])
    for b in range(2):
        own = sum(np.exp(q[b, h] @ kn[b, 0] * 8 ** -0.5 - lse[b, h]) for h in range(2))
        assert np.isclose(np.nansum(w[b]), 2 - own)
    assert w[0, 0, 2] == 0 and np.isnan(w[0, 0, 6])


def test_evict_hand_worked():
    """Slots 0 1 4 5 hold keys of weights 1 5 3 5; three stay: slots 1 and 5 (5), 4
    (3).  Slots 4 and 5 move to the free slots 0 and 2."""
    p = pages()
    w = np.array([[[1, 5, 9, 9, 3, 5, 0, 0]], [[2, 2, 2, 0, 0, 0, 0, 0]]], np.float32)
    k, v, wo, po, lens = S.evict(p, w, 3)
    assert lens.tolist() == [3, 3]
    assert wo[0, 0].tolist() == [3, 5, 5, 0, 0, 0, 0, 0]
    assert po[0, 0].tolist() == [4, 1, 5, -1, -1, -1, -1, -1]
    assert np.array_equal(k[[12, 13, 14], 0], p.k[[4, 13, 5], 0])
    assert po[1, 0].tolist() == [0, 1, 2, -1, -1, -1, -1, -1]


def test_evict_ties_and_protection():
    p = pages()
    w = np.array([[[2, 2, 9, 9, 2, 2, 0, 0]], [[np.nan, -1, np.nan, 0, 0, 0, 0, 0]]], np.float32)
    _, _, _, po, _ = S.evict(p, w, 2)
    assert po[0, 0, :2].tolist() == [0, 1]             # ties: the lowest slots
    assert sorted(po[1, 0, :2].tolist()) == [0, 1]     # a number before NaN, then the lowest NaN
    _, _, _, po, _ = S.evict(p, w, 2, sinks=1, recent=1)
    assert sorted(po[0, 0, :2].tolist()) == [0, 5]
