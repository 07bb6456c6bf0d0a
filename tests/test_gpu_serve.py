"""GPU: a batch of prompts through prefill, cut, drafted trees and a second cut
(serve.PromptCache), against the fp64 formulas over the keys that it kept."""

from __future__ import annotations

import numpy as np
import pytest

from oracle import serve_oracle as S

pytestmark = pytest.mark.gpu
TOL = {"bf16": 2e-2, "f32": 1e-5}      # outputs: as the sparse attention's tests
PROMPTS = [[130, 64, 1, 40], [77, 20], [5], [300, 31, 64, 16]]


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("sparse", [True, False])
@pytest.mark.parametrize("budget", [48, 1000])
def test_prompts_to_answers(dtype, d, sparse, budget):
    import torch
    from paper_2606_09441_amd.serve import PromptCache
    hq, hkv, g = 4, 2, 2
    so, ps = [0], [0]
    for p in PROMPTS:
        for n in p:
            so.append(so[-1] + n)
        ps.append(len(so) - 1)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator("cuda").manual_seed(3)
    draw = lambda n, h: torch.randn(n, h, d, generator=gen, device="cuda").to(dt)  # noqa: E731
    host = lambda t: t.double().cpu().numpy()  # noqa: E731
    score = {} if sparse else dict(cap=10.0, slopes=torch.tensor([.5, .1, .02, .3], device="cuda"))
    slopes = [0.0] * 4 if sparse else score["slopes"].tolist()
    q, k, v = draw(so[-1], hq), draw(so[-1], hkv), draw(so[-1], hkv)
    with PromptCache(so, ps, hq, hkv, d, page=32, room=64, max_rows=4, dtype=dt) as c:
        bits = [torch.full((c.plan.info[x],), 255, dtype=torch.uint8, device="cuda")
                for x in ("la_bytes", "ca_bytes")] if sparse else (None, None)
        out = c.prefill(q, k, v, *bits, **score)
        want, lse = S.dense(host(q), host(k), host(v), so, ps, "causal", None, score.get("cap", 0.0),
                            slopes)
        assert np.max(np.abs(host(out) - want)) <= TOL[dtype]

        # the weights that the query's tokens give, by position; who has to stay
        all_k = [host(k)[so[ps[b]]:so[ps[b + 1]]] for b in range(4)]
        all_v = [host(v)[so[ps[b]]:so[ps[b + 1]]] for b in range(4)]
        docs = [so[ps[b + 1] - 1] - so[ps[b]] for b in range(4)]
        c.cut(budget, sinks=2, recent=3)
        for b in range(4):
            n, first = int(c.pages.lens[b]), so[ps[b + 1] - 1]
            own = so[ps[b + 1]] - first
            assert n == min(docs[b], budget) + own
            assert c.next_pos[b] == docs[b] + own
            pos = c.pages.key_pos[b, :, :n].cpu().numpy()
            for h in range(hkv):
                w = np.zeros(docs[b])
                for i in range(first, first + own):
                    for x in range(h * g, h * g + g):
                        dist = i - so[ps[b]] - np.arange(docs[b])
                        s = S.scores(host(q)[i, x], all_k[b][:docs[b], h], d ** -0.5,
                                     score.get("cap", 0.0), slopes[x], dist)
                        w += np.exp(s - lse[i, x])
                kept = set(pos[h, :n - own].tolist())
                assert len(kept) == n - own and kept <= set(range(docs[b]))
                assert pos[h, n - own:].tolist() == list(range(docs[b], docs[b] + own))
                near = docs[b] + own - 3       # protected: the last three positions
                free = [j for j in range(docs[b]) if 2 <= j < near]
                assert all(j in kept for j in range(docs[b]) if j not in free)
                lost = [w[j] for j in free if j not in kept]
                stay = [w[j] for j in free if j in kept]
                if lost and stay:
                    assert max(lost) <= min(stay) * (1 + 1e-2)   # 2^-8 of a bf16 score's terms


        mask = torch.tensor([1, 3, 5, 11] * 4, device="cuda").view(16, 1)
        sees = [[0], [0, 1], [0, 2], [0, 1, 3]]
        depth = torch.tensor([0, 1, 1, 2] * 4, dtype=torch.int32, device="cuda")
        for _ in range(2):
            qn, kn, vn = draw(16, hq), draw(16, hkv), draw(16, hkv)
            at = (c.next_pos.repeat_interleave(4) + depth).int()
            out, lse = c.step(qn, kn, vn, tree_mask=mask, row_pos=at)
            for b in range(4):
                n = int(c.pages.lens[b])
                pos = c.pages.key_pos[b, :, :n].cpu().numpy()
                for i in range(4):
                    r, new = 4 * b + i, [4 * b + j for j in sees[i]]
                    for x in range(hq):
                        kk = np.concatenate([all_k[b][pos[x // g], x // g], host(kn)[new, x // g]])
                        vv = np.concatenate([all_v[b][pos[x // g], x // g], host(vn)[new, x // g]])
                        there = np.concatenate([pos[x // g], at.cpu().numpy()[new]])
                        y, _ = S.attend(host(qn)[r, x], kk, vv, d ** -0.5, score.get("cap", 0.0),
                                        slopes[x], int(at[r]) - there)
                        assert np.max(np.abs(host(out)[r, x] - y)) <= TOL[dtype]
            accepted = torch.tensor([0, 1, 3, 4, 8, 9], device="cuda")   # none of the last prompt
            c.append(qn, kn, vn, lse, accepted, row_pos=at)
            for r in accepted.tolist():
                all_k[r // 4] = np.concatenate([all_k[r // 4], host(kn)[r:r + 1]])
                all_v[r // 4] = np.concatenate([all_v[r // 4], host(vn)[r:r + 1]])
        before = c.pages.lens.tolist()
        c.cut(40, sinks=2, recent=8)
        assert c.pages.lens.tolist() == [min(n, 40) for n in before]
        for b in range(4):
            n = int(c.pages.lens[b])
            pos = c.pages.key_pos[b, :, :n].cpu().numpy()
            last = int(c.next_pos[b])
            for h in range(hkv):
                assert set(range(max(0, last - 8), last)) <= set(pos[h].tolist())
                rows = c.pages.page_table[b].cpu().numpy()
                at = [rows[i // 32] * 32 + i % 32 for i in range(n)]
                assert np.array_equal(host(c.pages.k_pages)[at, h], all_k[b][pos[h], h])
                assert np.array_equal(host(c.pages.v_pages)[at, h], all_v[b][pos[h], h])


def test_the_example_runs(capsys):
    from paper_2606_09441_amd import serve
    serve.main()
    out = capsys.readouterr().out
    assert "cut: [602, 559]" in out and "cut: [512, 512]" in out


def test_refusals():
    import torch
    from paper_2606_09441_amd import SiftError
    from paper_2606_09441_amd.serve import PromptCache
    q = torch.randn(40, 2, 64, device="cuda").bfloat16()
    with PromptCache([0, 30, 40], [0, 2], 2, 2, 64, page=16, room=8, max_rows=2) as c:
        bits = [torch.zeros(c.plan.info[x], dtype=torch.uint8, device="cuda")
                for x in ("la_bytes", "ca_bytes")]
        with pytest.raises(SiftError):
            c.prefill(q, q, q, *bits, cap=5.0)
        c.prefill(q, q, q, cap=5.0)
        with pytest.raises(SiftError):     # the query is not in the cache yet
            c.step(q[:1], q[:1], q[:1])
        c.cut(100)
        with pytest.raises(SiftError):     # no room
            for _ in range(40):
                _, lse = c.step(q[:2], q[:2], q[:2])
                c.append(q[:2], q[:2], q[:2], lse, torch.arange(2, device="cuda"))


def test_room_counts_each_prompts_own_rows():
    """Queries and answers fill their own prompt's slots: many prompts do not use up the
    room of one."""
    import torch
    from paper_2606_09441_amd.serve import PromptCache
    so, ps = [0], [0]
    for _ in range(6):
        so += [so[-1] + 64, so[-1] + 80]
        ps.append(len(so) - 1)
    x = torch.randn(so[-1], 2, 64, device="cuda").bfloat16()
    with PromptCache(so, ps, 2, 2, 64, page=16, room=16, max_rows=4) as c:
        c.prefill(x, x, x)
        c.cut(64)
        assert c.pages.lens.tolist() == [80] * 6
        for _ in range(15):                      # a token of each of four rows is accepted
            _, lse = c.step(x[:24], x[:24], x[:24])
            c.append(x[:24], x[:24], x[:24], lse, torch.arange(0, 24, 4, device="cuda"))
        assert c.pages.lens.tolist() == [95] * 6


def test_order_of_the_calls():
    import torch
    from paper_2606_09441_amd import SiftError
    from paper_2606_09441_amd.serve import PromptCache
    x = torch.randn(40, 2, 64, device="cuda").bfloat16()
    with PromptCache([0, 30, 40], [0, 2], 2, 2, 64, page=16, room=8, max_rows=2) as c:
        for call in (lambda: c.cut(8), lambda: c.step(x[:1], x[:1], x[:1])):
            with pytest.raises(SiftError) as e:
                call()
            assert e.value.status == 6
        c.prefill(x, x, x)
        with pytest.raises(SiftError) as e:
            c.prefill(x, x, x)
        assert e.value.status == 6


def test_answers_follow_the_first_cut():
    """A row taken in before it would lie behind a document's last page, where nothing
    sees it."""
    import torch
    from paper_2606_09441_amd import SiftError
    from paper_2606_09441_amd.serve import PromptCache
    x = torch.randn(40, 2, 64, device="cuda").bfloat16()
    lse, rows = torch.zeros(2, 2, device="cuda"), torch.arange(2, device="cuda")
    with PromptCache([0, 30, 40], [0, 2], 2, 2, 64, page=16, room=8, max_rows=2) as c:
        for prefilled in (False, True):
            with pytest.raises(SiftError) as e:
                c.append(x[:2], x[:2], x[:2], lse, rows)
            assert e.value.status == 6
            if not prefilled:
                c.prefill(x, x, x)
        assert c.pages.lens.tolist() == [30] and c.next_pos.tolist() == [40]


def test_a_refused_append_changes_nothing():
    """It can be made again after a cut, and then gives what it would have given."""
    import torch
    from paper_2606_09441_amd import SiftError
    from paper_2606_09441_amd.serve import PromptCache
    gen = torch.Generator("cuda").manual_seed(4)
    draw = lambda n: torch.randn(n, 2, 64, generator=gen, device="cuda").bfloat16()  # noqa: E731
    rows = torch.arange(2, device="cuda")
    x, steps = draw(40), [draw(2) for _ in range(30)]
    state = lambda c: [t.clone() for t in (c.weights, c.pages.lens, c.pages.key_pos, c.next_pos,  # noqa: E731
                                           c.pages.k_pages, c.pages.v_pages)] + [c.used]
    same = lambda a, b: all(torch.equal(s, t) for s, t in zip(a[:-1], b[:-1])) and a[-1] == b[-1]  # noqa: E731

    def run(cut_at):
        """The states after each step; cuts before step cut_at, or where a step is refused."""
        after, refused = [], None
        with PromptCache([0, 30, 40], [0, 2], 2, 2, 64, page=16, room=8, max_rows=2) as c:
            c.prefill(x, x, x)
            c.cut(100)
            for i, q in enumerate(steps[:16]):
                _, lse = c.step(q, q, q)
                if i == cut_at:
                    c.cut(20)
                before = state(c)
                try:
                    c.append(q, q, q, lse, rows, decay=0.5)
                except SiftError as e:
                    assert e.status == 5 and refused is None and same(before, state(c))
                    refused = i
                    c.cut(20)
                    c.append(q, q, q, lse, rows, decay=0.5)
                after.append(state(c))
        return after, refused

    first, at = run(None)
    assert at is not None
    again, none = run(at)
    assert none is None
    assert all(same(a, b) for a, b in zip(first, again))


def test_append_checks_its_rows_first():
    import torch
    from paper_2606_09441_amd import SiftError
    from paper_2606_09441_amd.serve import PromptCache
    x = torch.randn(40, 2, 64, device="cuda").bfloat16()
    rows = torch.arange(2, device="cuda")
    with PromptCache([0, 30, 40], [0, 2], 2, 2, 64, page=16, room=8, max_rows=2) as c:
        c.prefill(x, x, x)
        c.cut(100)
        _, lse = c.step(x[:2], x[:2], x[:2])
        before = c.weights.clone()
        for k, v in ((x[:2].float(), x[:2]), (x[:2], x[:2, :1])):
            with pytest.raises(SiftError) as e:
                c.append(x[:2], k, v, lse, rows)
            assert e.value.status == 2 and torch.equal(before, c.weights)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("dense", [False, True])
def test_new_keys_enter_with_the_weights_they_have_drawn(dtype, d, dense):
    """A query's or an answer's token has the weight that it and the later tokens of
    its prompt, taken in with it, give it."""
    import torch
    from paper_2606_09441_amd.serve import PromptCache
    hq, hkv, g = 6, 2, 3
    so, ps = [0], [0]
    for p in PROMPTS:
        for n in p:
            so.append(so[-1] + n)
        ps.append(len(so) - 1)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator("cuda").manual_seed(6)
    draw = lambda n, h: torch.randn(n, h, d, generator=gen, device="cuda").to(dt)  # noqa: E731
    host = lambda t: t.double().cpu().numpy()  # noqa: E731
    slopes = [.5, .1, .02, .3, .05, .01] if dense else [0.0] * 6
    cap = 10.0 if dense else 0.0
    score = dict(cap=cap, slopes=torch.tensor(slopes, device="cuda"), scale=0.2) if dense else {}
    scale = 0.2 if dense else d ** -0.5
    # scores and log sums are within 1e-4 (tests of the operators), weights so relative to them
    REL = 2e-4

    def drawn(q, k, lse, pos):
        """[n, Hkv] of a prompt's new tokens."""
        w = np.zeros((len(q), hkv))
        for i in range(len(q)):
            for h in range(hq):
                s = S.scores(q[i, h], k[:i + 1, h // g], scale, cap, slopes[h], pos[i] - pos[:i + 1])
                w[:i + 1, h // g] += np.exp(s - lse[i, h])
        return w

    q, k, v = draw(so[-1], hq), draw(so[-1], hkv), draw(so[-1], hkv)
    with PromptCache(so, ps, hq, hkv, d, page=32, room=64, max_rows=4, dtype=dt) as c:
        bits = [torch.full((c.plan.info[x],), 255, dtype=torch.uint8, device="cuda")
                for x in ("la_bytes", "ca_bytes")] if not dense else (None, None)
        c.prefill(q, k, v, *bits, **score)
        _, lse = S.dense(host(q), host(k), host(v), so, ps, "causal", scale, cap, slopes)
        c.cut(24, sinks=2)
        for b in range(4):
            n, a, z = int(c.pages.lens[b]), so[ps[b + 1] - 1], so[ps[b + 1]]
            want = drawn(host(q)[a:z], host(k)[a:z], lse[a:z], np.arange(a, z))
            got = host(c.weights[b, :, n - (z - a):n]).T
            assert np.max(np.abs(got / want - 1)) <= REL
            assert not bool(c.weights[b, :, n:].any())
        for accepted in ([0, 1, 3, 4, 5, 8], [7], [1, 2, 12, 13, 14, 15]):
            before, lens = c.weights.clone(), c.pages.lens.tolist()
            qn, kn, vn = draw(16, hq), draw(16, hkv), draw(16, hkv)
            _, lse = c.step(qn, kn, vn)
            at = c.next_pos.cpu().numpy().repeat(4) + np.arange(16) % 4
            rows = torch.tensor(accepted, device="cuda")
            c.append(qn, kn, vn, lse, rows, decay=0.5)
            for b in range(4):
                r = [x for x in accepted if x // 4 == b]
                want = drawn(host(qn)[r], host(kn)[r], host(lse)[r], at[r])
                got = host(c.weights[b, :, lens[b]:lens[b] + len(r)]).T
                assert int(c.pages.lens[b]) == lens[b] + len(r)
                assert not len(r) or np.max(np.abs(got / want - 1)) <= REL
                # the others' share of the accepted rows: no less than what decay leaves
                assert bool((c.weights[b, :, :lens[b]] >= 0.5 * before[b, :, :lens[b]]).all())


def test_answers_outlast_a_cut_without_protection():
    """Tokens that their own rows attend to are not the first to go."""
    import torch
    from paper_2606_09441_amd.serve import PromptCache
    gen = torch.Generator("cuda").manual_seed(7)
    draw = lambda n: torch.randn(n, 1, 64, generator=gen, device="cuda").bfloat16()  # noqa: E731
    x = draw(330)
    with PromptCache([0, 300, 330], [0, 2], 1, 1, 64, page=32, room=32, max_rows=1) as c:
        c.prefill(x, x, x)
        c.cut(100, sinks=0)
        for _ in range(10):
            q = 3 * draw(1)                   # 24 at itself, far above the others' scores
            _, lse = c.step(q, q, q)
            c.append(q, q, q, lse, torch.zeros(1, dtype=torch.int64, device="cuda"))
        c.cut(60, sinks=0)
        assert set(range(330, 340)) <= set(c.pages.key_pos[0, 0, :60].tolist())


@pytest.mark.parametrize("sparse", [True, False])
@pytest.mark.parametrize("prompts", [[[30, 0]], [[40, 7, 0], [5], [33, 0]]])
def test_prompts_without_a_query(prompts, sparse):
    """Documents alone: all keys draw nothing, the lowest slots stay."""
    import torch
    from paper_2606_09441_amd.serve import PromptCache
    so, ps = [0], [0]
    for p in prompts:
        for n in p:
            so.append(so[-1] + n)
        ps.append(len(so) - 1)
    x = torch.randn(so[-1], 2, 64, device="cuda")
    with PromptCache(so, ps, 2, 2, 64, page=16, room=8, max_rows=2,
                     dtype=torch.float32) as c:
        bits = [torch.full((c.plan.info[n],), 255, dtype=torch.uint8, device="cuda")
                for n in ("la_bytes", "ca_bytes")] if sparse else (None, None)
        c.prefill(x, x, x, *bits)
        c.cut(16, sinks=0)
        docs, query = [sum(p[:-1]) for p in prompts], [p[-1] for p in prompts]
        assert c.pages.lens.tolist() == [min(16, n) + m for n, m in zip(docs, query)]
        assert c.pages.key_pos[0, 0, :16].tolist() == list(range(16))
        out, lse = c.step(x[:2 * len(prompts)], x[:2 * len(prompts)], x[:2 * len(prompts)])
        assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())


def test_a_long_query_draws_weights_in_parts():
    """More scores than are made at a time."""
    import torch
    from paper_2606_09441_amd.serve import PromptCache
    n, hq, hkv, d = 2100, 8, 2, 64
    assert hq * n * n > 2 << 24
    gen = torch.Generator("cuda").manual_seed(8)
    draw = lambda h: torch.randn(n + 10, h, d, generator=gen, device="cuda")  # noqa: E731
    q, k, v = draw(hq), draw(hkv), draw(hkv)
    host = lambda t: t.double().cpu().numpy()  # noqa: E731
    with PromptCache([0, 10, n + 10], [0, 2], hq, hkv, d, page=64, dtype=torch.float32) as c:
        c.prefill(q, k, v)
        c.cut(10, sinks=0)
        got = host(c.weights[0, :, 10:n + 10])
    want = np.zeros((hkv, n))
    for h in range(hq):
        s = host(q[10:, h]) @ host(k[:, h // 4]).T * d ** -0.5
        s[:, 10:][np.triu_indices(n, 1)] = -np.inf
        m = s.max(1, keepdims=True)
        w = np.exp(s - m)
        want[h // 4] += (w / w.sum(1, keepdims=True))[:, 10:].sum(0)
    assert np.max(np.abs(got / want - 1)) <= 2e-4      # scores and log sums within 1e-4
