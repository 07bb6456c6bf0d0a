"""GPU: PromptCache with rotary positions of its own, and with keys held in e4m3 after the
cut."""

import numpy as np
import pytest
import torch

from oracle import serve_oracle as S

pytestmark = pytest.mark.gpu

PROMPTS = [[130, 64, 1, 40], [77, 20], [5], [300, 31, 64, 16]]
HQ, HKV, D = 4, 2, 128


def layout():
    so, ps = [0], [0]
    for p in PROMPTS:
        for n in p:
            so.append(so[-1] + n)
        ps.append(len(so) - 1)
    return so, ps


def make(seed, **kw):
    from paper_2606_09441_amd.serve import PromptCache
    so, ps = layout()
    gen = torch.Generator("cuda").manual_seed(seed)
    dt, d = kw.pop("dtype", torch.bfloat16), kw.pop("d", D)
    draw = lambda n, h: torch.randn(n, h, d, generator=gen, device="cuda").to(dt)  # noqa: E731
    cache = PromptCache(so, ps, HQ, HKV, d, page=32, room=64, max_rows=4, dtype=dt, **kw)
    return cache, so, ps, draw


def positions(so, ps):
    return torch.tensor([t - so[a] for a, z in zip(ps, ps[1:]) for t in range(so[a], so[z])],
                        dtype=torch.int32, device="cuda")


def rotary(interleaved=False, d=D):
    from paper_2606_09441_amd import Rotary, rotary_frequencies
    return Rotary(rotary_frequencies(d // 2, 10000.0)[0], interleaved)


MASK, SEES = [1, 3, 5, 11], [[0], [0, 1], [0, 2], [0, 1, 3]]


def bits_of(c):
    return [torch.full((c.plan.info[x],), 255, dtype=torch.uint8, device="cuda")
            for x in ("la_bytes", "ca_bytes")]


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.float32, 64)])
@pytest.mark.parametrize("sparse", [True, False])
def test_keys_turned_here_are_those_turned_before(dtype, d, sparse):
    """The same bits as with q and k turned by the caller."""
    r = rotary(True, d)
    mine, so, ps, draw = make(3, dtype=dtype, d=d, rotary=r)
    theirs, *_ = make(3, dtype=dtype, d=d)
    q, k, v = draw(so[-1], HQ), draw(so[-1], HKV), draw(so[-1], HKV)
    args = bits_of(mine) if sparse else [None, None]
    score = {} if sparse else {"cap": 10.0}
    out = [mine.prefill(q, k, v, *args, **score),
           theirs.prefill(*r.rotate(q, k, positions(so, ps)), v, *args, **score)]
    assert torch.equal(*out)
    for c in (mine, theirs):
        c.cut(48, sinks=2, recent=3)
    mask = torch.tensor(MASK * 4, device="cuda").view(16, 1)
    depth = torch.tensor([0, 1, 1, 2] * 4, dtype=torch.int32, device="cuda")
    accepted = torch.tensor([0, 1, 3, 4, 8, 9], device="cuda")
    for _ in range(2):
        q, k, v = draw(16, HQ), draw(16, HKV), draw(16, HKV)
        at = (mine.next_pos.repeat_interleave(4) + depth).int()
        qr, kr = r.rotate(q, k, at)
        a = mine.step(q, k, v, tree_mask=mask, row_pos=at)
        b = theirs.step(qr, kr, v, tree_mask=mask, row_pos=at)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        mine.append(q, k, v, a[1], accepted, row_pos=at)
        theirs.append(qr, kr, v, b[1], accepted, row_pos=at)
    mine.cut(40)
    theirs.cut(40)
    for x in ("k_pages", "v_pages", "lens", "key_pos"):
        assert torch.equal(getattr(mine.pages, x), getattr(theirs.pages, x))
    assert torch.equal(mine.weights, theirs.weights)
    mine.close()
    theirs.close()


def test_keys_held_in_codes():
    """From prompts to answers over e4m3 pages.  The codes are near the keys,
    and the outputs those of the
    attention over the numbers that they stand for, to bf16's 2e-2."""
    r = rotary()
    held, so, ps, draw = make(5, rotary=r, held=torch.float8_e4m3fn)
    plain, *_ = make(5, rotary=r)
    q, k, v = draw(so[-1], HQ), draw(so[-1], HKV), draw(so[-1], HKV)
    assert torch.equal(held.prefill(q, k, v, *bits_of(held)), plain.prefill(q, k, v, *bits_of(plain)))
    for c in (held, plain):
        c.cut(48, sinks=2, recent=3)
    assert held.pages.k_pages.dtype is torch.float8_e4m3fn
    assert held.pages.k_pages.numel() < plain.pages.k_pages.numel()
    host = lambda t: t.float().cpu().numpy()  # noqa: E731

    def numbers(c, name):
        x = getattr(c.pages, name + "_pages").float()
        if c.pages.k_scales is None:
            return host(x)
        s = getattr(c.pages, name + "_scales")
        return host((x.view(-1, 32, HKV, D) * s[:, None, :, None]).view(-1, HKV, D))

    def rows(c, b):
        n, t = int(c.pages.lens[b]), c.pages.page_table[b].cpu().numpy()
        return np.array([t[i // 32] * 32 + i % 32 for i in range(n)], np.int64)

    def same_keys(slack):
        assert held.pages.lens.tolist() == plain.pages.lens.tolist()
        for b in range(4):
            n = int(held.pages.lens[b])
            assert torch.equal(held.pages.key_pos[b, :, :n], plain.pages.key_pos[b, :, :n])
            for x in "kv":
                a, z = numbers(held, x)[rows(held, b)], numbers(plain, x)[rows(plain, b)]
                s = host(getattr(held.pages, x + "_scales"))[rows(held, b) // 32]
                half = np.maximum(np.abs(z) * 2.0 ** -4, s[..., None] * 2.0 ** -10)
                worst = float((np.abs(a - z) / half).max())
                assert worst <= slack

    # A key's first rounding is half a step, max(|z| 2^-4, s_1 2^-10).  Where its page's scale
    # grows, at least doubling, it is rounded again by s_i 2^-10 at most: s_2 2^-10 + .. + s
    # 2^-10 < 2 s 2^-10.  So within 3 max(|z| 2^-4, s 2^-10); and z itself is a bf16, off by
    # 2^-8 of it from what an appended key is turned to: 2^-4 more.
    slack = 3 + 2.0 ** -4 + 2.0 ** -8
    same_keys(slack)
    mask = torch.tensor(MASK * 4, device="cuda").view(16, 1)
    depth = torch.tensor([0, 1, 1, 2] * 4, dtype=torch.int32, device="cuda")
    accepted = torch.tensor([0, 1, 3, 4, 8, 9], device="cuda")
    for step in range(6):
        q, k, v = draw(16, HQ), draw(16, HKV), draw(16, HKV)
        at = (held.next_pos.repeat_interleave(4) + depth).int()
        out, lse = held.step(q, k, v, tree_mask=mask, row_pos=at)
        qr, kr = r.rotate(q, k, at)
        pages = S.Pages(numbers(held, "k"), numbers(held, "v"), held.pages.page_table.cpu().numpy(),
                        held.pages.lens.cpu().numpy(), 32)
        sees = np.zeros((4, 4), bool)
        for i, x in enumerate(SEES):
            sees[i, x] = True
        ref, ref_lse = S.cache_attention(host(qr), host(kr), host(v), pages, np.arange(0, 17, 4),
                                         [sees] * 4)
        assert np.abs(host(out) - ref).max() <= 2e-2
        assert np.abs(host(lse) - ref_lse).max() <= 1e-4
        _, other = plain.step(q, k, v, tree_mask=mask, row_pos=at)
        held.append(q, k, v, lse, accepted, row_pos=at)
        plain.append(q, k, v, other, accepted, row_pos=at)
        assert held.next_pos.tolist() == plain.next_pos.tolist()
        same_keys(slack)
    from paper_2606_09441_amd import SiftError
    with pytest.raises(SiftError) as e:
        held.cut(40)
    assert e.value.status == 4
    held.close()
    plain.close()


def test_refused_types():
    from paper_2606_09441_amd import SiftError
    from paper_2606_09441_amd.serve import PromptCache
    so, ps = layout()
    for dtype, held in ((torch.float32, torch.float8_e4m3fn), (torch.bfloat16, torch.float16),
                        (torch.bfloat16, torch.float32)):
        with pytest.raises(SiftError) as e:
            PromptCache(so, ps, HQ, HKV, 64, dtype=dtype, held=held)
        assert e.value.status == 4


def test_views_that_are_no_plain_buffers():
    """Keys cut from a wider tensor, and from one that begins anywhere."""
    a, so, ps, draw = make(7)
    b, *_ = make(7)
    n = so[-1]
    wide = draw(n, HKV + 1)
    v = draw(n, HKV)
    odd = torch.empty(v.numel() + 1, dtype=v.dtype, device=v.device)[1:].view(v.shape).copy_(v)
    q = draw(n, HQ)
    out = [a.prefill(q, wide[:, 1:], odd, *bits_of(a)),
           b.prefill(q, wide[:, 1:].contiguous(), v, *bits_of(b))]
    assert torch.equal(*out)
    a.close()
    b.close()


def test_the_example_holds_codes(capsys):
    from paper_2606_09441_amd import serve
    serve.main()
    out = capsys.readouterr().out
    assert "of torch.bfloat16" in out and "of torch.float8_e4m3fn" in out
