"""GPU: attention over e4m3 pages whose scales lie at the ends of their range, 2^-100 and
2^120 (sift_cache_attention with SIFT_E4M3 pools): what a page's scale is changes neither
the weights of its keys nor their sums; and appends to pages whose scales lie beyond.

In the former all sequences have the same pages, so that there are as many units as workgroups and one
goes over a sequence from its first key to its last, with the reference that its first
tiles left.  Every new token sees the cache and itself."""

import numpy as np
import pytest
import torch

from gpu_helpers import device, max_abs, say

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn
LSE_TOL = 1e-4
Q = 8.0625      # of dim 0; the scale is 1 / 8, so a score is 1.0078125 times a key's dim 0
D = 64

# (sequences, new tokens, query heads of the one kv head): narrow units and wide ones
UNITS = {"narrow": (512, 1, 1), "wide": (64, 32, 32)}


class Shared:
    """n slots of dims 0 k0 [n] and codes v [n, D], with scales for each page."""

    def __init__(self, units, page, k0, v, k_scale, v_scale, q=Q):
        from paper_2606_09441_amd import Cache, CachePages
        self.B, self.new, self.hq = UNITS[units]
        dev, n = device(), len(k0)
        pages = -(-n // page)
        f32 = lambda x: torch.as_tensor(np.asarray(x, np.float32)).to(dev)  # noqa: E731
        k = np.zeros((pages * page, D), np.float32)
        k[:n, 0] = k0
        codes = np.zeros((pages * page, D), np.float32)
        codes[:n] = v
        self.k0, self.q = np.asarray(k0, np.float64), q
        self.v = np.asarray(v, np.float64) * np.repeat(np.asarray(v_scale, np.float64), page)[:n, None]
        self.scales = [f32(x).view(pages, 1) for x in (k_scale, v_scale)]
        per_row = self.scales[0].repeat_interleave(page, 0)
        self.codes = [(f32(k) / per_row).to(E4M3).view(-1, 1, D), f32(codes).to(E4M3).view(-1, 1, D)]
        assert torch.equal(self.codes[0].float().view(-1, D) * per_row, f32(k))
        assert torch.equal(self.codes[1].float().view(-1, D), f32(codes))
        table = torch.arange(pages, dtype=torch.int32, device=dev).expand(self.B, -1).contiguous()
        self.lens = torch.full((self.B,), n, dtype=torch.int32, device=dev)
        self.kv = CachePages(*self.codes, table, self.lens, k_scales=self.scales[0],
                             v_scales=self.scales[1])
        self.cache = Cache(self.B, self.hq, 1, D, page=page, max_pages=pages, max_rows=self.new)

    def attention(self, own, **score):
        """(out, lse) of a sequence, on the host; `own`: the new tokens' values."""
        rows, dev = self.B * self.new, device()
        q = torch.zeros(rows, self.hq, D, dtype=torch.bfloat16, device=dev)
        q[..., 0] = self.q
        k_new = torch.zeros(rows, 1, D, dtype=torch.bfloat16, device=dev)
        mask = torch.tensor([1 << i for i in range(self.new)] * self.B, device=dev).view(rows, 1)
        lse = torch.full((rows, self.hq), 7.0, device=dev)
        out = self.cache.attention(q, k_new, torch.full_like(k_new, own), self.kv, tree_mask=mask,
                                   lse=lse, **score)
        torch.cuda.synchronize()
        self.cache.close()
        shape = (self.B, self.new, self.hq)
        out, lse = out.float().view(*shape, D), lse.view(shape)
        assert torch.equal(out, out[:1].expand_as(out)) or torch.isnan(out).any()
        return out[0].double().cpu().numpy(), lse[0].double().cpu().numpy()

    def exact(self, own, cap=0.0, slopes=None):
        """(out, lse, sum w |v|) in 64 bits, [new, hq, ..]."""
        n, i = len(self.k0), np.arange(self.new)
        s = np.concatenate([self.k0, [0.0]]) * (self.q / 8)
        if cap:
            s = cap * np.tanh(s / cap)
        s = np.broadcast_to(s, (self.new, self.hq, n + 1)).copy()
        if slopes is not None:
            far = np.concatenate([n + i[:, None] - np.arange(n), np.zeros((self.new, 1))], 1)
            s -= np.asarray(slopes, np.float64)[None, :, None] * far[:, None]
        top = s.max(-1, keepdims=True)
        w = np.exp(s - top)
        lse = (top + np.log(w.sum(-1, keepdims=True)))[..., 0]
        w /= w.sum(-1, keepdims=True)
        v = np.concatenate([self.v, np.full((1, D), own)])
        return w @ v, lse, w @ np.abs(v)


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("units,n", [("narrow", 131072), ("wide", 32768)])
def test_light_keys_of_pages_whose_values_are_zero(units, n, page):
    """One heavy key, then n - 1 of weights 2^-26.2 of its: their pages' V is all zero, so
    that its scale is the least, and their part of a row's sum is the sum of as many weights
    all the same, 4e-4 of it for those of a wavefront.

    Tolerance: of the log sum that of other caches, 1e-4, and the additions of light weights
    to a sum of 1 or more and below 2, each off by 2^-24 at most.  There is one addition
    for 16 keys (narrow, 8 of them in each of two lanes; a wavefront has a quarter of the
    tiles) or for a page's part of 64 keys (wide)."""
    k0 = np.zeros(n)
    k0[0] = 18.0
    pages = n // page
    k_scale = np.full(pages, 2.0 ** -100)
    k_scale[0] = 2.0 ** -4
    x = Shared(units, page, k0, np.zeros((n, D)), k_scale, np.full(pages, 2.0 ** -100))
    out, lse = x.attention(1.0)
    ref, ref_lse, _ = x.exact(1.0)
    adds = n // 64 if units == "narrow" else n // min(page, 64)
    tol = LSE_TOL + adds * 2.0 ** -24
    say(f"[scales] {units} {page}: lse {max_abs(lse, ref_lse):.2e} of {tol:.2e}")
    some = n / 4 if units == "narrow" else n             # light keys of a wavefront
    assert some * np.exp(-18.0 * Q / 8) > 1.5 * tol      # it shows where they are left out
    assert max_abs(lse, ref_lse) <= tol
    # the new token's weight, in bf16 over such a sum, and the output in bf16
    assert (np.abs(out - ref) <= ref * (2.0 ** -8 + 2.0 ** -8 + tol)).all()


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("score", ["plain", "cap", "bias"])
@pytest.mark.parametrize("scale", [2.0 ** -100, 1.5 * 2.0 ** -99, 2.0 ** -60, 2.0 ** 60, 2.0 ** 100,
                                   1.75 * 2.0 ** 100, 1.5 * 2.0 ** 119, 2.0 ** 120])
@pytest.mark.parametrize("units,n", [("narrow", 300), ("wide", 1030)])
def test_values_at_the_ends_of_the_range(units, n, scale, score, page):
    """Values of 2^-9 to 2^-6 scales, so that 2^13 times the largest is a number too: with
    scores that grow by 5, 7.3 in powers of 2, after the first 128 keys, the weights
    reach 2^7.3 of the reference that those left, and their sum stays below 2^13 of it.

    The weights are rounded to bf16, 2^-8, in the numerator and the denominator, and the
    output by 2^-8; scores in fp32 are off by less than 1e-5, which is as much of a weight."""
    rng = np.random.default_rng(5)
    k0 = np.where(np.arange(n) < 128, 0.0, 5.0)
    v = rng.choice([-1.0, 1.0], (n, D)) * np.exp2(rng.integers(-9, -5, (n, D)))
    pages = -(-n // page)
    x = Shared(units, page, k0, v, np.full(pages, 2.0 ** -5), np.full(pages, scale))
    kw = {"cap": dict(cap=30.0), "bias": dict(slopes=np.full(x.hq, 2.0 ** -10, np.float32)),
          "plain": {}}[score]
    ref, ref_lse, size = x.exact(0.0, **kw)
    if score == "bias":
        kw = dict(slopes=torch.from_numpy(kw["slopes"]).to(device()))
    out, lse = x.attention(0.0, **kw)
    e = float((np.abs(out - ref) / (np.abs(ref) * 2.0 ** -8 + size * (2.0 ** -7 + 2e-5))).max())
    say(f"[scales] {units} {page} {score} {scale:.3g}: {e:.2f} of the bound, lse "
        f"{max_abs(lse, ref_lse):.2e}")
    assert max_abs(lse, ref_lse) <= LSE_TOL
    assert e <= 1


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("score", ["plain", "cap", "bias"])
@pytest.mark.parametrize("scale", [2.0 ** -100, 1.5 * 2.0 ** -99, 2.0 ** 100, 2.0 ** 120])
@pytest.mark.parametrize("units,n", [("narrow", 300), ("wide", 1030)])
def test_keys_at_the_ends_of_the_range(units, n, scale, score, page):
    """The same for K: queries as small as the keys are large leave the scores what they
    are, and the bounds with them."""
    rng = np.random.default_rng(6)
    k0 = np.where(np.arange(n) < 128, 0.0, rng.choice([2.0, 5.0, -7.0], n))
    v = rng.integers(-7, 8, (n, D)) / 4.0
    pages = -(-n // page)
    x = Shared(units, page, k0 * scale, v, np.full(pages, scale), np.ones(pages),
               Q / 2.0 ** np.floor(np.log2(scale)))
    kw = {"cap": dict(cap=30.0), "bias": dict(slopes=np.full(x.hq, 2.0 ** -10, np.float32)),
          "plain": {}}[score]
    ref, ref_lse, size = x.exact(0.0, **kw)
    if score == "bias":
        kw = dict(slopes=torch.from_numpy(kw["slopes"]).to(device()))
    out, lse = x.attention(0.0, **kw)
    e = float((np.abs(out - ref) / (np.abs(ref) * 2.0 ** -8 + size * (2.0 ** -7 + 2e-5))).max())
    say(f"[scales] {units} {page} {score} K {scale:.3g}: {e:.2f} of the bound, lse "
        f"{max_abs(lse, ref_lse):.2e}")
    assert max_abs(lse, ref_lse) <= LSE_TOL
    assert e <= 1


@pytest.mark.parametrize("page,d", [(16, 64), (64, 128)])
@pytest.mark.parametrize("scale,taken", [
    (0.0, 2.0 ** -100), (-1.0, 2.0 ** -100), (2.0 ** -110, 2.0 ** -100), (np.nan, 2.0 ** -100),
    (1e-40, 2.0 ** -100), (2.0 ** 121, 2.0 ** 120), (1.5 * 2.0 ** 127, 2.0 ** 120),
    (np.inf, 2.0 ** 120), (2.0 ** -100, 2.0 ** -100), (2.0 ** 120, 2.0 ** 120)])
def test_appends_take_a_scale_as_the_attention_does(scale, taken, page, d):
    """A page begun under a scale out of range: new rows of zeros leave the keys that it
    holds what they were, to the bit, and its scale becomes the one in range."""
    from paper_2606_09441_amd import Cache, CachePages
    dev, hkv, held, new = device(), 2, 9, 5
    rng = np.random.default_rng(1)
    x = rng.choice([-1.0, 1.0], (2, page, hkv, d)) * np.exp2(rng.integers(-9, -5, (2, page, hkv, d)))
    was = torch.from_numpy(x.astype(np.float32)).to(dev)
    k, v = (t.to(E4M3) for t in was)
    scales = [torch.full((1, hkv), scale, device=dev) for _ in range(2)]
    lens = torch.tensor([held], dtype=torch.int32, device=dev)
    kv = CachePages(k, v, torch.zeros(1, 1, dtype=torch.int32, device=dev), lens,
                    k_scales=scales[0], v_scales=scales[1])
    none = torch.zeros(1, hkv, d, dtype=torch.bfloat16, device=dev)
    zeros = torch.zeros(new, hkv, d, dtype=torch.bfloat16, device=dev)
    with Cache(1, hkv, hkv, d, page=page, max_pages=1, max_rows=1) as cache:
        before = cache.attention(none, none, none, kv)   # the values' mean
        grown = cache.append(kv, zeros, zeros)
        after = cache.attention(none, none, none, kv)
        torch.cuda.synchronize()
    assert grown.tolist() == [held + new]
    mean = was[1, :held].double().sum(0) * taken / (held + 1)
    # weights in bf16 over their own sum are the same; fp32 sums and the output in bf16
    size = was[1, :held].double().abs().sum(0) * taken / (held + 1)
    assert ((before[0].double() - mean).abs() <= mean.abs() * 2.0 ** -8 + size * 2.0 ** -20).all()
    assert torch.equal(before, after)
    for t, codes, now in zip(was, (k, v), scales):
        assert now.tolist() == [[taken] * hkv]
        assert torch.equal(codes[:held].float(), t[:held])
        assert not codes[held:held + new].float().any()
