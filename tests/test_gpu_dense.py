"""GPU tests of the dense attention with transformed scores (sift_plan_dense)
against the fp64 oracle, element by element."""

from __future__ import annotations

import numpy as np
import pytest

from gpu_helpers import device, max_abs, say
from oracle import serve_oracle as S

pytestmark = pytest.mark.gpu

# Inputs are N(0, 1) with a few keys four times as long.  Outputs: the project's
# bars.  The log sum: a score is a sum of up to 128 products in fp32 (error at
# most 128 * 2^-24 * sum|q k| * scale, about 1e-4 at |s| ~ 16 and 1e-5 in
# practice); the hardware's exp2 and the polynomial add a few 2^-24 of it.
TOL = {"f32": 1e-5, "bf16": 2e-2}
LSE_TOL = 1e-4

LAYOUTS = {
    # prompts as lists of segment lengths, the query last
    "one_token": [[1, 0]],
    "edges": [[64, 63, 65, 1, 33], [1, 128, 1], [127, 129, 32, 0]],
    "long": [[200, 300, 77]],
    "query_only": [[130], [1]],
}


def layout(prompts):
    so, ps = [0], [0]
    for p in prompts:
        for n in p:
            so.append(so[-1] + n)
        ps.append(len(so) - 1)
    return so, ps


def inputs(n, hq, hkv, d, dtype, seed=0):
    import torch
    rng = np.random.default_rng(seed)
    q = rng.standard_normal((n, hq, d)).astype(np.float32)
    k = rng.standard_normal((n, hkv, d)).astype(np.float32)
    k *= np.where(rng.random((n, hkv, 1)) < 0.05, 4.0, 1.0).astype(np.float32)
    v = rng.standard_normal((n, hkv, d)).astype(np.float32)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    dev = [torch.from_numpy(x).to(device()).to(dt) for x in (q, k, v)]
    return dev, [x.float().cpu().numpy() for x in dev]


def run(prompts, hq, hkv, d, dtype, mask, cap=0.0, bias=False, scale=None, seed=0, tile=64,
        by_head=False, want_lse=True, slope=None):
    """(out, lse) of the library and of the oracle."""
    import torch
    from paper_2606_09441_amd import Plan
    so, ps = layout(prompts)
    n = so[-1]
    (q, k, v), (qn, kn, vn) = inputs(n, hq, hkv, d, dtype, seed)
    slopes = (2.0 ** (-4.0 * np.arange(1, hq + 1) / hq)).astype(np.float32) if bias else None
    if slope is not None:
        slopes = (slope * np.arange(1, hq + 1) / hq).astype(np.float32)
    lse = torch.full((n, hq), 7.0, device=q.device)
    with Plan(so, ps, hq, hkv, d, tile) as plan:
        out = plan.dense(q, k, v, mask=mask, scale=scale, cap=cap, lse=lse if want_lse else None,
                         slopes=None if slopes is None else torch.from_numpy(slopes).to(q.device))
        torch.cuda.synchronize()
    want = (S.dense_by_head if by_head else S.dense)(qn, kn, vn, so, ps, mask, scale, cap, slopes)
    return out.float().cpu().numpy(), lse.cpu().numpy(), *want


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("mask", ["causal", "document", "prefix"])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (2.0, False), (50.0, False), (0.0, True),
                                      (20.0, True)])
def test_masks_and_scores(dtype, d, mask, cap, bias):
    for name, prompts in LAYOUTS.items():
        out, lse, ref, ref_lse = run(prompts, 6, 2, d, dtype, mask, cap, bias)
        e, el = max_abs(out, ref), max_abs(lse, ref_lse)
        say(f"{name} {dtype} {d} {mask} cap {cap} bias {bias}: {e:.2e}, lse {el:.2e}")
        assert e <= TOL[dtype] and el <= LSE_TOL


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("mask", ["causal", "document", "prefix"])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (2.0, False), (50.0, False), (0.0, True),
                                      (20.0, True)])
def test_many_heads(dtype, d, mask, cap, bias):
    """Enough records and heads for the 128-row workgroups; with and without lse."""
    prompts = [[64, 63, 65, 1, 33], [1, 128, 1], [300, 129, 77], [200, 0]]
    out, lse, ref, ref_lse = run(prompts, 24, 8, d, dtype, mask, cap, bias, by_head=True)
    bare = run(prompts, 24, 8, d, dtype, mask, cap, bias, by_head=True, want_lse=False)[0]
    e, el = max_abs(out, ref), max_abs(lse, ref_lse)
    say(f"{dtype} {d} {mask} cap {cap} bias {bias}: {e:.2e}, lse {el:.2e}")
    assert e <= TOL[dtype] and el <= LSE_TOL
    assert max_abs(bare, ref) <= TOL[dtype]


@pytest.mark.parametrize("hq,hkv", [(4, 2), (40, 8)])
@pytest.mark.parametrize("slope", [-0.7, -3.0, 5.0, 300.0])
def test_steep_and_negative_slopes(hq, hkv, slope):
    """Far keys favoured, and weights that vanish within a tile."""
    for dtype in ("bf16", "f32"):
        for mask in ("causal", "prefix"):
            out, lse, ref, ref_lse = run([[150, 300, 77], [130, 5]], hq, hkv, 64, dtype, mask,
                                         bias=True, by_head=True, slope=slope)
            assert max_abs(out, ref) <= TOL[dtype]
            # |slope| * distance in fp32: relative 2^-23
            assert np.max(np.abs(lse - ref_lse) / np.maximum(1.0, np.abs(ref_lse) / 30)) <= LSE_TOL


@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 8), (5, 5), (6, 3), (16, 16), (12, 4)])
def test_head_layouts(hq, hkv):
    """Every assignment of records and heads to workgroups."""
    for dtype in ("bf16", "f32"):
        out, lse, ref, ref_lse = run([[130, 70, 40], [20, 5]], hq, hkv, 64, dtype, "causal")
        assert max_abs(out, ref) <= TOL[dtype] and max_abs(lse, ref_lse) <= LSE_TOL


def test_scale():
    out, lse, ref, ref_lse = run([[100, 30]], 2, 1, 128, "bf16", "causal", scale=0.03)
    assert max_abs(out, ref) <= TOL["bf16"] and max_abs(lse, ref_lse) <= LSE_TOL


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("hq,hkv", [(2, 1), (72, 1)])
def test_unseen_keys_do_not_matter(dtype, value, hq, hkv):
    """A key with such values only reaches the rows that see it: under the causal
    mask the rows from it on, and no other prompt's."""
    import torch
    from paper_2606_09441_amd import Plan
    so, ps = layout([[90, 60], [40, 10]])
    n, bad = so[-1], 70
    (q, k, v), (qn, kn, vn) = inputs(n, hq, hkv, 128, dtype)
    k[bad], v[bad] = value, value
    v[bad, :, 3:] = 0.5         # the other dims of a visible key stay as they are ...
    k[bad] = 0.25               # ... where its scores are finite
    kn, vn = k.float().cpu().numpy(), v.float().cpu().numpy()
    with Plan(so, ps, hq, hkv, 128, 64) as plan:
        out = plan.dense(q, k, v).float().cpu().numpy()
        k[bad] = value          # and a score that is none
        worse = plan.dense(q, k, v).float().cpu().numpy()
    rows = np.r_[0:bad, 150:n]
    with np.errstate(all="ignore"):
        ref, _ = S.dense(qn, kn, vn, so, ps, "causal")
    assert max_abs(out[rows], ref[rows]) <= TOL[dtype]
    assert max_abs(worse[rows], ref[rows]) <= TOL[dtype]
    assert max_abs(out[bad:150, :, 3:], ref[bad:150, :, 3:]) <= TOL[dtype]
    got, want = out[bad:150, :, :3], ref[bad:150, :, :3]
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got[~np.isnan(got)], want[~np.isnan(want)])


def test_same_as_sparse_path():
    """All-ones bits make the sparse attention dense causal: the two agree, on a
    plan that has run both in turn."""
    import torch
    import workloads as W
    from gpu_helpers import DevWorkload
    wl = W.all_ones(W.custom([[200, 64, 70], [96, 33]], tile=64, hq=4, hkv=2, d=128, dtype="bf16",
                             seed=1))
    dw = DevWorkload(wl)
    a = dw.run().clone()
    b = dw.plan.dense(dw.q, dw.k, dw.v)
    c = dw.run()
    torch.cuda.synchronize()
    dw.close()
    assert torch.equal(a, c)
    assert max_abs(a.float().cpu(), b.float().cpu()) <= TOL["bf16"]


def test_streams_and_repeats():
    """The same bits on another stream, in a captured graph and on its replays."""
    import torch
    from paper_2606_09441_amd import Plan
    so, ps = layout([[150, 60], [33, 0]])
    (q, k, v), _ = inputs(so[-1], 4, 2, 128, "bf16")
    with Plan(so, ps, 4, 2, 128, 64) as plan:
        first = plan.dense(q, k, v, mask="prefix", cap=30.0)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        out = torch.zeros_like(q)
        with torch.cuda.stream(side):
            plan.dense(q, k, v, mask="prefix", cap=30.0, out=out)
        side.synchronize()
        assert torch.equal(out, first)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            plan.dense(q, k, v, mask="prefix", cap=30.0, out=out)
        for _ in range(3):
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, first)


def test_refusals():
    import torch
    from paper_2606_09441_amd import Plan, SiftError
    so, ps = layout([[100, 30]])
    (q, k, v), _ = inputs(130, 4, 2, 128, "bf16")
    with Plan(so, ps, 4, 2, 128, 64) as plan:
        def refused(status, *a, **kw):
            with pytest.raises(SiftError) as e:
                plan.dense(*a, **kw)
            assert e.value.status == status
        refused(4, q, k, v, mask="sideways")
        refused(4, q, k, v, cap=-1.0)
        refused(4, q, k, v, cap=float("nan"))
        refused(4, q, k, v, cap=float("inf"))
        refused(2, q[:-1], k, v)
        refused(2, q, k[:, :1].contiguous(), v)
        refused(4, q, k.float(), v)
        refused(4, q, k, v, out=q.float())
        refused(5, q, k, v, slopes=torch.zeros(3, device=q.device))
        refused(4, q, k, v, slopes=torch.zeros(4))
        refused(5, q, k, v, lse=torch.zeros(130, 3, device=q.device))
        odd = torch.empty(q.numel() + 1, dtype=q.dtype, device=q.device)[1:].view_as(q)
        refused(4, odd, k, v)


def test_offsets_beyond_32_bits():
    """Queries and outputs of more than 2^31 elements: the last prompt's rows equal
    those of the same prompt alone."""
    import torch
    from paper_2606_09441_amd import Plan
    one = [128] * 54 + [16]
    so, ps = layout([one] * 51)
    n, hq, hkv, d = so[-1], 48, 8, 128
    assert n * hq * d > 1 << 31
    gen = torch.Generator(device=device()).manual_seed(1)
    q = torch.empty(n, hq, d, dtype=torch.bfloat16, device=device())
    for i in range(0, n, 1 << 16):
        q[i:i + (1 << 16)].normal_(generator=gen)
    k = torch.randn(n, hkv, d, generator=gen, device=device()).to(torch.bfloat16)
    v = torch.randn(n, hkv, d, generator=gen, device=device()).to(torch.bfloat16)
    with Plan(so, ps, hq, hkv, d, 128) as plan:
        out = plan.dense(q, k, v, mask="document", cap=50.0)
    a = so[ps[-2]]
    so1, ps1 = layout([one])
    with Plan(so1, ps1, hq, hkv, d, 128) as plan:
        alone = plan.dense(q[a:].contiguous(), k[a:].contiguous(), v[a:].contiguous(),
                           mask="document", cap=50.0)
    torch.cuda.synchronize()
    assert torch.equal(out[a:], alone)


def lse_error(lse, ref):
    """Largest error of log sums, |slope| * distance in fp32 among their terms
    (relative 2^-23)."""
    return np.max(np.abs(lse - ref) / np.maximum(1.0, np.abs(ref) / 30))


@pytest.mark.parametrize("cap", [0.0, 300.0])
@pytest.mark.parametrize("mask", ["causal", "document", "prefix"])
@pytest.mark.parametrize("slope", [2.0, 4.0, -3.0])
def test_bias_beside_widely_spread_products(slope, mask, cap):
    """Scores of standard deviation 9 (36 for some keys) under slopes that no key's
    neighbours share: the largest product and the largest bias of a tile are of
    different keys, hundreds apart."""
    for d in (64, 128):
        out, lse, ref, ref_lse = run([[150, 300, 77], [130, 5]], 40, 8, d, "bf16", mask, cap, True,
                                     scale=9 * d ** -0.5, by_head=True, slope=slope)
        say(f"slope {slope} {mask} cap {cap} {d}: {max_abs(out, ref):.2e}, {lse_error(lse, ref_lse):.2e}")
        assert max_abs(out, ref) <= TOL["bf16"] and lse_error(lse, ref_lse) <= LSE_TOL


@pytest.mark.parametrize("slope,score", [(1.5, 90.0), (2.0, 100.0), (2.0, 120.0), (-1.5, 90.0)])
def test_a_far_key_with_a_large_score(slope, score):
    """It is the largest product of a tile whose nearest key has the largest bias."""
    import torch
    from paper_2606_09441_amd import Plan
    so, ps = layout([[300, 20]])
    n, hq, hkv, d = so[-1], 128, 8, 64
    (q, k, v), _ = inputs(n, hq, hkv, d, "bf16", 5)
    unit = q[256].view(hkv, hq // hkv, d)[:, 0].float()
    k[192] = (unit * (score * d ** 0.5 / (unit * unit).sum(1, keepdim=True))).to(k.dtype)
    slopes = torch.full((hq,), slope, device=q.device)
    lse = torch.empty(n, hq, device=q.device)
    with Plan(so, ps, hq, hkv, d, 64) as plan:
        out = plan.dense(q, k, v, slopes=slopes, lse=lse)
    f = lambda x: x.float().cpu().numpy()  # noqa: E731
    ref, ref_lse = S.dense_by_head(f(q), f(k), f(v), so, ps, "causal", None, 0.0, f(slopes))
    assert max_abs(f(out), ref) <= TOL["bf16"] and lse_error(f(lse), ref_lse) <= LSE_TOL


def test_scales_and_caps_that_fp32_does_not_hold():
    """Their coefficients would be infinite, and a score of 0 no number."""
    import torch
    from paper_2606_09441_amd import Plan, SiftError
    so, ps = layout([[40, 10]])
    (q, k, v), (qn, kn, vn) = inputs(50, 2, 1, 128, "f32")
    q[:, 0], qn[:, 0] = 0, 0
    with Plan(so, ps, 2, 1, 128, 64) as plan:
        for kw in (dict(cap=5e-7), dict(cap=1e-20), dict(scale=3e38), dict(scale=1e30, cap=1.0)):
            with pytest.raises(SiftError) as e:
                plan.dense(q, k, v, **kw)
            assert e.value.status == 4
        for kw in (dict(cap=1e-6), dict(cap=1e15), dict(scale=1e30)):
            out = plan.dense(q, k, v, **kw).cpu().numpy()
            ref = S.dense(qn, kn, vn, so, ps, "causal", **kw)[0]
            assert max_abs(out[:, 0], ref[:, 0]) <= TOL["f32"]
            if "cap" in kw:
                assert max_abs(out, ref) <= TOL["f32"]
