"""GPU: rotary positions (sift_rotate, Rotary) against a plain computation in 64 bits.

An output is m (x cos a - y sin a), rounded once.  Off by at most
  bf16: |out| 2^-8 of the rounding, and (|x| + |y|) m 2^-16 of the hardware's cosine and
        sine (a fraction of a turn in fp32 is off by 2^-25, times 2 pi; the function and
        the products by some 2^-20)
  fp32: |out| 2^-24, and (|x| + |y|) m 2^-22: cosine and sine off by 2^-23 (the angle's
        rest rounded, its polynomial, the magnitude), two products and their sum by 2^-24
        each
"""

import numpy as np
import pytest
import torch

import workloads as W
from gpu_helpers import device, oracle_layout, say
from oracle import layer_oracle as LO

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def turned(x, positions, inv_freq, interleaved, magnitude=1.0, back=False):
    """(out, |x| + |y| of every dim's pair, 0 where it does not turn), in 64 bits."""
    x = x.double().cpu()
    a = positions.double().cpu()[:, None] * inv_freq.double().cpu()
    a = (-a if back else a)[:, None]
    half = inv_freq.numel()
    out, size = x.clone(), torch.zeros_like(x)
    re, im = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (
        slice(0, half), slice(half, 2 * half))
    u, w = x[..., re], x[..., im]
    out[..., re] = magnitude * (u * a.cos() - w * a.sin())
    out[..., im] = magnitude * (w * a.cos() + u * a.sin())
    size[..., re] = size[..., im] = magnitude * (u.abs() + w.abs())
    return out, size


def check(tag, got, x, positions, inv_freq, interleaved, magnitude=1.0, back=False):
    ref, size = turned(x, positions, inv_freq, interleaved, magnitude, back)
    step, angle = (2.0 ** -8, 2.0 ** -16) if x.dtype == torch.bfloat16 else (2.0 ** -24, 2.0 ** -22)
    err = (got.double().cpu() - ref).abs()
    worst = (err / (ref.abs() * step + size * angle + 1e-40)).max().item() if err.numel() else 0.0
    say(f"[rotary] {tag}: {worst:.3f} of the bound")
    assert worst <= 1.0
    return ref


def inputs(tokens, hq, hk, d, rot, dtype, far, seed=0, base=10000.0):
    dev = device()
    gen = torch.Generator(dev).manual_seed(seed)
    normal = lambda h: torch.randn(tokens, h, d, generator=gen, device=dev).to(DTYPES[dtype])  # noqa: E731
    pos = torch.randint(-far // 8, far, (tokens,), generator=gen, device=dev, dtype=torch.int32)
    i = torch.arange(rot // 2, dtype=torch.float64, device=dev)
    return normal(hq), normal(hk) if hk else None, pos, (base ** (-2 * i / rot)).float()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,hq,hk,d,rot,far", [
    (1, 1, 0, 2, 2, 100),          # a pair
    (1, 32, 8, 128, 128, 16640),   # a token
    (7, 5, 1, 64, 64, 1 << 20),
    (33, 4, 2, 64, 32, 1 << 20),   # part of the head
    (65, 9, 3, 128, 80, 70000),    # odd chunks of a half
    (19, 3, 1, 128, 66, 5000),     # halves of no whole chunks
    (13, 2, 2, 20, 6, 5000),       # heads of no whole chunks
    (3, 130, 70, 128, 96, 5000),   # many heads; items that do not fill a wavefront
    (2, 2, 1, 1024, 1024, 5000),   # wide heads
    (9000, 2, 1, 64, 64, 1 << 30), # far positions
])
def test_rotation(tokens, hq, hk, d, rot, far, dtype, interleaved):
    from paper_2606_09441_amd import Rotary
    q, k, pos, f = inputs(tokens, hq, hk, d, rot, dtype, far)
    r = Rotary(f, interleaved=interleaved)
    keep = q.clone(), None if k is None else k.clone()
    for back in (False, True):
        qo, ko = r.rotate(q, k, pos, back=back)
        check(f"q back={back}", qo, q, pos, f, interleaved, back=back)
        if hk:
            check(f"k back={back}", ko, k, pos, f, interleaved, back=back)
        else:
            assert ko is None
    assert torch.equal(q, keep[0]) and (k is None or torch.equal(k, keep[1]))
    # in place, and from a buffer that is aligned to nothing
    apart = torch.empty(q.numel() + 1, dtype=q.dtype, device=q.device)[1:].view(q.shape).copy_(q)
    want = r.rotate(q, None, pos)[0]
    odd = r.rotate(apart, None, pos)[0]
    check("not aligned", odd, q, pos, f, interleaved)
    r.rotate_(q, k, pos)
    assert torch.equal(q, want)


def test_no_tokens():
    from paper_2606_09441_amd import Rotary
    q, k, pos, f = inputs(0, 4, 2, 64, 64, "bf16", 10)
    qo, ko = Rotary(f).rotate(q, k, pos)
    assert qo.shape == (0, 4, 64) and ko.shape == (0, 2, 64)


def test_position_zero_and_magnitude():
    from paper_2606_09441_amd import Rotary
    q, k, pos, f = inputs(40, 4, 2, 64, 32, "f32", 10)
    pos.zero_()
    qo, ko = Rotary(f, interleaved=True).rotate(q, k, pos)
    assert torch.equal(qo, q) and torch.equal(ko, k)   # cos 0 = 1, sin 0 = 0
    pos += torch.arange(40, device=pos.device, dtype=torch.int32) * 3
    for back in (False, True):
        qo, ko = Rotary(f, magnitude=1.25).rotate(q, k, pos, back=back)
        check("magnitude", qo, q, pos, f, False, 1.25, back)


def test_not_finite_stays_in_its_pair():
    from paper_2606_09441_amd import Rotary
    q, _, pos, f = inputs(3, 2, 0, 64, 32, "bf16", 1000)
    clean = Rotary(f).rotate(q, None, pos)[0]
    q[1, 0, 3], q[1, 1, 50] = float("inf"), float("nan")
    got = Rotary(f).rotate(q, None, pos)[0]
    bad = ~got.isfinite()
    where = torch.zeros_like(bad)
    where[1, 0, 3] = where[1, 0, 19] = where[1, 1, 50] = True   # a pair; a dim that stays
    assert torch.equal(bad, where)
    assert torch.equal(got[~where], clean[~where])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_than_two_to_the_31_bytes(dtype):
    """The last rows of a tensor whose byte offsets pass 32 bits."""
    from paper_2606_09441_amd import Rotary
    tokens = (1 << 31) // (128 * 128) // (4 if dtype == "f32" else 2) * 2 + 5
    dev = device()
    q = torch.zeros(tokens, 128, 128, dtype=DTYPES[dtype], device=dev)
    few, _, pos, f = inputs(5, 128, 0, 128, 128, dtype, 9000)
    q[-5:] = few
    every = torch.zeros(tokens, dtype=torch.int32, device=dev)
    every[-5:] = pos
    Rotary(f).rotate_(q, None, every)
    check("far rows", q[-5:], few, pos, f, False)
    assert not q[:-5].any()


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradients(interleaved):
    """The formula's gradient, and differences: the call is linear, so along a direction
    they are the call of that direction, up to the rounding of its outputs."""
    from paper_2606_09441_amd import Rotary
    q, k, pos, f = inputs(37, 6, 2, 64, 48, "f32", 50000, seed=3)
    r = Rotary(f, interleaved=interleaved, magnitude=1.1)
    q.requires_grad_()
    k.requires_grad_()
    qo, ko = r(q, k, pos)
    gq, gk = torch.randn_like(qo), torch.randn_like(ko)
    dq, dk = torch.autograd.grad((qo, ko), (q, k), (gq, gk))
    check("dq", dq, gq, pos, f, interleaved, 1.1, back=True)
    check("dk", dk, gk, pos, f, interleaved, 1.1, back=True)
    # <g, f(x + t) - f(x)> = <f'(g), t>
    t = torch.randn_like(q)
    diff = ((r.rotate(q.detach() + t, None, pos)[0] - qo.detach()).double() * gq.double()).sum()
    along = (dq.double() * t.double()).sum()
    # both calls' errors times |g|, and q + t's rounding; that of dq times |t|
    off = 2.0 ** -22 + 3 * 2.0 ** -24
    each = [turned(y, pos, f, interleaved, 1.1)[1] + 1.1 * y.detach().double().abs().cpu()
            for y in (q, q + t, gq)]
    size = (gq.double().abs().cpu() * (each[0] + each[1])).sum()
    size += (t.double().abs().cpu() * each[2]).sum()
    assert abs(diff - along).item() <= off * size.item()
    # expanded and missing gradients, one output alone, and the gradient of a gradient
    qo, ko = r(q, k, pos)
    dq, = torch.autograd.grad(qo.sum(), (q,), create_graph=False)
    check("expanded", dq, torch.ones_like(q), pos, f, interleaved, 1.1, back=True)
    g = torch.randn_like(q).requires_grad_()
    qo, _ = r(q, None, pos)
    dq, = torch.autograd.grad(qo, (q,), g, create_graph=True)
    ddg, = torch.autograd.grad(dq, (g,), t)
    check("twice", ddg, t, pos, f, interleaved, 1.1)


def test_one_leaf_for_both():
    """q and k cut from one projection: their gradients meet in it."""
    from paper_2606_09441_amd import Rotary
    x, _, pos, f = inputs(21, 6, 0, 64, 64, "bf16", 900)
    x.requires_grad_()
    q, k = x[:, :4].contiguous(), x[:, 4:].contiguous()
    qo, ko = Rotary(f)(q, k, pos)
    g = torch.randn_like(x)
    torch.autograd.backward((qo, ko), (g[:, :4], g[:, 4:]))
    check("leaf", x.grad, g, pos, f, False, back=True)


def test_streams_and_graphs():
    """On another stream than the tensors' own, and captured: every replay with new
    inputs gives what a call outside gives."""
    from paper_2606_09441_amd import Rotary
    q, k, pos, f = inputs(200, 8, 2, 128, 128, "bf16", 5000)
    r = Rotary(f)
    want = r.rotate(q, k, pos)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = r.rotate(q, k, pos, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    g = torch.randn_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fwd = r.rotate(q, k, pos)
        bwd = r.rotate(g, None, pos, back=True)[0]
    for i in range(3):
        q.copy_(torch.randn_like(q))
        pos += 17
        graph.replay()
        torch.cuda.synchronize()
        now = r.rotate(q, k, pos)
        assert torch.equal(fwd[0], now[0]) and torch.equal(fwd[1], now[1])
        assert torch.equal(bwd, r.rotate(g, None, pos, back=True)[0])


def test_no_gradients_in_a_captured_graph():
    """Refused before anything is recorded; without gradients such a call is as any."""
    from paper_2606_09441_amd import Rotary, SiftError
    q, k, pos, f = inputs(50, 4, 2, 64, 64, "bf16", 300)
    r = Rotary(f)
    want = r.rotate(q, k, pos)
    leaf = k.clone().requires_grad_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(SiftError, match="captured"):
            r(q, leaf, pos)
        got = r(q, k, pos)
        with torch.no_grad():
            again = r(q, leaf, pos)
    for _ in range(3):
        for x in got + again:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got + again, want + want))


def test_moved_keys():
    """Keys turned back from their document's positions and on to the prompt's are, to
    two roundings and both cosines' errors, those turned at once."""
    from paper_2606_09441_amd import Rotary
    _, k, pos, f = inputs(300, 1, 8, 128, 128, "f32", 2000)
    r = Rotary(f)
    pos.abs_()
    at = r.rotate(k, None, pos)[0]
    moved = r.rotate(r.rotate(at, None, pos, back=True)[0], None, pos + 7000)[0]
    once, size = turned(k, pos + 7000, f, False)
    assert ((moved.double().cpu() - once).abs() <= 3 * 1.5 * (2.0 ** -22 + 2.0 ** -24) * size).all()


def test_layer_with_a_rotary():
    """The decoder layer's slice, to its own tolerance (2% of max |out|)."""
    from paper_2606_09441_amd import Plan, Rotary
    from paper_2606_09441_amd.layer import PrefillLayer
    hq, hkv, d = 4, 2, 128
    wl = W.custom([[300, 129, 75]], tile=64, hq=hq, hkv=hkv, d=d, dtype="bf16", seed=5, p_la=0.5,
                  p_ca=0.4)
    w = W.layer_weights(hq * d, hq, hkv, d, 2 * hq * d, seed=1)
    x = W.layer_input(wl.tokens, hq * d, seed=2)
    pos = W.prompt_positions(wl.seg_offsets, wl.prompt_seg_ptr)
    f = W.rope_inv_freq(d)
    up = lambda a: torch.from_numpy(a).to(device())  # noqa: E731
    layer = PrefillLayer({n: up(v).bfloat16() for n, v in w.items()}, hq, hkv, d, Rotary(up(f)))
    with Plan(wl.seg_offsets, wl.prompt_seg_ptr, hq, hkv, d, 64) as plan:
        out = layer.forward(up(x).bfloat16(), plan, up(pos), up(wl.la), up(wl.ca))
        torch.cuda.synchronize()
    ref = LO.layer_slice(oracle_layout(wl), x, w, wl.la, wl.ca, pos, f, hq, hkv, d)
    assert np.abs(out.float().cpu().numpy() - ref).max() <= 0.02 * np.abs(ref).max()
