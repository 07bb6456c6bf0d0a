"""GPU: what Rotary's calls in place and its gradient leave to autograd: no gradient is
silently another call's."""

import pytest
import torch

from gpu_helpers import device

pytestmark = pytest.mark.gpu

TOKENS, D = 7, 64


def inputs():
    from paper_2606_09441_amd import Rotary, rotary_frequencies
    gen = torch.Generator().manual_seed(3)
    q, k = (torch.randn(TOKENS, h, D, generator=gen).to(device()) for h in (4, 2))
    pos = torch.arange(TOKENS, dtype=torch.int32, device=device()) * 11
    return q, k, pos, Rotary(rotary_frequencies(D)[0])


@pytest.mark.parametrize("which", ["q", "k"])
@pytest.mark.parametrize("leaf", [True, False])
def test_nothing_in_a_graph_is_written(which, leaf):
    from paper_2606_09441_amd import SiftError
    q, k, pos, r = inputs()
    mine = (q if which == "q" else k).requires_grad_()
    if not leaf:
        mine = mine * 2
    was = mine.detach().clone()
    q, k = (mine, k) if which == "q" else (q, mine)
    with pytest.raises(SiftError) as e:
        r.rotate_(q, k, pos)
    assert e.value.status == 4
    with pytest.raises(SiftError) as e:
        r.rotate(q.detach(), k.detach(), pos, q_out=q, k_out=k)
    assert e.value.status == 4
    assert torch.equal(mine.detach(), was)
    want = r.rotate(q.detach(), k.detach(), pos)
    with torch.no_grad():   # as any operation in place
        got = r.rotate_(q, k, pos)
    assert torch.equal(got[0].detach(), want[0]) and torch.equal(got[1].detach(), want[1])


def test_a_tensor_saved_for_a_gradient_and_then_turned():
    q, k, pos, r = inputs()
    w = torch.ones_like(q, requires_grad=True)
    y = (w * q).sum()
    r.rotate_(q, k, pos)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    z = torch.empty_like(k)
    y = (w[:, :2] * z).sum()
    r.rotate(q, k, pos, k_out=z)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_a_table_changed_between_a_call_and_its_gradient():
    q, k, pos, r = inputs()
    q.requires_grad_()
    out, _ = r(q, k, pos)
    r.inv_freq.mul_(2)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()


def test_in_inference_mode():
    q, k, pos, r = inputs()
    want = r.rotate(q, k, pos)
    with torch.inference_mode():
        a, b = q.clone(), k.clone()
        r.rotate_(a, b, pos)
    assert torch.equal(a, want[0]) and torch.equal(b, want[1])
    a, b = r.rotate_(a, b, pos, back=True)   # and outside of it
    assert torch.allclose(a, q, atol=1e-5) and torch.allclose(b, k, atol=1e-5)


def test_a_layer_whose_weights_require_gradients():
    """Runs as without: the attention records none."""
    from paper_2606_09441_amd.layer import PrefillLayer
    hq, hkv, d = 4, 2, D
    gen = torch.Generator().manual_seed(1)
    draw = lambda *s: (torch.randn(*s, generator=gen) / 16).bfloat16().to(device())  # noqa: E731
    *_, pos, r = inputs()
    w = {"w_in": draw(hq * d), "Wqkv": draw((hq + 2 * hkv) * d, hq * d), "Wo": draw(hq * d, hq * d)}
    x = draw(TOKENS, hq * d)

    class Plan:
        def run(self, q, k, v, la, ca):
            seen.append((q.detach(), k.detach()))
            return q.detach()

    outs, seen = [], []
    for grad in (False, True):
        # (the norm's stays as it is: recorded, another path rounds elsewhere)
        mine = {n: t.clone().requires_grad_(grad and n != "w_in") for n, t in w.items()}
        layer = PrefillLayer(mine, hq, hkv, d, r)
        outs.append(layer.attention_block(x, Plan(), pos, None, None).detach())
    assert torch.equal(*outs) and all(torch.equal(a, b) for a, b in zip(*seen))
