"""What PromptCache refuses before anything is written, on the host: its handles are
stand-ins that record their calls."""

import pytest
import torch

from paper_2606_09441_amd import SiftError
from paper_2606_09441_amd.serve import PromptCache

HQ, HKV, D, TOKENS = 4, 2, 64, 40


class Calls:
    """Takes any call, and remembers it."""

    hq, hkv, d, num_seqs, slots = HQ, HKV, D, 2, 64
    device = torch.device("cpu")

    def __init__(self, names):
        self.names = names

    def __getattr__(self, name):
        return lambda *a, **kw: self.names.append(name)


def prompts(rotary=False):
    """Two prompts of 15 and 5, and of 12 and 8 tokens, not prefilled; the calls."""
    names = []
    p = object.__new__(PromptCache)
    p.cache = p.plan = p._queries = p.pages = Calls(names)
    p.rotary = Calls(names) if rotary else None
    p.weights, p._pending, p._codes, p._dtype = None, None, False, torch.bfloat16
    p._slots = torch.arange(TOKENS, dtype=torch.int32)
    p._token_ptr = torch.tensor([0, 20, 40], dtype=torch.int32)
    p._token_pos = torch.arange(TOKENS, dtype=torch.int32) % 20
    p._query = torch.tensor([*range(15, 20), *range(32, 40)])
    p._query_ptr, p._query_rows = torch.tensor([0, 5, 13], dtype=torch.int32), [0, 5, 13]
    p._tile_page = p._query_pos = p._slots
    return p, names


def tensors(**other):
    return {n: torch.zeros(other.get(n, (TOKENS, HQ if n == "q" else HKV, D)),
                           dtype=other.get("dtype", torch.bfloat16)) for n in "qkv"}


WRONG = [{n: s for n in names} for names in ("q", "k", "v", "kv", "qkv")
         for s in [(TOKENS - 1, HQ if names == "q" else HKV, D)]]
WRONG += [{"k": (0, HKV, D), "v": (0, HKV, D)}, {"k": (TOKENS + 1, HKV, D)}, {"k": (TOKENS, 1, D)},
          {"v": (TOKENS, HKV, 2 * D)}, {"q": (TOKENS, HQ - 1, D)}, {"q": (TOKENS, HQ * D)}]


@pytest.mark.parametrize("rotary", [False, True])
@pytest.mark.parametrize("sparse", [False, True])
@pytest.mark.parametrize("wrong", WRONG + [{"dtype": torch.float32}])
def test_prefill_takes_the_prompts_tokens(wrong, sparse, rotary):
    p, names = prompts(rotary)
    bits = torch.zeros(8, dtype=torch.uint8)
    with pytest.raises(SiftError) as e:
        p.prefill(**tensors(**wrong), **(dict(la=bits, ca=bits) if sparse else {}))
    assert e.value.status == 2 and names == []


def test_prefill_takes_tensors_of_its_device():
    for one in "qkv":
        p, names = prompts()
        t = tensors()
        t[one] = t[one].to("meta")
        with pytest.raises(SiftError) as e:
            p.prefill(**t)
        assert e.value.status == 7 and names == []


def test_prefill_goes_on_with_the_right_ones():
    p, names = prompts()
    p.prefill(**tensors())
    assert names == ["append", "dense", "accumulate"]


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("short", ["k_new", "v_new", "lse", "row_pos"])
def test_append_takes_as_many_rows_as_the_step(short, codes):
    """rows are indexes into all of them."""
    p, names = prompts()
    p.weights, p._codes, p.used, p.max_rows = torch.zeros(2, HKV, 64), codes, 0, 8
    p.next_pos = torch.zeros(2, dtype=torch.int32)
    p.pages.k_pages, p.pages.lens = torch.zeros(128, HKV, D), p.next_pos
    p._score = dict(scale=None, cap=0.0, slopes=None)
    t = {"k_new": torch.zeros(8, HKV, D), "v_new": torch.zeros(8, HKV, D),
         "row_pos": torch.arange(8, dtype=torch.int32)}
    t = {n: x.to(torch.bfloat16) if x.dim() == 3 else x for n, x in t.items()}
    t |= {"q": torch.zeros(8, HQ, D, dtype=torch.bfloat16), "lse": torch.zeros(8, HQ)}
    p.append(**t, rows=torch.tensor([0, 5, 7]))
    assert names == (["append"] if codes else ["accumulate", "append"])
    names.clear()
    t[short] = t[short][:7]
    if codes and short == "lse":     # not read
        p.append(**t, rows=torch.tensor([0, 5, 7]))
        return
    with pytest.raises(SiftError) as e:
        p.append(**t, rows=torch.tensor([0, 5, 7]))
    assert e.value.status == 2 and names == []
